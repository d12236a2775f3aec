// Rows of a table of embeddings, and the table's gradient.
//
//   out_t = s E[token_t]                 dE[v] = s sum_{t: token_t = v} dy_t
//
// Both move bytes and compute next to nothing, so what bounds them is memory where they are large and the latency of launches
// where they are small.  The gradient sorts the tokens (stable, so that a row's terms are added in the order of t), finds where each token's run of
// rows begins and ends, and then writes every row of the gradient once: zeros, or the sum of its run.  Runs of more than 64 rows (frequent tokens have
// thousands) would leave one wavefront working for long: they are summed beforehand by parts of up to 64 rows.
#include <type_traits>

#include "rfast_operators.h"

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 64;  // sorted rows whose sum a wavefront makes beforehand

struct Lookup {
  const void* table;
  const int32_t* tokens;
  void* out;
  int64_t ld_table, ld_out;
  int32_t rows, vocabulary, d;
  float scale;
};

// LANES lanes take a row, eight columns each at a time; wide rows are cut into slabs of 512 columns, a wavefront each.
template <class IN, class OUT, int LANES> __global__ void __launch_bounds__(kThreads) rfast_embedding_kernel(Lookup a, int slabs) {
  const int64_t unit = (((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kThreads + threadIdx.x) / LANES;
  const int64_t row = unit / slabs;
  if (row >= a.rows) return;
  const int col = ((int)(unit % slabs) * LANES + threadIdx.x % LANES) * 8;
  if (col >= a.d) return;
  const int32_t token = a.tokens[row];
  float v[8] = {};
  if ((uint32_t)token < (uint32_t)a.vocabulary) {
    load_eight<false>((const IN*)a.table + token * a.ld_table + col, a.d - col, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= a.scale;
  }
  store_eight<false>((OUT*)a.out + row * a.ld_out + col, a.d - col, v);
}

struct Back {
  const void* dy;
  const int32_t* sorted;  // [rows] tokens in order, `vocabulary` for padding
  const int32_t* order;   // [rows] the row of dy
  int32_t* begin;         // [vocabulary] of the tokens that are there; the others' hold anything
  int32_t* end;
  float* part;            // [chunks][2][d]
  void* grad;
  int64_t ld_dy, ld_grad;
  int32_t rows, vocabulary, d, slabs;
  float scale;
};

// Sum of dy over sorted positions [lo, hi), eight columns of a lane.
template <class IN> __device__ inline void sum_rows(const Back& a, int32_t lo, int32_t hi, int col, float* v) {
  const IN* dy = (const IN*)a.dy + col;
#pragma unroll 4
  for (int32_t p = lo; p < hi; ++p) {
    float t[8];
    load_eight<false>(dy + a.order[p] * a.ld_dy, a.d - col, t);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += t[j];
  }
}

// A wavefront per chunk of 64 sorted positions and slab of 512 columns: where runs begin and end, and the sums of the chunk's parts of long runs.
// A run of more than 64 rows that has a part of this chunk has its first or its last position, so there are at most two.
template <class IN> __global__ void __launch_bounds__(kThreads) rfast_embedding_runs(Back a) {
  const int64_t unit = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (kThreads / 64) + threadIdx.x / 64;
  const int64_t chunk = unit / a.slabs, first = chunk * kChunk;
  if (first >= a.rows) return;
  const int slab = (int)(unit % a.slabs), lane = threadIdx.x & 63;
  const int64_t p = first + lane;
  const int count = (int)min((int64_t)kChunk, a.rows - first);
  const int32_t mine = p < a.rows ? a.sorted[p] : -1;
  const int32_t back = chunk > 0 ? a.sorted[p - kChunk] : -1;             // the chunk before
  const int32_t ahead = p + kChunk < a.rows ? a.sorted[p + kChunk] : -1;  // the chunk behind
  const int32_t before = __shfl_up(mine, 1, 64), after = __shfl_down(mine, 1, 64);
  const int32_t last = __shfl(back, 63, 64), next = __shfl(ahead, 0, 64);
  const int32_t left = lane > 0 ? before : last, right = lane < 63 ? after : next;
  const bool token = mine >= 0 && mine < a.vocabulary;
  if (slab == 0 && token) {
    if (left != mine) a.begin[mine] = (int32_t)p;
    if (right != mine) a.end[mine] = (int32_t)p + 1;
  }
  const int col = (slab * 64 + lane) * 8;
  const int32_t head = __shfl(mine, 0, 64), tail = __shfl(mine, count - 1, 64);
  const uint64_t in_head = __ballot(mine == head), in_tail = __ballot(mine == tail);
  const int behind = __popcll(__ballot(back == head)), beyond = __popcll(__ballot(ahead == tail));
  const int n_head = __popcll(in_head), n_tail = __popcll(in_tail);
  // (where one run has the whole chunk, both counts apply)
  if (head != a.vocabulary && behind + n_head + (head == tail ? beyond : 0) > kChunk && col < a.d) {
    float v[8] = {};
    sum_rows<IN>(a, (int32_t)first, (int32_t)first + n_head, col, v);
    store_eight<false>(a.part + (2 * chunk) * a.d + col, a.d - col, v);
  }
  if (tail != head && tail != a.vocabulary && n_tail + beyond > kChunk && col < a.d) {
    float v[8] = {};
    sum_rows<IN>(a, (int32_t)first + count - n_tail, (int32_t)first + count, col, v);
    store_eight<false>(a.part + (2 * chunk + 1) * a.d + col, a.d - col, v);
  }
}

// LANES lanes per row of the gradient (or, where it is accumulated, per sorted position, of which the first of a run works).
template <class IN, class OUT, int LANES, bool ADD> __global__ void __launch_bounds__(kThreads) rfast_embedding_grad(Back a, int64_t units) {
  const int64_t unit = (((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kThreads + threadIdx.x) / LANES;
  if (unit >= units) return;
  const int64_t at = unit / a.slabs;
  const int col = ((int)(unit % a.slabs) * LANES + threadIdx.x % LANES) * 8;
  if (col >= a.d) return;
  int32_t token, lo = 0, hi = 0;
  if constexpr (ADD) {
    token = a.sorted[at];
    if (token >= a.vocabulary || (at > 0 && a.sorted[at - 1] == token)) return;
    lo = (int32_t)at;
    hi = a.end[token];
  } else {
    token = (int32_t)at;
    // begin[] is not cleared: a number counts only if a run of this very token begins there, whatever was in memory
    const int32_t b = a.begin[at];
    if ((uint32_t)b < (uint32_t)a.rows && a.sorted[b] == token && (b == 0 || a.sorted[b - 1] != token)) lo = b, hi = a.end[at];
  }
  float v[8] = {};
  if (hi - lo > kChunk) {
    const float* part = a.part + col;
    for (int32_t c = lo / kChunk; c <= (hi - 1) / kChunk; ++c) {
      float t[8];
      load_eight<false>(part + (2 * (int64_t)c + (lo > c * kChunk)) * a.d, a.d - col, t);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += t[j];
    }
  } else {
    sum_rows<IN>(a, lo, hi, col, v);
  }
  OUT* grad = (OUT*)a.grad + token * a.ld_grad + col;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] *= a.scale;
  if constexpr (ADD) {
    float had[8];
    load_eight<false>(grad, a.d - col, had);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += had[j];
  }
  store_eight<false>(grad, a.d - col, v);
}

// Lanes per row of d columns, eight of them each: a power of two from 8 to 64.
template <class F> hipError_t by_lanes(int32_t d, F go) {
  using std::integral_constant;
  if (d <= 64) return go(integral_constant<int, 8>());
  if (d <= 128) return go(integral_constant<int, 16>());
  if (d <= 256) return go(integral_constant<int, 32>());
  return go(integral_constant<int, 64>());
}
int slabs_of(int32_t d) { return (d + 511) / 512; }

size_t up(size_t b) { return (b + 255) / 256 * 256; }
struct Layout {
  size_t order, sorted, begin, end, part, sort, total;
  Layout(int32_t rows, int32_t vocabulary, int32_t d) {
    size_t at = 0;
    const auto take = [&](size_t bytes) {
      const size_t here = at;
      at += up(bytes);
      return here;
    };
    order = take((size_t)rows * 4);
    sorted = take((size_t)rows * 4);
    begin = take((size_t)vocabulary * 4);
    end = take((size_t)vocabulary * 4);
    part = take(rows > kChunk ? ((size_t)rows + kChunk - 1) / kChunk * 2 * d * 4 : 0);
    sort = take(rfast_sort_bytes(rows, vocabulary));
    total = at;
  }
};

bool sizes_ok(int32_t rows, int32_t vocabulary, int32_t d) { return rows >= 0 && vocabulary >= 1 && d >= 1 && d <= 0x7ffffc00; }  // (columns of whole slabs stay within 32 bits)

}  // namespace

extern "C" int rfast_embedding(int32_t rows, int32_t vocabulary, int32_t d, const void* table, int32_t table_type, int64_t ld_table,
                               const int32_t* tokens, float scale, void* out, int32_t out_type, int64_t ld_out, void* hip_stream) {
  if (!sizes_ok(rows, vocabulary, d)) return rfast_refuse(RFAST_EINVAL, "need rows >= 0, vocabulary >= 1 and d 1 .. 2^31 - 1024");
  if (!rfast_type_ok(table_type) || !rfast_type_ok(out_type)) return rfast_refuse(RFAST_EINVAL, "types must be RFAST_F32 or RFAST_BF16");
  if (rows == 0) return RFAST_OK;
  if (!table || !tokens || !out) return rfast_refuse(RFAST_EINVAL, "NULL argument");
  if (ld_table < d || ld_out < d) return rfast_refuse(RFAST_EINVAL, "rows are at least d elements apart");
  const int tw = rfast_type_bytes(table_type), ow = rfast_type_bytes(out_type);
  if ((uintptr_t)table % tw || (uintptr_t)out % ow || (uintptr_t)tokens % 4)
    return rfast_refuse(RFAST_EINVAL, "an address is no multiple of its element's size");
  const RfastArea o = {out, rows, ld_out * ow, (int64_t)d * ow};
  if (rfast_overlap(o, {table, vocabulary, ld_table * tw, (int64_t)d * tw}) || rfast_overlap(o, {tokens, 1, 4 * (int64_t)rows, 4 * (int64_t)rows}))
    return rfast_refuse(RFAST_EINVAL, "the output overlaps an input");
  const Lookup a = {table, tokens, out, ld_table, ld_out, rows, vocabulary, d, scale};
  const hipStream_t s = (hipStream_t)hip_stream;
  const hipError_t e = by_lanes(d, [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    const int slabs = slabs_of(d);
    const dim3 grid = rfast_grid_of(((int64_t)rows * slabs * L + kThreads - 1) / kThreads);
    const bool tf = table_type == RFAST_F32, of = out_type == RFAST_F32;
    if (tf && of) hipLaunchKernelGGL((rfast_embedding_kernel<float, float, L>), grid, dim3(kThreads), 0, s, a, slabs);
    else if (tf) hipLaunchKernelGGL((rfast_embedding_kernel<float, u16, L>), grid, dim3(kThreads), 0, s, a, slabs);
    else if (of) hipLaunchKernelGGL((rfast_embedding_kernel<u16, float, L>), grid, dim3(kThreads), 0, s, a, slabs);
    else hipLaunchKernelGGL((rfast_embedding_kernel<u16, u16, L>), grid, dim3(kThreads), 0, s, a, slabs);
    return hipGetLastError();
  });
  return e == hipSuccess ? RFAST_OK : rfast_refuse_hip(e, "embedding launch");
}

extern "C" size_t rfast_embedding_backward_workspace_bytes(int32_t rows, int32_t vocabulary, int32_t d) {
  return sizes_ok(rows, vocabulary, d) ? Layout(rows, vocabulary, d).total : 0;
}

extern "C" int rfast_embedding_backward(int32_t rows, int32_t vocabulary, int32_t d, const void* dy, int32_t dy_type, int64_t ld_dy,
                                        const int32_t* tokens, float scale, void* grad, int32_t grad_type, int64_t ld_grad, int32_t accumulate,
                                        void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!sizes_ok(rows, vocabulary, d)) return rfast_refuse(RFAST_EINVAL, "need rows >= 0, vocabulary >= 1 and d 1 .. 2^31 - 1024");
  if (!rfast_type_ok(dy_type) || !rfast_type_ok(grad_type)) return rfast_refuse(RFAST_EINVAL, "types must be RFAST_F32 or RFAST_BF16");
  if (accumulate != 0 && accumulate != 1) return rfast_refuse(RFAST_EINVAL, "accumulate must be 0 or 1");
  if (!grad || (rows && (!dy || !tokens))) return rfast_refuse(RFAST_EINVAL, "NULL argument");
  if (ld_grad < d || (rows && ld_dy < d)) return rfast_refuse(RFAST_EINVAL, "rows are at least d elements apart");
  const int yw = rfast_type_bytes(dy_type), gw = rfast_type_bytes(grad_type);
  if ((rows && ((uintptr_t)dy % yw || (uintptr_t)tokens % 4)) || (uintptr_t)grad % gw)
    return rfast_refuse(RFAST_EINVAL, "an address is no multiple of its element's size");
  const Layout at(rows, vocabulary, d);
  if (!workspace || (uintptr_t)workspace % 256) return rfast_refuse(RFAST_EINVAL, "the workspace must be 256-byte aligned");
  if (workspace_bytes < at.total) return rfast_refuse(RFAST_ENOMEM, "workspace too small: need " + std::to_string(at.total) + " bytes");
  const RfastArea g = {grad, vocabulary, ld_grad * gw, (int64_t)d * gw}, y = {dy, rows, ld_dy * yw, (int64_t)d * yw},
                  t = {tokens, 1, 4 * (int64_t)rows, 4 * (int64_t)rows}, w = {workspace, 1, (int64_t)at.total, (int64_t)at.total};
  if (rfast_overlap(g, y) || (rows && rfast_overlap(g, t))) return rfast_refuse(RFAST_EINVAL, "the gradient overlaps an input");
  if (rfast_overlap(w, g) || rfast_overlap(w, y) || (rows && rfast_overlap(w, t))) return rfast_refuse(RFAST_EINVAL, "the workspace overlaps a tensor");
  if (rows == 0 && accumulate) return RFAST_OK;
  char* ws = (char*)workspace;
  const hipStream_t s = (hipStream_t)hip_stream;
  Back a = {dy, (int32_t*)(ws + at.sorted), (int32_t*)(ws + at.order), (int32_t*)(ws + at.begin), (int32_t*)(ws + at.end), (float*)(ws + at.part), grad,
            ld_dy, ld_grad, rows, vocabulary, d, slabs_of(d), scale};
  hipError_t e = hipSuccess;
  const bool yf = dy_type == RFAST_F32, gf = grad_type == RFAST_F32;
  if (rows) {
    e = rfast_sort({rows, vocabulary, tokens, nullptr, nullptr, (int32_t*)a.order, (int32_t*)a.sorted, ws + at.sort}, s);
    if (e != hipSuccess) return rfast_refuse_hip(e, "sort launch");
    const int64_t waves = ((int64_t)rows + kChunk - 1) / kChunk * a.slabs;
    const dim3 grid = rfast_grid_of((waves + kThreads / 64 - 1) / (kThreads / 64));
    if (yf) hipLaunchKernelGGL((rfast_embedding_runs<float>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((rfast_embedding_runs<u16>), grid, dim3(kThreads), 0, s, a);
  }
  e = by_lanes(d, [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    const int64_t units = (int64_t)(accumulate ? rows : vocabulary) * a.slabs;
    const dim3 grid = rfast_grid_of((units * L + kThreads - 1) / kThreads);
    const auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, a, units);
      return hipGetLastError();
    };
    if (accumulate) {
      if (yf) return gf ? go(rfast_embedding_grad<float, float, L, true>) : go(rfast_embedding_grad<float, u16, L, true>);
      return gf ? go(rfast_embedding_grad<u16, float, L, true>) : go(rfast_embedding_grad<u16, u16, L, true>);
    }
    if (yf) return gf ? go(rfast_embedding_grad<float, float, L, false>) : go(rfast_embedding_grad<float, u16, L, false>);
    return gf ? go(rfast_embedding_grad<u16, float, L, false>) : go(rfast_embedding_grad<u16, u16, L, false>);
  });
  return e == hipSuccess ? RFAST_OK : rfast_refuse_hip(e, "embedding gradient launch");
}
