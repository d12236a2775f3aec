// Softmax cross-entropy of rows of logits with its gradient.
//
//   lse = log sum exp l_k,  loss = lse - l_label,  grad_k = c (exp(l_k - lse) - [k == label])
//
// Some five operations per logit, so the bound is one read of the logits and one write of the gradient.  A row therefore stays in
// registers between the two: a wavefront's up to kWaveMost logits, a workgroup's of 256 or 1024 lanes beyond.  Rows longer than the registers
// of a workgroup are read twice, the second time through the caches, with a running maximum and sum per lane in the first pass.
// A row's maximum is taken out of its exponents before they are formed, so that nothing overflows; sums are in 32 bits,
// one per lane and then a tree.
#include <type_traits>

#include "rfast_operators.h"

namespace {

struct Args {
  const void* logits;
  const int32_t* labels;
  float* loss;
  float* lse;
  void* grad;
  const int32_t* d_rows;
  int64_t ld_logits, ld_grad;
  int32_t rows, K;
  float scale;
};

template <class T> constexpr int kGroup = 16 / (int)sizeof(T);  // logits per 16-byte load

// A group of logits from p on, of which `left` (1 or more) exist; the others are classes that are masked out.
__device__ inline void load_group(const float* p, int left, float* v) {
  if (left >= 4) load_four<false>(p, 4, v);
  else
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = q < left ? p[q] : -INFINITY;
}
__device__ inline void load_group(const u16* p, int left, float* v) {
  if (left >= 8) {
    const any_u32x4 t = *reinterpret_cast<const any_u32x4*>(p);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v[2 * q] = __uint_as_float(t[q] << 16);
      v[2 * q + 1] = __uint_as_float(t[q] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = q < left ? from_bf16(p[q]) : -INFINITY;
  }
}
template <int N> __device__ inline void store_group(float* p, int left, const float* v) {
#pragma unroll
  for (int q = 0; q < N; q += 4)
    if (left > q) store_four<false>(p + q, left - q, v + q);
}
template <int N> __device__ inline void store_group(u16* p, int left, const float* v) {
  if constexpr (N == 8) {
    if (left >= 8) {
      const any_u32x4 t = {to_bf16_pair(v[0], v[1]), to_bf16_pair(v[2], v[3]), to_bf16_pair(v[4], v[5]), to_bf16_pair(v[6], v[7])};
      *reinterpret_cast<any_u32x4*>(p) = t;
      return;
    }
  }
#pragma unroll
  for (int q = 0; q < N; q += 4)
    if (left > q) store_four<false>(p + q, left - q, v + q);
}

// over the row's lanes: those of a wavefront, or of the workgroup through `box` (two arrays used in turn)
template <int LANES, class F> __device__ inline float row_reduce(float v, float* box, F f) {
  v = wave_reduce(v, f);
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = v;
    __syncthreads();
    v = box[0];
#pragma unroll
    for (int w = 1; w < LANES / 64; ++w) v = f(v, box[w]);
  }
  return v;
}

// What a row comes to, from its largest logit (-infinity: none above it) and the sum of exp(l - shift)
struct RowEnd {
  float lse, inverse, shift, log_sum;  // probability of l = exp(l - shift) * inverse
};
__device__ inline float shift_of(float top) { return top == -INFINITY ? 0.f : top; }
__device__ inline RowEnd row_end(float shift, float sum) {
  if (sum == 0.f) return {-INFINITY, 0.f, 0.f, 0.f};  // every class is masked out
  const float l = logf(sum);
  return {shift + l, 1.f / sum, shift, l};
}
// (not lse - l_label: beside a large shift the logarithm would lose its digits)
__device__ inline float loss_of(const RowEnd& e, float label_logit) { return e.lse == -INFINITY ? 0.f : e.log_sum + (e.shift - label_logit); }
__device__ inline float grad_of(const RowEnd& e, float l, bool at_label, float scale) {
  if (e.lse == -INFINITY) return 0.f;
  return (__expf(l - e.shift) * e.inverse - (at_label ? 1.f : 0.f)) * scale;
}

template <class OUT> __device__ inline void zero_row(OUT* grad, int K, int lane, int lanes) {
  for (int k = lane; k < K; k += lanes) grad[k] = (OUT)0;
}

// LANES lanes hold a row, GROUPS groups of logits each.  LANES = 64: four rows per workgroup.
template <class IN, class OUT, int LANES, int GROUPS>
__global__ void __launch_bounds__(LANES == 64 ? 256 : LANES) rfast_xent_kernel(Args a) {
  constexpr int N = kGroup<IN>;
  __shared__ float box[2][16];
  const int lane = LANES == 64 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  const int64_t row = LANES == 64 ? block * 4 + (threadIdx.x >> 6) : block;
  if (row >= a.rows || (a.d_rows && row >= *a.d_rows)) return;
  const IN* l = (const IN*)a.logits + row * a.ld_logits;
  OUT* grad = a.grad ? (OUT*)a.grad + row * a.ld_grad : nullptr;
  const int label = a.labels[row];
  const bool counts = label >= 0 && label < a.K;
  if (!counts && !a.lse) {
    if (lane == 0 && a.loss) a.loss[row] = 0.f;
    if (grad) zero_row(grad, a.K, lane, LANES);
    return;
  }
  float v[GROUPS][N];
#pragma unroll
  for (int q = 0; q < GROUPS; ++q) {
    const int k = (q * LANES + lane) * N;
    if (k < a.K) load_group(l + k, a.K - k, v[q]);
    else
#pragma unroll
      for (int j = 0; j < N; ++j) v[q][j] = -INFINITY;
  }
  float own = 0.f;  // the label's logit, held by one lane
  if (counts) own = sizeof(IN) == 4 ? ((const float*)l)[label] : from_bf16(((const u16*)l)[label]);
  float top = -INFINITY;
#pragma unroll
  for (int q = 0; q < GROUPS; ++q)
#pragma unroll
    for (int j = 0; j < N; ++j) top = fmaxf(top, v[q][j]);
  const float shift = shift_of(row_reduce<LANES>(top, box[0], [](float x, float y) { return fmaxf(x, y); }));
  float sum = 0.f;
#pragma unroll
  for (int q = 0; q < GROUPS; ++q)
#pragma unroll
    for (int j = 0; j < N; ++j) sum += __expf(v[q][j] - shift);
  const RowEnd e = row_end(shift, row_reduce<LANES>(sum, box[1], [](float x, float y) { return x + y; }));
  if (lane == 0) {
    if (a.lse) a.lse[row] = e.lse;
    if (a.loss) a.loss[row] = counts ? loss_of(e, own) : 0.f;
  }
  if (!grad) return;
#pragma unroll
  for (int q = 0; q < GROUPS; ++q) {
    const int k = (q * LANES + lane) * N;
    if (k >= a.K) break;
    float g[N];
#pragma unroll
    for (int j = 0; j < N; ++j) g[j] = counts ? grad_of(e, v[q][j], k + j == label, a.scale) : 0.f;
    store_group<N>(grad + k, a.K - k, g);
  }
}

// Rows that no workgroup's registers hold.
template <class IN, class OUT>
__global__ void __launch_bounds__(1024) rfast_xent_long_kernel(Args a) {
  constexpr int N = kGroup<IN>;
  __shared__ float box[2][16];
  const int64_t row = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (row >= a.rows || (a.d_rows && row >= *a.d_rows)) return;
  const IN* l = (const IN*)a.logits + row * a.ld_logits;
  OUT* grad = a.grad ? (OUT*)a.grad + row * a.ld_grad : nullptr;
  const int label = a.labels[row];
  const bool counts = label >= 0 && label < a.K;
  if (!counts && !a.lse) {
    if (threadIdx.x == 0 && a.loss) a.loss[row] = 0.f;
    if (grad) zero_row(grad, a.K, threadIdx.x, 1024);
    return;
  }
  float own = 0.f;
  if (counts) own = sizeof(IN) == 4 ? ((const float*)l)[label] : from_bf16(((const u16*)l)[label]);
  float top = -INFINITY, sum = 0.f;  // of this lane's logits so far; sum of exp(l - shift_of(top))
  for (int64_t k = (int64_t)threadIdx.x * N; k < a.K; k += 1024 * N) {
    float v[N];
    load_group(l + k, (int)(a.K - k), v);
    float m = top;
#pragma unroll
    for (int j = 0; j < N; ++j) m = fmaxf(m, v[j]);
    const float shift = shift_of(m);
    sum *= top == -INFINITY ? 1.f : __expf(top - shift);  // (top = -infinity: the sum is 0, or NaN)
    top = m;
#pragma unroll
    for (int j = 0; j < N; ++j) sum += __expf(v[j] - shift);
  }
  const float shift = shift_of(row_reduce<1024>(top, box[0], [](float x, float y) { return fmaxf(x, y); }));
  sum *= top == -INFINITY ? 1.f : __expf(top - shift);
  const RowEnd e = row_end(shift, row_reduce<1024>(sum, box[1], [](float x, float y) { return x + y; }));
  if (threadIdx.x == 0) {
    if (a.lse) a.lse[row] = e.lse;
    if (a.loss) a.loss[row] = counts ? loss_of(e, own) : 0.f;
  }
  if (!grad) return;
  // (where the gradient takes the logits' place, `own` has been read before any lane writes: the reductions are barriers)
  for (int64_t k = (int64_t)threadIdx.x * N; k < a.K; k += 1024 * N) {
    float v[N], g[N];
    load_group(l + k, (int)(a.K - k), v);
#pragma unroll
    for (int j = 0; j < N; ++j) g[j] = counts ? grad_of(e, v[j], k + j == label, a.scale) : 0.f;
    store_group<N>(grad + k, (int)(a.K - k), g);
  }
}

dim3 grid_of(int64_t blocks) {  // a dimension of a launch has fewer than 2^32 lanes
  const int64_t x = blocks < 1 << 21 ? blocks : 1 << 21;
  return dim3((unsigned)x, (unsigned)((blocks + x - 1) / x));
}

template <class IN, class OUT> hipError_t launch(const Args& a, hipStream_t s) {
  constexpr int N = kGroup<IN>;
  const auto go = [&](auto lanes, auto groups) {
    constexpr int L = decltype(lanes)::value, G = decltype(groups)::value;
    hipLaunchKernelGGL((rfast_xent_kernel<IN, OUT, L, G>), grid_of(L == 64 ? ((int64_t)a.rows + 3) / 4 : a.rows), dim3(L == 64 ? 256 : L), 0, s, a);
    return hipGetLastError();
  };
  using std::integral_constant;
  const int64_t per64 = (a.K + 64 * N - 1) / (64 * N);  // groups per lane of a wavefront
  if (per64 <= 1) return go(integral_constant<int, 64>(), integral_constant<int, 1>());
  if (per64 <= 2) return go(integral_constant<int, 64>(), integral_constant<int, 2>());
  if (per64 <= 4) return go(integral_constant<int, 64>(), integral_constant<int, 4>());
  if (per64 <= 8) return go(integral_constant<int, 256>(), integral_constant<int, 2>());
  if (per64 <= 16) return go(integral_constant<int, 256>(), integral_constant<int, 4>());
  if (per64 <= 32) return go(integral_constant<int, 256>(), integral_constant<int, 8>());
  if (per64 <= 64) return go(integral_constant<int, 1024>(), integral_constant<int, 4>());
  if (per64 <= 128) return go(integral_constant<int, 1024>(), integral_constant<int, 8>());
  hipLaunchKernelGGL((rfast_xent_long_kernel<IN, OUT>), grid_of(a.rows), dim3(1024), 0, s, a);
  return hipGetLastError();
}

bool type_ok(int32_t t) { return t == RFAST_F32 || t == RFAST_BF16; }

}  // namespace

extern "C" int rfast_softmax_xent(int32_t rows, int32_t K, const void* logits, int32_t logits_type, int64_t ld_logits,
                                  const int32_t* labels, float grad_scale, float* loss, float* lse, void* grad, int32_t grad_type,
                                  int64_t ld_grad, const int32_t* d_rows, void* hip_stream) {
  if (rows < 0 || K < 1) return rfast_refuse(RFAST_EINVAL, "need rows >= 0 and K >= 1");
  if (!type_ok(logits_type) || (grad && !type_ok(grad_type))) return rfast_refuse(RFAST_EINVAL, "types must be RFAST_F32 or RFAST_BF16");
  if (rows == 0) return RFAST_OK;
  if (!logits || !labels) return rfast_refuse(RFAST_EINVAL, "NULL argument");
  if (ld_logits < K || (grad && ld_grad < K)) return rfast_refuse(RFAST_EINVAL, "rows are at least K elements apart");
  const int lw = logits_type == RFAST_F32 ? 4 : 2, gw = grad_type == RFAST_F32 ? 4 : 2;
  if ((uintptr_t)logits % lw || (uintptr_t)labels % 4 || (uintptr_t)loss % 4 || (uintptr_t)lse % 4 || (grad && (uintptr_t)grad % gw) ||
      (uintptr_t)d_rows % 4)
    return rfast_refuse(RFAST_EINVAL, "an address is no multiple of its element's size");
  if (grad) {
    const uintptr_t l0 = (uintptr_t)logits, l1 = l0 + ((size_t)(rows - 1) * ld_logits + K) * lw;
    const uintptr_t g0 = (uintptr_t)grad, g1 = g0 + ((size_t)(rows - 1) * ld_grad + K) * gw;
    if (g0 < l1 && l0 < g1 && !(g0 == l0 && lw == gw && ld_logits == ld_grad))
      return rfast_refuse(RFAST_EINVAL, "the gradient overlaps the logits without being in their place");
  }
  const Args a = {logits, labels, loss, lse, grad, d_rows, ld_logits, ld_grad, rows, K, grad_scale};
  const hipStream_t s = (hipStream_t)hip_stream;
  const bool lf = logits_type == RFAST_F32, gf = grad_type == RFAST_F32;
  const hipError_t e = lf ? (gf ? launch<float, float>(a, s) : launch<float, u16>(a, s)) : (gf ? launch<u16, float>(a, s) : launch<u16, u16>(a, s));
  return e == hipSuccess ? RFAST_OK : rfast_refuse_hip(e, "cross-entropy launch");
}
