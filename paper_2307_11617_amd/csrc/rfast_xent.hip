// Softmax cross-entropy of rows of logits with its gradient.
//
//   lse = log sum exp l_k,  loss = lse - l_label,  grad_k = c (exp(l_k - lse) - [k == label])
//
// Some five operations per logit, so the bound is one read of the logits and one write of the gradient.  A row therefore stays in
// registers between the two: of 8 to 64 lanes up to 1024 logits (2048 of bf16), of a workgroup of 256 to 1024 lanes beyond.  Rows longer than the registers
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

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;

// A group of neighbouring logits: what a 16-byte load holds.
template <class T> struct Group;
template <> struct Group<float> {
  static constexpr int N = 4;
  any_f32x4 raw;
  __device__ void load(const float* p) { raw = *reinterpret_cast<const any_f32x4*>(p); }
  __device__ void load(const float* p, int left) {
#pragma unroll
    for (int j = 0; j < N; ++j) raw[j] = j < left ? p[j] : -INFINITY;
  }
  __device__ float at(int j) const { return raw[j]; }
};
template <> struct Group<u16> {
  static constexpr int N = 8;
  any_u32x4 raw;
  __device__ void load(const u16* p) { raw = *reinterpret_cast<const any_u32x4*>(p); }
  __device__ void load(const u16* p, int left) {
#pragma unroll
    for (int j = 0; j < N; j += 2) raw[j >> 1] = (j < left ? p[j] : 0xFF80u) | (uint32_t)(j + 1 < left ? p[j + 1] : 0xFF80u) << 16;
  }
  __device__ float at(int j) const { return __uint_as_float(j & 1 ? raw[j >> 1] & 0xFFFF0000u : raw[j >> 1] << 16); }
};
template <int N> __device__ inline void store_group(float* p, const float* v) {
#pragma unroll
  for (int q = 0; q < N; q += 4) store_four<false>(p + q, 4, v + q);
}
template <int N> __device__ inline void store_group(u16* p, const float* v) {
  if constexpr (N == 8) {
    const any_u32x4 t = {to_bf16_pair(v[0], v[1]), to_bf16_pair(v[2], v[3]), to_bf16_pair(v[4], v[5]), to_bf16_pair(v[6], v[7])};
    *reinterpret_cast<any_u32x4*>(p) = t;
  } else {
    store_four<false>(p, 4, v);
  }
}

// Over the row's lanes: LANES neighbours of a wavefront, or a workgroup's through `box`.
template <int LANES, class F> __device__ inline float row_reduce(float v, float* box, F f) {
  if constexpr (LANES >= 64) {
    v = wave_reduce(v, f);
  } else {
    v = f(v, lane_of<0xB1>(v));
    v = f(v, lane_of<0x4E>(v));
    v = f(v, lane_of<0x141>(v));
    if constexpr (LANES >= 16) v = f(v, lane_of<0x140>(v));
    if constexpr (LANES >= 32) v = f(v, __shfl_xor(v, 16, 64));
  }
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = v;
    __syncthreads();
    v = box[0];
#pragma unroll
    for (int w = 1; w < LANES / 64; ++w) v = f(v, box[w]);
  }
  return v;
}

// exp(l - shift).  The difference is taken before the multiplication by log2(e): in one multiply-add the largest logit of a row would not come
// to exactly 1, nor the loss of a certain one to 0, and beside logits of 1e38 the product would overflow.
__device__ inline float power(float l, float shift) { return __builtin_amdgcn_exp2f((l - shift) * kLog2e); }
__device__ inline float shift_of(float top) { return top == -INFINITY ? 0.f : top; }  // (a row without a logit above -infinity: sum 0)
// loss = log sum - (l_label - shift), not lse - l_label: beside a large shift the logarithm would lose its digits
__device__ inline void finish_row(const Args& a, int64_t row, float shift, float sum, bool counts, float own) {
  const float log_sum = kLn2 * __builtin_amdgcn_logf(sum);  // sum is 0, or 1 and more, or NaN
  if (a.lse) a.lse[row] = sum == 0.f ? -INFINITY : shift + log_sum;
  if (a.loss) a.loss[row] = !counts || sum == 0.f ? 0.f : log_sum + (shift - own);
}

template <class OUT> __device__ inline void zero_row(OUT* grad, int K, int lane, int lanes) {
  for (int64_t k = lane; k < K; k += lanes) grad[k] = (OUT)0;  // (the last step of a row of nearly 2^31 passes 32 bits)
}

// LANES lanes hold a row, GROUPS groups of logits each.  LANES <= 64: 256 / LANES rows per workgroup.
// Every load is a whole group without a condition (a condition per load would have each of them waited for before the next is sent), so groups
// overlap at the ends of a row: group h begins at 8 h - m, moved into [0, K - 8] (4 instead of 8 in 32 bits), where m is how far a row of
// a workgroup's begins behind a multiple of 16 bytes, so that all but the first and last group are aligned (4096 rows of 50001: 184 us with
// m = 0, 152 so).  What a group shares with the one before is left out of its sum, and its gradient is written twice alike.
template <class IN, class OUT, int LANES, int GROUPS>
__global__ void __launch_bounds__(LANES <= 64 ? 256 : LANES, GROUPS >= 13 ? 4 : 1) rfast_xent_kernel(Args a) {
  constexpr int N = Group<IN>::N, ROWS = LANES <= 64 ? 256 / LANES : 1, SPAN = LANES * N;
  __shared__ float box[2][16];
  const int lane = threadIdx.x % LANES;
  const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * ROWS + threadIdx.x / LANES;
  // (of a wavefront that has several rows, those past the end leave: the others' lanes only look at each other)
  if (row >= a.rows || (a.d_rows && row >= *a.d_rows)) return;
  const IN* l = (const IN*)a.logits + row * a.ld_logits;
  OUT* grad = a.grad ? (OUT*)a.grad + row * a.ld_grad : nullptr;
  const int label = a.labels[row], last = a.K - N;  // last: where the last group begins (below 0: a row shorter than a group)
  const int m = LANES > 64 ? (int)((uintptr_t)l / sizeof(IN) % N) : 0;
  const bool counts = label >= 0 && label < a.K;
  if (!counts && !a.lse) {
    if (lane == 0 && a.loss) a.loss[row] = 0.f;
    if (grad) zero_row(grad, a.K, lane, LANES);
    return;
  }
  auto begin = [&](int h) { return max(min(h * N - m, last), 0); };
  Group<IN> v[GROUPS];
  if (LANES > 8 || GROUPS > 1 || last >= 0) {
#pragma unroll
    for (int q = 0; q < GROUPS; ++q) v[q].load(l + begin(q * LANES + lane));
  } else {
    v[0].load(l, a.K);
  }
  float own = 0.f;
  if (counts) own = sizeof(IN) == 4 ? ((const float*)l)[label] : from_bf16(((const u16*)l)[label]);
  float top = -INFINITY;
#pragma unroll
  for (int q = 0; q < GROUPS; ++q)
#pragma unroll
    for (int j = 0; j < N; ++j) top = fmaxf(top, v[q].at(j));
  const float shift = shift_of(row_reduce<LANES>(top, box[0], [](float x, float y) { return fmaxf(x, y); }));
  // The compiler would keep the unpacked logits of one pass for the next, at twice the registers of the packed ones.
  auto forget = [&] {
#pragma unroll
    for (int q = 0; q < GROUPS; ++q) asm volatile("" : "+v"(v[q].raw));
  };
  forget();
  float sum = 0.f;
#pragma unroll
  for (int q = 0; q < GROUPS; ++q) {
    if ((q + 1) * SPAN - m <= a.K && (q > 0 || m == 0)) {
#pragma unroll
      for (int j = 0; j < N; ++j) sum += power(v[q].at(j), shift);
    } else {
      const int h = q * LANES + lane, again = h > 0 ? begin(h - 1) + N - begin(h) : 0;  // what the group before has too
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float e = power(v[q].at(j), shift);
        sum += j >= again ? e : 0.f;
      }
    }
  }
  sum = row_reduce<LANES>(sum, box[1], [](float x, float y) { return x + y; });
  if (lane == 0) finish_row(a, row, shift, sum, counts, own);
  if (!grad) return;
  if (!counts || sum == 0.f) {
    zero_row(grad, a.K, lane, LANES);
    return;
  }
  const float c = a.scale / sum;
  forget();
#pragma unroll
  for (int q = 0; q < GROUPS; ++q) {
    const int h = q * LANES + lane, at = begin(h);
    float g[N];
#pragma unroll
    for (int j = 0; j < N; ++j) g[j] = power(v[q].at(j), shift) * c;
    if ((unsigned)(label - at) < (unsigned)N) {
#pragma unroll
      for (int j = 0; j < N; ++j) g[j] -= j == label - at ? a.scale : 0.f;
    }
    if (h * N - m >= a.K) continue;
    if (LANES > 8 || GROUPS > 1 || last >= 0) {
      store_group<N>(grad + at, g);
    } else {
#pragma unroll
      for (int j = 0; j < N; j += 4)
        if (a.K > j) store_four<false>(grad + j, a.K - j, g + j);
    }
  }
}

// Rows that no workgroup's registers hold.
template <class IN, class OUT>
__global__ void __launch_bounds__(1024) rfast_xent_long_kernel(Args a) {
  constexpr int N = Group<IN>::N, SPAN = 1024 * N;
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
  // this lane's largest logit so far and its sum of exp(l - that)
  float top = -INFINITY, sum = 0.f;
  const int64_t first = (int64_t)threadIdx.x * N;
  for (int64_t k = first; k < a.K; k += SPAN) {
    Group<IN> v;
    if (k + N <= a.K) v.load(l + k);
    else v.load(l + k, (int)(a.K - k));
    float m = top;
#pragma unroll
    for (int j = 0; j < N; ++j) m = fmaxf(m, v.at(j));
    const float shift = shift_of(m);
    if (m > top) sum *= power(top, shift);  // (top = -infinity: the sum is 0, or NaN)
    top = m;
#pragma unroll
    for (int j = 0; j < N; ++j) sum += power(v.at(j), shift);
  }
  const float shift = shift_of(row_reduce<1024>(top, box[0], [](float x, float y) { return fmaxf(x, y); }));
  if (shift > top) sum *= power(top, shift);
  sum = row_reduce<1024>(sum, box[1], [](float x, float y) { return x + y; });
  if (threadIdx.x == 0) finish_row(a, row, shift, sum, counts, own);
  if (!grad) return;
  // (where the gradient takes the logits' place, `own` has been read before any lane writes: the reductions are barriers)
  if (!counts || sum == 0.f) {
    zero_row(grad, a.K, threadIdx.x, 1024);
    return;
  }
  const float c = a.scale / sum;
  for (int64_t k = first; k < a.K; k += SPAN) {
    Group<IN> v;
    const bool whole = k + N <= a.K;
    if (whole) v.load(l + k);
    else v.load(l + k, (int)(a.K - k));
    float g[N];
#pragma unroll
    for (int j = 0; j < N; ++j) g[j] = power(v.at(j), shift) * c - (k + j == label ? a.scale : 0.f);
    if (whole) {
      store_group<N>(grad + k, g);
    } else {
#pragma unroll
      for (int j = 0; j < N; j += 4)
        if (a.K - k > j) store_four<false>(grad + k + j, a.K - k - j, g + j);
    }
  }
}

dim3 grid_of(int64_t blocks) {  // a dimension of a launch has fewer than 2^32 lanes
  const int64_t x = blocks < 1 << 21 ? blocks : 1 << 21;
  return dim3((unsigned)x, (unsigned)((blocks + x - 1) / x));
}

template <class IN, class OUT> hipError_t launch(const Args& a, hipStream_t s) {
  constexpr int N = Group<IN>::N;
  const auto go = [&](auto lanes, auto groups) {
    constexpr int L = decltype(lanes)::value, G = decltype(groups)::value, rows = L <= 64 ? 256 / L : 1;
    hipLaunchKernelGGL((rfast_xent_kernel<IN, OUT, L, G>), grid_of(((int64_t)a.rows + rows - 1) / rows), dim3(L <= 64 ? 256 : L), 0, s, a);
    return hipGetLastError();
  };
  using std::integral_constant;
  const auto fits = [&](int lanes, int groups) { return (int64_t)a.K + (lanes > 64 ? N - 1 : 0) <= (int64_t)lanes * groups * N; };
#define RFAST_TRY(L, G) \
  if (fits(L, G)) return go(integral_constant<int, L>(), integral_constant<int, G>())
  RFAST_TRY(8, 1);
  RFAST_TRY(8, 2);
  RFAST_TRY(16, 2);
  RFAST_TRY(32, 2);
  RFAST_TRY(64, 2);
  RFAST_TRY(64, 4);
  RFAST_TRY(256, 2);
  RFAST_TRY(256, 4);
  RFAST_TRY(256, 8);
  RFAST_TRY(512, 6);
  RFAST_TRY(512, 8);
  RFAST_TRY(512, 10);
  RFAST_TRY(512, 13);
  RFAST_TRY(512, 16);
  if constexpr (N == 4) {
    RFAST_TRY(1024, 16);
  }
#undef RFAST_TRY
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
    const RfastArea in = {logits, rows, ld_logits * lw, (int64_t)K * lw}, out = {grad, rows, ld_grad * gw, (int64_t)K * gw};
    if (rfast_overlap(in, out) && !(grad == logits && lw == gw && ld_logits == ld_grad))
      return rfast_refuse(RFAST_EINVAL, "the gradient overlaps the logits without being in their place");
  }
  const Args a = {logits, labels, loss, lse, grad, d_rows, ld_logits, ld_grad, rows, K, grad_scale};
  const hipStream_t s = (hipStream_t)hip_stream;
  const bool lf = logits_type == RFAST_F32, gf = grad_type == RFAST_F32;
  const hipError_t e = lf ? (gf ? launch<float, float>(a, s) : launch<float, u16>(a, s)) : (gf ? launch<u16, float>(a, s) : launch<u16, u16>(a, s));
  return e == hipSuccess ? RFAST_OK : rfast_refuse_hip(e, "cross-entropy launch");
}
