// AdamW over many tensors, moments in 32 bits or in 8.
//
// Elementwise; a coordinate in 32 bits moves 28 bytes (parameter, gradient, two moments in; all but the gradient out) for some 60
// vector instructions, so the kernel is bound by memory where the tensors are large and by latency where they are small.
//  - One launch for all tensors: the coordinates of every tensor are cut into chunks, a workgroup each, and a table says whose a chunk is.
//  - 8 bits: a block of 256 coordinates, which share a scale, is one wavefront's four coordinates per lane, so the largest magnitude is
//    found in registers and every byte is still moved once.
//  - Counters of steps are on the device (a replayed graph has to count).  Every workgroup reads them, and the last one to finish moves
//    them on; who is last is told by a word per group of workgroups and one for the groups, so that no word is hit by thousands.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "rfast_internal.h"
#include "rfast_operators.h"

namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 256;                    // coordinates per scale
constexpr int kSlice = kThreads / 64 * kBlock; // coordinates that the wavefronts of a workgroup take at a time
constexpr int kGroups = 64;                    // words for workgroups that are through
constexpr int kMostSteps = 0x7fffffff;         // where a counter stays
constexpr int kMostWorkgroups = 1 << 23;       // a launch has fewer than 2^32 lanes
constexpr float kCodeMost = 448.f;             // largest finite e4m3
constexpr float kCodeLeast = 0.001953125f;     // smallest e4m3 above zero, 2^-9
constexpr float kTopLeast = 0x1.cp-118f;       // 448 * 2^-126: below it a block's scale is no normal number
constexpr size_t kAlign = 256;
size_t up(size_t b) { return (b + kAlign - 1) / kAlign * kAlign; }

struct Row {
  void* param;
  const void* grad;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  u16* copy;
  int64_t count;
  int64_t first;  // its first chunk
  double decay;
};

struct Args {
  const Row* rows;
  const int32_t* whose;  // [chunks] tensor
  int32_t* steps;        // [tensors]
  unsigned* through;     // [kGroups * 16 + 1] workgroups that are through, 64 bytes apart
  const uint8_t* active;
  int32_t tensors, chunks;
  double gamma, log_beta1, log_beta2;
  float beta1, beta2, rest1, rest2, eps;  // rest = 1 - beta
};

// beta^t from log(beta) without the cancellation of 1 - beta^t
__device__ inline double one_less_power(double log_beta, int t) { return -expm1((double)t * log_beta); }

// a / b to about one unit in the last place: the step is not carried on like the moments, whose bits decide codes, and a division that
// is rounded correctly takes twice the instructions.  (b is at least eps, which is no denormal, so its reciprocal is finite; where b is infinite or
// the quotient is, the correction is no number and is left out.)
__device__ inline float over(float a, float b) {
  const float r = __builtin_amdgcn_rcpf(b);
  const float q = a * r;
  const float e = fmaf(-q, b, a);
  return fabsf(e) < INFINITY ? fmaf(e, r, q) : q;
}

__device__ inline float finite_magnitude(float v) {
  const float a = fabsf(v);
  return a < INFINITY ? a : 0.f;  // false for NaN too
}

// What a block whose largest magnitude is `top` is multiplied by to become codes.  Below kTopLeast the scale would lose its digits and its inverse
// be infinite (zeros times it NaN), as without a gradient a momentum gets there: by 0.9 a step from 1e-3 in some 700.  Such a block
// is held as zeros with a scale of zero; a root, whose square was a number of 32 bits, is 2^-75 and more or zero.
__device__ inline float inverse_of(float top) { return top >= kTopLeast ? 1.f / top * kCodeMost : 0.f; }
__device__ inline float scale_of(float top) { return top >= kTopLeast ? top * (1.f / kCodeMost) : 0.f; }

// Four values as e4m3 times scale; values that are not finite become NaN.
__device__ inline uint32_t codes_of(const float* v, float inverse, bool root) {
  float q[4];
  bool odd = false;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    q[j] = v[j] * inverse;
    if (root && v[j] > 0.f) q[j] = fmaxf(q[j], kCodeLeast);
    odd |= !(fabsf(v[j]) < INFINITY);
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true);
  if (odd) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (!(fabsf(v[j]) < INFINITY)) w |= 0x7F << (8 * j);
  }
  return (uint32_t)w;
}
__device__ inline void values_of(uint32_t w, float scale, float* v) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  v[0] = lo[0] * scale; v[1] = lo[1] * scale; v[2] = hi[0] * scale; v[3] = hi[1] * scale;
}

typedef unsigned int any_u32 __attribute__((aligned(1)));
template <bool STREAM> __device__ inline uint32_t load_codes(const uint8_t* p, int64_t left) {
  if (left >= 4) return wide_load<any_u32, STREAM>(p);
  uint32_t w = 0;
  for (int j = 0; j < 4; ++j)
    if (j < left) w |= (uint32_t)p[j] << (8 * j);
  return w;
}
template <bool STREAM> __device__ inline void store_codes(uint8_t* p, int64_t left, uint32_t w) {
  if (left >= 4) {
    wide_store<any_u32, STREAM>(p, w);
    return;
  }
  for (int j = 0; j < 4; ++j)
    if (j < left) p[j] = (uint8_t)(w >> (8 * j));
}

// The moments of four coordinates of a row: read, moved on, written.  With 8 bits all 64 lanes of the wavefront have to come
// along (they share the scale); lanes past the row's end have left <= 0.
template <int BITS, bool STREAM> struct Moments {
  float m[4], v[4];  // v: the root with 8 bits
  uint32_t cm, cv;
  float sm, sv;
  __device__ void read(const void* pm, const void* pv, const float* ms, const float* vs, int64_t k, int64_t left) {
    if constexpr (BITS == 32) {
      if (left > 0) {
        load_four<STREAM>((const float*)pm + k, left, m);
        load_four<STREAM>((const float*)pv + k, left, v);
      }
    } else {
      cm = cv = 0;
      if (left > 0) {
        cm = load_codes<STREAM>((const uint8_t*)pm + k, left);
        cv = load_codes<STREAM>((const uint8_t*)pv + k, left);
        sm = wide_load<float, false>(ms + k / kBlock);
        sv = wide_load<float, false>(vs + k / kBlock);
      }
    }
  }
  // root: sqrt(v) after the step
  __device__ void step(const float* g, float beta1, float rest1, float beta2, float rest2, float* root) {
    if constexpr (BITS == 8) {
      values_of(cm, sm, m);
      values_of(cv, sv, v);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = v[j] * v[j];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[j] = m[j] * beta1 + g[j] * rest1;
      v[j] = v[j] * beta2 + (g[j] * g[j]) * rest2;
      root[j] = sqrtf(v[j]);
    }
  }
  __device__ void write(void* pm, void* pv, float* ms, float* vs, int64_t k, int64_t left, const float* root) {
    if constexpr (BITS == 32) {
      if (left > 0) {
        store_four<STREAM>((float*)pm + k, left, m);
        store_four<STREAM>((float*)pv + k, left, v);
      }
    } else {
      float top_m = 0.f, top_v = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < left) {
          top_m = fmaxf(top_m, finite_magnitude(m[j]));
          top_v = fmaxf(top_v, finite_magnitude(root[j]));
        }
      top_m = wave_max(top_m);
      top_v = wave_max(top_v);
      if (left <= 0) return;
      store_codes<STREAM>((uint8_t*)pm + k, left, codes_of(m, inverse_of(top_m), false));
      store_codes<STREAM>((uint8_t*)pv + k, left, codes_of(root, inverse_of(top_v), true));
      if (k % kBlock == 0) {
        ms[k / kBlock] = scale_of(top_m);
        vs[k / kBlock] = scale_of(top_v);
      }
    }
  }
};

// Slices of a chunk of row r, this lane's coordinates from k0 on.  WHOLE: all of them exist, and their loads go out together without a condition;
// else each is looked at on its own.
template <class P, class G, int BITS, int U, bool STREAM, bool WHOLE>
__device__ inline void step_chunk(const Args& a, const Row& r, int t, int64_t k0) {
  Moments<BITS, STREAM> state[U];
  float p[U][4], g[U][4];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t k = k0 + u * kSlice, left = WHOLE ? 4 : r.count - k;
    if (left > 0) {
      load_four<STREAM>((const P*)r.param + k, left, p[u]);
      load_four<STREAM>((const G*)r.grad + k, left, g[u]);
    }
    state[u].read(r.m, r.v, r.m_scale, r.v_scale, k, left);
  }
  const float first = (float)(a.gamma / one_less_power(a.log_beta1, t));
  const float second = (float)(1.0 / sqrt(one_less_power(a.log_beta2, t)));
  const float keep = (float)(1.0 - a.gamma * r.decay);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t k = k0 + u * kSlice, left = WHOLE ? 4 : r.count - k;
    float root[4];
    state[u].step(g[u], a.beta1, a.rest1, a.beta2, a.rest2, root);
#pragma unroll
    for (int j = 0; j < 4; ++j) p[u][j] = p[u][j] * keep - over(state[u].m[j] * first, root[j] * second + a.eps);
    if (left > 0) {
      store_four<STREAM>((P*)r.param + k, left, p[u]);
      if (r.copy) store_four<STREAM>(r.copy + k, left, p[u]);
    }
    state[u].write(r.m, r.v, r.m_scale, r.v_scale, k, left, root);
  }
}

template <class P, class G, int BITS, int U, bool STREAM>
__global__ void __launch_bounds__(kThreads) rfast_adamw_kernel(Args a) {
  for (int chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
    const int i = __builtin_amdgcn_readfirstlane(a.whose[chunk]);
    if (a.active && a.active[i] == 0) continue;
    const Row r = a.rows[i];
    const int t = min(a.steps[i], kMostSteps - 1) + 1;
    const int64_t begin = (chunk - r.first) * (U * kSlice), k0 = begin + threadIdx.x * 4;
    if (begin + U * kSlice <= r.count) step_chunk<P, G, BITS, U, STREAM, true>(a, r, t, k0);
    else step_chunk<P, G, BITS, U, STREAM, false>(a, r, t, k0);
  }
  // The last workgroup moves the counters on.  No workgroup reads them any more: each has used what it read before it counts itself,
  // and nothing else is handed over, so the words need no ordering of memory (a release across the eight L2s writes them back:
  // with it, 256 small tensors took 48 us instead of 8).
  __shared__ bool last;
  __syncthreads();
  if (threadIdx.x == 0) {
    const unsigned group = blockIdx.x % kGroups;
    const unsigned in_group = (gridDim.x - group + kGroups - 1) / kGroups, groups = gridDim.x < kGroups ? gridDim.x : kGroups;
    last = false;
    if (__hip_atomic_fetch_add(a.through + group * 16, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == in_group - 1) {
      __hip_atomic_store(a.through + group * 16, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (__hip_atomic_fetch_add(a.through + kGroups * 16, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == groups - 1) {
        __hip_atomic_store(a.through + kGroups * 16, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last = true;
      }
    }
  }
  __syncthreads();
  if (!last) return;
  for (int i = threadIdx.x; i < a.tensors; i += kThreads)
    if (!a.active || a.active[i] != 0) a.steps[i] = min(a.steps[i], kMostSteps - 1) + 1;
}

// The AdamW variant of a round: the same moments, of the nodes about to act, from the tracked directions z; what the step would
// subtract, over gamma, is left for S1.  One workgroup per kSlice coordinates of a node.
struct RoundArgs {
  const float* z;
  int64_t z_stride;  // from node to node
  const float* x;
  float* dir;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  const int2* plan;  // {node, counter}, or NULL: every node
  const int32_t* t;
  int64_t p;
  double log_beta1, log_beta2;
  float beta1, beta2, rest1, rest2, eps, decay;
};

template <int BITS> __global__ void __launch_bounds__(kThreads) rfast_adamw_round_kernel(RoundArgs a) {
  int i = blockIdx.y, t;
  if (a.plan) {
    const int2 slot = a.plan[i];
    if (slot.x < 0) return;
    i = slot.x;
    t = slot.y + 1;
  } else {
    t = a.t[i] + 1;
  }
  const int64_t k = (int64_t)blockIdx.x * kSlice + threadIdx.x * 4, left = a.p - k;
  const int64_t row = (int64_t)i * a.p, blocks = (a.p + kBlock - 1) / kBlock;
  constexpr int WIDE = BITS / 8;
  void *m = (char*)a.m + row * WIDE, *v = (char*)a.v + row * WIDE;
  float* ms = BITS == 8 ? a.m_scale + i * blocks : nullptr;
  float* vs = BITS == 8 ? a.v_scale + i * blocks : nullptr;
  Moments<BITS, false> state;
  float g[4], x[4], root[4];
  if (left > 0) {
    load_four<false>(a.z + i * a.z_stride + k, left, g);
    load_four<false>(a.x + row + k, left, x);
  }
  state.read(m, v, ms, vs, k, left);
  const float first = (float)(1.0 / one_less_power(a.log_beta1, t));
  const float second = (float)(1.0 / sqrt(one_less_power(a.log_beta2, t)));
  state.step(g, a.beta1, a.rest1, a.beta2, a.rest2, root);
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = over(state.m[j] * first, root[j] * second + a.eps) + a.decay * x[j];
  if (left > 0) store_four<false>(a.dir + row + k, left, x);
  state.write(m, v, ms, vs, k, left, root);
}

struct Layout {
  size_t rows, whose, steps, through, total;
};
bool count_chunks(int32_t tensors, const rfast_adamw_tensor* t, int64_t slices, int64_t* chunks) {
  *chunks = 0;
  for (int32_t i = 0; i < tensors; ++i) {
    if (t[i].count < 0 || t[i].count > (int64_t)1 << 46) return false;
    *chunks += (t[i].count + slices * kSlice - 1) / (slices * kSlice);
    if (*chunks > 0x7fffffff - kMostWorkgroups) return false;  // (a workgroup's next chunk is still an int)
  }
  return true;
}
Layout layout_of(int32_t tensors, int64_t chunks) {
  Layout l;
  l.rows = 0;
  l.whose = up(l.rows + (size_t)tensors * sizeof(Row));
  l.steps = up(l.whose + (size_t)chunks * 4);
  l.through = up(l.steps + (size_t)tensors * 4);
  l.total = up(l.through + (kGroups * 16 + 1) * 4);
  return l;
}
// Slices per chunk.  32 bits: one (four loads per lane under way; 16 x 11.2 M coordinates 807 us, with two 875, with four 885).  8 bits,
// whose loads of the moments are short: four where there are chunks enough (507; 548 with two, 618 with one; 75 tensors of 200000 on
// average 41 / 40 / 47), else two (40 of 100000: 16.1; 17.6 with four, 17.7 with one).
int64_t slices_for(int32_t tensors, const rfast_adamw_tensor* t, int32_t bits, int64_t* chunks) {
  const int64_t most = bits == 32 ? 1 : 4;
  if (!count_chunks(tensors, t, most, chunks)) return 0;
  if (most == 1 || *chunks >= 2048) return most;
  return count_chunks(tensors, t, 2, chunks) ? 2 : 0;
}

}  // namespace

struct rfast_adamw {
  Args a;
  int param_type, grad_type, bits, slices;
  bool stream;
};

namespace {

template <class P, class G, int BITS> hipError_t launch(const rfast_adamw* h, const Args& a, hipStream_t s) {
  const dim3 grid((unsigned)std::min(std::max(a.chunks, 1), kMostWorkgroups)), block(kThreads);
  constexpr int MOST = BITS == 32 ? 1 : 4;
  if constexpr (MOST > 1) {
    if (h->slices == 2) {
      hipLaunchKernelGGL((rfast_adamw_kernel<P, G, BITS, 2, false>), grid, block, 0, s, a);
      return hipGetLastError();
    }
  }
  if (h->stream) hipLaunchKernelGGL((rfast_adamw_kernel<P, G, BITS, MOST, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((rfast_adamw_kernel<P, G, BITS, MOST, false>), grid, block, 0, s, a);
  return hipGetLastError();
}
template <class P, class G> hipError_t launch(const rfast_adamw* h, const Args& a, hipStream_t s) {
  return h->bits == 32 ? launch<P, G, 32>(h, a, s) : launch<P, G, 8>(h, a, s);
}

bool aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }

int create(rfast_adamw** out, int32_t tensors, const rfast_adamw_tensor* t, const rfast_adamw_options* o, void* d_workspace,
           size_t workspace_bytes, hipStream_t stream) {
  if (!t || !o || !d_workspace) return rfast_refuse(RFAST_EINVAL, "NULL argument");
  if (tensors < 1) return rfast_refuse(RFAST_EINVAL, "need at least one tensor");
  if ((o->param_type != RFAST_F32 && o->param_type != RFAST_BF16) || (o->grad_type != RFAST_F32 && o->grad_type != RFAST_BF16))
    return rfast_refuse(RFAST_EINVAL, "param_type and grad_type must be RFAST_F32 or RFAST_BF16");
  if (o->state_bits != 8 && o->state_bits != 32) return rfast_refuse(RFAST_EINVAL, "state_bits must be 8 or 32");
  if (!(o->beta1 >= 0 && o->beta1 < 1 && o->beta2 >= 0 && o->beta2 < 1)) return rfast_refuse(RFAST_ERANGE, "beta1 and beta2 must lie in [0, 1)");
  if (!rfast_adamw_eps_ok(o->eps)) return rfast_refuse(RFAST_ERANGE, "eps must lie in [2^-126, 1e30)");
  if (!aligned(d_workspace, kAlign)) return rfast_refuse(RFAST_EINVAL, "workspace must be 256-byte aligned");
  int64_t chunks;
  const int64_t slices = slices_for(tensors, t, o->state_bits, &chunks);
  if (slices == 0) return rfast_refuse(RFAST_EINVAL, "a tensor's count is out of range");
  const Layout l = layout_of(tensors, chunks);
  if (workspace_bytes < l.total) return rfast_refuse(RFAST_ENOMEM, "workspace too small");
  const size_t pw = o->param_type == RFAST_F32 ? 4 : 2, gw = o->grad_type == RFAST_F32 ? 4 : 2, sw = o->state_bits == 32 ? 4 : 1;
  std::vector<Row> rows((size_t)tensors);
  std::vector<int32_t> whose((size_t)chunks), steps((size_t)tensors);
  struct Span { uintptr_t at, end; bool written; };
  std::vector<Span> spans{{(uintptr_t)d_workspace, (uintptr_t)d_workspace + l.total, true}};
  int64_t first = 0, bytes = 0;
  for (int32_t i = 0; i < tensors; ++i) {
    const rfast_adamw_tensor& q = t[i];
    const std::string who = "tensor " + std::to_string(i) + ": ";
    if (!(q.weight_decay >= 0 && q.weight_decay < 1e30)) return rfast_refuse(RFAST_ERANGE, who + "weight_decay must be finite and >= 0");
    if (q.steps < 0 || q.steps > kMostSteps) return rfast_refuse(RFAST_ERANGE, who + "steps out of range");
    steps[i] = (int32_t)q.steps;
    rows[i] = {q.param, q.grad, q.m, q.v, q.m_scale, q.v_scale, (u16*)q.copy, q.count, first, q.weight_decay};
    const int64_t n = (q.count + slices * kSlice - 1) / (slices * kSlice);
    std::fill(whose.begin() + first, whose.begin() + first + n, i);
    first += n;
    if (q.count == 0) continue;
    if (!q.param || !q.grad || !q.m || !q.v) return rfast_refuse(RFAST_EINVAL, who + "NULL pointer");
    if (o->state_bits == 8 ? !q.m_scale || !q.v_scale : q.m_scale || q.v_scale)
      return rfast_refuse(RFAST_EINVAL, who + "scales are needed with states in 8 bits, and only there");
    if (!aligned(q.param, pw) || !aligned(q.grad, gw) || !aligned(q.m, sw) || !aligned(q.v, sw) || !aligned(q.m_scale, 4) ||
        !aligned(q.v_scale, 4) || !aligned(q.copy, 2))
      return rfast_refuse(RFAST_EINVAL, who + "an address is no multiple of its element's size");
    const size_t count = (size_t)q.count, blocks = (count + kBlock - 1) / kBlock;
    auto span = [&](const void* p, size_t len, bool written) {
      if (p) spans.push_back({(uintptr_t)p, (uintptr_t)p + len, written});
    };
    span(q.param, count * pw, true); span(q.grad, count * gw, false); span(q.m, count * sw, true); span(q.v, count * sw, true);
    span(q.m_scale, blocks * 4, true); span(q.v_scale, blocks * 4, true); span(q.copy, count * 2, true);
    bytes += q.count * (int64_t)(pw + gw + 2 * sw);
  }
  std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.at < b.at; });
  uintptr_t end = 0, end_written = 0;  // of what begins before
  for (const Span& s : spans) {
    if (s.at < end_written || (s.written && s.at < end))
      return rfast_refuse(RFAST_EINVAL, "memory that a step writes overlaps other memory of the step");
    end = std::max(end, s.end);
    if (s.written) end_written = std::max(end_written, s.end);
  }
  char* base = (char*)d_workspace;
  hipError_t e = hipMemcpyAsync(base + l.rows, rows.data(), rows.size() * sizeof(Row), hipMemcpyHostToDevice, stream);
  if (e == hipSuccess && chunks) e = hipMemcpyAsync(base + l.whose, whose.data(), whose.size() * 4, hipMemcpyHostToDevice, stream);
  if (e == hipSuccess) e = hipMemcpyAsync(base + l.steps, steps.data(), steps.size() * 4, hipMemcpyHostToDevice, stream);
  const std::vector<unsigned> none(kGroups * 16 + 1, 0u);
  if (e == hipSuccess) e = hipMemcpyAsync(base + l.through, none.data(), none.size() * 4, hipMemcpyHostToDevice, stream);
  if (e == hipSuccess) e = hipStreamSynchronize(stream);
  if (e != hipSuccess) return rfast_refuse_hip(e, "upload of the table of tensors");
  rfast_adamw* h = new rfast_adamw;
  h->param_type = o->param_type;
  h->grad_type = o->grad_type;
  h->bits = o->state_bits;
  h->slices = (int)slices;
  // What is read once a step streams past the caches where they would not hold it until the next: 16 x 11.2 M coordinates 910 -> 807 us,
  // 100 tensors of 200000 in 16 bits (240 MB) 81 -> 74; 20 tensors of 200000 (64 MB) 19.1 -> 20.7 with it, 90 MB with moments in 8 bits 47 -> 56.
  h->stream = bytes > (int64_t)160 << 20;
  h->a = {(const Row*)(base + l.rows), (const int32_t*)(base + l.whose), (int32_t*)(base + l.steps), (unsigned*)(base + l.through),
          nullptr, tensors, (int32_t)chunks, 0.0, std::log(o->beta1), std::log(o->beta2),
          (float)o->beta1, (float)o->beta2, (float)(1.0 - o->beta1), (float)(1.0 - o->beta2), (float)o->eps};
  *out = h;
  return RFAST_OK;
}

}  // namespace

hipError_t rfast_launch_adamw_round(rfast_ctx* c, bool sync, int parity) {
  const RfastDev& d = c->d;
  const RfastAdamwState& w = c->adamw;
  RoundArgs a = {d.z, d.p, d.x, d.mom, w.m, w.v, w.m_scale, w.v_scale, sync ? nullptr : d.active_plan, d.t, d.p, std::log(w.beta1),
                 std::log(w.beta2), (float)w.beta1, (float)w.beta2, (float)(1.0 - w.beta1), (float)(1.0 - w.beta2), (float)w.eps, (float)w.decay};
  if (sync && parity) {  // the current z is in slot 1 of the v ring
    a.z = d.v_ring + d.p;
    a.z_stride = (int64_t)d.M * d.p;
  }
  const dim3 grid((unsigned)((d.p + kSlice - 1) / kSlice), (unsigned)d.n);
  if (w.bits == 32) hipLaunchKernelGGL(rfast_adamw_round_kernel<32>, grid, dim3(kThreads), 0, c->stream, a);
  else hipLaunchKernelGGL(rfast_adamw_round_kernel<8>, grid, dim3(kThreads), 0, c->stream, a);
  return hipGetLastError();
}

extern "C" {

size_t rfast_adamw_workspace_bytes(int32_t tensors, const rfast_adamw_tensor* t) {
  int64_t with32, with8;  // chunks
  if (tensors < 1 || !t || slices_for(tensors, t, 32, &with32) == 0 || slices_for(tensors, t, 8, &with8) == 0) return 0;
  return layout_of(tensors, std::max(with32, with8)).total;
}

int rfast_adamw_create(rfast_adamw** out, int32_t tensors, const rfast_adamw_tensor* t, const rfast_adamw_options* o,
                       void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (!out) return rfast_refuse(RFAST_EINVAL, "out is NULL");
  *out = nullptr;
  try {
    return create(out, tensors, t, o, d_workspace, workspace_bytes, (hipStream_t)hip_stream);
  } catch (const std::exception&) {
    return rfast_refuse(RFAST_EINVAL, "host memory ran out");
  }
}

int rfast_adamw_step(rfast_adamw* h, double gamma, const uint8_t* d_active, void* hip_stream) {
  if (!h) return rfast_refuse(RFAST_EINVAL, "NULL handle");
  if (!(std::fabs(gamma) < 1e30)) return rfast_refuse(RFAST_ERANGE, "gamma must be finite");
  Args a = h->a;
  a.gamma = gamma;
  a.active = d_active;
  const hipStream_t s = (hipStream_t)hip_stream;
  const bool pf = h->param_type == RFAST_F32, gf = h->grad_type == RFAST_F32;
  const hipError_t e = pf ? (gf ? launch<float, float>(h, a, s) : launch<float, u16>(h, a, s))
                          : (gf ? launch<u16, float>(h, a, s) : launch<u16, u16>(h, a, s));
  return e == hipSuccess ? RFAST_OK : rfast_refuse_hip(e, "AdamW launch");
}

int rfast_adamw_steps(rfast_adamw* h, int32_t* host_steps, void* hip_stream) {
  if (!h || !host_steps) return rfast_refuse(RFAST_EINVAL, "NULL argument");
  hipError_t e = hipMemcpyAsync(host_steps, h->a.steps, (size_t)h->a.tensors * 4, hipMemcpyDeviceToHost, (hipStream_t)hip_stream);
  if (e == hipSuccess) e = hipStreamSynchronize((hipStream_t)hip_stream);
  return e == hipSuccess ? RFAST_OK : rfast_refuse_hip(e, "read of the counters");
}

int rfast_adamw_set_steps(rfast_adamw* h, const int32_t* host_steps, void* hip_stream) {
  if (!h || !host_steps) return rfast_refuse(RFAST_EINVAL, "NULL argument");
  for (int32_t i = 0; i < h->a.tensors; ++i)
    if (host_steps[i] < 0) return rfast_refuse(RFAST_ERANGE, "steps out of range");
  hipError_t e = hipMemcpyAsync(h->a.steps, host_steps, (size_t)h->a.tensors * 4, hipMemcpyHostToDevice, (hipStream_t)hip_stream);
  if (e == hipSuccess) e = hipStreamSynchronize((hipStream_t)hip_stream);
  return e == hipSuccess ? RFAST_OK : rfast_refuse_hip(e, "write of the counters");
}

void rfast_adamw_destroy(rfast_adamw* h) { delete h; }

}  // extern "C"
