// Gradient and loss of softmax regression through low-rank adapters: every node trains A (rank x d) and B (K x rank) beside a
// projection W0 that is frozen and the same for all (RFAST_OBJ_LORA_SOFTMAX).
//
// The nodes about to act are the requests of the operators on tensors: the sampled rows of the s-th of them are segment s, with the
// node's adapter, and the logits, their loss's gradient and the adapters' gradients are three calls (rfast_lora_forward,
// rfast_softmax_xent, rfast_lora_backward).  Around them one kernel gathers rows and rounds the adapters to bf16, and one puts the gradients, with the
// weight decay, into the slots of the stored samples.
#include <algorithm>

#include "rfast_internal.h"
#include "rfast_operators.h"

namespace {

constexpr int kThreads = 256;
constexpr size_t kAlign = 256;
size_t up(size_t b) { return (b + kAlign - 1) / kAlign * kAlign; }

int rows_per_node(const rfast_problem& p) { return p.batch > 0 ? p.batch : p.samples; }

rfast_lora_shape shape_of(int32_t n, const rfast_problem& p) {
  return {n * rows_per_node(p), n, n, p.d, p.K, p.rank, p.d, p.K, RFAST_F32, p.adapter_scale};
}

struct Scratch {
  u16 *a, *b;         // [n][rank][d], [n][K][rank]
  float *da, *db;
  u16* x;             // [n B][d] the round's rows, those of the s-th active node from s B on
  int32_t *label, *row_ptr, *node;  // [n B], [n + 1], [n] (-1: no segment)
  int32_t* all;       // [2] row_ptr of the loss: everything is one segment
  float* logits;      // [n B][K]
  u16* dy;            // [n B][K]
  float* loss;        // [n B]
  void* work;
  size_t work_bytes, total;
};

Scratch scratch_of(void* base, int32_t n, const rfast_problem& p) {
  Scratch s;
  char* at = (char*)base;
  auto take = [&](size_t bytes) { char* q = at; at += up(bytes); return (void*)q; };
  const size_t N = (size_t)n, B = (size_t)rows_per_node(p), d = (size_t)p.d, K = (size_t)p.K, r = (size_t)p.rank;
  const rfast_lora_shape shape = shape_of(n, p);
  s.a = (u16*)take(N * r * d * 2);
  s.b = (u16*)take(N * r * K * 2);
  s.da = (float*)take(N * r * d * 4);
  s.db = (float*)take(N * r * K * 4);
  s.x = (u16*)take(N * B * d * 2);
  s.label = (int32_t*)take(N * B * 4);
  s.row_ptr = (int32_t*)take((N + 1) * 4);
  s.node = (int32_t*)take(N * 4);
  s.all = (int32_t*)take(8);
  s.logits = (float*)take(N * B * K * 4);
  s.dy = (u16*)take(N * B * K * 2);
  s.loss = (float*)take(N * B * 4);
  s.work_bytes = std::max(rfast_lora_workspace_bytes(&shape, 0), rfast_lora_workspace_bytes(&shape, 1));
  s.work = take(s.work_bytes);
  s.total = (size_t)(at - (char*)base);
  return s;
}

// The node of work slot `slot` (as in rfast_softmax.hip): every node while the initial gradient is formed.
__device__ inline int pick_node(const RfastDev& s, bool init, int slot, int* t_old) {
  *t_old = -1;
  if (init) return slot;
  const int2 ap = s.active_plan[slot];
  *t_old = ap.y;
  return ap.x;
}

// blockIdx.y: work slot; blockIdx.x: its rows and its adapter, in strides of the grid.
__global__ void __launch_bounds__(kThreads) rfast_adapters_gather(RfastDev s, Scratch w, const int32_t* batch_idx, int B, bool init) {
  const int slot = blockIdx.y;
  int t_old;
  const int i = pick_node(s, init, slot, &t_old);
  const int active = init ? s.n : s.n_active[0];
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    w.row_ptr[slot] = min(slot, active) * B;
    w.node[slot] = i;
    if (slot == 0) w.row_ptr[s.n] = active * B;
  }
  if (i < 0) return;
  const int64_t lane = (int64_t)blockIdx.x * kThreads + threadIdx.x, lanes = (int64_t)gridDim.x * kThreads;
  const int d = s.prob.d;
  const int64_t pa = (int64_t)s.prob.rank * d, pb = (int64_t)s.prob.rank * s.prob.K;
  for (int64_t k = lane; k < s.p; k += lanes) {
    const u16 v = to_bf16(s.x[(int64_t)i * s.p + k]);
    if (k < pa) w.a[i * pa + k] = v;
    else w.b[i * pb + k - pa] = v;
  }
  const u16* pool = (const u16*)s.prob.data0 + (int64_t)i * s.prob.samples * d;
  const int32_t* labels = (const int32_t*)s.prob.data1 + (int64_t)i * s.prob.samples;
  for (int b = blockIdx.x; b < B; b += gridDim.x) {
    int row = batch_idx ? batch_idx[(int64_t)i * B + b] : b;
    if (row < 0 || row >= s.prob.samples) {
      if (threadIdx.x == 0 && atomicCAS(&s.err[0], 0, RFAST_ERANGE) == 0) {
        s.err[1] = s.n_active[1] - 1;  // the number of this round
        s.err[2] = 2;
        s.err[3] = i;
      }
      row = row < 0 ? 0 : s.prob.samples - 1;
    }
    const int64_t to = (int64_t)slot * B + b;
    if (threadIdx.x == 0) w.label[to] = labels[row];
    const u16* from = pool + (int64_t)row * d;
    for (int k = threadIdx.x * 4; k < d; k += kThreads * 4) {
      float v[4];
      load_four<false>(from + k, d - k, v);
      store_four<false>(w.x + to * d + k, d - k, v);
    }
  }
}

__global__ void __launch_bounds__(kThreads) rfast_adapters_put(RfastDev s, Scratch w, bool init) {
  int t_old;
  const int i = pick_node(s, init, blockIdx.y, &t_old);
  if (i < 0) return;
  const int64_t pa = (int64_t)s.prob.rank * s.prob.d, pb = (int64_t)s.prob.rank * s.prob.K;
  float* g = s.g + ((int64_t)((t_old + 1) & 1) * s.n + i) * s.p;
  for (int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x; k < s.p; k += (int64_t)gridDim.x * kThreads) {
    float v = k < pa ? w.da[i * pa + k] : w.db[i * pb + k - pa];
    if (s.wd != 0.f) v = fmaf(s.wd, s.x[(int64_t)i * s.p + k], v);
    g[k] = v;
  }
}

// The node average as the one adapter of the loss, and its row numbers.
__global__ void __launch_bounds__(kThreads) rfast_adapters_mean(RfastDev s, Scratch w) {
  const int64_t pa = (int64_t)s.prob.rank * s.prob.d;
  for (int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x; k < s.p; k += (int64_t)gridDim.x * kThreads) {
    const u16 v = to_bf16(s.xbar[k]);
    if (k < pa) w.a[k] = v;
    else w.b[k - pa] = v;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    w.all[0] = 0;
    w.all[1] = 0x7fffffff;
  }
}

// *out += scale * sum of loss[0 .. rows): one workgroup, in an order that the sizes alone decide
__global__ void __launch_bounds__(1024) rfast_adapters_sum(const float* loss, int rows, double scale, double* out) {
  __shared__ double part[16];
  double v = 0.0;
  for (int r = threadIdx.x; r < rows; r += 1024) v += loss[r];
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int q = 1; q < 16; ++q) v += part[q];
    *out += scale * v;
  }
}

// (arguments are checked when the context is made: what is left to fail is a launch)
hipError_t status(int code) { return code == RFAST_OK ? hipSuccess : hipErrorLaunchFailure; }

}  // namespace

bool rfast_adapters_shape_ok(int32_t n, int64_t p, const rfast_problem* prob) {
  if (prob->rank < 1 || prob->d < 1 || prob->K < 1 || (int64_t)prob->rank * ((int64_t)prob->d + prob->K) != p) return false;
  if ((int64_t)n * rows_per_node(*prob) > 1 << 27 || !(fabsf(prob->adapter_scale) < 1e30f)) return false;
  const rfast_lora_shape s = shape_of(n, *prob);
  return rfast_lora_workspace_bytes(&s, 1) > 0;
}

size_t rfast_adapters_scratch_bytes(int32_t n, const rfast_problem* prob) {
  return prob->kind == RFAST_OBJ_LORA_SOFTMAX ? scratch_of(nullptr, n, *prob).total : 0;
}

hipError_t rfast_adapters_gradient(rfast_ctx* c, const int32_t* batch_idx, bool init) {
  const RfastDev& d = c->d;
  const rfast_problem& p = d.prob;
  const int B = rows_per_node(p);
  const Scratch w = scratch_of(d.gscratch, d.n, p);
  const rfast_lora_shape s = shape_of(d.n, p);
  rfast_lora_shape back = s;
  back.y_type = RFAST_BF16;
  // eight workgroups per compute unit over all nodes
  const unsigned each = (unsigned)std::min<int64_t>((2048 + d.n - 1) / d.n, std::max<int64_t>(B, (d.p + kThreads - 1) / kThreads));
  hipLaunchKernelGGL(rfast_adapters_gather, dim3(each, d.n), dim3(kThreads), 0, c->stream, d, w, p.batch > 0 ? batch_idx : nullptr, B, init);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess) e = status(rfast_lora_forward(&s, w.x, p.data2, w.a, w.b, w.row_ptr, w.node, w.logits, w.work, w.work_bytes, c->stream));
  if (e == hipSuccess)
    e = status(rfast_softmax_xent(s.rows, p.K, w.logits, RFAST_F32, p.K, w.label, 1.0f / (float)B, nullptr, nullptr, w.dy, RFAST_BF16, p.K,
                                  w.row_ptr + d.n, c->stream));
  if (e == hipSuccess)
    e = status(rfast_lora_backward(&back, w.x, p.data2, w.a, w.b, w.row_ptr, w.node, w.dy, nullptr, w.da, w.db, w.work, w.work_bytes, c->stream));
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(rfast_adapters_put, dim3(each, d.n), dim3(kThreads), 0, c->stream, d, w, init);
  return hipGetLastError();
}

// Adds sum_i f_i(xbar) over the whole pools to *d_out, as many rows at a time as a round may have.
hipError_t rfast_adapters_loss(rfast_ctx* c, double* d_out) {
  const RfastDev& d = c->d;
  const rfast_problem& p = d.prob;
  const Scratch w = scratch_of(d.gscratch, d.n, p);
  rfast_lora_shape s = shape_of(d.n, p);
  s.segments = s.adapters = 1;
  const int64_t total = (int64_t)d.n * p.samples, most = s.rows;
  hipLaunchKernelGGL(rfast_adapters_mean, dim3((unsigned)std::min<int64_t>(1024, (d.p + kThreads - 1) / kThreads)), dim3(kThreads), 0, c->stream, d, w);
  hipError_t e = hipGetLastError();
  for (int64_t r0 = 0; r0 < total && e == hipSuccess; r0 += most) {
    s.rows = (int32_t)std::min(most, total - r0);
    e = status(rfast_lora_forward(&s, (const u16*)p.data0 + r0 * p.d, p.data2, w.a, w.b, w.all, nullptr, w.logits, w.work, w.work_bytes, c->stream));
    if (e == hipSuccess)
      e = status(rfast_softmax_xent(s.rows, p.K, w.logits, RFAST_F32, p.K, (const int32_t*)p.data1 + r0, 1.f, w.loss, nullptr, nullptr, RFAST_F32, p.K,
                                    nullptr, c->stream));
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(rfast_adapters_sum, dim3(1), dim3(1024), 0, c->stream, w.loss, s.rows, 1.0 / (double)p.samples, d_out);
    e = hipGetLastError();
  }
  return e;
}
