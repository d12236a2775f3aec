// Stable sort of whole numbers by counting: rows by the expert they go to, tokens by their number.
//
// A pass takes one digit of the numbers: how often each value of it occurs (per workgroup, over contiguous parts), where each value of each
// part begins (sums over values and parts), and every element behind the earlier ones of its part that have the same digit.  So the order of equal
// numbers is kept and the result does not depend on who runs first.  Numbers up to 2^10 take one pass, up to 2^20 two.
// Counting takes some 4 bytes per element and pass from memory: what bounds it is the latency of the launches.
#include <type_traits>

#include "rfast_operators.h"

namespace {

constexpr int kWaves = 16, kThreads = kWaves * 64;
constexpr int kChunks = 4;                     // of 64 neighbours that a wavefront takes at a time
constexpr int kTile = kThreads * kChunks;      // elements that a workgroup takes at a time
constexpr int kDigitMost = 10;
constexpr int kPartsMost = 256;

struct Part {
  const int32_t* key;   // of this pass, in its order
  const int32_t* index; // NULL: the identity
  int32_t* out_key;
  int32_t* out_index;
  int32_t* counts;      // [parts][bins]
  int32_t* row_ptr;
  int32_t* place;
  int32_t* order;
  int32_t count, keys, per_part;
  int shift;            // this pass's bits begin there
  bool first, last;
};

__device__ inline int clip_key(int32_t k, int32_t keys) { return (uint32_t)k < (uint32_t)keys ? k : keys; }

template <int DIGIT>
__global__ void __launch_bounds__(kThreads) rfast_sort_count(Part a) {
  constexpr int bins = 1 << DIGIT;
  __shared__ int32_t hist[bins];
  for (int b = threadIdx.x; b < bins; b += kThreads) hist[b] = 0;
  __syncthreads();
  const int64_t lo = (int64_t)blockIdx.x * a.per_part, hi = min(lo + a.per_part, (int64_t)a.count);
  for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) {
    const int k = a.first ? clip_key(a.key[i], a.keys) : a.key[i];
    atomicAdd(&hist[(k >> a.shift) & (bins - 1)], 1);
  }
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kThreads) a.counts[(int64_t)blockIdx.x * bins + b] = hist[b];
}

// Exclusive sums over the workgroup's threads.
__device__ inline int32_t before_me(int32_t v, int32_t* box) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int32_t s = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int32_t o = __shfl_up(s, d, 64);
    if (lane >= d) s += o;
  }
  if (lane == 63) box[wave] = s;
  __syncthreads();
  int32_t off = 0;
  for (int w = 0; w < wave; ++w) off += box[w];
  return off + s - v;
}

template <int DIGIT>
__global__ void __launch_bounds__(kThreads) rfast_sort_place(Part a, int parts) {
  constexpr int bins = 1 << DIGIT;
  __shared__ int32_t start[bins];          // where the next element of each digit of this part goes
  __shared__ int32_t hist[kWaves * bins];  // per wavefront: elements of each digit so far, then where they begin
  __shared__ int32_t box[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int me = blockIdx.x, b = threadIdx.x;
  int32_t total = 0, before = 0;
  if (b < bins) {
    for (int p = 0; p < parts; p += 16) {  // (sixteen loads under way; those past the last part read it again)
      int32_t c[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) c[i] = a.counts[(int64_t)min(p + i, parts - 1) * bins + b];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        total += p + i < parts ? c[i] : 0;
        before += p + i < me ? c[i] : 0;
      }
    }
  }
  const int32_t at = before_me(total, box);
  if (b < bins) start[b] = at + before;
  if (a.row_ptr && me == 0 && b <= a.keys) a.row_ptr[b] = at;  // (one pass: bins > keys)
  const int64_t lo = (int64_t)me * a.per_part, hi = min(lo + a.per_part, (int64_t)a.count);
  const uint64_t below = (1ull << lane) - 1;
  for (int64_t tile = lo; tile < hi; tile += kTile) {
    for (int i = threadIdx.x; i < kWaves * bins; i += kThreads) hist[i] = 0;
    __syncthreads();
    int32_t key[kChunks], rank[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const int64_t i = tile + wave * (64 * kChunks) + c * 64 + lane;
      key[c] = i < hi ? (a.first ? clip_key(a.key[i], a.keys) : a.key[i]) : -1;
    }
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const bool is = key[c] >= 0;
      const int digit = (key[c] >> a.shift) & (bins - 1);
      uint64_t same = __ballot(is);
#pragma unroll
      for (int k = 0; k < DIGIT; ++k) {
        const uint64_t one = __ballot((digit >> k) & 1);
        same &= (digit >> k) & 1 ? one : ~one;
      }
      rank[c] = 0;
      if (is) {
        const int32_t had = hist[wave * bins + digit];
        rank[c] = had + __popcll(same & below);
        __builtin_amdgcn_wave_barrier();
        if ((same & below) == 0) hist[wave * bins + digit] = had + __popcll(same);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
    if (b < bins) {
      int32_t run = start[b];
      for (int w = 0; w < kWaves; ++w) {
        const int32_t h = hist[w * bins + b];
        hist[w * bins + b] = run;
        run += h;
      }
      start[b] = run;
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const int64_t i = tile + wave * (64 * kChunks) + c * 64 + lane;
      if (i >= hi) continue;
      const int digit = (key[c] >> a.shift) & (bins - 1);
      const int32_t to = hist[wave * bins + digit] + rank[c];
      const int32_t from = a.index ? a.index[i] : (int32_t)i;
      if (a.out_key) a.out_key[to] = key[c];
      if (a.out_index) a.out_index[to] = from;
      if (a.last) {
        if (a.order) a.order[to] = key[c] < a.keys ? from : -1;
        if (a.place) a.place[from] = key[c] < a.keys ? to : -1;
      }
    }
    __syncthreads();
  }
}

// row_ptr where numbers take several passes: how many of the sorted ones are below each
__global__ void __launch_bounds__(256) rfast_sort_bounds(const int32_t* sorted, int32_t count, int32_t keys, int32_t* row_ptr) {
  const int64_t v = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
  if (v > keys) return;
  int32_t lo = 0, hi = count;
  while (lo < hi) {
    const int32_t mid = lo + (hi - lo) / 2;
    if (sorted[mid] < v) lo = mid + 1;
    else hi = mid;
  }
  row_ptr[v] = lo;
}

size_t up(size_t b) { return (b + 255) / 256 * 256; }

struct Plan {
  int passes, digit, parts;
  int32_t per_part;
  Plan(int32_t count, int32_t keys) {
    int bits = 1;
    while (bits < 31 && (keys >> bits) != 0) ++bits;  // `keys` itself is a number too: that of elements outside
    passes = (bits + kDigitMost - 1) / kDigitMost;
    digit = (bits + passes - 1) / passes;
    digit = digit <= 6 ? 6 : digit < 8 ? 8 : digit;  // (forms of the kernels)
    const int64_t tiles = ((int64_t)count + kTile - 1) / kTile;
    const int64_t per = (tiles + kPartsMost - 1) / kPartsMost;
    per_part = (int32_t)(per * kTile < 0x7fffffff ? per * kTile : 0x7fffffff);
    parts = count ? (int)(((int64_t)count + per_part - 1) / per_part) : 0;
  }
};

}  // namespace

size_t rfast_sort_bytes(int32_t count, int32_t keys) {
  const Plan p(count, keys);
  return up((size_t)p.parts << (p.digit + 2)) + (p.passes > 1 ? 4 : 0) * up((size_t)count * 4) + 256;
}

hipError_t rfast_sort(const RfastSort& s, hipStream_t stream) {
  const Plan p(s.count, s.keys);
  char* ws = (char*)s.workspace;
  int32_t* counts = (int32_t*)ws;
  ws += up((size_t)p.parts << (p.digit + 2));
  int32_t* buffer[4] = {};
  if (p.passes > 1) {
    for (int i = 0; i < 4; ++i) buffer[i] = (int32_t*)ws, ws += up((size_t)s.count * 4);
  }
  const int32_t* sorted = nullptr;
  for (int pass = 0; pass < p.passes && s.count; ++pass) {
    Part a = {};
    a.first = pass == 0;
    a.last = pass == p.passes - 1;
    a.count = s.count;
    a.keys = s.keys;
    a.per_part = p.per_part;
    a.counts = counts;
    a.shift = pass * p.digit;
    a.key = a.first ? s.key : buffer[(pass & 1) ^ 1];
    a.index = a.first ? nullptr : buffer[2 + ((pass & 1) ^ 1)];
    a.out_key = a.last ? s.sorted : buffer[pass & 1];
    a.out_index = a.last ? nullptr : buffer[2 + (pass & 1)];
    if (a.last && !a.out_key && s.row_ptr && p.passes > 1) a.out_key = buffer[pass & 1];
    if (a.last) {
      a.order = s.order;
      a.place = s.place;
      a.row_ptr = p.passes == 1 ? s.row_ptr : nullptr;
      sorted = a.out_key;
    }
    const auto go = [&](auto digit) {
      constexpr int D = decltype(digit)::value;
      hipLaunchKernelGGL((rfast_sort_count<D>), dim3(p.parts), dim3(kThreads), 0, stream, a);
      hipLaunchKernelGGL((rfast_sort_place<D>), dim3(p.parts), dim3(kThreads), 0, stream, a, p.parts);
    };
    using std::integral_constant;
    if (p.digit == 6) go(integral_constant<int, 6>());
    else if (p.digit == 8) go(integral_constant<int, 8>());
    else if (p.digit == 9) go(integral_constant<int, 9>());
    else go(integral_constant<int, 10>());
  }
  if (s.row_ptr && (p.passes > 1 || !s.count))
    hipLaunchKernelGGL(rfast_sort_bounds, rfast_grid_of(((int64_t)s.keys + 256) / 256), dim3(256), 0, stream, sorted, s.count, s.keys, s.row_ptr);
  return hipGetLastError();
}
