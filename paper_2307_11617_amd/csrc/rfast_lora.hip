// Low-rank adapters beside a shared projection, forward and backward.
//
//   u_t = A_a x_t,  y_t = W x_t + s B_a u_t;   e_t = s B_a^T dy_t,  dA_a = sum e_t x_t^T,  dB_a = s sum dy_t u_t^T,
//   dx_t = W^T dy_t + A_a^T e_t,   a = the adapter of row t
//
// Three kinds of products, all bf16 on the matrix cores with sums in 32 bits (v_mfma_f32_16x16x32_bf16):
//   down   rows times an adapter: [rows][c] x [c][rank].  Reads its rows once and is bound by that.
//   up     rows times the projection, with the adapter's second product as some more steps of the same contraction: the shared
//          product's accumulators take s B_a u_t before they are rounded, so that the adapters cost no pass over y.
//   sums   gradients of the adapters: [c][rows] x [rows][rank], contracted over an adapter's rows.  Bound by reading the rows.
// What down hands on (u, e) is held as three bf16, the value and twice what rounding left over, which together are its 24 bits: the
// products that read it are so small beside the others that this costs little, and sums of 32 bits are as good as if it were held in 32.
//
// Operand layout of the 16x16x32 instruction (lane l of 64): A: row l%16, contraction indices 8(l/16) .. +7;  B: column l%16, the
// same indices;  C/D: column l%16, rows 4(l/16) + v for v = 0..3.
#include <algorithm>

#include "rfast_operators.h"

namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int kMostRank = 64;
constexpr int kTileRows = 128, kTileOuts = 128, kStep = 64;  // of `up`
constexpr int kNone = -1, kBehind = -2;  // row without an adapter, row behind the last segment
constexpr size_t kAlign = 256;
size_t up(size_t b) { return (b + kAlign - 1) / kAlign * kAlign; }

__device__ inline f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Eight neighbours from p on, of which `left` exist (any number); zeros for the others.
__device__ inline u32x4 load_eight(const u16* p, int64_t left) {
  if (left >= 8) {
    const any_u32x4 t = *reinterpret_cast<const any_u32x4*>(p);
    return u32x4{t.x, t.y, t.z, t.w};
  }
  u32x4 t = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 7; ++j)
    if (j < left) t[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
  return t;
}

struct Segments {
  const int32_t* row_ptr;
  const int32_t* adapter;
  int32_t count, adapters, rows;
  __device__ int begin(int s) const { return min(max(row_ptr[s], 0), rows); }
  __device__ int end_of_all() const { return begin(count); }
  __device__ int adapter_of(int s) const {
    const int a = adapter ? adapter[s] : s;
    return a >= 0 && a < adapters ? a : kNone;
  }
  // The last segment that does not begin behind `row` (the one that holds it, if any does), found by 64 probes at a time.
  __device__ int find(int row) const {
    int lo = 0, hi = count;
    while (hi - lo > 1) {
      const int step = (hi - lo + 63) / 64, at = lo + (threadIdx.x & 63) * step;
      const int before = __popcll(__ballot(at < hi && row_ptr[at] <= row));
      lo += (before > 0 ? before - 1 : 0) * step;
      hi = min(lo + step, hi);
    }
    return lo;
  }
};

constexpr int tiles_of(int RP) { return RP < 16 ? 1 : RP / 16; }
constexpr int kPieces = 3;  // bf16 that a value of u or e is held as

// ------------------------------------------------------------------------------------------------------------- down
// out = scale * (rows of z) x (adapter's matrix m [rank][cols]) in kPieces bf16:
//   out_rows [rows][kPieces][RP]    what `up` reads
//   out_cols [kPieces][RP][pitch]   what `sums` reads: the same by columns
// One workgroup per 16 rows, its wavefronts share the contraction; rows of several segments are taken one segment after the other, or
// by several workgroups (gridDim.y) where there are so few rows that a segment is one or two of them.
struct Down {
  const u16* z;
  const u16* m;
  u16* out_rows;
  u16* out_cols;
  int32_t* ids;  // [rows] adapter of each row, kNone or kBehind
  Segments seg;
  int64_t ld, pitch;
  int32_t cols, rank;
  float scale;
};

template <int RP>
__global__ void __launch_bounds__(kThreads) rfast_lora_down(Down a) {
  constexpr int NT = tiles_of(RP);
  __shared__ f32x4 part[kWaves][NT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
  const int row0 = blockIdx.x * 16, end = min(row0 + 16, a.seg.rows), behind = a.seg.end_of_all();
  int run = 0;
  for (int r0 = row0, r1; r0 < end; r0 = r1, ++run) {
    int id = kBehind;
    r1 = end;
    if (r0 < behind) {
      const int s = a.seg.find(r0);
      const int stop = a.seg.begin(s + 1);
      id = stop > r0 ? a.seg.adapter_of(s) : kNone;
      r1 = min(stop > r0 ? stop : r0 + 1, end);
    }
    if (run % gridDim.y != blockIdx.y) continue;
    if (a.ids && threadIdx.x < r1 - r0) a.ids[r0 + threadIdx.x] = id;
    if (id == kBehind) break;
    f32x4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4{0, 0, 0, 0};
    if (id >= 0) {
      const bool mine = row0 + n >= r0 && row0 + n < r1;
      const u16* z = a.z + (int64_t)(row0 + n) * a.ld;
      const u16* m = a.m + (int64_t)id * a.rank * a.cols;
      for (int c = wave * 128 + g * 8; c < a.cols + g * 8; c += kWaves * 128) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int left = a.cols - (c + 32 * q);
          const u32x4 zf = load_eight(z + c + 32 * q, mine ? left : 0);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const int k = t * 16 + n;
            acc[t] = mfma(zf, load_eight(m + (int64_t)k * a.cols + c + 32 * q, k < a.rank ? left : 0), acc[t]);
          }
        }
      }
    }
    __syncthreads();  // the sums of the run before have been read
#pragma unroll
    for (int t = 0; t < NT; ++t) part[wave][t][lane] = acc[t];
    __syncthreads();
    if (wave < NT) {
      f32x4 v = part[0][wave][lane];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v += part[w][wave][lane];
      const int k = wave * 16 + n;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int row = row0 + 4 * g + q;
        if (k >= RP || row < r0 || row >= r1) continue;
        float f = v[q] * a.scale;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          const u16 piece = to_bf16(f);
          f -= from_bf16(piece);
          if (!(fabsf(f) < INFINITY)) f = 0.f;  // the value is not finite: the first piece says so, and the others must not undo it
          if (a.out_rows) a.out_rows[((int64_t)row * kPieces + i) * RP + k] = piece;
          if (a.out_cols) a.out_cols[(int64_t)(i * RP + k) * a.pitch + row] = piece;
        }
      }
    }
  }
}

// --------------------------------------------------------------------------------------------------------------- up
// y = (rows of z) x W^T + u x (adapter's matrix b [outs][rank])^T.  W [outs][cols].
struct Up {
  const u16* z;
  const u16* w;
  const u16* b;
  const u16* u;        // [rows][kPieces][RP]
  const int32_t* ids;
  void* y;
  int64_t ld_z, ld_y;
  int32_t rows, cols, outs, rank;
};

// The adapters' part for 16 rows from row0 on (B operand) and 16 outputs from out0 on (A operand): one step per adapter that
// the rows have.  A column of the result is one row's, so that the others of a step are left out there and nothing of an adapter
// (an infinity, say) reaches rows that have another.
template <int RP> __device__ inline f32x4 add_adapters(const Up& a, int row0, int out0, f32x4 acc) {
  constexpr int WIDE = kPieces * RP, STEPS = (WIDE + 31) / 32;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int row = row0 + n, out = out0 + n;
  const int id = row < a.rows ? a.ids[row] : kNone;
  uint64_t pending = __ballot(id >= 0) & 0xFFFF;
  u32x4 u[STEPS];
#pragma unroll
  for (int q = 0; q < STEPS; ++q) {
    const int k = 32 * q + 8 * g;
    u[q] = load_eight(a.u + (int64_t)row * WIDE + k, id >= 0 && k < WIDE ? 8 : 0);
  }
  while (pending) {
    const int who = __builtin_amdgcn_readlane(id, __builtin_ctzll(pending));
    const bool mine = id == who;
    pending &= ~__ballot(mine);
    const u16* b = a.b + ((int64_t)who * a.outs + out) * a.rank;
    f32x4 own = {0, 0, 0, 0};
#pragma unroll
    for (int q = 0; q < STEPS; ++q) {
      const int k = (32 * q + 8 * g) % RP;
      const u32x4 bf = load_eight(b + k, out < a.outs && 32 * q + 8 * g < WIDE ? a.rank - k : 0);
      own = mfma(bf, u[q], own);
    }
    if (mine) acc += own;
  }
  return acc;
}

// Four outputs from `out` on of one row
template <class Y> __device__ inline void store_outs(const Up& a, int row, int out, f32x4 v) {
  if (row >= a.rows || out >= a.outs || a.ids[row] == kBehind) return;
  const float f[4] = {v.x, v.y, v.z, v.w};
  store_four<false>((Y*)a.y + (int64_t)row * a.ld_y + out, a.outs - out, f);
}


// Many rows: a workgroup's tile of 128 outputs x 128 rows, 64 x 64 per wavefront, both operands through two buffers in LDS.  Chunks of
// 16 bytes are put at (chunk ^ row % 8) of their row, so that the 16 rows of an operand fall on all banks.
template <int RP, class Y>
__global__ void __launch_bounds__(kThreads) rfast_lora_up(Up a, int row_tiles) {
  __shared__ u32x4 tile[2][2][128 * kStep / 8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
  const int row0 = (blockIdx.x % row_tiles) * kTileRows, out0 = (blockIdx.x / row_tiles) * kTileOuts;
  const int wo = (wave >> 1) * 64, wr = (wave & 1) * 64;
  f32x4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
  u32x4 next[2][4];
  auto fetch = [&](int c0) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int r = (threadIdx.x >> 3) + 32 * q, c = c0 + (threadIdx.x & 7) * 8;
      next[0][q] = load_eight(a.w + (int64_t)(out0 + r) * a.cols + c, out0 + r < a.outs ? a.cols - c : 0);
      next[1][q] = load_eight(a.z + (int64_t)(row0 + r) * a.ld_z + c, row0 + r < a.rows ? a.cols - c : 0);
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int r = (threadIdx.x >> 3) + 32 * q, at = r * 8 + ((threadIdx.x & 7) ^ (r & 7));
      tile[buf][0][at] = next[0][q];
      tile[buf][1][at] = next[1][q];
    }
  };
  fetch(0);
  put(0);
  __syncthreads();
  for (int c0 = 0, buf = 0; c0 < a.cols; c0 += kStep, buf ^= 1) {
    const bool more = c0 + kStep < a.cols;
    if (more) fetch(c0 + kStep);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      u32x4 wf[4], zf[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ro = wo + 16 * i + n, rr = wr + 16 * i + n;
        wf[i] = tile[buf][0][ro * 8 + ((4 * q + g) ^ (ro & 7))];
        zf[i] = tile[buf][1][rr * 8 + ((4 * q + g) ^ (rr & 7))];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = mfma(wf[i], zf[j], acc[i][j]);
    }
    if (more) put(buf ^ 1);
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = row0 + wr + 16 * j, o = out0 + wo + 16 * i;
      if (r >= a.rows || o >= a.outs) continue;
      store_outs<Y>(a, r + n, o + 4 * g, add_adapters<RP>(a, r, o, acc[i][j]));
    }
}

// Up to 64 rows: bound by one read of W, which goes from memory to the registers of one wavefront and no further.  A workgroup has 16
// outputs, its wavefronts share the contraction.
constexpr int kFewRows = 64;
template <int RP, class Y, int RT>
__global__ void __launch_bounds__(kThreads) rfast_lora_up_few(Up a) {
  __shared__ f32x4 part[kWaves][RT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
  const int out0 = blockIdx.x * 16;
  f32x4 acc[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) acc[t] = f32x4{0, 0, 0, 0};
  const u16* w = a.w + (int64_t)(out0 + n) * a.cols;
  for (int c = wave * 128 + g * 8; c < a.cols + g * 8; c += kWaves * 128) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int left = a.cols - (c + 32 * q);
      const u32x4 wf = load_eight(w + c + 32 * q, out0 + n < a.outs ? left : 0);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const int row = 16 * t + n;
        acc[t] = mfma(wf, load_eight(a.z + (int64_t)row * a.ld_z + c + 32 * q, row < a.rows ? left : 0), acc[t]);
      }
    }
  }
#pragma unroll
  for (int t = 0; t < RT; ++t)
    if (wave == t) acc[t] = add_adapters<RP>(a, 16 * t, out0, acc[t]);
#pragma unroll
  for (int t = 0; t < RT; ++t) part[wave][t][lane] = acc[t];
  __syncthreads();
  if (wave < RT) {
    f32x4 v = part[0][wave][lane];
#pragma unroll
    for (int q = 1; q < kWaves; ++q) v += part[q][wave][lane];
    store_outs<Y>(a, 16 * wave + n, out0 + 4 * g, v);
  }
}

// ------------------------------------------------------------------------------------------------------------- sums
// out of adapter i = scale * sum over its rows of (row of z) x (row of s): [cols][rank], or [rank][cols] (RANK_MAJOR).
// A lane reads eight columns of eight rows, 16 bytes a row, and turns that block over in registers (one byte permutation per pair of
// elements), so that it has eight rows of each of its columns: operands without LDS.  Column 8 m + j is row m of operand j.
struct Sums {
  const u16* z;
  const u16* s;  // [kPieces][RP][pitch]
  float* out;
  Segments seg;
  int64_t ld, pitch;
  int32_t cols, rank;
  float scale;
};

// operands that the pieces of 16 ranks come in: one each, or, of 8 ranks, the first two pieces side by side and the third alone
template <int RP> constexpr int kFrags = RP == 8 ? 2 : kPieces;

template <int RP, bool RANK_MAJOR>
__global__ void __launch_bounds__(kThreads) rfast_lora_sums(Sums a) {
  constexpr int NT = tiles_of(RP);
  __shared__ f32x4 part[2][8][NT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
  const int who = blockIdx.y, c0 = blockIdx.x * 128;
  f32x4 acc[8][NT];
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[j][t] = f32x4{0, 0, 0, 0};
  auto segment = [&](int s) {
    const int end = a.seg.begin(s + 1);
    for (int t0 = a.seg.begin(s) + wave * 32; t0 < end; t0 += kWaves * 32) {
      const int r = t0 + 8 * g, c = c0 + 8 * n;
      u32x4 z[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = load_eight(a.z + (int64_t)(r + i) * a.ld + c, r + i < end ? a.cols - c : 0);
      u32x4 sf[NT][kFrags<RP>];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < kFrags<RP>; ++i) {
          const int k = (RP == 8 ? 16 * i : RP * i + 16 * t) + n;
          sf[t][i] = load_eight(a.s + (int64_t)k * a.pitch + r, k < kPieces * RP ? end - r : 0);
        }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        u32x4 zf;
#pragma unroll
        for (int q = 0; q < 4; ++q) zf[q] = __builtin_amdgcn_perm(z[2 * q + 1][j >> 1], z[2 * q][j >> 1], j & 1 ? 0x07060302 : 0x05040100);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < kFrags<RP>; ++i) acc[j][t] = RANK_MAJOR ? mfma(sf[t][i], zf, acc[j][t]) : mfma(zf, sf[t][i], acc[j][t]);
      }
    }
  };
  if (!a.seg.adapter) {
    if (who < a.seg.count) segment(who);
  } else {
    for (int s0 = 0; s0 < a.seg.count; s0 += 64) {
      uint64_t hit = __ballot(s0 + lane < a.seg.count && a.seg.adapter[s0 + lane] == who);
      for (; hit; hit &= hit - 1) segment(s0 + __builtin_ctzll(hit));
    }
  }
  // the wavefronts' sums, two and two
#pragma unroll
  for (int half = 2; half >= 1; half >>= 1) {
    __syncthreads();
    if (wave >= half && wave < 2 * half)
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int t = 0; t < NT; ++t) part[wave - half][j][t][lane] = acc[j][t];
    __syncthreads();
    if (wave < half)
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[j][t] += part[wave][j][t][lane];
  }
  if (wave != 0) return;
  if (RP == 8) {  // ranks 8 to 15 are second pieces of 0 to 7
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v) acc[j][0][v] += __shfl_xor(acc[j][0][v], RANK_MAJOR ? 32 : 8, 64);
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (RANK_MAJOR) {
      const int c = c0 + 8 * n;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int k = t * 16 + 4 * g + v;
        if (k >= a.rank || c >= a.cols) continue;
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = acc[j][t][v] * a.scale;
        float* to = a.out + ((int64_t)who * a.rank + k) * a.cols + c;
        store_four<false>(to, a.cols - c, f);
        if (a.cols - c > 4) store_four<false>(to + 4, a.cols - c - 4, f + 4);
      }
    } else {
      const int k = t * 16 + n;
      if (k >= a.rank) continue;
#pragma unroll
      for (int v = 0; v < 4; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int c = c0 + 8 * (4 * g + v) + j;
          if (c < a.cols) a.out[((int64_t)who * a.cols + c) * a.rank + k] = acc[j][t][v] * a.scale;
        }
    }
  }
}

// -------------------------------------------------------------------------------------------------------- transposes
// out [batch][cols][rows] = in [batch][rows][cols]
__global__ void __launch_bounds__(kThreads) rfast_lora_transpose(const u16* in, u16* out, int rows, int cols) {
  __shared__ u16 t[64][66];
  const int64_t at = (int64_t)blockIdx.z * rows * cols;
  const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64, x = threadIdx.x & 63;
  for (int q = threadIdx.x >> 6; q < 64; q += 4)
    if (r0 + q < rows && c0 + x < cols) t[q][x] = in[at + (int64_t)(r0 + q) * cols + c0 + x];
  __syncthreads();
  for (int q = threadIdx.x >> 6; q < 64; q += 4)
    if (c0 + q < cols && r0 + x < rows) out[at + (int64_t)(c0 + q) * rows + r0 + x] = t[x][q];
}

// ------------------------------------------------------------------------------------------------------------- host
int padded_rank(int rank) { return rank <= 8 ? 8 : rank <= 16 ? 16 : rank <= 32 ? 32 : 64; }

struct Layout {
  size_t ids, u_rows, u_cols, e_rows, e_cols, bt, at, wt, total;
  int64_t pitch;
};
Layout layout_of(const rfast_lora_shape& s, int pass) {
  Layout l;
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t at = off; off += up(bytes); return at; };
  const size_t T = (size_t)s.rows, wide = kPieces * (size_t)padded_rank(s.rank), d = (size_t)s.d, K = (size_t)s.K, r = (size_t)s.rank, n = (size_t)s.adapters;
  l.pitch = ((int64_t)s.rows + 7) / 8 * 8;
  l.ids = take(T * 4);
  l.u_rows = take(pass == 0 ? T * wide * 2 : 0);
  l.u_cols = take(pass != 0 ? wide * (size_t)l.pitch * 2 : 0);
  l.e_cols = take(pass != 0 ? wide * (size_t)l.pitch * 2 : 0);
  l.bt = take(pass != 0 ? n * K * r * 2 : 0);
  l.e_rows = take(pass == 2 ? T * wide * 2 : 0);
  l.at = take(pass == 2 ? n * d * r * 2 : 0);
  l.wt = take(pass == 2 ? d * K * 2 : 0);
  l.total = off;
  return l;
}

bool shape_ok(const rfast_lora_shape* s) {
  if (!s || s->rows < 0 || s->segments < 1 || s->adapters < 1 || s->d < 1 || s->K < 1 || s->rank < 1 || s->rank > kMostRank) return false;
  if (s->rows > 1 << 27 || s->d > 1 << 22 || s->K > 1 << 22 || s->adapters > 65535 || s->segments == 0x7fffffff) return false;
  // a launch has fewer than 2^32 lanes
  return ((int64_t)s->rows / kTileRows + 1) * (std::max(s->d, s->K) / kTileOuts + 1) < (int64_t)1 << 24;
}

template <class F> hipError_t by_rank(int rank, F f) {
  switch (padded_rank(rank)) {
    case 8: return f(std::integral_constant<int, 8>());
    case 16: return f(std::integral_constant<int, 16>());
    case 32: return f(std::integral_constant<int, 32>());
    default: return f(std::integral_constant<int, 64>());
  }
}

hipError_t launch_down(const Down& a, hipStream_t st) {
  // with few rows the segments of 16 of them go to workgroups of their own
  const int spread = a.seg.rows <= 1024 ? std::min(16, a.seg.count) : 1;
  return by_rank(a.rank, [&](auto rp) {
    hipLaunchKernelGGL((rfast_lora_down<decltype(rp)::value>), dim3((a.seg.rows + 15) / 16, spread), dim3(kThreads), 0, st, a);
    return hipGetLastError();
  });
}

template <class Y> hipError_t launch_up(const Up& a, hipStream_t st) {
  return by_rank(a.rank, [&](auto rp) {
    constexpr int RP = decltype(rp)::value;
    if (a.rows <= kFewRows) {
      const dim3 grid((unsigned)((a.outs + 15) / 16));
      if (a.rows <= 16) hipLaunchKernelGGL((rfast_lora_up_few<RP, Y, 1>), grid, dim3(kThreads), 0, st, a);
      else if (a.rows <= 32) hipLaunchKernelGGL((rfast_lora_up_few<RP, Y, 2>), grid, dim3(kThreads), 0, st, a);
      else hipLaunchKernelGGL((rfast_lora_up_few<RP, Y, 4>), grid, dim3(kThreads), 0, st, a);
    } else {
      const int row_tiles = (a.rows + kTileRows - 1) / kTileRows, out_tiles = (a.outs + kTileOuts - 1) / kTileOuts;
      hipLaunchKernelGGL((rfast_lora_up<RP, Y>), dim3((unsigned)row_tiles * out_tiles), dim3(kThreads), 0, st, a, row_tiles);
    }
    return hipGetLastError();
  });
}

template <bool RANK_MAJOR> hipError_t launch_sums(const Sums& a, hipStream_t st) {
  return by_rank(a.rank, [&](auto rp) {
    hipLaunchKernelGGL((rfast_lora_sums<decltype(rp)::value, RANK_MAJOR>), dim3((a.cols + 127) / 128, a.seg.adapters), dim3(kThreads), 0, st, a);
    return hipGetLastError();
  });
}

hipError_t launch_transpose(const u16* in, u16* out, int batch, int rows, int cols, hipStream_t st) {
  hipLaunchKernelGGL(rfast_lora_transpose, dim3((cols + 63) / 64, (rows + 63) / 64, batch), dim3(kThreads), 0, st, in, out, rows, cols);
  return hipGetLastError();
}

bool at_multiple(const void* p, size_t to) { return (uintptr_t)p % to == 0; }

int check(const rfast_lora_shape* s, int pass, const void* x, const void* W, const void* A, const void* B, const int32_t* row_ptr,
          const int32_t* adapter, const void* y, const void* workspace, size_t workspace_bytes) {
  if (!shape_ok(s)) return rfast_refuse(RFAST_EINVAL, "sizes out of range (rank 1 .. 64)");
  if (s->ld_x < s->d || s->ld_y < s->K) return rfast_refuse(RFAST_EINVAL, "rows are at least their length apart");
  if (s->y_type != RFAST_BF16 && !(pass == 0 && s->y_type == RFAST_F32)) return rfast_refuse(RFAST_EINVAL, "y_type: RFAST_BF16, or RFAST_F32 forward");
  if (!(s->scale > -1e30f && s->scale < 1e30f)) return rfast_refuse(RFAST_ERANGE, "scale must be finite");
  if (!W || !A || !B || !row_ptr || !workspace || (s->rows > 0 && (!x || !y))) return rfast_refuse(RFAST_EINVAL, "NULL argument");
  if (!at_multiple(workspace, kAlign)) return rfast_refuse(RFAST_EINVAL, "workspace must be 256-byte aligned");
  if (!at_multiple(x, 2) || !at_multiple(W, 2) || !at_multiple(A, 2) || !at_multiple(B, 2) || !at_multiple(row_ptr, 4) || !at_multiple(adapter, 4) ||
      !at_multiple(y, s->y_type == RFAST_F32 ? 4 : 2))
    return rfast_refuse(RFAST_EINVAL, "an address is no multiple of its element's size");
  if (workspace_bytes < layout_of(*s, pass).total) return rfast_refuse(RFAST_ENOMEM, "workspace too small");
  return RFAST_OK;
}

}  // namespace

extern "C" {

size_t rfast_lora_workspace_bytes(const rfast_lora_shape* s, int32_t pass) {
  if (!shape_ok(s) || pass < 0 || pass > 2) return 0;
  return layout_of(*s, pass).total;
}

int rfast_lora_forward(const rfast_lora_shape* s, const void* x, const void* W, const void* A, const void* B, const int32_t* row_ptr,
                       const int32_t* adapter, void* y, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int rc = check(s, 0, x, W, A, B, row_ptr, adapter, y, workspace, workspace_bytes);
  if (rc != RFAST_OK || s->rows == 0) return rc;
  const hipStream_t st = (hipStream_t)hip_stream;
  const Layout l = layout_of(*s, 0);
  char* ws = (char*)workspace;
  const Segments seg = {row_ptr, adapter, s->segments, s->adapters, s->rows};
  hipError_t e = launch_down({(const u16*)x, (const u16*)A, (u16*)(ws + l.u_rows), nullptr, (int32_t*)(ws + l.ids), seg, s->ld_x, 0, s->d, s->rank, s->scale}, st);
  if (e != hipSuccess) return rfast_refuse_hip(e, "adapter launch");
  const Up u = {(const u16*)x, (const u16*)W, (const u16*)B, (const u16*)(ws + l.u_rows), (const int32_t*)(ws + l.ids), y, s->ld_x, s->ld_y, s->rows, s->d, s->K, s->rank};
  e = s->y_type == RFAST_F32 ? launch_up<float>(u, st) : launch_up<u16>(u, st);
  return e == hipSuccess ? RFAST_OK : rfast_refuse_hip(e, "projection launch");
}

int rfast_lora_backward(const rfast_lora_shape* s, const void* x, const void* W, const void* A, const void* B, const int32_t* row_ptr,
                        const int32_t* adapter, const void* dy, void* dx, float* dA, float* dB, void* workspace, size_t workspace_bytes,
                        void* hip_stream) {
  const int pass = dx ? 2 : 1;
  const int rc = check(s, pass, x, W, A, B, row_ptr, adapter, dy, workspace, workspace_bytes);
  if (rc != RFAST_OK) return rc;
  if (!dA || !dB) return rfast_refuse(RFAST_EINVAL, "NULL argument");
  if (!at_multiple(dA, 4) || !at_multiple(dB, 4) || !at_multiple(dx, 2)) return rfast_refuse(RFAST_EINVAL, "an address is no multiple of its element's size");
  const hipStream_t st = (hipStream_t)hip_stream;
  const Layout l = layout_of(*s, pass);
  char* ws = (char*)workspace;
  const Segments seg = {row_ptr, adapter, s->segments, s->adapters, s->rows};
  u16 *u_cols = (u16*)(ws + l.u_cols), *e_cols = (u16*)(ws + l.e_cols), *bt = (u16*)(ws + l.bt);
  u16* e_rows = dx ? (u16*)(ws + l.e_rows) : nullptr;
  int32_t* ids = (int32_t*)(ws + l.ids);
  hipError_t e = hipSuccess;
  if (s->rows > 0) {
    e = launch_transpose((const u16*)B, bt, s->adapters, s->K, s->rank, st);
    if (e == hipSuccess) e = launch_down({(const u16*)x, (const u16*)A, nullptr, u_cols, nullptr, seg, s->ld_x, l.pitch, s->d, s->rank, 1.f}, st);
    if (e == hipSuccess) e = launch_down({(const u16*)dy, bt, e_rows, e_cols, ids, seg, s->ld_y, l.pitch, s->K, s->rank, s->scale}, st);
  }
  if (e == hipSuccess) e = launch_sums<true>({(const u16*)x, e_cols, dA, seg, s->ld_x, l.pitch, s->d, s->rank, 1.f}, st);
  if (e == hipSuccess) e = launch_sums<false>({(const u16*)dy, u_cols, dB, seg, s->ld_y, l.pitch, s->K, s->rank, s->scale}, st);
  if (e == hipSuccess && dx && s->rows > 0) {
    u16 *wt = (u16*)(ws + l.wt), *at = (u16*)(ws + l.at);
    e = launch_transpose((const u16*)W, wt, 1, s->K, s->d, st);
    if (e == hipSuccess) e = launch_transpose((const u16*)A, at, s->adapters, s->rank, s->d, st);
    if (e == hipSuccess) e = launch_up<u16>({(const u16*)dy, wt, at, e_rows, ids, dx, s->ld_y, s->ld_x, s->rows, s->K, s->d, s->rank}, st);
  }
  return e == hipSuccess ? RFAST_OK : rfast_refuse_hip(e, "adapter gradient launch");
}

}  // extern "C"
