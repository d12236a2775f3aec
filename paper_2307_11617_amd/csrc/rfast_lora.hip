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
#include <type_traits>

#include "rfast_operators.h"

namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int kMostRank = 64;
constexpr int kStep = 64;                 // contraction indices of a stage of `up`
constexpr int kNone = -1, kBehind = -2;  // row without an adapter, row behind the last segment
constexpr size_t kAlign = 256;
size_t up(size_t b) { return (b + kAlign - 1) / kAlign * kAlign; }

__device__ inline f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Eight neighbours from p on.
__device__ inline u32x4 load_eight(const u16* p) {
  const any_u32x4 t = *reinterpret_cast<const any_u32x4*>(p);
  return u32x4{t.x, t.y, t.z, t.w};
}
// ... of which `left` exist (any number); zeros for the others.  For the ends of rows: a condition per load has it waited for before the next
// is sent, so wherever all of them exist the loads go out without one.
__device__ inline u32x4 load_eight(const u16* p, int64_t left) {
  if (left >= 8) return load_eight(p);
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
// A workgroup has 16 RT rows, its WAVES wavefronts share the contraction; rows of several segments are taken one segment after the other,
// or by several workgroups (gridDim.y) where there are so few rows that a segment is one or two of them.  Rows and ranks that do not
// exist or belong to another segment are read as the nearest that do, and what comes of them is left out.
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

template <int RP, int RT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) rfast_lora_down(Down a) {
  constexpr int NT = tiles_of(RP), CHUNK = 128;
  __shared__ f32x4 part[WAVES][RT * NT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int row0 = blockIdx.x * (16 * RT), end = min(row0 + 16 * RT, a.seg.rows), behind = a.seg.end_of_all();
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
    f32x4 acc[RT][NT];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[i][t] = f32x4{0, 0, 0, 0};
    if (id >= 0) {
      const u16 *z[RT], *m[NT];
#pragma unroll
      for (int i = 0; i < RT; ++i) z[i] = a.z + (int64_t)min(max(row0 + 16 * i + n, r0), r1 - 1) * a.ld + g * 8;
#pragma unroll
      for (int t = 0; t < NT; ++t) m[t] = a.m + ((int64_t)id * a.rank + min(t * 16 + n, a.rank - 1)) * a.cols + g * 8;
      const int whole = a.cols / CHUNK * CHUNK;
      auto chunk = [&](int c, auto load) {
        u32x4 zf[4][RT], mf[4][NT];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
#pragma unroll
          for (int i = 0; i < RT; ++i) zf[q][i] = load(z[i], c + 32 * q);
#pragma unroll
          for (int t = 0; t < NT; ++t) mf[q][t] = load(m[t], c + 32 * q);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[i][t] = mfma(zf[q][i], mf[q][t], acc[i][t]);
      };
      for (int c = wave * CHUNK; c < whole; c += WAVES * CHUNK) chunk(c, [&](const u16* p, int at) { return load_eight(p + at); });
      if (whole < a.cols && wave == whole / CHUNK % WAVES)
        chunk(whole, [&](const u16* p, int at) { return load_eight(p + at, a.cols - at - g * 8); });
    }
    __syncthreads();  // the sums of the run before have been read
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int t = 0; t < NT; ++t) part[wave][i * NT + t][lane] = acc[i][t];
    __syncthreads();
    for (int u = wave; u < RT * NT; u += WAVES) {
      f32x4 v = part[0][u][lane];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) v += part[w][u][lane];
      const int k = u % NT * 16 + n, first = row0 + u / NT * 16 + 4 * g;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int row = first + q;
        if (k >= RP || row < r0 || row >= r1) continue;
        float f = k < a.rank ? v[q] * a.scale : 0.f;
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

template <int RP> struct Pieces {  // of u for 16 rows, as B operand
  static constexpr int WIDE = kPieces * RP, STEPS = (WIDE + 31) / 32;
  u32x4 f[STEPS];
  __device__ void load(const Up& a, int row) {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int q = 0; q < STEPS; ++q) {
      const int k = 32 * q + 8 * g;
      f[q] = load_eight(a.u + (int64_t)row * WIDE + min(k, WIDE - 8));
      if (k >= WIDE) f[q] = u32x4{0, 0, 0, 0};
    }
  }
};
template <int RP> struct Factor {  // b of adapter `who` for 16 outputs from out0 on, as A operand
  static constexpr int WIDE = kPieces * RP, STEPS = (WIDE + 31) / 32;
  u32x4 f[STEPS];
  __device__ void load(const Up& a, int who, int out0) {
    const int lane = threadIdx.x & 63, out = min(out0 + (lane & 15), a.outs - 1);
    const u16* b = a.b + ((int64_t)who * a.outs + out) * a.rank;
#pragma unroll
    for (int q = 0; q < STEPS; ++q) {
      const int k = 32 * q + 8 * (lane >> 4);
      if (a.rank == RP) f[q] = k < WIDE ? load_eight(b + k % RP) : u32x4{0, 0, 0, 0};
      else f[q] = load_eight(b + k % RP, k < WIDE ? a.rank - k % RP : 0);
    }
  }
};

// The adapters' part for 16 rows (their pieces u, their adapters id: lane n has row n's) and 16 outputs from out0 on: one step per adapter
// that the rows have.  A column of the result is one row's, so that the others of a step are left out there and nothing of an adapter (an
// infinity, say) reaches rows that have another.
template <int RP> __device__ inline f32x4 add_adapters(const Up& a, const Pieces<RP>& u, int id, int out0, f32x4 acc) {
  uint64_t pending = __ballot(id >= 0) & 0xFFFF;
  while (pending) {
    const int who = __builtin_amdgcn_readlane(id, __builtin_ctzll(pending));
    const bool mine = id == who;
    pending &= ~__ballot(mine);
    Factor<RP> b;
    b.load(a, who, out0);
    f32x4 own = {0, 0, 0, 0};
#pragma unroll
    for (int q = 0; q < Factor<RP>::STEPS; ++q) own = mfma(b.f[q], u.f[q], own);
    if (mine) acc += own;
  }
  return acc;
}

// Four outputs from `out` on of one row
template <class Y> __device__ inline void store_outs(const Up& a, int row, int id, int out, f32x4 v) {
  if (row >= a.rows || out >= a.outs || id == kBehind) return;
  const float f[4] = {v.x, v.y, v.z, v.w};
  store_four<false>((Y*)a.y + (int64_t)row * a.ld_y + out, a.outs - out, f);
}

// Many rows: a workgroup's tile of TO outputs x TR rows, shared by WO x WR wavefronts, both operands through two buffers in LDS.  A row of a
// stage is eight chunks of 16 bytes; chunk c is put at place c ^ row % 8, so that the 16 rows of an operand fall on all banks.
// DIRECT: rows begin at multiples of 16 bytes, and stages go from memory to LDS without passing through registers (a wavefront's load
// fills 1 KB, eight rows, in the order of its lanes, so each lane fetches the chunk that belongs to its place); else, and for a last stage
// that is not whole, through registers.
// TURNED: w is [cols][outs] instead, as the gradient of the rows reads it.  A lane fetches eight rows of four outputs and turns that block
// over in registers, one byte permutation per pair of elements.
template <int RP, class Y, int TO, int TR, int WO, int WR, bool DIRECT, bool TURNED>
__global__ void __launch_bounds__(64 * WO * WR) rfast_lora_up(Up a, int row_tiles, int out_tiles) {
  constexpr int WAVES = WO * WR, THREADS = 64 * WAVES, OI = TO / WO / 16, RJ = TR / WR / 16;
  constexpr int WL = TO / 8 / WAVES, ZL = TR / 8 / WAVES;  // loads of 16 bytes per lane and stage
  static_assert(WL * 8 * WAVES == TO && ZL * 8 * WAVES == TR && TO * kStep / 32 == THREADS * (TO * kStep / 32 / THREADS), "tile");
  constexpr int TL = TURNED ? TO * kStep / 32 / THREADS : 1;  // blocks of 8 x 4 per lane
  __shared__ u32x4 w_tile[2][TO * 8], z_tile[2][TR * 8];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  // Workgroups are dealt to the eight XCDs by turns: one XCD gets consecutive tiles, which share rows and outputs in its L2.
  const int tiles = row_tiles * out_tiles;
  int t = blockIdx.x;
  if (tiles % 8 == 0) t = t % 8 * (tiles / 8) + t / 8;
  // bands of eight tiles of rows, within a band output by output
  const int band = t / (8 * out_tiles), in_band = t - band * 8 * out_tiles, high = min(8, row_tiles - 8 * band);
  const int row0 = (band * 8 + in_band % high) * TR, out0 = in_band / high * TO;
  const int wo = wave / WR * (TO / WO), wr = wave % WR * (TR / WR);

  f32x4 acc[OI][RJ];
#pragma unroll
  for (int i = 0; i < OI; ++i)
#pragma unroll
    for (int j = 0; j < RJ; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

  // this lane's place of a load: row lane / 8 of eight, and the chunk that goes there
  const int lr = lane >> 3, lc = ((lane & 7) ^ lr) * 8;
  const u16* zp[ZL];
  const u16* wp[WL];
#pragma unroll
  for (int q = 0; q < ZL; ++q) zp[q] = a.z + (int64_t)min(row0 + (q * WAVES + wave) * 8 + lr, a.rows - 1) * a.ld_z + lc;
#pragma unroll
  for (int q = 0; q < WL; ++q) wp[q] = a.w + (int64_t)min(out0 + (q * WAVES + wave) * 8 + lr, a.outs - 1) * a.cols + lc;
  u32x4 zr[ZL], wr_[WL];
  any_u32x2 tr[TL][8];
  const bool outs_whole = out0 + TO <= a.outs;

  auto send = [&](u32x4* to, const u16* from) {
    __builtin_amdgcn_global_load_lds((const RFAST_GLOBAL void*)(uintptr_t)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
  };
  auto fetch = [&](int c0, int buf) {  // stage from c0 on: into LDS, or into registers for `put`
    const bool whole = c0 + kStep <= a.cols;
    if (DIRECT && whole) {
#pragma unroll
      for (int q = 0; q < ZL; ++q) send(&z_tile[buf][(q * WAVES + wave) * 64], zp[q] + c0);
      if constexpr (!TURNED) {
#pragma unroll
        for (int q = 0; q < WL; ++q) send(&w_tile[buf][(q * WAVES + wave) * 64], wp[q] + c0);
      }
    } else if (whole) {
#pragma unroll
      for (int q = 0; q < ZL; ++q) zr[q] = load_eight(zp[q] + c0);
      if constexpr (!TURNED) {
#pragma unroll
        for (int q = 0; q < WL; ++q) wr_[q] = load_eight(wp[q] + c0);
      }
    } else {
#pragma unroll
      for (int q = 0; q < ZL; ++q) zr[q] = load_eight(zp[q] + c0, a.cols - c0 - lc);
      if constexpr (!TURNED) {
#pragma unroll
        for (int q = 0; q < WL; ++q) wr_[q] = load_eight(wp[q] + c0, a.cols - c0 - lc);
      }
    }
    if constexpr (TURNED) {
#pragma unroll
      for (int q = 0; q < TL; ++q) {
        const int b = q * THREADS + threadIdx.x, k = c0 + b / (TO / 4) * 8, o = out0 + b % (TO / 4) * 4;
        const u16* p = a.w + (int64_t)k * a.outs + o;
        if (whole && outs_whole) {
#pragma unroll
          for (int i = 0; i < 8; ++i) tr[q][i] = *reinterpret_cast<const any_u32x2*>(p + (int64_t)i * a.outs);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const u32x4 v = load_eight(p + (int64_t)i * a.outs, k + i < a.cols ? min(a.outs - o, 4) : 0);
            tr[q][i] = any_u32x2{v.x, v.y};
          }
        }
      }
    }
  };
  auto put = [&](int c0, int buf) {
    if (!DIRECT || c0 + kStep > a.cols) {
#pragma unroll
      for (int q = 0; q < ZL; ++q) z_tile[buf][(q * WAVES + wave) * 64 + lane] = zr[q];
      if constexpr (!TURNED) {
#pragma unroll
        for (int q = 0; q < WL; ++q) w_tile[buf][(q * WAVES + wave) * 64 + lane] = wr_[q];
      }
    }
    if constexpr (TURNED) {
#pragma unroll
      for (int q = 0; q < TL; ++q) {
        const int b = q * THREADS + threadIdx.x, c = b / (TO / 4), o = b % (TO / 4) * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          u32x4 v;
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_perm(tr[q][2 * i + 1][j >> 1], tr[q][2 * i][j >> 1], j & 1 ? 0x07060302 : 0x05040100);
          w_tile[buf][(o + j) * 8 + (c ^ ((o + j) & 7))] = v;
        }
      }
    }
  };
  // (all of a wavefront's loads into LDS have arrived, then all wavefronts')
  auto meet = [&] {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };

  fetch(0, 0);
  put(0, 0);
  meet();
  for (int c0 = 0, buf = 0; c0 < a.cols; c0 += kStep, buf ^= 1) {
    const bool more = c0 + kStep < a.cols;
    if (more) fetch(c0 + kStep, buf ^ 1);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      u32x4 wf[OI], zf[RJ];
#pragma unroll
      for (int j = 0; j < RJ; ++j) zf[j] = z_tile[buf][(wr + 16 * j + n) * 8 + ((4 * q + g) ^ (n & 7))];
#pragma unroll
      for (int i = 0; i < OI; ++i) wf[i] = w_tile[buf][(wo + 16 * i + n) * 8 + ((4 * q + g) ^ (n & 7))];
#pragma unroll
      for (int i = 0; i < OI; ++i)
#pragma unroll
        for (int j = 0; j < RJ; ++j) acc[i][j] = mfma(wf[i], zf[j], acc[i][j]);
    }
    if (more) put(c0 + kStep, buf ^ 1);
    meet();
  }

  // The adapters' part.  Usually all rows of a wavefront have the same adapter, whose factors are then fetched once for all of them.
  int id[RJ];
  Pieces<RP> u[RJ];
  bool alike = true;
#pragma unroll
  for (int j = 0; j < RJ; ++j) {
    const int row = row0 + wr + 16 * j + n;
    id[j] = row < a.rows ? a.ids[row] : kBehind;
    u[j].load(a, min(row, a.rows - 1));
  }
  const int who = __builtin_amdgcn_readfirstlane(id[0]);
#pragma unroll
  for (int j = 0; j < RJ; ++j) alike = alike && __all(id[j] == who);
#pragma unroll
  for (int i = 0; i < OI; ++i) {
    const int o = out0 + wo + 16 * i;
    if (o >= a.outs) break;
    if (alike) {
      if (who >= 0) {
        Factor<RP> b;
        b.load(a, who, o);
#pragma unroll
        for (int j = 0; j < RJ; ++j)
#pragma unroll
          for (int q = 0; q < Factor<RP>::STEPS; ++q) acc[i][j] = mfma(b.f[q], u[j].f[q], acc[i][j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < RJ; ++j) acc[i][j] = add_adapters<RP>(a, u[j], id[j], o, acc[i][j]);
    }
#pragma unroll
    for (int j = 0; j < RJ; ++j) store_outs<Y>(a, row0 + wr + 16 * j + n, id[j], o + 4 * g, acc[i][j]);
  }
}

// Up to 64 rows: bound by one read of W, which goes from memory to the registers of one wavefront and no further.  A workgroup has 16 OT
// outputs, its WAVES wavefronts share the contraction.
constexpr int kFewRows = 64;
template <int RP, class Y, int OT, int RT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) rfast_lora_up_few(Up a) {
  constexpr int CHUNK = 128;
  __shared__ f32x4 part[WAVES][OT * RT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int out0 = blockIdx.x * (16 * OT);
  f32x4 acc[OT][RT];
  const u16 *w[OT], *z[RT];
#pragma unroll
  for (int o = 0; o < OT; ++o) {
    w[o] = a.w + (int64_t)min(out0 + 16 * o + n, a.outs - 1) * a.cols + g * 8;
#pragma unroll
    for (int t = 0; t < RT; ++t) acc[o][t] = f32x4{0, 0, 0, 0};
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) z[t] = a.z + (int64_t)min(16 * t + n, a.rows - 1) * a.ld_z + g * 8;
  const int whole = a.cols / CHUNK * CHUNK;
  auto chunk = [&](int c, auto load) {
    u32x4 wf[4][OT], zf[4][RT];
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int o = 0; o < OT; ++o) wf[q][o] = load(w[o], c + 32 * q);
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int t = 0; t < RT; ++t) zf[q][t] = load(z[t], c + 32 * q);
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int o = 0; o < OT; ++o)
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[o][t] = mfma(wf[q][o], zf[q][t], acc[o][t]);
  };
  for (int c = wave * CHUNK; c < whole; c += WAVES * CHUNK) chunk(c, [&](const u16* p, int at) { return load_eight(p + at); });
  if (whole < a.cols && wave == whole / CHUNK % WAVES)
    chunk(whole, [&](const u16* p, int at) { return load_eight(p + at, a.cols - at - g * 8); });
  // the adapters' part of a tile is one wavefront's, so that the tiles' go on beside each other
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int o = 0; o < OT; ++o)
      if (wave == (t * OT + o) % WAVES && out0 + 16 * o < a.outs) {
        const int row = 16 * t + n;
        Pieces<RP> u;
        u.load(a, min(row, a.rows - 1));
        acc[o][t] = add_adapters<RP>(a, u, row < a.rows ? a.ids[row] : kBehind, out0 + 16 * o, acc[o][t]);
      }
#pragma unroll
  for (int o = 0; o < OT; ++o)
#pragma unroll
    for (int t = 0; t < RT; ++t) part[wave][o * RT + t][lane] = acc[o][t];
  __syncthreads();
  for (int u = wave; u < OT * RT; u += WAVES) {
    f32x4 v = part[0][u][lane];
#pragma unroll
    for (int q = 1; q < WAVES; ++q) v += part[q][u][lane];
    const int row = 16 * (u % RT) + n;
    store_outs<Y>(a, row, row < a.rows ? a.ids[row] : kBehind, out0 + 16 * (u / RT) + 4 * g, v);
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
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int who = blockIdx.y, c0 = blockIdx.x * 128;
  f32x4 acc[8][NT];
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[j][t] = f32x4{0, 0, 0, 0};
  // A lane's first column, moved back where a tile ends with the row (what it computes twice is written twice alike).
  const bool wide = a.cols >= 8;
  const int c = wide ? min(c0 + 8 * n, a.cols - 8) : 0;
  auto block = [&](int t0, int end, auto whole) {  // 32 rows from t0 on; whole: all of them exist, and rows have eight columns
    constexpr bool WHOLE = decltype(whole)::value;
    const int r = t0 + 8 * g;
    u32x4 z[8], sf[NT][kFrags<RP>];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const u16* p = a.z + (int64_t)(r + i) * a.ld + c;
      z[i] = WHOLE ? load_eight(p) : load_eight(p, r + i < end ? min(a.cols - c, 8) : 0);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < kFrags<RP>; ++i) {
        const int k = (RP == 8 ? 16 * i : RP * i + 16 * t) + n;
        const u16* p = a.s + (int64_t)min(k, kPieces * RP - 1) * a.pitch + r;
        sf[t][i] = WHOLE ? load_eight(p) : load_eight(p, end - r);
        if (k >= kPieces * RP) sf[t][i] = u32x4{0, 0, 0, 0};
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
  };
  auto segment = [&](int s) {
    const int end = a.seg.begin(s + 1);
    for (int t0 = a.seg.begin(s) + wave * 32; t0 < end; t0 += kWaves * 32) {
      if (wide && t0 + 32 <= end) block(t0, end, std::true_type());
      else block(t0, end, std::false_type());
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
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int k = t * 16 + 4 * g + v;
        if (k >= a.rank) continue;
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
          const int at = (wide ? min(c0 + 8 * (4 * g + v), a.cols - 8) : 0) + j;
          if (at < a.cols) a.out[((int64_t)who * a.cols + at) * a.rank + k] = acc[j][t][v] * a.scale;
        }
    }
  }
}

// -------------------------------------------------------------------------------------------------------- transposes
// out [batch][cols][rows] = in [batch][rows][cols], of one adapter's matrix or both
struct Transpose {
  const u16* in;
  u16* out;
  int32_t rows, cols, tiles_x, tiles;  // tiles of 64 x 64 per matrix
};
__global__ void __launch_bounds__(kThreads) rfast_lora_transpose(Transpose a, Transpose b) {
  __shared__ u16 t[64][66];
  const bool second = (int)blockIdx.x >= a.tiles;
  const Transpose q = second ? b : a;
  const int tile = blockIdx.x - (second ? a.tiles : 0);
  const int64_t at = (int64_t)blockIdx.y * q.rows * q.cols;
  const int r0 = tile / q.tiles_x * 64, c0 = tile % q.tiles_x * 64, x = threadIdx.x & 63, high = min(64, q.rows - r0), wide = min(64, q.cols - c0);
  if (q.cols < 64) {  // (rows are shorter than a wavefront: their elements follow each other)
    for (int i = threadIdx.x; i < high * wide; i += kThreads) t[i / wide][i % wide] = q.in[at + (int64_t)r0 * q.cols + i];
  } else {
    for (int i = threadIdx.x >> 6; i < high; i += 4)
      if (x < wide) t[i][x] = q.in[at + (int64_t)(r0 + i) * q.cols + c0 + x];
  }
  __syncthreads();
  for (int i = threadIdx.x >> 6; i < wide; i += 4)
    if (x < high) q.out[at + (int64_t)(c0 + i) * q.rows + r0 + x] = t[x][i];
}

// ------------------------------------------------------------------------------------------------------------- host
int padded_rank(int rank) { return rank <= 8 ? 8 : rank <= 16 ? 16 : rank <= 32 ? 32 : 64; }

struct Layout {
  size_t ids, u_rows, u_cols, e_rows, e_cols, bt, at, total;
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
  l.total = off;
  return l;
}

bool shape_ok(const rfast_lora_shape* s) {
  if (!s || s->rows < 0 || s->segments < 1 || s->adapters < 1 || s->d < 1 || s->K < 1 || s->rank < 1 || s->rank > kMostRank) return false;
  if (s->rows > 1 << 27 || s->d > 1 << 22 || s->K > 1 << 22 || s->adapters > 65535 || s->segments == 0x7fffffff) return false;
  // a launch has fewer than 2^32 lanes
  return ((int64_t)s->rows / 128 + 1) * (std::max(s->d, s->K) / 64 + 1) < (int64_t)1 << 23;
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
  return by_rank(a.rank, [&](auto rp) {
    constexpr int RP = decltype(rp)::value;
    const auto go = [&](auto rt, auto waves, int spread) {
      constexpr int RT = decltype(rt)::value, W = decltype(waves)::value;
      hipLaunchKernelGGL((rfast_lora_down<RP, RT, W>), dim3((a.seg.rows + 16 * RT - 1) / (16 * RT), spread), dim3(64 * W), 0, st, a);
      return hipGetLastError();
    };
    using std::integral_constant;
    // with few rows the segments of 16 of them go to workgroups of their own
    if (a.seg.rows <= 1024) return go(integral_constant<int, 1>(), integral_constant<int, 8>(), std::min(16, a.seg.count));
    if (a.seg.rows <= 8192) return go(integral_constant<int, 1>(), integral_constant<int, 8>(), 1);
    return go(integral_constant<int, 2>(), integral_constant<int, 4>(), 1);
  });
}

template <int RP, class Y, int TO, int TR, int WO, int WR, bool TURNED> hipError_t launch_up_tiles(const Up& a, hipStream_t st) {
  const int row_tiles = (a.rows + TR - 1) / TR, out_tiles = (a.outs + TO - 1) / TO;
  const dim3 grid((unsigned)row_tiles * out_tiles), block(64 * WO * WR);
  const bool direct = a.ld_z % 8 == 0 && (uintptr_t)a.z % 16 == 0 && (TURNED || (a.cols % 8 == 0 && (uintptr_t)a.w % 16 == 0));
  if (direct) hipLaunchKernelGGL((rfast_lora_up<RP, Y, TO, TR, WO, WR, true, TURNED>), grid, block, 0, st, a, row_tiles, out_tiles);
  else hipLaunchKernelGGL((rfast_lora_up<RP, Y, TO, TR, WO, WR, false, TURNED>), grid, block, 0, st, a, row_tiles, out_tiles);
  return hipGetLastError();
}

// turned: w is [cols][outs]
template <class Y, bool TURNED> hipError_t launch_up(const Up& a, hipStream_t st) {
  return by_rank(a.rank, [&](auto rp) {
    constexpr int RP = decltype(rp)::value;
    if constexpr (!TURNED) {
      if (a.rows <= kFewRows) {
        const dim3 grid((unsigned)((a.outs + 15) / 16));
        if (a.rows <= 16) hipLaunchKernelGGL((rfast_lora_up_few<RP, Y, 1, 1, 8>), grid, dim3(512), 0, st, a);
        else if (a.rows <= 32) hipLaunchKernelGGL((rfast_lora_up_few<RP, Y, 1, 2, 8>), grid, dim3(512), 0, st, a);
        else hipLaunchKernelGGL((rfast_lora_up_few<RP, Y, 1, 4, 8>), grid, dim3(512), 0, st, a);
        return hipGetLastError();
      }
    }
    const int64_t large = ((int64_t)a.rows + 255) / 256 * ((a.outs + 255) / 256);
    if (large >= 192) return launch_up_tiles<RP, Y, 256, 256, 2, 4, TURNED>(a, st);
    return launch_up_tiles<RP, Y, 128, 128, 2, 2, TURNED>(a, st);
  });
}

template <bool RANK_MAJOR> hipError_t launch_sums(const Sums& a, hipStream_t st) {
  return by_rank(a.rank, [&](auto rp) {
    hipLaunchKernelGGL((rfast_lora_sums<decltype(rp)::value, RANK_MAJOR>), dim3((a.cols + 127) / 128, a.seg.adapters), dim3(kThreads), 0, st, a);
    return hipGetLastError();
  });
}

Transpose transpose_of(const u16* in, u16* out, int rows, int cols) {
  const int x = (cols + 63) / 64;
  return {in, out, rows, cols, x, x * ((rows + 63) / 64)};
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
  e = s->y_type == RFAST_F32 ? launch_up<float, false>(u, st) : launch_up<u16, false>(u, st);
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
    u16* at = (u16*)(ws + l.at);
    const Transpose tb = transpose_of((const u16*)B, bt, s->K, s->rank);
    Transpose ta = transpose_of((const u16*)A, at, s->rank, s->d);
    if (!dx) ta.tiles = 0;
    hipLaunchKernelGGL(rfast_lora_transpose, dim3(tb.tiles + ta.tiles, s->adapters), dim3(kThreads), 0, st, tb, ta);
    e = hipGetLastError();
    if (e == hipSuccess) e = launch_down({(const u16*)x, (const u16*)A, nullptr, u_cols, nullptr, seg, s->ld_x, l.pitch, s->d, s->rank, 1.f}, st);
    if (e == hipSuccess) e = launch_down({(const u16*)dy, bt, e_rows, e_cols, ids, seg, s->ld_y, l.pitch, s->K, s->rank, s->scale}, st);
    if (e == hipSuccess && dx)
      e = launch_up<u16, true>({(const u16*)dy, (const u16*)W, at, e_rows, ids, dx, s->ld_y, s->ld_x, s->rows, s->K, s->d, s->rank}, st);
  }
  if (e == hipSuccess) e = launch_sums<true>({(const u16*)x, e_cols, dA, seg, s->ld_x, l.pitch, s->d, s->rank, 1.f}, st);
  if (e == hipSuccess) e = launch_sums<false>({(const u16*)dy, u_cols, dB, seg, s->ld_y, l.pitch, s->K, s->rank, s->scale}, st);
  return e == hipSuccess ? RFAST_OK : rfast_refuse_hip(e, "adapter gradient launch");
}

}  // extern "C"
