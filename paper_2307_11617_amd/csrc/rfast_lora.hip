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
// ... of which `left` exist (any number); zeros for the others.  For rows of fewer than eight: a condition per load has it waited for before the
// next is sent, so everywhere else the loads go out without one.
__device__ inline u32x4 load_few(const u16* p, int64_t left) {
  u32x4 t = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < left) t[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
  return t;
}
// v without its first n elements (n >= 0), zeros behind the others
__device__ inline u32x4 drop_first(u32x4 v, int n) {
  const uint64_t lo = (uint64_t)v.y << 32 | v.x, hi = (uint64_t)v.w << 32 | v.z;
  const int b = 16 * n;
  const uint64_t l = b < 64 ? lo >> b | (b > 0 ? hi << (64 - b) : 0) : b < 128 ? hi >> (b - 64) : 0, h = b < 64 ? hi >> b : 0;
  return u32x4{(uint32_t)l, (uint32_t)(l >> 32), (uint32_t)h, (uint32_t)(h >> 32)};
}
// the first n elements of v (any n), zeros behind them
__device__ inline u32x4 keep_first(u32x4 v, int n) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = 2 * i + 1 < n ? v[i] : 2 * i < n ? v[i] & 0xFFFF : 0;
  return v;
}
// Eight neighbours from p on in a row of at least eight that ends at p + left, before p or behind it: the row's last eight are read and moved
// to their places, so p + left has to be the row's end whatever is wanted of it.
__device__ inline u32x4 load_eight(const u16* p, int64_t left) {
  const int there = (int)min(left, (int64_t)8);
  return drop_first(load_eight(left < 8 ? p + left - 8 : p), 8 - max(there, 0));
}
__device__ inline u32x4 load_eight(const u16* p, int64_t left, bool wide) { return wide ? load_eight(p, left) : load_few(p, left); }

// Takes chunks first, first + step, .. below end through load(chunk, operands) and use(operands), the loads of one chunk under way while
// the one before is used.  (Left to itself the compiler reuses a load's registers as soon as it can, and has a third of a chunk under way.)
template <class Operands, class Load, class Use> __device__ inline void pipelined(int first, int end, int step, Load load, Use use) {
  Operands x, y;
  if (first < end) load(first, x);
  for (int c = first; c < end; c += 2 * step) {
    if (c + step < end) load(c + step, y);
    __builtin_amdgcn_sched_barrier(0);
    use(x);
    if (c + step >= end) break;
    if (c + 2 * step < end) load(c + 2 * step, x);
    __builtin_amdgcn_sched_barrier(0);
    use(y);
  }
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
  // Blocks of R rows that no segment shares: segment s has the numbers from begin(s) / R + s on, which is enough for all of its rows before
  // those of the next one begin (and leaves some numbers without rows).  What is behind the last segment counts as one more.
  static __host__ __device__ int64_t blocks(int rows, int segments, int R) { return (int64_t)rows / R + segments + 2; }
  // The segment of block `block`: the last whose numbers do not begin behind it, found by 64 probes at a time.
  __device__ int find(int block, int R) const {
    int lo = 0, hi = count + 1;
    while (hi - lo > 1) {
      const int step = (hi - lo + 63) / 64, at = lo + (threadIdx.x & 63) * step;
      const int before = __popcll(__ballot(at < hi && begin(min(at, count)) / R + at <= block));
      lo += (before > 0 ? before - 1 : 0) * step;
      hi = min(lo + step, hi);
    }
    return lo;
  }
};

constexpr int tiles_of(int RP) { return RP < 16 ? 1 : RP / 16; }
constexpr int kPieces = 3;  // bf16 that a value of u or e is held as

// -------------------------------------------------------------------------------------------------------- transposes
// out [batch][cols][rows] = in [batch][rows][cols], up to three at once.  A wavefront turns 64 x 64 over: a lane reads eight neighbours of
// eight rows and writes eight neighbours of eight columns, turned over in registers, so that eight lanes cover a line both ways.
struct Transpose {
  const u16* in;
  u16* out;
  int32_t rows, cols, tiles_x, tiles;  // tiles of 64 x 64 per matrix
  int32_t batch;
};
struct Transposes {
  Transpose t[3];
};
__device__ inline void turn_over(const Transposes& a, int64_t tile) {
  Transpose q = a.t[0];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (tile >= (int64_t)q.tiles * q.batch) {
      tile -= (int64_t)q.tiles * q.batch;
      q = a.t[i + 1];
    }
  if (tile >= (int64_t)q.tiles * q.batch) return;
  const int lane = threadIdx.x & 63, in_matrix = (int)(tile % q.tiles);
  const int64_t at = tile / q.tiles * q.rows * q.cols;
  const int r = in_matrix / q.tiles_x * 64 + lane / 8 * 8, c = in_matrix % q.tiles_x * 64 + lane % 8 * 8;
  const u16* from = q.in + at + (int64_t)r * q.cols + c;
  u16* to = q.out + at + (int64_t)c * q.rows + r;
  u32x4 v[8];
  const bool whole = r + 8 <= q.rows && c + 8 <= q.cols;
  if (whole) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = load_eight(from + (int64_t)i * q.cols);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = load_few(from + (int64_t)i * q.cols, r + i < q.rows ? q.cols - c : 0);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    any_u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_perm(v[2 * i + 1][j >> 1], v[2 * i][j >> 1], j & 1 ? 0x07060302 : 0x05040100);
    if (whole) {
      *reinterpret_cast<any_u32x4*>(to + (int64_t)j * q.rows) = w;
    } else if (c + j < q.cols) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r + i < q.rows) to[(int64_t)j * q.rows + i] = (u16)(w[i >> 1] >> (16 * (i & 1)));
    }
  }
}

// ------------------------------------------------------------------------------------------------------------- down
// out = scale * (rows of z) x (adapter's matrix m [rank][cols]) in kPieces bf16:
//   out_rows [rows][kPieces][RP]    what `up` reads
//   out_cols [kPieces][RP][pitch]   what `sums` reads: the same by columns
// A workgroup has up to 16 RT rows of one segment, its WAVES wavefronts share the contraction.  Rows and ranks that do not exist are read as
// the nearest that do, and what comes of them is left out.
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
  int32_t blocks;  // workgroups (in x) for rows; those behind them turn matrices over that the next launch needs
  Transposes turn;
};

template <int RP, int RT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) rfast_lora_down(Down a) {
  constexpr int NT = tiles_of(RP), CHUNK = 128;
  __shared__ f32x4 part[WAVES][RT * NT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  if ((int)blockIdx.x >= a.blocks) {
    turn_over(a.turn, (int64_t)((int)blockIdx.x - a.blocks) * WAVES + wave);
    return;
  }
  constexpr int R = 16 * RT;
  const int s = a.seg.find(blockIdx.x, R), begin = a.seg.begin(s), stop = s < a.seg.count ? a.seg.begin(s + 1) : a.seg.rows;
  const int row0 = begin + ((int)blockIdx.x - s - begin / R) * R;
  if (row0 < begin || row0 >= stop) return;
  const int r1 = min(row0 + R, stop), id = s < a.seg.count ? a.seg.adapter_of(s) : kBehind;
  if (a.ids && threadIdx.x < r1 - row0) a.ids[row0 + threadIdx.x] = id;
  if (id == kBehind) return;
  f32x4 acc[RT][NT];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[i][t] = f32x4{0, 0, 0, 0};
  if (id >= 0) {
    const u16 *z[RT], *m[NT];
#pragma unroll
    for (int i = 0; i < RT; ++i) z[i] = a.z + (int64_t)min(row0 + 16 * i + n, r1 - 1) * a.ld + g * 8;
#pragma unroll
    for (int t = 0; t < NT; ++t) m[t] = a.m + ((int64_t)id * a.rank + min(t * 16 + n, a.rank - 1)) * a.cols + g * 8;
    const int whole = a.cols / CHUNK * CHUNK;
    struct Operands {
      u32x4 z[4][RT], m[4][NT];
    };
    auto fetch = [&](int c, Operands& o, auto load) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
#pragma unroll
        for (int i = 0; i < RT; ++i) o.z[q][i] = load(z[i], c + 32 * q);
#pragma unroll
        for (int t = 0; t < NT; ++t) o.m[q][t] = load(m[t], c + 32 * q);
      }
    };
    auto use = [&](const Operands& o) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int t = 0; t < NT; ++t) acc[i][t] = mfma(o.z[q][i], o.m[q][t], acc[i][t]);
    };
    // (several workgroups are on a compute unit: what waits in one, another does, and a chunk ahead in registers is none the faster)
    for (int c = wave * CHUNK; c < whole; c += WAVES * CHUNK) {
      Operands o;
      fetch(c, o, [&](const u16* p, int at) { return load_eight(p + at); });
      __builtin_amdgcn_sched_barrier(0);
      use(o);
    }
    if (whole < a.cols && wave == whole / CHUNK % WAVES) {
      Operands o;
      if (a.cols >= 8) fetch(whole, o, [&](const u16* p, int at) { return load_eight(p + at, a.cols - at - g * 8); });
      else fetch(whole, o, [&](const u16* p, int at) { return load_few(p + at, a.cols - at - g * 8); });
      use(o);
    }
  }
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
      if (k >= RP || row >= r1) continue;
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
  int32_t rows, cols, outs, rank, adapters;
  // rfast_lora_up with FUSED: u is formed there, from the first factors
  const u16* m;  // [adapters][rank][cols]
  Segments seg;
  float scale;
  float* partials;  // [splits][rows][pitch_of(outs)], where the contraction is split over workgroups
  // (where row numbers are out of order a row's may never have been written)
  __device__ int id(int row) const {
    const int i = row < rows ? ids[row] : kBehind;
    return i < adapters ? i : kNone;
  }
};

int64_t __host__ __device__ pitch_of(int outs) { return ((int64_t)outs + 3) / 4 * 4; }

// Where chunk c of row o of a matrix of CH chunks a row is put in LDS: at c ^ swizzle.
template <int CH> __device__ inline int swizzle(int o) { return CH == 4 ? o >> 1 & 3 : CH == 8 ? o & 7 : CH == 2 ? o >> 2 & 1 : 0; }

template <int RP> struct Pieces {  // of u for 16 rows, as B operand
  static constexpr int WIDE = kPieces * RP, STEPS = (WIDE + 31) / 32;
  u32x4 f[STEPS];
  __device__ void load(const u16* pieces, int row) {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int q = 0; q < STEPS; ++q) {
      const int k = 32 * q + 8 * g;
      f[q] = load_eight(pieces + (int64_t)row * WIDE + min(k, WIDE - 8));
      if (k >= WIDE) f[q] = u32x4{0, 0, 0, 0};
    }
  }
  __device__ void load(const Up& a, int row) { load(a.u, row); }
};
template <int RP> struct Factor {  // b of adapter `who` for 16 outputs from out0 on, as A operand
  static constexpr int WIDE = kPieces * RP, STEPS = (WIDE + 31) / 32;
  u32x4 f[STEPS];
  __device__ void load(const Up& a, int who, int out0) {
    const int lane = threadIdx.x & 63, out = min(out0 + (lane & 15), a.outs - 1);
    const u16* b = a.b + ((int64_t)who * a.outs + out) * a.rank;
#pragma unroll
    for (int q = 0; q < STEPS; ++q) {
      const int k = 32 * q + 8 * (lane >> 4), at = k % RP;  // (where k is past the pieces, what it would repeat is read and dropped)
      f[q] = a.rank == RP ? load_eight(b + at) : load_eight(b + at, a.rank - at, a.rank >= 8);
      if (k >= WIDE) f[q] = u32x4{0, 0, 0, 0};
    }
  }
};

// The adapters' part for 16 rows (their pieces u, their adapters id: lane n has row n's) and 16 outputs from out0 on, as far as it is
// wavefront `share` of SHARES'; four adapters' factors are under way at a time.  A column of the result is one row's, so that the others of a step are
// left out there and nothing of an adapter (an infinity, say) reaches rows that have another.
template <int RP, int SHARES> __device__ inline f32x4 add_adapters(const Up& a, const Pieces<RP>& u, int id, int out0, int share, f32x4 acc) {
  uint64_t pending = __ballot(id >= 0) & 0xFFFF;
  for (int turn = 0; pending;) {
    int who[4], found = 0;
    for (; pending && found < 4; ++turn) {
      const int w = __builtin_amdgcn_readlane(id, __builtin_ctzll(pending));
      pending &= ~__ballot(id == w);
      if (turn % SHARES != share) continue;
      if (found == 0) who[0] = who[1] = who[2] = who[3] = w;
      else if (found == 1) who[1] = w;
      else if (found == 2) who[2] = w;
      else who[3] = w;
      ++found;
    }
    if (!found) break;
    Factor<RP> b[4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (q < found) b[q].load(a, who[q], out0);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (q >= found) break;
      f32x4 own = {0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < Factor<RP>::STEPS; ++s) own = mfma(b[q].f[s], u.f[s], own);
      if (id == who[q]) acc += own;
    }
  }
  return acc;
}

// Four outputs from `out` on of one row
template <class Y> __device__ inline void store_outs(const Up& a, int row, int id, int out, f32x4 v) {
  if (row >= a.rows || out >= a.outs || id == kBehind) return;
  const float f[4] = {v.x, v.y, v.z, v.w};
  store_four<false>((Y*)a.y + (int64_t)row * a.ld_y + out, a.outs - out, f);
}

// Many rows: a workgroup's tile of TO outputs x TR rows, shared by WO x WR wavefronts, both operands staged in LDS, kStep contraction indices
// at a time, kStages of them in turn.  A row of a stage is four chunks of 16 bytes; chunk c is put at place c ^ row / 2 % 4, so that the
// 16 rows of an operand fall on all banks.
// What bounds it is how far ahead the stages are sent for: with two buffers of 64 indices (the next one under way while one is
// multiplied) the matrix cores were busy for 38 % of the time; 54 % as it is (8001 x 4096 x 4096).  So stage s + 4 is sent for when the operands of stage s are in
// registers, and the operands of stage s + 1 are read from LDS while those of stage s are multiplied; one barrier per stage says both that stage s + 1
// has arrived and that nobody reads stage s any more.  A contraction that is no multiple of kStep begins with what is over.
// DIRECT: rows begin at multiples of 16 bytes, and stages go from memory to LDS without passing through registers (a wavefront's load
// fills 1 KB, sixteen rows, in the order of its lanes, so each lane fetches the chunk that belongs to its place).  Else they go through
// registers, one stage ahead.
// FUSED: few outputs (one tile of them), so that the pass of `down` over the rows would cost as much as this one.  A workgroup has rows of one
// segment only, the first factors of its adapter are some more rows of w, and what they come to is handed on through LDS: 32768 rows of 128 nodes, 1024 x
// 128, rank 8: 21 + 22 us in two passes, 32 so.
// SPLIT: few tiles, so that their stages one after the other would be all there is to wait for: workgroups (in y) share the contraction and
// write what they have; rfast_lora_join adds it up, and the adapters' part.
constexpr int kStep = 32, kStages = 4;
enum Mode { kWhole, kFused, kSplit };

template <int RP, class Y, int TO, int TR, int WO, int WR, bool DIRECT, Mode MODE>
__global__ void __launch_bounds__(64 * WO * WR) rfast_lora_up(Up a, int row_tiles, int out_tiles) {
  constexpr bool FUSED = MODE == kFused;
  constexpr int WAVES = WO * WR, OI = TO / WO / 16, RJ = TR / WR / 16;
  constexpr int UT = FUSED ? tiles_of(RP) : 0, UJ = RJ / WO;                    // blocks of ranks; blocks of rows whose u a wavefront forms
  constexpr int WL = TO / 16 / WAVES, ZL = TR / 16 / WAVES, L = WL + ZL + UT;  // loads per lane and stage, of 16 bytes (of u: 4)
  static_assert(WL * 16 * WAVES == TO && ZL * 16 * WAVES == TR, "every wavefront fetches the same number of rows");
  static_assert(!FUSED || (DIRECT && WAVES == 4 && RJ % WO == 0 && TR * kPieces * RP * 2 <= kStages * TR * 64), "fused");
  __shared__ u32x4 w_tile[kStages][TO * 4], z_tile[kStages][TR * 4], m_tile[FUSED ? kStages : 1][FUSED ? UT * 64 : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  int row0, out0, rows_end, own = kNone;
  if (FUSED) {
    const int q = a.seg.find(blockIdx.x, TR), begin = a.seg.begin(q), stop = q < a.seg.count ? a.seg.begin(q + 1) : begin;
    row0 = begin + ((int)blockIdx.x - q - begin / TR) * TR;
    if (row0 < begin || row0 >= stop) return;
    rows_end = min(row0 + TR, stop);
    out0 = 0;
    own = a.seg.adapter_of(q);
  } else {
    // Workgroups are dealt to the eight XCDs by turns: one XCD gets consecutive tiles, which share rows and outputs in its L2.
    const int tiles = row_tiles * out_tiles;
    int t = blockIdx.x;
    if (tiles % 8 == 0) t = t % 8 * (tiles / 8) + t / 8;
    // bands of eight tiles of rows, within a band output by output
    const int band = t / (8 * out_tiles), in_band = t - band * 8 * out_tiles, high = min(8, row_tiles - 8 * band);
    row0 = (band * 8 + in_band % high) * TR;
    out0 = in_band / high * TO;
    rows_end = a.rows;
  }
  const int wo = wave / WR * (TO / WO), wr = wave % WR * (TR / WR);

  f32x4 acc[OI][RJ];
#pragma unroll
  for (int i = 0; i < OI; ++i)
#pragma unroll
    for (int j = 0; j < RJ; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

  // this lane's place of a load: row lane / 4 of sixteen, and the chunk that goes there; rows that do not exist are the last one
  const int lr = lane >> 2, lc = ((lane & 3) ^ (lr >> 1 & 3)) * 8;
  const char* z0 = (const char*)(a.z + (int64_t)row0 * a.ld_z);
  const char* w0 = (const char*)(a.w + (int64_t)out0 * a.cols);
  uint32_t zo[ZL], wofs[WL];  // bytes behind these (the launcher sees to it that they fit)
#pragma unroll
  for (int q = 0; q < ZL; ++q) zo[q] = (uint32_t)(min((q * WAVES + wave) * 16 + lr, rows_end - 1 - row0) * (uint32_t)a.ld_z + lc) * 2;
#pragma unroll
  for (int q = 0; q < WL; ++q) wofs[q] = (uint32_t)(min((q * WAVES + wave) * 16 + lr, a.outs - 1 - out0) * (uint32_t)a.cols + lc) * 2;
  auto send = [&](u32x4* to, const char* from) {
    __builtin_amdgcn_global_load_lds((const RFAST_GLOBAL void*)(uintptr_t)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
  };
  // of 16 ranks a wavefront fetches four, four bytes per lane
  const char* m0 = nullptr;
  uint32_t mo[FUSED ? UT : 1];
  if (FUSED) {
    m0 = (const char*)(a.m + (int64_t)max(own, 0) * a.rank * a.cols);
#pragma unroll
    for (int q = 0; q < UT; ++q) {
      const int k = 4 * wave + (lane >> 4), chunk = (lane >> 2 & 3) ^ (k >> 1 & 3);
      mo[q] = (uint32_t)min(16 * q + k, a.rank - 1) * (uint32_t)a.cols * 2 + chunk * 16 + (lane & 3) * 4;
    }
  }
  const int all_stages = (a.cols + kStep - 1) / kStep, splits = MODE == kSplit ? gridDim.y : 1, split = MODE == kSplit ? blockIdx.y : 0;
  const int first = all_stages * split / splits, stages = all_stages * (split + 1) / splits - first;  // stage s here is first + s of all
  const int all_over = a.cols % kStep, over = first == 0 ? all_over : 0;                              // (the first of all takes what is over)
  auto begin = [&](int s) { return all_over ? (first + s == 0 ? a.cols - all_over : (first + s - 1) * kStep) : (first + s) * kStep; };
  auto fetch = [&](int s) {
    const int64_t c = (int64_t)begin(s) * 2;
#pragma unroll
    for (int q = 0; q < ZL; ++q) send(&z_tile[s % kStages][(q * WAVES + wave) * 64], z0 + c + zo[q]);
#pragma unroll
    for (int q = 0; q < WL; ++q) send(&w_tile[s % kStages][(q * WAVES + wave) * 64], w0 + c + wofs[q]);
#pragma unroll
    for (int q = 0; q < UT; ++q)
      __builtin_amdgcn_global_load_lds((const RFAST_GLOBAL void*)(uintptr_t)(m0 + c + mo[q]),
                                       (__attribute__((address_space(3))) void*)&m_tile[s % kStages][q * 64 + wave * 16], 4, 0, 0);
  };
  u32x4 zr[ZL], wg[WL], mg[FUSED ? UT : 1];
  auto take = [&](int s) {
    const int64_t c = (int64_t)begin(s) * 2;
    if (s > 0 || !over) {
#pragma unroll
      for (int q = 0; q < ZL; ++q) zr[q] = load_eight((const u16*)(z0 + c + zo[q]));
#pragma unroll
      for (int q = 0; q < WL; ++q) wg[q] = load_eight((const u16*)(w0 + c + wofs[q]));
    } else {
#pragma unroll
      for (int q = 0; q < ZL; ++q) zr[q] = load_eight((const u16*)(z0 + c + zo[q]), over - lc, a.cols >= 8);
#pragma unroll
      for (int q = 0; q < WL; ++q) wg[q] = load_eight((const u16*)(w0 + c + wofs[q]), over - lc, a.cols >= 8);
#pragma unroll
      for (int q = 0; q < UT; ++q)  // (every wavefront fetches and puts all sixteen ranks of a block here)
        mg[q] = load_eight((const u16*)(m0 + c) + (int64_t)min(16 * q + lr, a.rank - 1) * a.cols + lc, over - lc, a.cols >= 8);
    }
  };
  auto put = [&](int s) {
#pragma unroll
    for (int q = 0; q < ZL; ++q) z_tile[s % kStages][(q * WAVES + wave) * 64 + lane] = zr[q];
#pragma unroll
    for (int q = 0; q < WL; ++q) w_tile[s % kStages][(q * WAVES + wave) * 64 + lane] = wg[q];
#pragma unroll
    for (int q = 0; q < UT; ++q) m_tile[s % kStages][q * 64 + lane] = mg[q];
  };
  // Stage s + 1 has arrived, for all wavefronts (stages s + 2 and s + 3 may be under way; loads return in order), and what was read
  // from LDS or written there before is done.
  auto meet = [&](int s) {
    if (!DIRECT) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else if (s + 3 < stages) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * L) : "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  };
  const int place = g ^ (n >> 1 & 3);
  auto z_of = [&](int s, int j) { return z_tile[s % kStages][(wr + 16 * j + n) * 4 + place]; };
  auto w_of = [&](int s, int i) { return w_tile[s % kStages][(wo + 16 * i + n) * 4 + place]; };
  struct Operands {
    u32x4 w[OI], z[RJ], m[FUSED ? UT : 1];
  } x, y;
  auto m_of = [&](int s, int t) { return m_tile[s % kStages][(16 * t + n) * 4 + place]; };
  const int first_j = FUSED ? wave / WR * UJ : 0;  // the blocks of rows whose u this wavefront forms
  f32x4 form[FUSED ? UT : 1][UJ];
#pragma unroll
  for (int t = 0; t < UT; ++t)
#pragma unroll
    for (int j = 0; j < UJ; ++j) form[t][j] = f32x4{0, 0, 0, 0};
  // (what is read ahead of the last stage is whatever is there, and not used)
  auto stage = [&](int s, const Operands& now, Operands& next) {
    meet(s);
    if (DIRECT) {
      if (s + kStages < stages) fetch(s + kStages);
    } else {
      if (s + 2 < stages) put(s + 2);
      if (s + 3 < stages) take(s + 3);
    }
#pragma unroll
    for (int j = 0; j < RJ; ++j) next.z[j] = z_of(s + 1, j);
#pragma unroll
    for (int i = 0; i < OI; ++i) next.w[i] = w_of(s + 1, i);
#pragma unroll
    for (int t = 0; t < UT; ++t) next.m[t] = m_of(s + 1, t);
#pragma unroll
    for (int i = 0; i < OI; ++i)
#pragma unroll
      for (int j = 0; j < RJ; ++j) acc[i][j] = mfma(now.w[i], now.z[j], acc[i][j]);
#pragma unroll
    for (int t = 0; t < UT; ++t)
#pragma unroll
      for (int j = 0; j < UJ; ++j) form[t][j] = mfma(now.m[t], first_j == 0 ? now.z[j] : now.z[UJ + j], form[t][j]);
    // reads and products by turns, so that the reads are through before the products are
#pragma unroll
    for (int i = 0; i < OI + RJ; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, OI * RJ / (OI + RJ + 2), 0);
    }
  };
  if (DIRECT) {
    if (over) {
      take(0);
      put(0);
    } else {
      fetch(0);
    }
    for (int s = 1; s < kStages; ++s)
      if (s < stages) fetch(s);
  } else {
    take(0);
    put(0);
    if (stages > 1) {
      take(1);
      put(1);
    }
    if (stages > 2) take(2);
  }
  meet(-1);
#pragma unroll
  for (int j = 0; j < RJ; ++j) x.z[j] = z_of(0, j);
#pragma unroll
  for (int i = 0; i < OI; ++i) x.w[i] = w_of(0, i);
#pragma unroll
  for (int t = 0; t < UT; ++t) x.m[t] = m_of(0, t);
  int s = 0;
  for (; s + 1 < stages; s += 2) {
    stage(s, x, y);
    stage(s + 1, y, x);
  }
  if (s < stages) stage(s, x, y);
  if constexpr (MODE == kSplit) {
#pragma unroll
    for (int i = 0; i < OI; ++i)
#pragma unroll
      for (int j = 0; j < RJ; ++j) {
        const int row = row0 + wr + 16 * j + n, out = out0 + wo + 16 * i + 4 * g;
        if (row < a.rows && out < a.outs) *reinterpret_cast<f32x4*>(a.partials + ((int64_t)split * a.rows + row) * pitch_of(a.outs) + out) = acc[i][j];
      }
    return;
  }

  // The adapters' part, one run of rows with the same adapter after the other: its factors for the tile's outputs come through LDS (those of
  // the next run are under way meanwhile), and every wavefront that has rows of the run takes them up.  A column of a product is one
  // row's, so that the others are left out there and nothing of an adapter (an infinity, say) reaches rows that have another.
  // (Every wavefront fetching the factors of its own outputs from memory took 100 us of 340 for 8001 x 4096 x 4096, rank 32.)
  constexpr int CH = RP / 8, MINE = (TO * CH + 64 * WAVES - 1) / (64 * WAVES);  // chunks of an output's factors; chunks of a lane
  u32x4* factors = &w_tile[0][0];                                              // [TO][CH]
  int* tile_ids = (int*)&z_tile[0][0];                                         // [TR]
  static_assert(TO * CH <= kStages * TO * 4, "the factors fit the stages they take the place of");
  int id[RJ];
#pragma unroll
  for (int j = 0; j < RJ; ++j) {
    const int row = row0 + wr + 16 * j + n;
    id[j] = !FUSED ? a.id(row) : row < rows_end ? own : kBehind;
  }
  Pieces<RP> u[RJ];
  if (RP <= 32 && !FUSED) {
#pragma unroll
    for (int j = 0; j < RJ; ++j) u[j].load(a, min(row0 + wr + 16 * j + n, a.rows - 1));
  }
  __syncthreads();  // nobody reads the stages any more
  if (FUSED) {
    u16* pieces = (u16*)&z_tile[0][0];  // [TR][kPieces][RP]
#pragma unroll
    for (int t = 0; t < UT; ++t)
#pragma unroll
      for (int j = 0; j < UJ; ++j)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int k = 16 * t + 4 * g + v;
          float f = k < a.rank ? form[t][j][v] * a.scale : 0.f;
#pragma unroll
          for (int i = 0; i < kPieces; ++i) {
            const u16 piece = to_bf16(f);
            f -= from_bf16(piece);
            if (!(fabsf(f) < INFINITY)) f = 0.f;
            if (k < RP) pieces[((wr + 16 * (first_j + j) + n) * kPieces + i) * RP + k] = piece;
          }
        }
  } else {
    for (int r = threadIdx.x; r < TR; r += 64 * WAVES) tile_ids[r] = a.id(row0 + r);
  }
  __syncthreads();
  if (FUSED) {
#pragma unroll
    for (int j = 0; j < RJ; ++j) u[j].load((const u16*)&z_tile[0][0], wr + 16 * j + n);
  }
  auto run_end = [&](int r) {  // where the run that begins at r ends
    if (FUSED) return TR;
    const int who = tile_ids[r];
    for (int q = r; q < TR; q += 64) {
      const uint64_t other = __ballot(q + lane < TR && tile_ids[min(q + lane, TR - 1)] != who);
      if (other) return q + __builtin_ctzll(other);
    }
    return TR;
  };
  u32x4 mine[MINE];
  auto take_factors = [&](int who) {
#pragma unroll
    for (int q = 0; q < MINE; ++q) {
      const int c = q * 64 * WAVES + threadIdx.x, out = min(out0 + c / CH, a.outs - 1), k = c % CH * 8;
      const u16* b = a.b + ((int64_t)who * a.outs + out) * a.rank + k;
      mine[q] = a.rank == RP ? load_eight(b) : load_eight(b, a.rank - k, a.rank >= 8);
    }
  };
  int r = 0, who = FUSED ? own : tile_ids[0], stop = run_end(0);
  if (who >= 0) take_factors(who);
  while (r < TR) {
    if (who >= 0) {
#pragma unroll
      for (int q = 0; q < MINE; ++q) {
        const int c = q * 64 * WAVES + threadIdx.x, o = c / CH;
        if (c < TO * CH) factors[o * CH + (c % CH ^ swizzle<CH>(o))] = mine[q];
      }
    }
    const int next = stop < TR ? tile_ids[stop] : kNone, next_stop = stop < TR ? run_end(stop) : TR;
    __syncthreads();
    if (next >= 0) take_factors(next);
    if (who >= 0 && r < wr + 16 * RJ && stop > wr) {
#pragma unroll
      for (int j = 0; j < RJ; ++j) {
        const int first = wr + 16 * j;
        if (r >= first + 16 || stop <= first) continue;
        if (RP > 32 && !FUSED) u[j].load(a, min(row0 + first + n, a.rows - 1));
        const bool in = first + n >= r && first + n < stop;
#pragma unroll
        for (int i = 0; i < OI; ++i) {
          f32x4 own = {0, 0, 0, 0};
#pragma unroll
          for (int q = 0; q < Pieces<RP>::STEPS; ++q) {
            const int o = wo + 16 * i + n, k = (32 * q + 8 * g) % RP / 8;
            own = mfma(factors[o * CH + (k ^ swizzle<CH>(o))], u[j].f[q], own);
          }
          if (in) acc[i][j] += own;
        }
      }
    }
    __syncthreads();
    r = stop;
    who = next;
    stop = next_stop;
  }
#pragma unroll
  for (int i = 0; i < OI; ++i)
#pragma unroll
    for (int j = 0; j < RJ; ++j) store_outs<Y>(a, row0 + wr + 16 * j + n, id[j], out0 + wo + 16 * i + 4 * g, acc[i][j]);
}

// y = the sum of the partial products + the adapters' part.  A wavefront has 16 rows and 16 outputs.
template <int RP, class Y> __global__ void __launch_bounds__(kThreads) rfast_lora_join(Up a, int splits) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int out0 = (blockIdx.x * kWaves + wave) * 16, row = blockIdx.y * 16 + n;
  if (out0 >= a.outs) return;
  const int id = a.id(row), out = min(out0 + 4 * g, (int)pitch_of(a.outs) - 4);
  Pieces<RP> u;
  u.load(a, min(row, a.rows - 1));
  const float* p = a.partials + min(row, a.rows - 1) * pitch_of(a.outs) + out;
  f32x4 acc = {0, 0, 0, 0};
#pragma unroll 4
  for (int q = 0; q < splits; ++q) acc += *reinterpret_cast<const f32x4*>(p + q * a.rows * pitch_of(a.outs));
  acc = add_adapters<RP, 1>(a, u, id, out0, 0, acc);
  store_outs<Y>(a, row, id, out0 + 4 * g, acc);
}

// Up to 64 rows: bound by one read of W, which goes from memory to the registers of one wavefront and no further.  A workgroup has 16 OT
// outputs, its WAVES wavefronts share the contraction.
template <int RP, class Y, int OT, int RT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) rfast_lora_up_few(Up a) {
  constexpr int Q = 4, CHUNK = 32 * Q;
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
  struct Operands {
    u32x4 w[Q][OT], z[Q][RT];
  };
  auto fetch = [&](int c, Operands& f, auto load) {
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int o = 0; o < OT; ++o) f.w[q][o] = load(w[o], c + 32 * q);
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int t = 0; t < RT; ++t) f.z[q][t] = load(z[t], c + 32 * q);
  };
  auto use = [&](const Operands& f) {
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int o = 0; o < OT; ++o)
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[o][t] = mfma(f.w[q][o], f.z[q][t], acc[o][t]);
  };
  pipelined<Operands>(wave * CHUNK, whole, WAVES * CHUNK, [&](int c, Operands& f) { fetch(c, f, [&](const u16* p, int at) { return load_eight(p + at); }); }, use);
  if (whole < a.cols && wave == whole / CHUNK % WAVES) {
    Operands f;
    if (a.cols >= 8) fetch(whole, f, [&](const u16* p, int at) { return load_eight(p + at, a.cols - at - g * 8); });
    else fetch(whole, f, [&](const u16* p, int at) { return load_few(p + at, a.cols - at - g * 8); });
    use(f);
  }
  // (the adapters of a tile are dealt to the wavefronts)
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int row = 16 * t + n, id = a.id(row);
    Pieces<RP> u;
    u.load(a, min(row, a.rows - 1));
#pragma unroll
    for (int o = 0; o < OT; ++o)
      if (out0 + 16 * o < a.outs) acc[o][t] = add_adapters<RP, WAVES>(a, u, id, out0 + 16 * o, (wave + t) % WAVES, acc[o][t]);
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
    store_outs<Y>(a, row, a.id(row), out0 + 16 * (u / RT) + 4 * g, v);
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

template <int RP, bool RANK_MAJOR, int WAVES>
__device__ inline void sums_of(const Sums& a, int tile, f32x4 (*part)[8][tiles_of(RP)][64]) {
  constexpr int NT = tiles_of(RP);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int who = blockIdx.y, c0 = tile * 128;
  f32x4 acc[8][NT];
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[j][t] = f32x4{0, 0, 0, 0};
  // A lane's first column, moved back where a tile ends with the row (what it computes twice is written twice alike).
  const bool wide = a.cols >= 8;
  const int c = wide ? min(c0 + 8 * n, a.cols - 8) : 0;
  struct Operands {
    u32x4 z[8], s[NT][kFrags<RP>];
  };
  auto fetch = [&](int t0, int end, Operands& o, auto whole) {  // 32 rows from t0 on; whole: all of them exist, and rows have eight columns
    constexpr bool WHOLE = decltype(whole)::value;
    const int r = t0 + 8 * g, from = WHOLE ? r : min((int64_t)r, a.pitch - 8);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const u16* p = a.z + (int64_t)(WHOLE ? r + i : min(r + i, end - 1)) * a.ld + c;
      o.z[i] = wide ? load_eight(p) : load_few(p, a.cols - c);
      if (!WHOLE && r + i >= end) o.z[i] = u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < kFrags<RP>; ++i) {
        const int k = (RP == 8 ? 16 * i : RP * i + 16 * t) + n;
        o.s[t][i] = load_eight(a.s + (int64_t)min(k, kPieces * RP - 1) * a.pitch + from);
        if (!WHOLE) o.s[t][i] = keep_first(drop_first(o.s[t][i], r - from), end - r);
      }
  };
  auto use = [&](const Operands& o) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      u32x4 zf;
#pragma unroll
      for (int q = 0; q < 4; ++q) zf[q] = __builtin_amdgcn_perm(o.z[2 * q + 1][j >> 1], o.z[2 * q][j >> 1], j & 1 ? 0x07060302 : 0x05040100);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < kFrags<RP>; ++i) {
          u32x4 sf = o.s[t][i];
          if (RP == 8 && i == 1 && n >= 8) sf = u32x4{0, 0, 0, 0};  // (the third piece has no neighbour)
          acc[j][t] = RANK_MAJOR ? mfma(sf, zf, acc[j][t]) : mfma(zf, sf, acc[j][t]);
        }
    }
  };
  bool shared = false;  // more than the first wavefront have a part
  auto segment = [&](int s) {
    const int begin = a.seg.begin(s), end = a.seg.begin(s + 1);
    shared |= end - begin > 32;
    const int whole = wide && end > begin ? begin + (end - begin) / 32 * 32 : begin;
    pipelined<Operands>(begin + wave * 32, whole, WAVES * 32, [&](int t0, Operands& o) { fetch(t0, end, o, std::true_type()); }, use);
    for (int t0 = whole; t0 < end; t0 += 32)
      if (wave == (t0 - begin) / 32 % WAVES) {
        Operands o;
        fetch(t0, end, o, std::false_type());
        use(o);
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
  if (!shared && wave != 0) return;
#pragma unroll
  for (int half = WAVES / 2; half >= 1 && shared; half >>= 1) {
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

// dA and dB in one launch: the first `tiles_a` tiles of columns are dA's
template <int RP, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) rfast_lora_sums(Sums a, Sums b, int tiles_a) {
  __shared__ f32x4 part[WAVES / 2][8][tiles_of(RP)][64];
  if ((int)blockIdx.x < tiles_a) sums_of<RP, true, WAVES>(a, blockIdx.x, part);
  else sums_of<RP, false, WAVES>(b, blockIdx.x - tiles_a, part);
}

// ------------------------------------------------------------------------------------------------------------- host
int padded_rank(int rank) { return rank <= 8 ? 8 : rank <= 16 ? 16 : rank <= 32 ? 32 : 64; }

// Workgroups that share the contraction of one tile of 128 x 128, where there are fewer tiles than compute units: a stage of 32 takes a
// lone workgroup 0.45 us.  4096 x 4096, rank 16, whole and split: 128 rows 73 and 31 us, 512 rows 72 and 48; 8192 x 512, 1024 rows 130 and
// 44; 1024 x 1024, 300 rows 29 and 19.
constexpr int kFewRows = 64;
int splits_of(int64_t rows, int64_t outs, int64_t cols) {
  const int64_t tiles = (rows + 127) / 128 * ((outs + 127) / 128), stages = (cols + kStep - 1) / kStep;
  if (rows <= kFewRows || tiles > 128) return 0;
  return (int)std::max<int64_t>(1, std::min({256 / tiles, stages / 8, (int64_t)16}));
}
// Where rows over a multiple of 256 would have the card do one more round of tiles that are mostly empty, they are a launch of their own:
// 4100 rows, 4096 x 4096, 202 us in 17 x 16 tiles, 125 + 9 so.
int whole_rows(int64_t rows, int64_t outs) {
  const int64_t columns = (outs + 255) / 256, units = 256, whole = rows / 256 * 256;
  return (int)(whole > 0 && (whole / 256 * columns + units - 1) / units < ((rows + 255) / 256 * columns + units - 1) / units ? whole : rows);
}
// What the partial products of `rows` rows, or of any fewer, take at most: a workspace for many rows does for few.  (Tiles of rows times splits
// are at most 256 / tiles of outputs, as splits_of divides them.)
size_t partials_bytes(int64_t rows, int64_t outs, int64_t cols) {
  const int64_t columns = (outs + 127) / 128, most = std::max<int64_t>(1, std::min<int64_t>(16, (cols + kStep - 1) / kStep / 8));
  if (rows <= kFewRows || columns > 128) return 0;
  return (size_t)(128 * std::min(256 / columns, (rows + 127) / 128 * most) * pitch_of((int)outs) * 4);
}

struct Layout {
  size_t ids, u_rows, u_cols, e_rows, e_cols, bt, at, wt, partials, total;
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
  l.partials = take(pass == 0 ? partials_bytes(s.rows, s.K, s.d) : pass == 2 ? partials_bytes(s.rows, s.d, s.K) : 0);
  l.total = off;
  return l;
}

bool shape_ok(const rfast_lora_shape* s) {
  if (!s || s->rows < 0 || s->segments < 1 || s->adapters < 1 || s->d < 1 || s->K < 1 || s->rank < 1 || s->rank > kMostRank) return false;
  if (s->segments > 1 << 22 || s->rows > 1 << 26 || s->ld_x > 1 << 22 || s->ld_y > 1 << 22 || s->d > 1 << 22 || s->K > 1 << 22 || s->adapters > 65535) return false;
  // a launch has fewer than 2^32 lanes, also one that turns the matrices over: 64 for each of their tiles beside 512 for a block of rows, of which
  // there are up to 66 more than segments (with more than 1024 rows 256 lanes, of up to 2^22 + 2^21 + 2)
  const int64_t tiles = (int64_t)s->adapters * ((s->K + 63) / 64 + (s->d + 63) / 64) + (int64_t)((s->K + 63) / 64) * ((s->d + 63) / 64);
  if (tiles >= (int64_t)1 << 25 || tiles + 8 * ((int64_t)s->segments + 67) >= (int64_t)1 << 26) return false;
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

Transpose transpose_of(const void* in, void* out, int rows, int cols, int batch) {
  const int x = (cols + 63) / 64;
  return {(const u16*)in, (u16*)out, rows, cols, x, x * ((rows + 63) / 64), batch};
}
int64_t tiles_of(const Transpose& t) { return (int64_t)t.tiles * t.batch; }

hipError_t launch_down(const Down& a, hipStream_t st) {
  return by_rank(a.rank, [&](auto rp) {
    constexpr int RP = decltype(rp)::value;
    const auto go = [&](auto rt, auto waves) {
      constexpr int RT = decltype(rt)::value, W = decltype(waves)::value;
      Down b = a;
      b.blocks = (int32_t)Segments::blocks(a.seg.rows, a.seg.count, 16 * RT);
      const int64_t tiles = tiles_of(a.turn.t[0]) + tiles_of(a.turn.t[1]) + tiles_of(a.turn.t[2]);
      hipLaunchKernelGGL((rfast_lora_down<RP, RT, W>), dim3((unsigned)(b.blocks + (tiles + W - 1) / W)), dim3(64 * W), 0, st, b);
      return hipGetLastError();
    };
    using std::integral_constant;
    if (a.seg.rows <= 1024) return go(integral_constant<int, 1>(), integral_constant<int, 8>());
    return go(integral_constant<int, 2>(), integral_constant<int, 4>());
  });
}

template <int RP, class Y, int TO, int TR, int WO, int WR, bool DIRECT> hipError_t launch_up_tiles(const Up& a, hipStream_t st) {
  const int row_tiles = (a.rows + TR - 1) / TR, out_tiles = (a.outs + TO - 1) / TO;
  const dim3 grid((unsigned)row_tiles * out_tiles), block(64 * WO * WR);
  hipLaunchKernelGGL((rfast_lora_up<RP, Y, TO, TR, WO, WR, DIRECT, kWhole>), grid, block, 0, st, a, row_tiles, out_tiles);
  return hipGetLastError();
}
template <int RP, class Y> hipError_t launch_up_split(const Up& a, int splits, bool direct, hipStream_t st) {
  const int row_tiles = (a.rows + 127) / 128, out_tiles = (a.outs + 127) / 128;
  const dim3 grid((unsigned)row_tiles * out_tiles, splits);
  if (direct) hipLaunchKernelGGL((rfast_lora_up<8, float, 128, 128, 2, 2, true, kSplit>), grid, dim3(kThreads), 0, st, a, row_tiles, out_tiles);
  else hipLaunchKernelGGL((rfast_lora_up<8, float, 128, 128, 2, 2, false, kSplit>), grid, dim3(kThreads), 0, st, a, row_tiles, out_tiles);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((rfast_lora_join<RP, Y>), dim3((unsigned)((a.outs + 16 * kWaves - 1) / (16 * kWaves)), (unsigned)((a.rows + 15) / 16)), dim3(kThreads), 0, st,
                     a, splits);
  return hipGetLastError();
}

template <class Y> hipError_t launch_up_rows(const Up& a, hipStream_t st) {
  return by_rank(a.rank, [&](auto rp) {
    constexpr int RP = decltype(rp)::value;
    if (a.rows <= kFewRows) {
      const auto few = [&](auto ot, auto rt) {
        constexpr int OT = decltype(ot)::value, RT = decltype(rt)::value;
        hipLaunchKernelGGL((rfast_lora_up_few<RP, Y, OT, RT, 8>), dim3((unsigned)((a.outs + 16 * OT - 1) / (16 * OT))), dim3(512), 0, st, a);
        return hipGetLastError();
      };
      using std::integral_constant;
      // Two blocks of outputs per workgroup read the rows, from L2, half as often, but there have to be workgroups enough: 48 rows, 4096 x 8192
      // (without adapters) 34 us with one, 29 with two, 45 with four (15 without the rows).
      const auto by_rows = [&](auto ot) {
        if (a.rows <= 16) return few(ot, integral_constant<int, 1>());
        if (a.rows <= 32) return few(ot, integral_constant<int, 2>());
        return a.rows <= 48 ? few(ot, integral_constant<int, 3>()) : few(ot, integral_constant<int, 4>());
      };
      return a.outs >= 32 * 256 ? by_rows(integral_constant<int, 2>()) : by_rows(integral_constant<int, 1>());
    }
    const int64_t large = ((int64_t)a.rows + 255) / 256 * ((a.outs + 255) / 256);
    const bool direct = a.ld_z % 8 == 0 && (uintptr_t)a.z % 16 == 0 && a.cols % 8 == 0 && (uintptr_t)a.w % 16 == 0;
    const int splits = splits_of(a.rows, a.outs, a.cols);
    if (splits > 0) return launch_up_split<RP, Y>(a, splits, direct, st);
    if (!direct) return launch_up_tiles<RP, Y, 128, 128, 2, 2, false>(a, st);
    if (large >= 192) return launch_up_tiles<RP, Y, 256, 256, 2, 4, true>(a, st);
    return launch_up_tiles<RP, Y, 128, 128, 2, 2, true>(a, st);
  });
}

// Few outputs go in one launch, where its workgroups, one or more per segment, are all on the card at once or their tiles are half full at
// least: 32768 rows, 1024 x 128, rank 8, two launches and one: 128 segments 45 and 32 us, 2048 segments 56 and 106; 4096 rows of 256
// segments 34 and 25.  Long rows of few tiles are better split: one segment of 512 rows, 4096 x 128, rank 16, 26 us, and 59 in one launch; 8192
// rows 53 and 60; but 16384 rows, 2048 x 128, 48 and 36; 1000 rows, 784 x 10, 18.5 and 17.
bool fused_pays(const Up& a) {
  const int64_t segments = a.seg.count;
  return a.outs <= 128 && a.rank <= 32 && a.rows > kFewRows && (a.rows / 128 + segments <= 512 || a.rows >= 64 * segments) && a.ld_z % 8 == 0 &&
         (uintptr_t)a.z % 16 == 0 && a.cols % 8 == 0 && (a.cols <= 1024 || splits_of(a.rows, a.outs, a.cols) < 4) && (uintptr_t)a.w % 16 == 0 &&
         (uintptr_t)a.m % 16 == 0;
}
template <class Y> hipError_t launch_fused(const Up& a, hipStream_t st) {
  return by_rank(a.rank, [&](auto rp) {
    constexpr int RP = decltype(rp)::value <= 32 ? decltype(rp)::value : 32;
    hipLaunchKernelGGL((rfast_lora_up<RP, Y, 128, 128, 2, 2, true, kFused>), dim3((unsigned)Segments::blocks(a.rows, a.seg.count, 128)), dim3(kThreads), 0,
                       st, a, 0, 0);
    return hipGetLastError();
  });
}

template <class Y> hipError_t launch_up(const Up& all, hipStream_t st) {
  Up a = all;
  const int whole = whole_rows(a.rows, a.outs);
  if (whole < a.rows) {
    a.rows = whole;
    Up rest = all;
    rest.rows -= whole;
    rest.z += (int64_t)whole * a.ld_z;
    rest.u += (int64_t)whole * kPieces * padded_rank(a.rank);
    rest.ids += whole;
    rest.y = (Y*)a.y + (int64_t)whole * a.ld_y;
    const hipError_t e = launch_up_rows<Y>(rest, st);
    if (e != hipSuccess) return e;
  }
  return launch_up_rows<Y>(a, st);
}

hipError_t launch_sums(const Sums& a, const Sums& b, hipStream_t st) {
  return by_rank(a.rank, [&](auto rp) {
    constexpr int WAVES = 4;
    const int tiles_a = (a.cols + 127) / 128, tiles_b = (b.cols + 127) / 128;
    hipLaunchKernelGGL((rfast_lora_sums<decltype(rp)::value, WAVES>), dim3(tiles_a + tiles_b, a.seg.adapters), dim3(64 * WAVES), 0, st, a, b, tiles_a);
    return hipGetLastError();
  });
}

bool at_multiple(const void* p, size_t to) { return (uintptr_t)p % to == 0; }

RfastArea flat(const void* p, int64_t bytes) { return {p, 1, bytes, bytes}; }

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
  {
    const int64_t n = s->adapters, r = s->rank, d = s->d, K = s->K, wide = s->y_type == RFAST_F32 ? 4 : 2;
    const RfastArea out = {y, s->rows, s->ld_y * wide, K * wide}, work = flat(workspace, (int64_t)layout_of(*s, 0).total);
    const RfastArea read[] = {{x, s->rows, s->ld_x * 2, d * 2}, flat(W, K * d * 2), flat(A, n * r * d * 2), flat(B, n * r * K * 2),
                              flat(row_ptr, ((int64_t)s->segments + 1) * 4), flat(adapter, (int64_t)s->segments * 4)};
    for (const RfastArea& in : read)
      if (rfast_overlap(out, in) || rfast_overlap(work, in)) return rfast_refuse(RFAST_EINVAL, "memory that is written overlaps an argument");
    if (rfast_overlap(out, work)) return rfast_refuse(RFAST_EINVAL, "memory that is written overlaps an argument");
  }
  const hipStream_t st = (hipStream_t)hip_stream;
  const Layout l = layout_of(*s, 0);
  char* ws = (char*)workspace;
  const Segments seg = {row_ptr, adapter, s->segments, s->adapters, s->rows};
  const Up u = {(const u16*)x, (const u16*)W, (const u16*)B, (const u16*)(ws + l.u_rows), (const int32_t*)(ws + l.ids), y, s->ld_x, s->ld_y, s->rows, s->d, s->K, s->rank,
                s->adapters, (const u16*)A, seg, s->scale, (float*)(ws + l.partials)};
  hipError_t e = hipSuccess;
  if (fused_pays(u)) {
    e = s->y_type == RFAST_F32 ? launch_fused<float>(u, st) : launch_fused<u16>(u, st);
    return e == hipSuccess ? RFAST_OK : rfast_refuse_hip(e, "projection launch");
  }
  e = launch_down({(const u16*)x, (const u16*)A, (u16*)(ws + l.u_rows), nullptr, (int32_t*)(ws + l.ids), seg, s->ld_x, 0, s->d, s->rank, s->scale, 0, {}}, st);
  if (e != hipSuccess) return rfast_refuse_hip(e, "adapter launch");
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
  {
    const int64_t T = s->rows, n = s->adapters, r = s->rank, d = s->d, K = s->K;
    const RfastArea written[] = {{dx, T, s->ld_x * 2, d * 2}, flat(dA, n * r * d * 4), flat(dB, n * r * K * 4), flat(workspace, (int64_t)layout_of(*s, pass).total)};
    const RfastArea read[] = {{x, T, s->ld_x * 2, d * 2}, {dy, T, s->ld_y * 2, K * 2}, flat(W, K * d * 2), flat(A, n * r * d * 2), flat(B, n * r * K * 2),
                              flat(row_ptr, ((int64_t)s->segments + 1) * 4), flat(adapter, (int64_t)s->segments * 4)};
    for (int i = 0; i < 4; ++i) {
      for (const RfastArea& in : read)
        if (rfast_overlap(written[i], in)) return rfast_refuse(RFAST_EINVAL, "memory that is written overlaps an argument");
      for (int j = 0; j < i; ++j)
        if (rfast_overlap(written[i], written[j])) return rfast_refuse(RFAST_EINVAL, "memory that is written overlaps an argument");
    }
  }
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
    Transposes t = {{transpose_of(B, bt, s->K, s->rank, s->adapters), {}, {}}};
    if (dx) {
      t.t[1] = transpose_of(A, ws + l.at, s->rank, s->d, s->adapters);
      t.t[2] = transpose_of(W, ws + l.wt, s->K, s->d, 1);
    }
    e = launch_down({(const u16*)x, (const u16*)A, nullptr, u_cols, nullptr, seg, s->ld_x, l.pitch, s->d, s->rank, 1.f, 0, t}, st);
    if (e == hipSuccess) e = launch_down({(const u16*)dy, bt, e_rows, e_cols, ids, seg, s->ld_y, l.pitch, s->K, s->rank, s->scale, 0, {}}, st);
    if (e == hipSuccess && dx)
      e = launch_up<u16>({(const u16*)dy, (const u16*)(ws + l.wt), (const u16*)(ws + l.at), e_rows, ids, dx, s->ld_y, s->ld_x, s->rows, s->K, s->d, s->rank, s->adapters, nullptr, {}, 1.f, (float*)(ws + l.partials)}, st);
  }
  if (e == hipSuccess)
    e = launch_sums({(const u16*)x, e_cols, dA, seg, s->ld_x, l.pitch, s->d, s->rank, 1.f},
                    {(const u16*)dy, u_cols, dB, seg, s->ld_y, l.pitch, s->K, s->rank, s->scale}, st);
  return e == hipSuccess ? RFAST_OK : rfast_refuse_hip(e, "adapter gradient launch");
}

}  // extern "C"
