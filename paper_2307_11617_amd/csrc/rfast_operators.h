// Shared by the operators that take no context (rfast_adamw.hip, rfast_xent.hip, rfast_lora.hip) and by the rounds that call them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <string>

#include "rfast.h"

int rfast_refuse(int code, const std::string& msg);  // text for rfast_last_error(NULL)
int rfast_refuse_hip(hipError_t e, const char* what);
// AdamW divides by sqrt(v) + eps in 32 bits: a denormal has no finite reciprocal, and 0 / eps would be no number
inline bool rfast_adamw_eps_ok(double eps) { return eps >= 0x1p-126 && eps < 1e30; }

// Memory of a call: rows of `wide` bytes, `apart` bytes apart.  Other columns of the same rows are other memory.
struct RfastArea {
  const void* p;
  int64_t rows, apart, wide;
};
inline bool rfast_overlap(const RfastArea& a, const RfastArea& b) {
  if (!a.p || !b.p || a.rows < 1 || b.rows < 1) return false;
  const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p, a1 = a0 + (a.rows - 1) * a.apart + a.wide, b1 = b0 + (b.rows - 1) * b.apart + b.wide;
  if (a1 <= b0 || b1 <= a0) return false;
  if (a.apart != b.apart || a.rows < 2 || b.rows < 2) return true;
  const int64_t behind = (int64_t)(b0 > a0 ? (b0 - a0) % a.apart : (a.apart - (a0 - b0) % a.apart) % a.apart);  // other columns of the same rows?
  return behind < a.wide || behind + b.wide > a.apart;
}

typedef unsigned short u16;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
// At any element's address: the memory system takes wide accesses at every byte address, so that a matrix whose rows start
// anywhere costs one more cache line per row and no other path.
typedef unsigned int any_u32x4 __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned int any_u32x2 __attribute__((ext_vector_type(2), aligned(2)));
typedef float any_f32x4 __attribute__((ext_vector_type(4), aligned(4)));

__device__ inline float from_bf16(u16 b) { return __uint_as_float((uint32_t)b << 16); }
__device__ inline u16 to_bf16(float f) { return __builtin_bit_cast(u16, (__bf16)f); }
__device__ inline uint32_t to_bf16_pair(float a, float b) { return to_bf16(a) | ((uint32_t)to_bf16(b) << 16); }

// (pointers that come out of a table in memory would be taken for ones of any address space)
#define RFAST_GLOBAL __attribute__((address_space(1)))
template <class V, bool STREAM> __device__ inline V wide_load(const void* p) {
  const RFAST_GLOBAL V* g = (const RFAST_GLOBAL V*)(uintptr_t)p;
  if constexpr (STREAM) return __builtin_nontemporal_load(g);
  else return *g;
}
template <class V, bool STREAM> __device__ inline void wide_store(void* p, V v) {
  RFAST_GLOBAL V* g = (RFAST_GLOBAL V*)(uintptr_t)p;
  if constexpr (STREAM) __builtin_nontemporal_store(v, g);
  else *g = v;
}

// Four neighbours of an array of `T` (float or u16 = bf16) from p on, as floats; `left` (1 or more) of them exist.
template <bool STREAM> __device__ inline void load_four(const float* p, int64_t left, float* v) {
  if (left >= 4) {
    const any_f32x4 t = wide_load<any_f32x4, STREAM>(p);
    v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
  } else {
    for (int j = 0; j < 4; ++j) v[j] = j < left ? p[j] : 0.f;
  }
}
template <bool STREAM> __device__ inline void load_four(const u16* p, int64_t left, float* v) {
  if (left >= 4) {
    const any_u32x2 t = wide_load<any_u32x2, STREAM>(p);
    v[0] = __uint_as_float(t.x << 16); v[1] = __uint_as_float(t.x & 0xFFFF0000u);
    v[2] = __uint_as_float(t.y << 16); v[3] = __uint_as_float(t.y & 0xFFFF0000u);
  } else {
    for (int j = 0; j < 4; ++j) v[j] = j < left ? from_bf16(p[j]) : 0.f;
  }
}
template <bool STREAM> __device__ inline void store_four(float* p, int64_t left, const float* v) {
  if (left >= 4) {
    const any_f32x4 t = {v[0], v[1], v[2], v[3]};
    wide_store<any_f32x4, STREAM>(p, t);
  } else {
    for (int j = 0; j < 4; ++j)
      if (j < left) p[j] = v[j];
  }
}
template <bool STREAM> __device__ inline void store_four(u16* p, int64_t left, const float* v) {
  if (left >= 4) {
    const any_u32x2 t = {to_bf16_pair(v[0], v[1]), to_bf16_pair(v[2], v[3])};
    wide_store<any_u32x2, STREAM>(p, t);
  } else {
    for (int j = 0; j < 4; ++j)
      if (j < left) p[j] = to_bf16(v[j]);
  }
}

// Reductions over the 64 lanes of a wavefront, the result in every lane: within rows of 16 by the data-parallel primitives of
// the vector unit (a lane reads another's register as an operand), across rows by a shuffle.
template <int CTRL> __device__ inline float lane_of(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
template <class F> __device__ inline float wave_reduce(float v, F f) {
  v = f(v, lane_of<0xB1>(v));   // the neighbour
  v = f(v, lane_of<0x4E>(v));   // the other pair of four
  v = f(v, lane_of<0x141>(v));  // the other four of eight (mirrored)
  v = f(v, lane_of<0x140>(v));  // the other eight of sixteen (mirrored)
  v = f(v, __shfl_xor(v, 16, 64));
  return f(v, __shfl_xor(v, 32, 64));
}
__device__ inline float wave_max(float v) {
  return wave_reduce(v, [](float a, float b) { return fmaxf(a, b); });
}
