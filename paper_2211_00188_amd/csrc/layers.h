// What the operators of a model's layers share: element types, groups of rows, checks of arguments.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/adacgd.h"
#include "devutil.h"

namespace adacgd {

// Sets the calling thread's last error and returns `code` (engine.hip).
int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

constexpr int64_t kMaxCount = (int64_t(1) << 31) - 1;     // rows, groups, strides
constexpr int64_t kMaxColumns = int64_t(1) << 24;

inline int64_t dtype_size(int32_t t) { return t == ADACGD_FP32 ? 4 : 2; }

// A matrix argument of `rows` rows (of each group, if it is a grouped one).
inline int check_tensor(const adacgd_tensor* t, const char* name, int64_t rows, int64_t columns, bool grouped, bool may_share) {
  if (!t) return fail(ADACGD_ERR_ARG, "%s is null", name);
  if (t->dtype < 0 || t->dtype > ADACGD_FP16) return fail(ADACGD_ERR_ARG, "%s: unknown type %d", name, t->dtype);
  if (t->pad != 0) return fail(ADACGD_ERR_ARG, "%s: pad must be 0", name);
  if (rows > 0 && !t->data) return fail(ADACGD_ERR_ARG, "%s: data is null", name);
  if ((uintptr_t)t->data % dtype_size(t->dtype)) return fail(ADACGD_ERR_ARG, "%s: data is not aligned to its type", name);
  if (rows > 1 && (t->stride < columns || t->stride > kMaxCount))
    return fail(ADACGD_ERR_ARG, "%s: stride must be in [%lld, 2^31), got %lld", name, (long long)columns, (long long)t->stride);
  if (grouped && t->group_stride < 0) return fail(ADACGD_ERR_ARG, "%s: group_stride must not be negative", name);
  if (grouped && !may_share && t->group_stride < (rows > 1 ? (rows - 1) * t->stride : 0) + columns)
    return fail(ADACGD_ERR_ARG, "%s: group_stride is smaller than a matrix", name);
  return ADACGD_OK;
}
inline int check_count(const char* name, int64_t v, int64_t lo, int64_t hi) {
  if (v < lo || v > hi) return fail(ADACGD_ERR_ARG, "%s must be in [%lld, %lld], got %lld", name, (long long)lo, (long long)hi, (long long)v);
  return ADACGD_OK;
}
inline int check_workspace(const void* w, int64_t have, int64_t need) {
  if (need == 0) return ADACGD_OK;
  if (!w || (uintptr_t)w % 256 || have < need)
    return fail(ADACGD_ERR_ALLOC, "workspace of %lld bytes, 256-byte aligned, needed; %lld given", (long long)need, (long long)(w ? have : 0));
  return ADACGD_OK;
}
// After a launch.
inline int launched(const char* name) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ADACGD_OK : fail(ADACGD_ERR_DEVICE, "%s: launch failed: %s", name, hipGetErrorString(e));
}
#define ADACGD_TRY(call)          \
  do {                            \
    const int rc_ = (call);       \
    if (rc_) return rc_;          \
  } while (0)

// Rows are cut into slices of at most 2^SHIFT, none across two groups.  Slice j of group g has number
// (offsets[g] >> SHIFT) + g + j: these numbers ascend without a prefix sum (a group of `len` rows that begins at o ends at
// or below ((o + len) >> SHIFT) + 1), every group has one at least, and (rows >> shift) + groups bounds them, which is all
// that the host knows.  Numbers that no slice has are left out by whoever gets them.
// offsets are clamped where they are read, so that no value of theirs leads outside the matrices.
struct Slice {
  int64_t group;        // -1: none
  int64_t begin, end;   // rows; empty only for an empty group
  int64_t first, last;  // rows of the whole group
};
__host__ __device__ inline int64_t slice_numbers(int64_t rows, int64_t groups, int shift) { return (rows >> shift) + groups; }
// First number of a group's slices.
__host__ __device__ inline int64_t first_number(int64_t first_row, int64_t group, int shift) { return (first_row >> shift) + group; }

// Where partial sums are kept for the slices of groups of more than 2^shift rows only: from 2 (first row >> shift) on.  The
// next such group begins behind the last slice, and the number of places does not depend on the number of groups.
__host__ __device__ inline int64_t part_number(int64_t first, int shift) { return 2 * (first >> shift); }
__host__ __device__ inline int64_t part_numbers(int64_t rows, int shift) { return 2 * (rows >> shift) + 1; }

__device__ __forceinline__ int64_t offset_at(const int64_t* offsets, int64_t i, int64_t rows) {
  const int64_t o = offsets[i];
  return o < 0 ? 0 : o > rows ? rows : o;
}
// All lanes of a wavefront call it with the same arguments: 64 groups are looked at with one load.  `each` entries of
// offsets make one group.
__device__ __forceinline__ Slice find_slice(const int64_t* offsets, int64_t groups, int64_t rows, int64_t each, int shift, int64_t number) {
  Slice s{-1, 0, 0, 0, 0};
  if (!offsets) {                                         // one group of all rows
    s.last = rows;
    s.begin = number << shift;
    if (s.begin >= rows && number > 0) return s;
    s.group = 0;
    s.end = s.begin + (int64_t(1) << shift) < rows ? s.begin + (int64_t(1) << shift) : rows;
    return s;
  }
  int64_t low = 0, count = groups;
  const int lane = (int)lane_id();
  for (;;) {
    const int64_t step = (count + 63) / 64;
    const bool here = lane * step < count;
    const int64_t g = low + (here ? lane * step : 0);
    const uint64_t m = ballot(here && first_number(offset_at(offsets, g * each, rows), g, shift) <= number);
    if (m == 0) return s;
    const int64_t hit = 63 - __builtin_clzll(m);          // (the last of them)
    low += hit * step;
    count = count - hit * step < step ? count - hit * step : step;
    if (step == 1) break;
  }
  s.first = offset_at(offsets, low * each, rows);
  s.last = offset_at(offsets, (low + 1) * each, rows);
  if (s.last < s.first) s.last = s.first;
  const int64_t j = number - first_number(s.first, low, shift);
  s.begin = s.first + (j << shift);
  if (s.begin >= s.last && j > 0) return s;
  s.group = low;
  s.end = s.begin + (int64_t(1) << shift) < s.last ? s.begin + (int64_t(1) << shift) : s.last;
  return s;
}

// The last group that begins at or before `row` (0 if none does), 64 of them looked at with one load.  For all lanes of a wavefront.
__device__ __forceinline__ int64_t group_of(const int64_t* offsets, int64_t groups, int64_t rows, int64_t row) {
  const int lane = (int)lane_id();
  int64_t low = 0, count = groups;
  while (count > 1) {
    const int64_t step = (count + 63) / 64;
    const bool here = lane * step < count;
    const uint64_t m = ballot(here && offset_at(offsets, low + (here ? lane * step : 0), rows) <= row);
    const int64_t hit = m ? 63 - __builtin_clzll(m) : 0;
    low += hit * step;
    count = count - hit * step < step ? count - hit * step : step;
  }
  return low;
}


template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_or0f(float v) { return __uint_as_float(dpp_or0<CTRL, ROWS>(__float_as_uint(v))); }
// Sum over 16 neighbouring lanes, in all of them (by rotations of such a row).
__device__ __forceinline__ float row16_sumf(float v) {
  v += dpp_or0f<0x128, 0xf>(v);
  v += dpp_or0f<0x124, 0xf>(v);
  v += dpp_or0f<0x122, 0xf>(v);
  v += dpp_or0f<0x121, 0xf>(v);
  return v;
}
// Sum over the wavefront, in every lane.
__device__ __forceinline__ float wave_sumf(float v) {
  v += dpp_or0f<kDppShr + 1, 0xf>(v);
  v += dpp_or0f<kDppShr + 2, 0xf>(v);
  v += dpp_or0f<kDppShr + 4, 0xf>(v);
  v += dpp_or0f<kDppShr + 8, 0xf>(v);
  v += dpp_or0f<kDppBcast15, 0xa>(v);
  v += dpp_or0f<kDppBcast31, 0xc>(v);
  return __uint_as_float(lane_value(__float_as_uint(v), 63));
}

// Element types: what is stored, and its value as a float.
template <typename T>
__device__ __forceinline__ float to_float(T v) { return (float)v; }
template <typename T>
__device__ __forceinline__ T from_float(float v) { return (T)v; }      // (to nearest, ties to even)

// 16 bytes of a row at any alignment; a vector that passes the row's end is taken element by element (`missing` behind it).  Kept as
// words: where elements of the two ways to load it met, the compiler would wait for the load at once to take them apart.
typedef uint32_t word4 __attribute__((ext_vector_type(4)));
template <typename T>
struct Vec {
  static constexpr int kElems = 16 / sizeof(T);
  word4 w;
  __device__ __forceinline__ float get(int j) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[j]);
    else if constexpr (__is_same(T, __bf16)) return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
    else return to_float(__builtin_bit_cast(T, (uint16_t)(j & 1 ? w[j / 2] >> 16 : w[j / 2])));
  }
  __device__ __forceinline__ void put(const float (&f)[kElems]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(f[j]);
    } else {
      typedef T pair __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = __builtin_bit_cast(uint32_t, pair{from_float<T>(f[2 * j]), from_float<T>(f[2 * j + 1])});
    }
  }
  static __device__ __forceinline__ uint32_t bits(T v) {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(uint32_t, v);
    else return __builtin_bit_cast(uint16_t, v);
  }
  __device__ __forceinline__ void load(const T* p, int64_t have, float missing = 0.f) {
    if (have >= kElems) {
      __builtin_memcpy(&w, p, 16);
      return;
    }
    w = word4{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < kElems; ++j) {
      const uint32_t u = bits(j < have ? p[j] : from_float<T>(missing));
      if constexpr (sizeof(T) == 4) w[j] = u;
      else w[j / 2] |= u << (16 * (j & 1));
    }
  }
  // What was computed from the elements is computed again after this, not kept in registers of twice their size.
  __device__ __forceinline__ void again() { asm volatile("" : "+v"(w)); }
  __device__ __forceinline__ void store(T* p, int64_t have) const {
    if (have >= kElems) {
      __builtin_memcpy(p, &w, 16);
      return;
    }
#pragma unroll
    for (int j = 0; j < kElems; ++j) {
      if (j >= have) break;
      if constexpr (sizeof(T) == 4) p[j] = __uint_as_float(w[j]);
      else p[j] = __builtin_bit_cast(T, (uint16_t)(w[j / 2] >> (16 * (j & 1))));
    }
  }
};

// f(type tag) for the C type of a dtype.
template <typename F>
inline int by_dtype(int32_t dtype, F f) {
  if (dtype == ADACGD_FP32) return f(float());
  if (dtype == ADACGD_BF16) return f(__bf16());
  return f(_Float16());
}

}  // namespace adacgd
