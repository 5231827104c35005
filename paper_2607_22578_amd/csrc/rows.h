// Device helpers shared by the row-table kernels: decoding of table columns to
// fp32 and rounding of fp32 to the output types.
#pragma once

#include "common.h"

namespace hs {

typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4v_t __attribute__((ext_vector_type(4)));
// The same with no alignment beyond that of the elements: global accesses need none, so
// rows of any width and start are read and written 16 bytes at a time.
typedef uint32_t u32x4e_t __attribute__((ext_vector_type(4), aligned(2)));
template <int N>
struct __attribute__((packed)) WordsAt {
  uint32_t w[N];
};
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float bf16_to_f32(uint32_t b) { return __uint_as_float(b << 16); }

// Two fp32 -> two bf16 (round to nearest even), `a` in the low half.
__device__ __forceinline__ uint32_t f32_to_bf16x2(float a, float b) {
  const bf16x2_t v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ uint16_t f32_to_bf16(float a) {
  return __builtin_bit_cast(uint16_t, (__bf16)a);
}

// C (4 or 8) consecutive columns of a row from column `col` (FP4: a multiple of C),
// undecoded: as loaded, so that several can be in flight.
template <int DT, int C>
struct RawCols {
  static constexpr int kBytes = DT == HS_F32 ? 4 * C : DT == HS_BF16 ? 2 * C
                              : DT == HS_FP8_E4M3 ? C : C / 2;
  static constexpr int kWords = kBytes < 4 ? 1 : kBytes / 4;
  uint32_t w[kWords];

  __device__ __forceinline__ void load(const uint8_t *row, int64_t col) {
    const uint8_t *p = row + col * kBytes / C;
    if constexpr (kBytes == 2) {
      w[0] = *(const uint16_t *)p;
    } else {
      constexpr int N = kWords < 4 ? kWords : 4;
#pragma unroll
      for (int i = 0; i < kWords / N; ++i) {
        const WordsAt<N> v = ((const WordsAt<N> *)p)[i];
#pragma unroll
        for (int j = 0; j < N; ++j) w[N * i + j] = v.w[j];
      }
    }
  }

  __device__ __forceinline__ void decode(float *v) const {
    if constexpr (DT == HS_F32) {
#pragma unroll
      for (int i = 0; i < C; ++i) v[i] = __uint_as_float(w[i]);
    } else if constexpr (DT == HS_BF16) {
#pragma unroll
      for (int i = 0; i < C / 2; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    } else if constexpr (DT == HS_FP8_E4M3) {
#pragma unroll
      for (int i = 0; i < C / 4; ++i) {
        const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false);
        const f32x2_t b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
        v[4 * i] = a[0];
        v[4 * i + 1] = a[1];
        v[4 * i + 2] = b[0];
        v[4 * i + 3] = b[1];
      }
    } else {
      // (two codes a byte; the byte is an immediate of the conversion)
      f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], 1.0f, 0);
      v[0] = a[0];
      v[1] = a[1];
      a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], 1.0f, 1);
      v[2] = a[0];
      v[3] = a[1];
      if constexpr (C == 8) {
        a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], 1.0f, 2);
        v[4] = a[0];
        v[5] = a[1];
        a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], 1.0f, 3);
        v[6] = a[0];
        v[7] = a[1];
      }
    }
  }
};

// One column, for the ends of rows.
template <int DT>
__device__ __forceinline__ float load_col(const uint8_t *row, int64_t col) {
  if constexpr (DT == HS_F32) {
    return ((const float *)row)[col];
  } else if constexpr (DT == HS_BF16) {
    return bf16_to_f32(((const uint16_t *)row)[col]);
  } else if constexpr (DT == HS_FP8_E4M3) {
    return __builtin_amdgcn_cvt_f32_fp8((int)row[col], 0);
  } else {
    const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)row[col >> 1], 1.0f, 0);
    return col & 1 ? a[1] : a[0];
  }
}

// C consecutive outputs (16 bytes of them) rounded to the output type.
template <int OT, int C>
__device__ __forceinline__ u32x4v_t round_cols(const float *v) {
  static_assert(C == (OT == HS_F32 ? 4 : 8), "16 bytes");
  u32x4v_t o;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (OT == HS_F32) {
      o[i] = __float_as_uint(v[i]);
    } else {
      o[i] = f32_to_bf16x2(v[2 * i], v[2 * i + 1]);
    }
  }
  return o;
}

__device__ __forceinline__ void store_cols(void *at, u32x4v_t v) { *(u32x4e_t *)at = v; }

// (past the caches: for outputs that the kernel does not read again)
__device__ __forceinline__ void stream_cols(void *at, u32x4v_t v) {
  __builtin_nontemporal_store((u32x4e_t)v, (u32x4e_t *)at);
}

template <int OT>
__device__ __forceinline__ void store_col(void *row, int64_t col, float v) {
  if constexpr (OT == HS_F32) {
    ((float *)row)[col] = v;
  } else {
    ((uint16_t *)row)[col] = f32_to_bf16(v);
  }
}

template <int DT>
__device__ __forceinline__ int64_t row_bytes(int64_t dim) {
  return DT == HS_F32 ? dim * 4 : DT == HS_BF16 ? dim * 2 : DT == HS_FP8_E4M3 ? dim : dim / 2;
}

// Orders a wave's LDS accesses (its lanes run together: only the compiler has to).
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ int64_t load_id(const void *ids, int is64, int64_t i) {
  return is64 ? ((const int64_t *)ids)[i] : (int64_t)((const int32_t *)ids)[i];
}

}  // namespace hs
