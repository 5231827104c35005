// Products of a few rows with every row of a packed table (E2M1 codes, a scale per
// group of columns):
//   out[m][r] = sum_g scale[r][g] * sum_{c in g} x[m][c] * code[r][c].
//
// The codes become bf16 by the hardware's conversion (two a time, exact), so the
// products run on the bf16 matrix cores: mfma_f32_16x16x32_bf16 with 16 rows of x as
// the left and 16 table rows as the right operand.  The sums of one group are scaled
// and added in fp32.  fp32 rows of x are split into three bf16 parts (the top 8, the
// next 8 and the last 8 significant bits: exact).
//
// A wave loads 16 bytes (32 columns) per lane: lane l has row l % 16 and piece l / 16 of
// 128 columns.  One MFMA takes 8 columns from each of the four lane groups, so without
// more it would mix the four pieces: right for groups of 128.  For groups of 64 and 32
// the pieces' words are exchanged between the lane groups (two swaps of lane halves,
// two more of lane quarters for 32), and x is read in the same order.
// Floor: the table, read once.
#include "rows.h"

namespace hs {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int kNT = 4;   // 16-row tiles of the table per wave

__device__ __forceinline__ bf16x8_t decode_codes(uint32_t w) {
  bf16x8_t b;
  const bf16x2_t p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0);
  const bf16x2_t p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1);
  const bf16x2_t p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2);
  const bf16x2_t p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3);
  b[0] = p0[0]; b[1] = p0[1];
  b[2] = p1[0]; b[3] = p1[1];
  b[4] = p2[0]; b[5] = p2[1];
  b[6] = p3[0]; b[7] = p3[1];
  return b;
}

__device__ __forceinline__ void swap_halves(uint32_t &a, uint32_t &b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}

__device__ __forceinline__ void swap_quarters(uint32_t &a, uint32_t &b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}

// After the exchange, word j of lane group p holds columns
// piece_of(j, p) * 32 + word_of(j, p) * 8 .. + 8 of the 128, all of word j within
// one group of columns.
template <int GROUP>
__device__ __forceinline__ void exchange(uint32_t *w) {
  if constexpr (GROUP <= 64) {
    swap_halves(w[0], w[1]);
    swap_halves(w[2], w[3]);
  }
  if constexpr (GROUP == 32) {
    swap_quarters(w[0], w[2]);
    swap_quarters(w[1], w[3]);
  }
}

template <int GROUP>
__device__ __forceinline__ int first_col(int j, int p) {
  if constexpr (GROUP == 128) return p * 32 + j * 8;
  // halves exchanged: words 0, 2 hold pieces 0 and 1, words 1, 3 pieces 2 and 3
  if constexpr (GROUP == 64) return ((j & 1) * 2 + (p & 1)) * 32 + ((j & 2) + (p >> 1)) * 8;
  // quarters too: words 0, 2, 1, 3 hold pieces 0, 1, 2, 3, their words in the order 0, 2, 1, 3
  return ((j & 1) * 2 + (j >> 1)) * 32 + ((p & 1) * 2 + (p >> 1)) * 8;
}

// Group (of the 128 / GROUP in the block) that word j belongs to.
template <int GROUP>
__device__ __forceinline__ constexpr int group_of(int j) {
  return GROUP == 128 ? 0 : GROUP == 64 ? (j & 1) : (j & 1) * 2 + (j >> 1);
}

// The eight columns of x for one lane and MFMA, as PARTS bf16 vectors.
template <int XT, int PARTS>
__device__ __forceinline__ void load_x(const uint8_t *row, int col, bool in, bf16x8_t *part) {
  if constexpr (XT == HS_BF16) {
    part[0] = in ? *(const bf16x8_t *)(row + (int64_t)col * 2) : bf16x8_t{};
  } else {
    uint32_t h[8] = {};
    if (in) {
      RawCols<HS_F32, 8> raw;
      raw.load(row, col);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = raw.w[i];
    }
    uint32_t w[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // truncation, so that nothing overflows; each rest is exact
      uint32_t t[3][2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float f = __uint_as_float(h[2 * i + e]);
#pragma unroll
        for (int p = 0; p < 3; ++p) {
          t[p][e] = __float_as_uint(f) & 0xFFFF0000u;
          f -= __uint_as_float(t[p][e]);
        }
      }
#pragma unroll
      for (int p = 0; p < 3; ++p) w[p][i] = (t[p][0] >> 16) | t[p][1];
    }
#pragma unroll
    for (int p = 0; p < 3; ++p)
      part[p] = __builtin_bit_cast(bf16x8_t, u32x4v_t{w[p][0], w[p][1], w[p][2], w[p][3]});
  }
}

// One workgroup of four waves: KS of them share the columns (their sums are joined in
// LDS, in wave order), 4 / KS have 64 table rows each.  MT tiles of 16 rows of x.
template <int XT, int GROUP, int MT>
__global__ __launch_bounds__(256) void score_packed_kernel(
    const uint8_t *__restrict__ codes, const void *__restrict__ scales, int scale_bf16,
    int64_t rows, int dim, const uint8_t *__restrict__ x, int64_t n_x, int ks, int64_t row_blocks,
    int64_t items, void *__restrict__ out, int out_f32, int64_t out_stride) {
  constexpr int PARTS = XT == HS_F32 ? 3 : 1;
  constexpr int XB = XT == HS_F32 ? 4 : 2;
  constexpr int NG = 128 / GROUP;
  __shared__ f32x4_t joined[3][kNT * MT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int i16 = lane & 15, p = lane >> 4;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t mb = item / row_blocks;
    const int64_t rb = item - mb * row_blocks;
    const int64_t n0 = (rb * (4 / ks) + wave / ks) * (16 * kNT);
    const int64_t m0 = mb * (16 * MT);
    const int part_of = wave % ks;
    const int blocks = (dim + 127) / 128;
    const int k0 = part_of * blocks / ks, k1 = (part_of + 1) * blocks / ks;
    const int64_t cb = dim / 2, groups = dim / GROUP;
    f32x4_t tot[kNT][MT];
  #pragma unroll
    for (int t = 0; t < kNT; ++t)
  #pragma unroll
      for (int m = 0; m < MT; ++m) tot[t][m] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    const uint8_t *row[kNT];
    int64_t srow[kNT];
  #pragma unroll
    for (int t = 0; t < kNT; ++t) {
      int64_t r = n0 + t * 16 + i16;
      if (r >= rows) r = rows - 1;
      row[t] = codes + r * cb;
      srow[t] = r * groups;
    }
    const uint8_t *xrow[MT];
    bool xin[MT];
  #pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int64_t r = m0 + m * 16 + i16;
      xin[m] = r < n_x;
      xrow[m] = x + (xin[m] ? r : 0) * dim * XB;
    }
    for (int kb = k0; kb < k1; ++kb) {
      const int c0 = kb * 128;
      uint32_t w[kNT][4];
      float sc[kNT][NG];
  #pragma unroll
      for (int t = 0; t < kNT; ++t) {
        u32x4v_t v = {0u, 0u, 0u, 0u};
        if (c0 + p * 32 < dim) v = *(const u32x4v_t *)(row[t] + (c0 + p * 32) / 2);
  #pragma unroll
        for (int j = 0; j < 4; ++j) w[t][j] = v[j];
  #pragma unroll
        for (int g = 0; g < NG; ++g) {
          const int64_t at = srow[t] + c0 / GROUP + g;
          sc[t][g] = c0 + g * GROUP >= dim ? 0.0f
                     : scale_bf16 ? bf16_to_f32(((const uint16_t *)scales)[at])
                                  : ((const float *)scales)[at];
        }
      }
  #pragma unroll
      for (int t = 0; t < kNT; ++t) exchange<GROUP>(w[t]);
  #pragma unroll
      for (int g = 0; g < NG; ++g) {
        f32x4_t acc[kNT][MT];
  #pragma unroll
        for (int t = 0; t < kNT; ++t)
  #pragma unroll
          for (int m = 0; m < MT; ++m) acc[t][m] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  #pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (group_of<GROUP>(j) != g) continue;
          const int col = c0 + first_col<GROUP>(j, p);
          bf16x8_t xa[MT][PARTS];
  #pragma unroll
          for (int m = 0; m < MT; ++m) load_x<XT, PARTS>(xrow[m], col, xin[m] && col < dim, xa[m]);
  #pragma unroll
          for (int t = 0; t < kNT; ++t) {
            const bf16x8_t b = decode_codes(w[t][j]);
  #pragma unroll
            for (int m = 0; m < MT; ++m)
  #pragma unroll
              for (int q = PARTS - 1; q >= 0; --q)   // (small parts first)
                acc[t][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xa[m][q], b, acc[t][m], 0, 0, 0);
          }
        }
  #pragma unroll
        for (int t = 0; t < kNT; ++t)
  #pragma unroll
          for (int m = 0; m < MT; ++m)
  #pragma unroll
            for (int i = 0; i < 4; ++i)
              tot[t][m][i] = __builtin_fmaf(sc[t][g], acc[t][m][i], tot[t][m][i]);
      }
    }
    // (ks = 4: waves 1-3 into wave 0; ks = 2: waves 1 and 3 into 0 and 2)
    if (ks > 1) {
      if (part_of > 0) {
  #pragma unroll
        for (int t = 0; t < kNT; ++t)
  #pragma unroll
          for (int m = 0; m < MT; ++m) joined[wave - 1][t * MT + m][lane] = tot[t][m];
      }
      __syncthreads();
      for (int q = 1; q < ks && part_of == 0; ++q) {
  #pragma unroll
        for (int t = 0; t < kNT; ++t)
  #pragma unroll
          for (int m = 0; m < MT; ++m) {
            const f32x4_t o = joined[wave + q - 1][t * MT + m][lane];
  #pragma unroll
            for (int i = 0; i < 4; ++i) tot[t][m][i] += o[i];
          }
      }
    }
    if (part_of == 0) {
    // lane l holds table row l % 16 of a tile and rows 4 (l / 16) .. + 3 of x
  #pragma unroll
    for (int m = 0; m < MT; ++m)
  #pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t r = m0 + m * 16 + p * 4 + i;
        if (r >= n_x) continue;
  #pragma unroll
        for (int t = 0; t < kNT; ++t) {
          const int64_t n = n0 + t * 16 + i16;
          if (n >= rows) continue;
          if (out_f32)
            ((float *)out)[r * out_stride + n] = tot[t][m][i];
          else
            ((uint16_t *)out)[r * out_stride + n] = f32_to_bf16(tot[t][m][i]);
        }
      }
    }
    if (ks > 1) __syncthreads();   // (the next item reuses `joined`)
  }
}

template <int XT, int GROUP>
hipError_t launch_packed_t(const hs_row_table *t, const void *x, int64_t n_x, void *out,
                           int out_dtype, int64_t out_stride, hipStream_t st) {
  const int mt = n_x <= 16 ? 1 : n_x <= 32 ? 2 : 4;
  const int64_t mblocks = (n_x + 16 * mt - 1) / (16 * mt);
  const int64_t waves = (t->rows + 63) / 64 * mblocks;
  // the columns shared by up to four waves while there are fewer than 4,096 (16 per CU)
  int ks = 1;
  while (ks < 4 && waves * ks < 4096 && t->dim > 128 * ks) ks *= 2;
  const int64_t row_blocks = (t->rows + 64 * (4 / ks) - 1) / (64 * (4 / ks));
  auto kernel = mt == 1   ? score_packed_kernel<XT, GROUP, 1>
                : mt == 2 ? score_packed_kernel<XT, GROUP, 2>
                          : score_packed_kernel<XT, GROUP, 4>;
  const int64_t items = row_blocks * mblocks;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(items < (1 << 22) ? items : (1 << 22))), dim3(256), 0, st,
                     (const uint8_t *)t->data, t->scale, (int)(t->scale_dtype == HS_BF16), t->rows,
                     (int)t->dim, (const uint8_t *)x, n_x, ks, row_blocks, items, out,
                     (int)(out_dtype == HS_F32), out_stride);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_score_packed(const hs_row_table *t, const void *x, int x_dtype, int64_t n_x,
                               void *out, int out_dtype, int64_t out_stride, hipStream_t st) {
  if (n_x <= 0 || t->rows <= 0) return hipSuccess;
#define HS_PACKED(G)                                                                        \
  (x_dtype == HS_F32 ? launch_packed_t<HS_F32, G>(t, x, n_x, out, out_dtype, out_stride, st) \
                     : launch_packed_t<HS_BF16, G>(t, x, n_x, out, out_dtype, out_stride, st))
  return t->group == 32 ? HS_PACKED(32) : t->group == 64 ? HS_PACKED(64) : HS_PACKED(128);
#undef HS_PACKED
}

}  // namespace hs
