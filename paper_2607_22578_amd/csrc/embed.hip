// Embedding lookup with scaling, out[i] = scale * T[ids[i]], from a table of fp32,
// bf16, fp8 (a scale per row) or packed fp4 (a scale per group of columns) rows; and
// the packing of rows into four bits.
#include "rows.h"

namespace hs {

// ---------------------------------------------------------------- lookup
//
// A group of threads makes one row; a thread makes 16 bytes of it at a time, so a wave
// stores whole row segments, as the byte gather does (hs_scatter).  Bound by the bytes:
// 65,536 tokens from a 131,072 x 4,096 table in four bits (583 MB): 90 us, 6.5 TB/s.
template <int DT, int OT>
__global__ __launch_bounds__(256) void embed_kernel(
    const uint8_t *__restrict__ data, const void *__restrict__ scales, int scale_bf16,
    int64_t rows, int dim, int gshift, const void *__restrict__ ids, int is64, int64_t n,
    float mul, int64_t pad, int group, uint8_t *__restrict__ out) {
  constexpr int C = OT == HS_F32 ? 4 : 8;
  constexpr int OB = OT == HS_F32 ? 4 : 2;
  const int per_block = 256 / group;
  const int sub = threadIdx.x / group, lane = threadIdx.x % group;
  // (a row's last access ends with the row: it may make columns once more)
  const int vpr = dim >= C ? (dim + C - 1) / C : 0;
  for (int64_t i = (int64_t)blockIdx.x * per_block + sub; i < n;
       i += (int64_t)gridDim.x * per_block) {
    const int64_t id = load_id(ids, is64, i);
    const bool token = id >= 0 && id < rows && id != pad;
    const uint8_t *row = data + (token ? id : 0) * row_bytes<DT>(dim);
    uint8_t *dst = out + i * (int64_t)dim * OB;
    const float rs = DT == HS_FP8_E4M3 && token ? ((const float *)scales)[id] : 1.0f;
    const int64_t gs = DT == HS_FP4_E2M1 && token ? id * (dim >> gshift) : 0;
    for (int a = lane; a < vpr; a += group) {
      const int c = a * C + C <= dim ? a * C : dim - C;
      float v[C];
      if (token) {
        float s = rs;
        if constexpr (DT == HS_FP4_E2M1) {
          const int64_t g = gs + (c >> gshift);
          s = scale_bf16 ? bf16_to_f32(((const uint16_t *)scales)[g]) : ((const float *)scales)[g];
        }
        RawCols<DT, C> raw;
        raw.load(row, c);
        raw.decode(v);
#pragma unroll
        for (int j = 0; j < C; ++j) v[j] = (DT >= HS_FP8_E4M3 ? v[j] * s : v[j]) * mul;
      } else {
#pragma unroll
        for (int j = 0; j < C; ++j) v[j] = 0.0f;
      }
      stream_cols(dst + (int64_t)c * OB, round_cols<OT, C>(v));
    }
    // rows of less than an access (packed ones are longer)
    if constexpr (DT != HS_FP4_E2M1) {
      for (int c = vpr > 0 ? dim : lane; c < dim; c += group) {
        float v = 0.0f;
        if (token) v = (DT == HS_FP8_E4M3 ? load_col<DT>(row, c) * rs : load_col<DT>(row, c)) * mul;
        store_col<OT>(dst, c, v);
      }
    }
  }
}

template <int DT, int OT>
static hipError_t launch_embed_t(const hs_row_table *t, const void *ids, int is64, int64_t n,
                                 float scale, int64_t pad, void *out, hipStream_t st) {
  constexpr int C = OT == HS_F32 ? 4 : 8;
  const int gshift = t->group == 128 ? 7 : t->group == 64 ? 6 : 5;
  const int vpr = (int)((t->dim + C - 1) / C);
  int group = 1;
  while (group < vpr && group < 256) group <<= 1;
  const int per_block = 256 / group;
  int64_t blocks = (n + per_block - 1) / per_block;
  if (blocks > 65536) blocks = 65536;
  hipLaunchKernelGGL((embed_kernel<DT, OT>),
                     dim3((unsigned)blocks), dim3(256), 0, st, (const uint8_t *)t->data, t->scale,
                     (int)(t->scale_dtype == HS_BF16), t->rows, (int)t->dim, gshift, ids, is64, n,
                     scale, pad, group, (uint8_t *)out);
  return hipGetLastError();
}

hipError_t launch_embed(const hs_row_table *t, const void *ids, int is64, int64_t n, float scale,
                        int64_t pad, void *out, int out_dtype, hipStream_t st) {
  if (n <= 0) return hipSuccess;
#define HS_EMBED(DT)                                                                   \
  case DT:                                                                             \
    return out_dtype == HS_F32 ? launch_embed_t<DT, HS_F32>(t, ids, is64, n, scale, pad, out, st) \
                               : launch_embed_t<DT, HS_BF16>(t, ids, is64, n, scale, pad, out, st)
  switch (t->dtype) {
    HS_EMBED(HS_F32);
    HS_EMBED(HS_BF16);
    HS_EMBED(HS_FP8_E4M3);
    default:
      HS_EMBED(HS_FP4_E2M1);
  }
#undef HS_EMBED
}

// ---------------------------------------------------------------- packing
//
// A thread packs eight columns (one word of codes); the group's largest magnitude
// goes over the group's 4, 8 or 16 neighbouring lanes.  The thresholds are the
// midpoints between neighbouring E2M1 values; a midpoint goes to the even code.
// 131,072 x 4,096 bf16 rows (1,376 MB): 466 us, 3.0 TB/s, less than a copy's 4.8 for its
// divisions and comparisons.
__device__ __forceinline__ uint32_t e2m1_code(float q) {
  const float a = fabsf(q);
  const uint32_t m = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) +
                     (a >= 3.5f) + (a > 5.0f);
  return q < 0.0f ? m | 8u : m;
}

template <int DT>
__global__ __launch_bounds__(256) void pack_rows_kernel(const uint8_t *__restrict__ src,
                                                        int64_t words, int lanes, int scale_bf16,
                                                        uint32_t *__restrict__ codes,
                                                        void *__restrict__ scales) {
  // (groups never straddle a wave: 64 is a multiple of their lanes, and `words` of
  // them too, so a group's lanes all take part or none does)
  for (int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x; w < words;
       w += (int64_t)gridDim.x * 256) {
    RawCols<DT, 8> raw;
    float v[8];
    raw.load(src, w * 8);
    raw.decode(v);
    float amax = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf(v[j]));
    for (int d = 1; d < lanes; d <<= 1) amax = fmaxf(amax, __shfl_xor(amax, d));
    float s = amax / 6.0f;
    if (scale_bf16) s = bf16_to_f32(f32_to_bf16(s));
    uint32_t word = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t c = s > 0.0f ? e2m1_code(v[j] / s) : 0u;
      word |= c << (4 * j);
    }
    codes[w] = word;
    if ((threadIdx.x & (lanes - 1)) == 0) {
      const int64_t g = w / lanes;
      if (scale_bf16)
        ((uint16_t *)scales)[g] = f32_to_bf16(s);
      else
        ((float *)scales)[g] = s;
    }
  }
}

hipError_t launch_pack_rows(const void *src, int src_dtype, int64_t rows, int64_t dim, int group,
                            int scale_dtype, void *codes, void *scales, hipStream_t st) {
  const int64_t words = rows * (dim / 8);
  if (words <= 0) return hipSuccess;
  int64_t blocks = (words + 255) / 256;
  if (blocks > 65536) blocks = 65536;
  hipLaunchKernelGGL(
      (src_dtype == HS_F32 ? pack_rows_kernel<HS_F32> : pack_rows_kernel<HS_BF16>),
      dim3((unsigned)blocks), dim3(256), 0, st, (const uint8_t *)src, words, group / 8,
      (int)(scale_dtype == HS_BF16), (uint32_t *)codes, scales);
  return hipGetLastError();
}

}  // namespace hs
