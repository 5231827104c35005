// Adjustments of rows of scores: penalties for repeated tokens, biases, allow masks.
//
// One workgroup per (row, tile of columns).  It marks the tile's seen tokens and
// biased columns in LDS from the row's lists (counts by integer atomics, the last bias
// entry by an atomic max: no order of the entries matters), then streams the tile:
// each score is read once and written once.  Bound by those bytes; every tile of a row
// reads the row's lists again, from L2.
#include "rows.h"

namespace hs {

namespace {

constexpr int kThreads = 512;
constexpr int kTile = 8192;        // columns: two LDS arrays of 32 KiB
constexpr int kTileSmall = 2048;   // where larger ones would leave CUs idle

__device__ __forceinline__ float adjusted(float x, uint32_t mark, uint32_t entry, bool allow,
                                          float rep, float freq, float pres,
                                          const float *__restrict__ bias) {
  if (mark) {
    x = x > 0.0f ? x / rep : x * rep;
    const uint32_t n = mark & 0x7FFFFFFFu;
    if (n) x = (x - freq * (float)n) - pres;
  }
  if (entry) x += bias[entry - 1];
  return allow ? x : -__builtin_inff();
}

template <int DT, bool WIDE>
__global__ __launch_bounds__(kThreads) void adjust_kernel(
    hs_adjust a, const uint8_t *__restrict__ in, int64_t stride, uint8_t *__restrict__ out,
    int64_t out_stride, int64_t n_cols, int tile, int64_t tiles, int64_t items) {
  extern __shared__ uint32_t lds[];
  uint32_t *mark = lds, *entry = lds + tile;
  constexpr int ES = DT == HS_F32 ? 4 : 2, C = 16 / ES;
  const int tid = threadIdx.x;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t r = item / tiles, c0 = (item - r * tiles) * tile;
    const int cols = (int)(n_cols - c0 < tile ? n_cols - c0 : tile);
    int64_t s0 = 0, s1 = 0, b0 = 0, b1 = 0;
    if (a.seen_off) {
      s0 = a.seen_off[r];
      s1 = a.seen_off[r + 1];
      s0 = s0 < 0 ? 0 : s0;
      s1 = s1 > a.n_seen ? a.n_seen : s1;
    }
    if (a.bias_off) {
      b0 = a.bias_off[r];
      b1 = a.bias_off[r + 1];
      b0 = b0 < 0 ? 0 : b0;
      b1 = b1 > a.n_bias ? a.n_bias : b1;
    }
    const bool lists = s0 < s1 || b0 < b1;
    if (lists) {
      for (int i = tid; i < tile; i += kThreads) {
        mark[i] = 0u;
        entry[i] = 0u;
      }
      __syncthreads();
      const int64_t late = s0 + (a.prompt_len ? a.prompt_len[r] : 0);
      for (int64_t e = s0 + tid; e < s1; e += kThreads) {
        const int64_t c = (int64_t)a.seen[e] - c0;
        if (c >= 0 && c < cols) {
          if (e >= late)
            atomicAdd(&mark[c], 1u);
          else
            atomicOr(&mark[c], 0x80000000u);
        }
      }
      for (int64_t e = b0 + tid; e < b1; e += kThreads) {
        const int64_t c = (int64_t)a.bias_id[e] - c0;
        if (c >= 0 && c < cols) atomicMax(&entry[c], (uint32_t)(e - b0) + 1u);
      }
      __syncthreads();
    }
    const float rep = a.repetition ? a.repetition[r] : 1.0f;
    const float freq = a.frequency ? a.frequency[r] : 0.0f;
    const float pres = a.presence ? a.presence[r] : 0.0f;
    const float *bias = a.bias + b0;
    const uint32_t *allow = a.allow ? a.allow + r * a.allow_stride + (c0 >> 5) : nullptr;
    const uint8_t *src = in + (r * stride + c0) * ES;
    uint8_t *dst = out + (r * out_stride + c0) * ES;
    if constexpr (WIDE) {
      const int vecs = cols / C;
      for (int v = tid; v < vecs; v += kThreads) {
        const int c = v * C;
        RawCols<DT, C> raw;
        float x[C];
        raw.load(src, c);
        const uint32_t bits = allow ? allow[c >> 5] >> (c & 31) : ~0u;
        raw.decode(x);
#pragma unroll
        for (int j = 0; j < C; ++j)
          x[j] = adjusted(x[j], lists ? mark[c + j] : 0u, lists ? entry[c + j] : 0u,
                          (bits >> j) & 1u, rep, freq, pres, bias);
        *(u32x4v_t *)(dst + (int64_t)c * ES) = round_cols<DT, C>(x);
      }
    }
    for (int c = (WIDE ? cols / C * C : 0) + tid; c < cols; c += kThreads) {
      const bool ok = !allow || ((allow[c >> 5] >> (c & 31)) & 1u);
      store_col<DT>(dst, c, adjusted(load_col<DT>(src, c), lists ? mark[c] : 0u,
                                     lists ? entry[c] : 0u, ok, rep, freq, pres, bias));
    }
    __syncthreads();   // (the next item clears the marks)
  }
}

}  // namespace

hipError_t launch_adjust(const hs_adjust *a, const void *in, int64_t stride, void *out,
                         int64_t out_stride, int dtype, int64_t n_rows, int64_t n_cols,
                         hipStream_t st) {
  if (n_rows <= 0 || n_cols <= 0) return hipSuccess;
  const int es = dtype == HS_F32 ? 4 : 2;
  const int tile = n_rows * ((n_cols + kTile - 1) / kTile) < 1024 ? kTileSmall : kTile;
  const int64_t tiles = (n_cols + tile - 1) / tile, items = n_rows * tiles;
  const bool wide = ((uintptr_t)in % 16) == 0 && ((uintptr_t)out % 16) == 0 &&
                    (n_rows == 1 || (stride * es % 16 == 0 && out_stride * es % 16 == 0));
  const dim3 g((unsigned)(items < (1 << 20) ? items : (1 << 20))), b(kThreads);
  const size_t lds = (size_t)tile * 8;
  auto kernel = dtype == HS_F32 ? (wide ? adjust_kernel<HS_F32, true> : adjust_kernel<HS_F32, false>)
                                : (wide ? adjust_kernel<HS_BF16, true>
                                        : adjust_kernel<HS_BF16, false>);
  hipLaunchKernelGGL(kernel, g, b, lds, st, *a, (const uint8_t *)in, stride, (uint8_t *)out,
                     out_stride, n_cols, tile, tiles, items);
  return hipGetLastError();
}

}  // namespace hs
