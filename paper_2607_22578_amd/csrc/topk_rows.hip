// The k best columns of materialised rows of scores.
//
// Phase 1: work items are (row, slice of columns) as in the score kernels
// (make_split).  A workgroup streams its slice in tiles and keeps, in LDS, the keys
// (ordered score, ~column) that may be among the slice's k best: those above a
// bound that starts as the k-th largest of the threads' maxima of the first tile and
// is made exact whenever the buffer has filled.  It leaves the slice's sorted k best.
// Phase 2: the merge of the score step (topk_merge_kernel).  With one slice per row
// phase 1 writes the results itself.
// Floor: the scores, read once.
#include "rows.h"

namespace hs {

namespace {

constexpr int kThreads = 512;
constexpr int kPer = 8;                      // columns per thread and tile
constexpr int kTile = kThreads * kPer;
constexpr int kKeep = 2048;                  // keys kept from one tile to the next, at most
constexpr int kBuf = kKeep + kTile;
constexpr int kPerBuf = kBuf / kThreads;
constexpr int kListMax = 8192;               // keys of one row's lists (the merge's LDS)

struct Shared {
  uint64_t buf[kBuf];
  uint32_t maxima[kThreads];
  uint32_t sums[2][kThreads / 64];
  uint32_t bound;
  int count;
};

// The k-th largest of the 512 maxima (ordered scores), found by wave 0 bit by bit
// from the top: eight values a lane, a ballot for each.
__device__ __forceinline__ uint32_t kth_maximum(const uint32_t *maxima, int lane, int k) {
  uint32_t v[kThreads / 64];
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) v[i] = maxima[i * 64 + lane];
  uint32_t t = 0u;
  for (int b = 31; b >= 0; --b) {
    const uint32_t c = t | (1u << b);
    int n = 0;
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) n += __popcll(__builtin_amdgcn_ballot_w64(v[i] >= c));
    if (n >= k) t = c;
    if (n == k) break;
  }
  return t;
}

// Cuts the buffer's m > k keys to the k largest (in any order); returns the k-th.
__device__ uint64_t cut(Shared &s, int m, int k) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint64_t key[kPerBuf];
#pragma unroll
  for (int i = 0; i < kPerBuf; ++i) {
    const int j = i * kThreads + tid;
    key[i] = j < m ? s.buf[j] : 0ull;
  }
  uint64_t t = 0ull;
  for (int b = 63; b >= 0; --b) {
    const uint64_t c = t | (1ull << b);
    uint32_t n = 0u;
#pragma unroll
    for (int i = 0; i < kPerBuf; ++i) n += __popcll(__builtin_amdgcn_ballot_w64(key[i] >= c));
    if (lane == 0) s.sums[b & 1][wave] = n;
    __syncthreads();
    n = 0u;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) n += s.sums[b & 1][w];
    if (n >= (uint32_t)k) t = c;
    if (n == (uint32_t)k) break;   // (the same for every thread)
  }
  __syncthreads();
  if (tid == 0) s.count = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kPerBuf; ++i)
    if (key[i] >= t) s.buf[atomicAdd(&s.count, 1)] = key[i];
  __syncthreads();
  return t;
}

template <int DT, bool WIDE>
__global__ __launch_bounds__(kThreads) void topk_rows_kernel(
    const uint8_t *__restrict__ scores, int64_t stride, int64_t n_rows, int64_t n_cols, int k,
    int64_t smax, int grid, uint64_t *__restrict__ part, float *__restrict__ out_s,
    int32_t *__restrict__ out_i) {
  __shared__ Shared s;
  constexpr int ES = DT == HS_F32 ? 4 : 2, C = 16 / ES;
  const Split sp = make_split(n_rows, n_cols, 1, kTile, grid, smax);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t items = n_rows * sp.S;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t r = item / sp.S, slice = item - r * sp.S;
    const int64_t t0 = slice * sp.ntiles / sp.S, t1 = (slice + 1) * sp.ntiles / sp.S;
    const uint8_t *row = scores + r * stride * ES;
    if (tid == 0) s.count = 0;
    uint64_t floor_key = 0ull;   // only keys above it are kept
    for (int64_t t = t0; t < t1; ++t) {
      const int64_t c0 = t * kTile;
      float v[kPer];
      int64_t col[kPer];
#pragma unroll
      for (int q = 0; q < kPer; ++q) {
        col[q] = WIDE ? c0 + (int64_t)(q / C * kThreads + tid) * C + q % C
                      : c0 + (int64_t)q * kThreads + tid;
      }
      if constexpr (WIDE) {
#pragma unroll
        for (int q = 0; q < kPer; q += C) {
          if (col[q] + C <= n_cols) {
            RawCols<DT, C> raw;
            raw.load(row, col[q]);
            raw.decode(v + q);
          } else {
#pragma unroll
            for (int j = 0; j < C; ++j)
              v[q + j] = col[q + j] < n_cols ? load_col<DT>(row, col[q + j]) : -__builtin_inff();
          }
        }
      } else {
#pragma unroll
        for (int q = 0; q < kPer; ++q)
          v[q] = col[q] < n_cols ? load_col<DT>(row, col[q]) : -__builtin_inff();
      }
      if (t == t0 && k <= kThreads) {
        float mx = -__builtin_inff();
#pragma unroll
        for (int q = 0; q < kPer; ++q) mx = fmaxf(mx, v[q]);   // (a NaN loses)
        s.maxima[tid] = ord_score(mx);
        __syncthreads();
        if (wave == 0) {
          const uint32_t b = kth_maximum(s.maxima, lane, k);
          if (lane == 0) s.bound = b;
        }
      }
      __syncthreads();
      // (a key's low word is above 0, so keys of the bound's own score stay)
      if (t == t0 && k <= kThreads) floor_key = (uint64_t)s.bound << 32;
#pragma unroll
      for (int q = 0; q < kPer; ++q) {
        const uint64_t key = make_key(v[q], (uint32_t)col[q]);
        const bool keep = v[q] > -__builtin_inff() && key > floor_key;
        const uint64_t mask = __builtin_amdgcn_ballot_w64(keep);
        if (mask) {
          int base = 0;
          if (lane == 0) base = atomicAdd(&s.count, __popcll(mask));
          base = __shfl(base, 0);
          if (keep) s.buf[base + __popcll(mask & ((1ull << lane) - 1ull))] = key;
        }
      }
      __syncthreads();
      const int m = s.count;
      __syncthreads();
      if (m > kKeep) floor_key = cut(s, m, k);
    }
    __syncthreads();
    int m = s.count;
    if (m > 2 * k + 256) {
      cut(s, m, k);
      m = k;
    }
    // rank = keys above (they are distinct)
    uint64_t *list = part + item * k;
    for (int u = tid; u < m; u += kThreads) {
      const uint64_t key = s.buf[u];
      int rank = 0;
      for (int j = 0; j < m; ++j) rank += s.buf[j] > key ? 1 : 0;
      if (rank < k) {
        if (sp.S == 1) {
          float sc;
          int32_t c;
          decode_key(key, sc, c);
          out_s[r * k + rank] = sc;
          out_i[r * k + rank] = c;
        } else {
          list[rank] = key;
        }
      }
    }
    for (int j = m + tid; j < k; j += kThreads) {
      if (sp.S == 1) {
        out_s[r * k + j] = -__builtin_inff();
        out_i[r * k + j] = -1;
      } else {
        list[j] = 0ull;
      }
    }
    __syncthreads();
  }
}

}  // namespace

int persistent_grid();
hipError_t launch_lists_merge(const void *part, int64_t n_rows, int64_t n_cols, int k, int nc,
                              int64_t smax, int grid, float *out_s, int32_t *out_i,
                              hipStream_t st);

static int64_t slices_max(int k) { return kListMax / k; }

size_t topk_rows_workspace_bytes(int64_t n_rows, int64_t n_cols, int k) {
  // make_split gives at most 8 rounds of a grid of at most 1,024 workgroups
  int64_t s = (n_cols + kTile - 1) / kTile;
  if (s > slices_max(k)) s = slices_max(k);
  if (s > 8192 / (n_rows > 0 ? n_rows : 1)) s = 8192 / (n_rows > 0 ? n_rows : 1);
  if (s < 1) s = 1;
  const int64_t b = n_rows * s * k * 8;
  return (size_t)(b < 256 ? 256 : (b + 255) & ~(int64_t)255);
}

hipError_t launch_topk_rows(const void *scores, int dtype, int64_t stride, int64_t n_rows,
                            int64_t n_cols, int k, float *out_s, int32_t *out_i, void *ws,
                            hipStream_t st) {
  if (n_rows <= 0) return hipSuccess;
  const int grid = 2 * persistent_grid();
  const int64_t smax = slices_max(k);
  const Split sp = make_split(n_rows, n_cols, 1, kTile, grid, smax);
  const int64_t items = n_rows * sp.S;
  const int es = dtype == HS_F32 ? 4 : 2;
  const bool wide = ((uintptr_t)scores % 16) == 0 && (n_rows == 1 || stride * es % 16 == 0);
  auto kernel = dtype == HS_F32
                    ? (wide ? topk_rows_kernel<HS_F32, true> : topk_rows_kernel<HS_F32, false>)
                    : (wide ? topk_rows_kernel<HS_BF16, true> : topk_rows_kernel<HS_BF16, false>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)(items < 65536 ? items : 65536)), dim3(kThreads), 0,
                     st, (const uint8_t *)scores, stride, n_rows, n_cols, k, smax, grid,
                     (uint64_t *)ws, out_s, out_i);
  if (sp.S > 1)
    return launch_lists_merge(ws, n_rows, n_cols, k, kTile, smax, grid, out_s, out_i, st);
  return hipGetLastError();
}

}  // namespace hs
