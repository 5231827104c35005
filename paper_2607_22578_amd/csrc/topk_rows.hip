// The k best columns of materialised rows of scores.
//
// Phase 1 (rows above 32,768 columns): the largest score of every strip of 32 or 64
// columns, and of every 64 strips; nothing but a stream over the scores.
// Phase 2: a workgroup per row.  A score that k of those maxima (or of its threads'
// maxima over them) reach is a lower bound of the k-th best, and a close one while
// there are many more of them than k; only the strips that reach it are read again, and
// the few columns in them that reach it are ranked by counting.  Shorter rows are their
// own maxima.  Where too many columns reach the bound (equal scores) the k-th best
// score is found bit by bit, and the columns that have it are taken in ascending order.
// Loops are short on purpose: with one workgroup on a CU, fetching straight-line code
// took longer than reading the maxima twice (17 against 11 us, 1 x 32,000, k = 50).
// Floor: the scores, read once.  24 x 1M fp32, k = 100 (96 MB): 17 us for the strips, 5.6
// TB/s, and 12 for the selection, which is latency: 24 workgroups, a few dependent
// passes.  1 x 32,000, k = 50: 10 us.  Above k = 256 the bound takes a pass for each bit: 24 x
// 1M, k = 1,024 102 us.  24 x 1M whose 5,000 equal best lie at the rows' ends: 586 us.
#include "rows.h"

namespace hs {

namespace {

constexpr int kRowCols = 32768;    // longest row done without strips
constexpr int kStripThreads = 256;
constexpr int kReads = 8;          // accesses of a strip, 16 bytes each
constexpr int kSuper = 64;         // strips that share a maximum of the second level: a wave's
constexpr int kListMax = 4096;     // strips, or groups of them, that reach the bound

// Ordered score; 0 (below every real one) for -inf and NaN, which are never taken.
__device__ __forceinline__ uint32_t taken_score(float v) {
  return v > -__builtin_inff() ? ord_score(v) : 0u;
}

template <int DT, bool WIDE>
constexpr __host__ __device__ int access_cols() {
  return WIDE ? (DT == HS_F32 ? 4 : 8) : 1;
}

// f(score, column) for the columns of U accesses (C columns from col[u] on, which may end
// past the row or lie past it).  All loads are in flight together: those outside are
// made at the row's start instead.  (Rows have at least C columns.)
template <int DT, bool WIDE, int U, class F>
__device__ __forceinline__ void visit(const uint8_t *row, const int64_t *col, int64_t n_cols,
                                      F f) {
  constexpr int C = access_cols<DT, WIDE>();
  if constexpr (WIDE) {
    RawCols<DT, WIDE ? C : 4> raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u].load(row, col[u] + C <= n_cols ? col[u] : 0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (col[u] + C <= n_cols) {
        float v[C];
        raw[u].decode(v);
#pragma unroll
        for (int j = 0; j < C; ++j) f(v[j], col[u] + j);
      } else {
#pragma unroll 1
        for (int64_t c = col[u]; c < n_cols; ++c) f(load_col<DT>(row, c), c);
      }
    }
  } else {
    float v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load_col<DT>(row, col[u] < n_cols ? col[u] : 0);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (col[u] < n_cols) f(v[u], col[u]);
  }
}

// ---------------------------------------------------------------- strips
//
// Strip j = 256 t + i of a row: accesses i, i + 256, ... of tile t.  The row's maxima in
// `maxima`: n1 of strips, then n1 / 64 of groups of 64 strips.
template <int DT>
__global__ __launch_bounds__(kStripThreads) void strip_maxima_kernel(
    const uint8_t *__restrict__ scores, int64_t stride, int64_t n_cols, int64_t tiles,
    int64_t items, uint32_t *__restrict__ maxima) {
  constexpr int ES = DT == HS_F32 ? 4 : 2, C = access_cols<DT, true>();
  const int64_t n1 = tiles * kStripThreads, per_row = n1 + n1 / kSuper;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t r = item / tiles, t = item - r * tiles;
    const uint8_t *row = scores + r * stride * ES;
    int64_t col[kReads];
#pragma unroll
    for (int i = 0; i < kReads; ++i)
      col[i] = ((t * kReads + i) * kStripThreads + threadIdx.x) * C;
    float mx = -__builtin_inff();
    visit<DT, true, kReads>(row, col, n_cols,
                            [&](float v, int64_t) { mx = fmaxf(mx, v); });   // (a NaN loses)
    uint32_t o = taken_score(mx);
    const int64_t j = t * kStripThreads + threadIdx.x;
    maxima[r * per_row + j] = o;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t other = __shfl_xor(o, d);
      o = other > o ? other : o;
    }
    if ((threadIdx.x & 63) == 0) maxima[r * per_row + n1 + j / kSuper] = o;
  }
}

// ---------------------------------------------------------------- selection

// A score that at least k of 64 E values reach, found by one wave bit by bit from the
// top until hardly more than k do.
template <int E>
__device__ __forceinline__ uint32_t bound_of(const uint32_t *v, int k) {
  uint32_t t = 0u;
#pragma unroll 1
  for (int b = 31; b >= 0; --b) {
    const uint32_t c = t | (1u << b);
    int n = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) n += __popcll(__builtin_amdgcn_ballot_w64(v[i] >= c));
    if (n >= k) {
      t = c;
      if (n <= k + k / 8) break;
    }
  }
  return t;
}

// The same for T maxima in LDS, combined first to the fewest that are 3 k or more: fewer
// ballots, and the bound still lets 1.2 k scores through, hardly more.
template <int T>
__device__ __forceinline__ uint32_t bound_of_maxima(const uint32_t *maxima, int lane, int k) {
  constexpr int E = T / 64;
  uint32_t v[E];
#pragma unroll
  for (int i = 0; i < E; ++i) v[i] = maxima[i * 64 + lane];
  if (E >= 16 && 3 * k > T / 2) return bound_of<E>(v, k);
#pragma unroll
  for (int i = 0; i < E / 2; ++i) v[i] = v[i] > v[i + E / 2] ? v[i] : v[i + E / 2];
  if (3 * k > T / 4) return bound_of<E / 2>(v, k);
#pragma unroll
  for (int i = 0; i < E / 4; ++i) v[i] = v[i] > v[i + E / 4] ? v[i] : v[i + E / 4];
  return bound_of<E / 4>(v, k);
}

// Workgroups of T threads, a row at a time.  LEVELS: 0, the row is its own maxima; 1 and
// 2, the maxima of n1 strips or of n1 / 64 groups of them are searched (n1 is a multiple
// of 256).
template <int DT, bool WIDE, int LEVELS, int T>
__global__ __launch_bounds__(T) void select_rows_kernel(
    const uint8_t *__restrict__ scores, int64_t stride, int64_t n_rows, int64_t n_cols, int k,
    const uint32_t *__restrict__ maxima, int64_t n1, float *__restrict__ out_s,
    int32_t *__restrict__ out_i) {
  constexpr int ES = DT == HS_F32 ? 4 : 2, C = access_cols<DT, WIDE>();
  constexpr int CAP = T * 6;   // (at least k - 1 keys and T columns of a tie)
  __shared__ uint64_t buf[CAP];
  __shared__ uint32_t group[T];
  __shared__ uint32_t strip[LEVELS > 0 ? kListMax : 1], super[LEVELS > 1 ? kListMax : 1];
  __shared__ uint32_t bound;
  __shared__ int count, strips, supers;
  const int tid = threadIdx.x, lane = tid & 63;
  for (int64_t r = blockIdx.x; r < n_rows; r += gridDim.x) {
    const uint8_t *row = scores + r * stride * ES;
    const uint32_t *strip_max = maxima + r * (n1 + n1 / kSuper), *super_max = strip_max + n1;
    // f(ordered score, column) for the thread's columns of the whole row
    auto each_of_row = [&](auto f) {
      for (int64_t i = (int64_t)tid * C; i < n_cols; i += 4 * T * C) {
        const int64_t col[4] = {i, i + T * C, i + 2 * T * C, i + 3 * T * C};
        visit<DT, WIDE, 4>(row, col, n_cols,
                           [&](float v, int64_t c) { f(taken_score(v), (uint32_t)c); });
      }
    };
    // f(ordered score, index) for the thread's maxima of the level that is searched
    auto each_max = [&](auto f) {
      if constexpr (LEVELS == 0) {
        each_of_row(f);
      } else {
        const uint32_t *m = LEVELS == 1 ? strip_max : super_max;
        const int64_t n = LEVELS == 1 ? n1 : n1 / kSuper;
        if (n <= 8 * T) {   // (one by one: as many threads as can have a maximum)
#pragma unroll 4
          for (int64_t i = tid; i < n; i += T) f(m[i], (uint32_t)i);
        } else {
#pragma unroll 4
          for (int64_t i = tid; i < n / 4; i += T) {   // (n1 / 64 is a multiple of 4, too)
            const WordsAt<4> w = ((const WordsAt<4> *)m)[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) f(w.w[j], (uint32_t)(4 * i + j));
          }
        }
      }
    };
    // f(ordered score, column) for the thread's columns that may reach the bound
    auto each_col = [&](auto f) {
      if (LEVELS == 0 || strips > kListMax) {
        each_of_row(f);
        return;
      }
      const int all = strips * kReads;
      for (int i0 = tid; i0 < all; i0 += 4 * T) {
        int64_t col[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int i = i0 + u * T;
          const uint32_t j = strip[i < all ? i / kReads : 0];
          const int64_t at = (int64_t)(j / kStripThreads) * kReads + i % kReads;
          col[u] = i < all ? (at * kStripThreads + j % kStripThreads) * C : n_cols;
        }
        visit<DT, WIDE, 4>(row, col, n_cols,
                           [&](float v, int64_t c) { f(taken_score(v), (uint32_t)c); });
      }
    };
    // How many of the scores that `each` visits pass f; `count` is left at that.
    auto tally = [&](auto each, auto f) {
      __syncthreads();
      if (tid == 0) count = 0;
      __syncthreads();
      int n = 0;
      each([&](uint32_t o, uint32_t) { n += f(o) ? 1 : 0; });
      if (n) atomicAdd(&count, n);
      __syncthreads();
      return count;
    };
    uint32_t b = 0u;
    if (k <= T / 4) {
      uint32_t mx = 0u;
      each_max([&](uint32_t o, uint32_t) { mx = o > mx ? o : mx; });
      group[tid] = mx;
      __syncthreads();
      if (tid < 64) {
        const uint32_t t = bound_of_maxima<T>(group, lane, k);
        if (lane == 0) bound = t;
      }
      __syncthreads();
      b = bound;
    } else {
#pragma unroll 1
      for (int i = 31; i >= 0; --i) {
        const uint32_t c = b | (1u << i);
        const int n = tally(each_max, [&](uint32_t o) { return o >= c; });
        if (n >= k) {
          b = c;
          if (n <= k + k / 8) break;   // (the same for every thread)
        }
      }
    }
    b = b > 0u ? b : 1u;
    // lists the strips that reach `least`
    auto gather = [&](uint32_t least) {
      __syncthreads();
      if (tid == 0) count = strips = supers = 0;
      __syncthreads();
      auto list = [&](uint32_t *to, int *n, uint32_t j) {
        const int at = atomicAdd(n, 1);
        if (at < kListMax) to[at] = j;
      };
      if constexpr (LEVELS == 1) {
        each_max([&](uint32_t o, uint32_t j) {
          if (o >= least) list(strip, &strips, j);
        });
        __syncthreads();
      }
      if constexpr (LEVELS == 2) {
        each_max([&](uint32_t o, uint32_t j) {
          if (o >= least) list(super, &supers, j);
        });
        __syncthreads();
        if (supers > kListMax) {
          if (tid == 0) strips = kListMax + 1;   // (the whole row)
        } else {
#pragma unroll 4
          for (int i = tid; i < supers * kSuper; i += T) {
            const uint32_t j = super[i / kSuper] * kSuper + i % kSuper;
            if (strip_max[j] >= least) list(strip, &strips, j);
          }
        }
        __syncthreads();
      }
    };
    gather(b);
    int m = CAP + 1;   // (more strips than the list holds: too many columns)
    if (LEVELS == 0 || strips <= kListMax) {
      each_col([&](uint32_t o, uint32_t c) {
        if (o >= b) {
          const int at = atomicAdd(&count, 1);
          if (at < CAP) buf[at] = (uint64_t)o << 32 | ~c;
        }
      });
      __syncthreads();
      m = count;
    }
    if (m > CAP || m > 2 * k + 512) {   // (or too many to rank: it takes m^2 reads)
      // t: the k-th best score; often the bound itself (equal scores).  Those above it are
      // in few strips.
      gather(b + 1u);
      uint32_t t = b;
      int above = tally(each_col, [&](uint32_t o) { return o > t; });
      if (above >= k) {
        t = 0u;
#pragma unroll 1
        for (int i = 31; i >= 0; --i) {
          const uint32_t c = t | (1u << i);
          if (tally(each_col, [&](uint32_t o) { return o >= c; }) >= k) t = c;
        }
      }
      __syncthreads();
      if (tid == 0) count = 0;
      __syncthreads();
      each_col([&](uint32_t o, uint32_t c) {
        if (o > t) buf[atomicAdd(&count, 1)] = (uint64_t)o << 32 | ~c;   // (below k of them)
      });
      __syncthreads();
      // columns of score t, in ascending chunks, until there are k keys
      for (int64_t c0 = 0; c0 < n_cols && count < k; c0 += 4 * T) {
        bool tie[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int64_t c = c0 + u * T + tid;
          tie[u] = c < n_cols && taken_score(load_col<DT>(row, c)) == t;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {   // (T columns at a time: few more than needed)
          __syncthreads();              // (everyone has seen the count)
          if (tie[u]) buf[atomicAdd(&count, 1)] = (uint64_t)t << 32 | ~(uint32_t)(c0 + u * T + tid);
          __syncthreads();
          if (count >= k) break;
        }
      }
      m = count;
    }
    // rank = keys above (they are distinct)
    for (int u = tid; u < m; u += T) {
      const uint64_t key = buf[u];
      int rank = 0;
#pragma unroll 8
      for (int j = 0; j < m; ++j) rank += buf[j] > key ? 1 : 0;
      if (rank < k) {
        float sc;
        int32_t c;
        decode_key(key, sc, c);
        out_s[r * k + rank] = sc;
        out_i[r * k + rank] = c;
      }
    }
    for (int j = m + tid; j < k; j += T) {
      out_s[r * k + j] = -__builtin_inff();
      out_i[r * k + j] = -1;
    }
    __syncthreads();
  }
}

int64_t strip_tiles(int64_t n_cols, int cols) {
  const int64_t tile = (int64_t)kStripThreads * cols;
  return (n_cols + tile - 1) / tile;
}

template <int DT, bool WIDE>
hipError_t launch_topk_t(const void *scores, int64_t stride, int64_t n_rows, int64_t n_cols, int k,
                         void *ws, float *out_s, int32_t *out_i, hipStream_t st) {
  const dim3 g((unsigned)(n_rows < 65536 ? n_rows : 65536));
  const uint8_t *in = (const uint8_t *)scores;
  if (n_cols <= kRowCols) {
    // (256 threads do for 4,096 columns while their maxima are four times k)
    if (n_cols <= 4096 && k <= 64)
      hipLaunchKernelGGL((select_rows_kernel<DT, WIDE, 0, 256>), g, dim3(256), 0, st, in,
                         stride, n_rows, n_cols, k, nullptr, 0, out_s, out_i);
    else
      hipLaunchKernelGGL((select_rows_kernel<DT, WIDE, 0, 1024>), g, dim3(1024), 0, st, in,
                         stride, n_rows, n_cols, k, nullptr, 0, out_s, out_i);
    return hipGetLastError();
  }
  if constexpr (WIDE) {   // (rows this long are)
    const int64_t tiles = strip_tiles(n_cols, access_cols<DT, WIDE>() * kReads);
    const int64_t items = n_rows * tiles, n1 = tiles * kStripThreads;
    hipLaunchKernelGGL((strip_maxima_kernel<DT>),
                       dim3((unsigned)(items < (1 << 20) ? items : (1 << 20))),
                       dim3(kStripThreads), 0, st, in, stride, n_cols, tiles, items,
                       (uint32_t *)ws);
    // (few strips are searched themselves: a step less, and a closer bound; groups of
    // them while there are four times k: below, their bound would be loose)
    if (n1 > 32768 && n1 / kSuper >= 4 * (int64_t)k)
      hipLaunchKernelGGL((select_rows_kernel<DT, WIDE, 2, 1024>), g, dim3(1024), 0, st, in, stride,
                         n_rows, n_cols, k, (const uint32_t *)ws, n1, out_s, out_i);
    else
      hipLaunchKernelGGL((select_rows_kernel<DT, WIDE, 1, 1024>), g, dim3(1024), 0, st, in, stride,
                         n_rows, n_cols, k, (const uint32_t *)ws, n1, out_s, out_i);
  }
  return hipGetLastError();
}

}  // namespace

size_t topk_rows_workspace_bytes(int64_t n_rows, int64_t n_cols, int k) {
  (void)k;
  if (n_cols <= kRowCols) return 256;
  // (strips of 32 columns; bf16 ones may have 64)
  const int64_t n1 = strip_tiles(n_cols, 32) * kStripThreads;
  return (size_t)(n_rows > 0 ? n_rows : 1) * (size_t)(n1 + n1 / kSuper) * 4;
}

hipError_t launch_topk_rows(const void *scores, int dtype, int64_t stride, int64_t n_rows,
                            int64_t n_cols, int k, float *out_s, int32_t *out_i, void *ws,
                            hipStream_t st) {
  if (n_rows <= 0) return hipSuccess;
  const int es = dtype == HS_F32 ? 4 : 2;
  const bool wide = n_cols >= 16 / es;
  auto launch = dtype == HS_F32 ? (wide ? launch_topk_t<HS_F32, true> : launch_topk_t<HS_F32, false>)
                                : (wide ? launch_topk_t<HS_BF16, true>
                                        : launch_topk_t<HS_BF16, false>);
  return launch(scores, stride, n_rows, n_cols, k, ws, out_s, out_i, st);
}

}  // namespace hs
