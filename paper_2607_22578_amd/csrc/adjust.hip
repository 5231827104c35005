// Adjustments of rows of scores: penalties for repeated tokens, biases, allow masks.
//
// A workgroup takes a range of a row's columns.  It gathers the row's seen tokens and
// biased columns of that range in an LDS hash table (counts by integer atomics, the
// last bias entry by an atomic max: no order of the entries matters), works out their
// adjusted scores, one thread for each, and marks them in a bitmap; then it streams the
// range without a barrier: each score is read once and written once, the marked ones
// replaced from the table.  A range with more marked columns than the table holds is
// taken in halves.
// Bound by the scores' bytes.  256 x 131,072 bf16, 1,000 tokens seen and 25 biases on
// average, a mask per row (140 MB): 39 us, 3.6 TB/s (35 without lists).  (Counts in two words per column of a
// 4,096-column tile took 53 to 70 us, with the chain of list, marks and scores paid
// for each tile.)  Each range reads all of its row's entries: 1 x 131,072 fp32 with 1,000, 10,000 and
// 100,000 of them 11, 18 and 105 us; 256 rows with 20,000 each, taken in halves too, 1,470 us.
#include "rows.h"

namespace hs {

int persistent_grid();

namespace {

constexpr int kThreads = 256;
constexpr int kRangeMax = 32768;   // columns of a workgroup: a bitmap of 4 KiB
constexpr int kRangeMin = 1024;    // where longer ones would leave CUs idle
constexpr int kSlots = 2048;       // of the table: 24 KiB
constexpr int kMarkedMax = 1536;   // entries that it takes
constexpr int kInFlight = 2;       // accesses of a thread (and as many of the next)

__device__ __forceinline__ float adjusted(float x, uint32_t mark, uint32_t entry, float rep,
                                          float freq, float pres,
                                          const float *__restrict__ bias) {
  if (mark) {
    x = x > 0.0f ? x / rep : x * rep;
    const uint32_t n = mark & 0x7FFFFFFFu;
    if (n) x = (x - freq * (float)n) - pres;
  }
  if (entry) x += bias[entry - 1];
  return x;
}

__device__ __forceinline__ uint32_t first_slot(uint32_t c) {
  return (c * 2654435761u) >> 21;   // (Fibonacci hashing to 2^11)
}

struct __align__(16) Table {
  uint32_t key[kSlots];     // column - lo + 1; 0: empty
  uint32_t mark[kSlots];    // times seen after the prompt and, in bit 31, in it; then the
                            // column's adjusted score
  uint32_t entry[kSlots];   // last bias entry + 1
  uint32_t marked[kRangeMax / 32];
  int count;

  // Slot of column c (entered if it is not there); -1 once the table is full.
  __device__ __forceinline__ int enter(uint32_t c) {
    uint32_t s = first_slot(c);
    for (;;) {
      uint32_t k = __hip_atomic_load(&key[s], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      if (k == 0u) {
        if (__hip_atomic_load(&count, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) >= kMarkedMax)
          return -1;   // (a few more than that may get in)
        k = atomicCAS(&key[s], 0u, c + 1u);
        if (k == 0u) {
          atomicAdd(&count, 1);
          return (int)s;
        }
      }
      if (k == c + 1u) return (int)s;
      s = (s + 1u) & (kSlots - 1);
    }
  }

  __device__ __forceinline__ float value(uint32_t c) const {
    uint32_t s = first_slot(c);
    while (key[s] != c + 1u) s = (s + 1u) & (kSlots - 1);
    return __uint_as_float(mark[s]);
  }
};
// threads that see room at the same time: the table never fills up, so searches end
static_assert(kMarkedMax + kThreads < kSlots, "an empty slot is always left");

// WIDE: rows have 16 bytes at least.
template <int DT, bool WIDE>
__global__ __launch_bounds__(kThreads) void adjust_kernel(
    hs_adjust a, const uint8_t *__restrict__ in, int64_t stride, uint8_t *__restrict__ out,
    int64_t out_stride, int64_t n_cols, int range, int64_t ranges, int64_t items) {
  __shared__ Table t;
  constexpr int ES = DT == HS_F32 ? 4 : 2, C = 16 / ES, U = kInFlight, L = 4;
  const int tid = threadIdx.x;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t r = item / ranges, first = (item - r * ranges) * range;
    const int64_t last = first + range < n_cols ? first + range : n_cols;
    int64_t s0 = 0, s1 = 0, b0 = 0, b1 = 0;
    if (a.seen_off) {
      s0 = a.seen_off[r];
      s1 = a.seen_off[r + 1];
      s0 = s0 < 0 ? 0 : s0;
      s1 = s1 > a.n_seen ? a.n_seen : s1;
      s0 = s0 > s1 ? s1 : s0;   // (entries are counted on from here: no overflow)
    }
    if (a.bias_off) {
      b0 = a.bias_off[r];
      b1 = a.bias_off[r + 1];
      b0 = b0 < 0 ? 0 : b0;
      b1 = b1 > a.n_bias ? a.n_bias : b1;
      b0 = b0 > b1 ? b1 : b0;
    }
    const bool lists = s0 < s1 || b0 < b1;
    const int64_t late = s0 + (a.prompt_len ? a.prompt_len[r] : 0);
    const float rep = a.repetition ? a.repetition[r] : 1.0f;
    const float freq = a.frequency ? a.frequency[r] : 0.0f;
    const float pres = a.presence ? a.presence[r] : 0.0f;
    const uint8_t *src = in + r * stride * ES;
    uint8_t *dst = out + r * out_stride * ES;
    const uint32_t *allow = a.allow ? a.allow + r * a.allow_stride : nullptr;
    // the first entries of the lists, and below the first scores of the range, are on
    // their way before the table is ready; accesses outside are made at the row's start
    int32_t id0[L], bias0 = -1;
    auto fetch = [&](int64_t e0, int32_t *id) {
#pragma unroll
      for (int u = 0; u < L; ++u) {
        const int64_t e = e0 + u * kThreads;
        id[u] = e < s1 ? a.seen[e] : -1;
      }
    };
    fetch(s0 + tid, id0);
    if (b0 + tid < b1) bias0 = a.bias_id[b0 + tid];
    RawCols<DT, C> raw[U];
    uint32_t bits[U];
    const uint32_t *words = allow ? allow : (const uint32_t *)(((uintptr_t)src + 3) & ~(uintptr_t)3);
    for (int64_t lo = first, hi = last; lo < last; lo = hi, hi = last) {
      auto load = [&](int v0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          int64_t c = lo + (int64_t)(v0 + u * kThreads) * C;
          c = c + C <= last ? c : 0;
          raw[u].load(src, c);
          bits[u] = words[c >> 5] >> (c & 31);
        }
      };
      if constexpr (WIDE) load(tid);
      // the marked columns of [lo, hi)
      while (lists) {
        const uint4 zero = {0u, 0u, 0u, 0u};
        for (int i = tid; i < kSlots / 4; i += kThreads)
          ((uint4 *)t.key)[i] = ((uint4 *)t.mark)[i] = ((uint4 *)t.entry)[i] = zero;
        for (int i = tid; i < (int)(hi - lo + 31) / 32; i += kThreads) t.marked[i] = 0u;
        if (tid == 0) t.count = 0;
        __syncthreads();
        for (int64_t e0 = s0 + tid; e0 < s1; e0 += L * kThreads) {
          int32_t id[L];
          if (e0 < s0 + kThreads) {
#pragma unroll
            for (int u = 0; u < L; ++u) id[u] = id0[u];
          } else {
            fetch(e0, id);
          }
#pragma unroll 1
          for (int u = 0; u < L; ++u) {
            int32_t c = id[0];
#pragma unroll
            for (int w = 0; w + 1 < L; ++w) id[w] = id[w + 1];
            if (c < lo || c >= hi) continue;   // (no id is below 0: lo >= 0)
            const int s = t.enter((uint32_t)(c - lo));
            if (s < 0) break;
            if (e0 + u * kThreads >= late)
              atomicAdd(&t.mark[s], 1u);
            else
              atomicOr(&t.mark[s], 0x80000000u);
          }
        }
        for (int64_t e = b0 + tid; e < b1; e += kThreads) {
          const int32_t c = e < b0 + kThreads ? bias0 : a.bias_id[e];
          if (c < lo || c >= hi) continue;
          const int s = t.enter((uint32_t)(c - lo));
          if (s < 0) break;
          atomicMax(&t.entry[s], (uint32_t)(e - b0) + 1u);
        }
        __syncthreads();
        if (t.count < kMarkedMax) break;
        // (a full table may lack entries; ranges of kRangeMin columns always fit)
        hi = lo + ((hi - lo) / 2 + 31) / 32 * 32;
        __syncthreads();
      }
      if (lists) {
        for (int i = tid; i < kSlots; i += kThreads) {
          const uint32_t k = t.key[i];
          if (k == 0u) continue;
          const uint32_t c = k - 1u;
          t.mark[i] = __float_as_uint(adjusted(load_col<DT>(src, lo + c), t.mark[i], t.entry[i],
                                               rep, freq, pres, a.bias + b0));
          atomicOr(&t.marked[c >> 5], 1u << (c & 31));
        }
        __syncthreads();
      }
      // the stream: the thread's next U accesses in flight while U are done
      const int cols = (int)(hi - lo), vecs = WIDE ? cols / C : 0;
      if constexpr (WIDE) {
        for (int v0 = tid; v0 < vecs; v0 += U * kThreads) {
          RawCols<DT, C> now[U];
          uint32_t ok[U];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            now[u] = raw[u];
            ok[u] = allow ? bits[u] : ~0u;
          }
          load(v0 + U * kThreads);
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int v = v0 + u * kThreads, c = v * C;
            if (v >= vecs) break;
            float x[C];
            now[u].decode(x);
            uint32_t here = lists ? t.marked[c >> 5] >> (c & 31) & ((1u << C) - 1u) : 0u;
            while (here) {
              const int j = __builtin_ctz(here);
              here &= here - 1u;
              const float y = t.value((uint32_t)(c + j));
#pragma unroll
              for (int w = 0; w < C; ++w) x[w] = w == j ? y : x[w];
            }
#pragma unroll
            for (int j = 0; j < C; ++j) x[j] = (ok[u] >> j) & 1u ? x[j] : -__builtin_inff();
            store_cols(dst + (lo + c) * ES, round_cols<DT, C>(x));
          }
        }
      }
      for (int c = vecs * C + tid; c < cols; c += kThreads) {
        const int64_t at = lo + c;
        const bool ok = !allow || ((allow[at >> 5] >> (at & 31)) & 1u);
        const bool here = lists && ((t.marked[c >> 5] >> (c & 31)) & 1u);
        const float x = here ? t.value((uint32_t)c) : load_col<DT>(src, at);
        store_col<DT>(dst, at, ok ? x : -__builtin_inff());
      }
      __syncthreads();   // (the next range clears the table)
    }
  }
}

}  // namespace

hipError_t launch_adjust(const hs_adjust *a, const void *in, int64_t stride, void *out,
                         int64_t out_stride, int dtype, int64_t n_rows, int64_t n_cols,
                         hipStream_t st) {
  if (n_rows <= 0 || n_cols <= 0) return hipSuccess;
  const int es = dtype == HS_F32 ? 4 : 2;
  // ranges: as long as leaves about five workgroups per CU (as many as the LDS holds)
  int64_t range = n_rows * n_cols / (5 * (int64_t)persistent_grid());
  range = (range + kRangeMin - 1) / kRangeMin * kRangeMin;
  range = range < kRangeMin ? kRangeMin : range > kRangeMax ? kRangeMax : range;
  const int64_t ranges = (n_cols + range - 1) / range, items = n_rows * ranges;
  const bool wide = n_cols * es >= 16;
  const dim3 g((unsigned)(items < (1 << 20) ? items : (1 << 20))), b(kThreads);
  auto kernel = dtype == HS_F32 ? (wide ? adjust_kernel<HS_F32, true> : adjust_kernel<HS_F32, false>)
                                : (wide ? adjust_kernel<HS_BF16, true>
                                        : adjust_kernel<HS_BF16, false>);
  hipLaunchKernelGGL(kernel, g, b, 0, st, *a, (const uint8_t *)in, stride, (uint8_t *)out,
                     out_stride, n_cols, (int)range, ranges, items);
  return hipGetLastError();
}

}  // namespace hs
