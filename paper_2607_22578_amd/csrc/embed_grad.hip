// Gradient of the embedding lookup, dT[v] = scale * sum_{i: ids[i] = v} dO[i], by
// tokens sorted together with their positions.
//
//   sort    LSD radix sort of (token, position), stable, so a token's positions come
//           in ascending order; positions that stand for no token take the key
//           `rows`, behind all others.  Up to kSmallMax positions in one workgroup;
//           above, two launches per digit (counts per tile, scatter).
//   sums    the sorted places in chunks of at most 64: a wave (or, of narrow rows, a few
//           lanes) adds up the rows of its chunk for one slice of columns, place after place, in registers, and
//           writes a row whenever the token changes.  The work per wave does not depend
//           on how often tokens occur.  Tokens that reach over a chunk's end leave
//           partial sums.
//   join    partial sums of the tokens over several chunks, in chunk order.
// Every row's additions are thus in an order that the sizes and ids fix.
// Floor: dO once, dT once; the keys are small beside them.  262,144 bf16 rows of 1,024
// columns for 131,072 tokens, fp32 gradient (1,075 MB): 265 us; the sums' launch (877 MB of
// it) 190 us, 4.6 TB/s, a copy's rate; the sort 40 us beside zeros.  10,007 fp32 rows of 771
// for 50,257 (186 MB): 49 us; 2,048 bf16 rows of 1,024 for 32,000 (70 MB): 25 us, of which
// 20 are the latency of three launches, whatever zeros are written beside them.  Added to a table:
// the first 290 us (50,772 tokens occur), the second 50.
#include "rows.h"

namespace hs {

namespace {

constexpr int kSmallMax = 10240;     // positions that one workgroup sorts: 152 KiB of LDS
constexpr int kSmallWaves = 16;
constexpr int kSortWaves = 16;       // per tile
constexpr int kRounds = 4;           // keys per lane held in registers
constexpr int kDigitBits = 9;        // most bits of a digit
constexpr int kDigits = 1 << kDigitBits;
static_assert(kSortWaves * 64 == 2 * kDigits, "two threads per digit");
constexpr int kTilesMax = 64;        // tiles of the sort
constexpr int kTileMin = 1024;       // positions that make another tile worth it
constexpr int kChunk = 64;           // sorted places of one wave, at most
constexpr int kSpanMany = 24;        // chunks that a workgroup instead of a wave joins
constexpr int kJoinWaves = 8;

struct GradWs {
  uint32_t *tok[2], *pos[2];   // [n] each: sorted keys and positions
  uint32_t *hist;              // [kTilesMax][kDigits]
  uint32_t *count;             // [1]: entries of the list
  uint32_t *many;              // [chunks]: chunks where a token over many chunks begins
  uint8_t *present;            // [rows, in fours]: 1 for tokens that occur
  float *part;                 // [2 x chunks][dim]: sums of the tokens over a chunk's
                               // start (0) and end (1)
};

__host__ __device__ int64_t up256(int64_t x) { return (x + 255) & ~(int64_t)255; }

// Places per chunk: 64, or fewer while the chunks, their column slices (of 512) and, of rows
// of up to 256 columns, the chunks that share a wave would not give 2,048 waves (8 per CU).
int chunk_places(int64_t n, int64_t dim) {
  int c = kChunk, share = 1;
  while (share < 64 && dim * share <= 256) share *= 2;
  while (c > 8 && (n + c - 1) / c * ((dim + 511) / 512) / share < 2048) c >>= 1;
  return c;
}

size_t layout(int64_t n, int64_t rows, int64_t dim, void *base, GradWs *w) {
  uint8_t *p = (uint8_t *)base;
  const int64_t kb = up256(n * 4);
  const int64_t chunks = (n + chunk_places(n, dim) - 1) / chunk_places(n, dim);
  int64_t at = 0;
  for (int i = 0; i < 2; ++i) {
    if (w) w->tok[i] = (uint32_t *)(p + at);
    at += kb;
    if (w) w->pos[i] = (uint32_t *)(p + at);
    at += kb;
  }
  if (w) w->hist = (uint32_t *)(p + at);
  at += (int64_t)kTilesMax * kDigits * 4;
  if (w) w->count = (uint32_t *)(p + at);
  at += 256;
  if (w) w->many = (uint32_t *)(p + at);
  at += up256(chunks * 4);
  if (w) w->present = p + at;
  at += up256(rows);
  if (w) w->part = (float *)(p + at);
  at += up256(chunks * 2 * dim * 4);
  return (size_t)at;
}

// ---------------------------------------------------------------- rows of zeros
//
// The sort's launches leave most CUs idle, so further workgroups of theirs, and some of the
// sums' and the join's, write the rows of tokens that do not occur.
struct Zeros {
  uint8_t *table;
  int64_t first, last;    // rows that are looked at, from a multiple of 4 on
  int dim, elem;
};

// Zeros for the absent ones among rows r0 .. r0 + 3: a set bit each in `absent`.
// Neighbours are written as one span, a wave's accesses at multiples of 1 KiB, so rows of
// any width fill whole cache lines but for the span's ends.
__device__ __forceinline__ void zero_four(const Zeros &z, int64_t r0, uint32_t absent) {
  const int64_t rb = (int64_t)z.dim * z.elem;
  const u32x4v_t zero = {0u, 0u, 0u, 0u};
  while (absent) {
    const int f = __builtin_ctz(absent), len = __builtin_ctz(~(absent >> f));
    absent &= ~(((1u << len) - 1u) << f);
    uint8_t *p = z.table + (r0 + f) * rb, *end = p + len * rb;
    uint8_t *at = (uint8_t *)((uintptr_t)p & ~(uintptr_t)1023) + (threadIdx.x & 63) * 16;
    for (; at < end; at += 1024) {
      if (at >= p && at + 16 <= end) {
        stream_cols(at, zero);
      } else {
#pragma unroll 1
        for (uint8_t *e = at < p ? p : at; e < at + 16 && e < end; e += z.elem) {
          if (z.elem == 4)
            *(uint32_t *)e = 0u;
          else
            *(uint16_t *)e = 0u;
        }
      }
    }
  }
}

// The share of workgroup `wg` of `wgs`, a wave for four rows.
__device__ __forceinline__ void zero_rows(const Zeros &z, const uint8_t *present, int64_t wg,
                                          int64_t wgs) {
  const int waves = blockDim.x / 64;
  for (int64_t r = z.first + (wg * waves + (threadIdx.x >> 6)) * 4; r < z.last;
       r += wgs * waves * 4) {
    const uint32_t here = *(const uint32_t *)(present + r);
    uint32_t absent = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      absent |= r + i < z.last && !((here >> (8 * i)) & 255u) ? 1u << i : 0u;
    zero_four(z, r, __builtin_amdgcn_readfirstlane(absent));
  }
}

// ---------------------------------------------------------------- sort

__device__ __forceinline__ uint32_t token_key(const void *ids, int is64, int64_t i, int64_t rows,
                                              int64_t pad) {
  const int64_t id = load_id(ids, is64, i);
  return (uint32_t)(id >= 0 && id < rows && id != pad ? id : rows);
}

// f(key, position) for the workgroup's positions below n: four loads of a thread are in
// flight, at position 0 where there is none.
template <class ID, class F>
__device__ __forceinline__ void each_key(const ID *__restrict__ ids, int n, int64_t rows,
                                         int64_t pad, F f) {
  const int step = blockDim.x;
  for (int i0 = threadIdx.x; i0 < n; i0 += 4 * step) {
    int64_t id[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) id[u] = (int64_t)ids[i0 + u * step < n ? i0 + u * step : 0];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i0 + u * step < n)
        f((uint32_t)(id[u] >= 0 && id[u] < rows && id[u] != pad ? id[u] : rows), i0 + u * step);
  }
}

// Lanes of the wave with the same digit as this one, among the lanes in `in`.  (Every bit
// that a digit can have: a loop over those in use took three times the instructions.)
__device__ __forceinline__ uint64_t same_digit(uint32_t d, bool in) {
  const uint64_t some = __builtin_amdgcn_ballot_w64(in);
  uint32_t lo = (uint32_t)some, hi = (uint32_t)(some >> 32);
#pragma unroll
  for (int b = 0; b < kDigitBits; ++b) {
    const uint32_t mine = (uint32_t)((int32_t)(d << (31 - b)) >> 31);   // the bit, 32 times
    const uint64_t v = __builtin_amdgcn_ballot_w64(mine != 0u);
    lo &= ~((uint32_t)v ^ mine);
    hi &= ~((uint32_t)(v >> 32) ^ mine);
  }
  return (uint64_t)hi << 32 | lo;
}

// Exclusive scan of one value per thread over the first kDigits threads of a
// workgroup; `sums` holds kDigits / 64 words.  Every thread of the workgroup calls it.
__device__ __forceinline__ uint32_t scan_digits(uint32_t v, uint32_t *sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t s = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(s, d);
    if (lane >= d) s += o;
  }
  if (lane == 63 && wave < kDigits / 64) sums[wave] = s;
  __syncthreads();
  uint32_t before = 0u;
#pragma unroll
  for (int w = 0; w < kDigits / 64; ++w) before += w < wave ? sums[w] : 0u;
  return before + s - v;
}

// All passes in one workgroup, keys and positions in LDS; 16 waves, each with a
// contiguous share and its own digit counters (made exclusive over digits and waves).
// The workgroups behind the first write the rows of zeros below z.last, slabs of `slab` rows
// each, and note the tokens that occur from there to `stop` for the sums' launch, slabs of
// `noted` rows each: they find the tokens of their slabs themselves.
__global__ __launch_bounds__(kSmallWaves * 64) void grad_sort_small(
    const void *__restrict__ ids, int is64, int n, int64_t rows, int64_t pad, int bits, int passes,
    uint32_t *__restrict__ tok, uint32_t *__restrict__ pos, uint32_t *__restrict__ count, Zeros z,
    int64_t stop, int slab, int noted, uint8_t *__restrict__ present) {
  __shared__ uint32_t key[2][kSmallMax];
  __shared__ uint16_t val[2][kSmallMax];
  __shared__ uint32_t cnt[kSmallWaves][kDigits];
  __shared__ uint32_t sums[kDigits / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (blockIdx.x == 0 && tid == 0) *count = 0u;
  if (blockIdx.x > 0) {
    uint32_t *occur = key[0], *later = key[1];   // a bit per row (at most 32 kSmallMax each)
    for (int64_t s = blockIdx.x - 1; s * slab < z.last || z.last + s * noted < stop;
         s += gridDim.x - 1) {
      const int64_t first = s * slab, last = first + slab < z.last ? first + slab : z.last;
      const int64_t from = z.last + s * noted, to = from + noted < stop ? from + noted : stop;
      for (int i = tid; i < slab / 32; i += kSmallWaves * 64) occur[i] = 0u;
      for (int i = tid; i < noted / 32; i += kSmallWaves * 64) later[i] = 0u;
      __syncthreads();
      auto mark = [&](uint32_t v, int) {
        if (v >= first && v < last)
          atomicOr(&occur[(v - first) >> 5], 1u << (v & 31));
        else if (v >= from && v < to)
          atomicOr(&later[(v - from) >> 5], 1u << (v & 31));
      };
      if (is64)
        each_key((const int64_t *)ids, n, rows, pad, mark);
      else
        each_key((const int32_t *)ids, n, rows, pad, mark);
      __syncthreads();
      for (int64_t r = from + tid * 4; r < to; r += kSmallWaves * 64 * 4) {
        const uint32_t here = later[(r - from) >> 5] >> (r & 31) & 15u;
        *(uint32_t *)(present + r) = here * 0x00204081u & 0x01010101u;   // (a byte per bit)
      }
      for (int64_t r = first + wave * 4; r < last; r += kSmallWaves * 4) {
        uint32_t absent = ~(occur[(r - first) >> 5] >> (r & 31)) & 15u;
        if (last - r < 4) absent &= (1u << (last - r)) - 1u;
        zero_four(z, r, __builtin_amdgcn_readfirstlane(absent));
      }
      __syncthreads();
    }
    return;
  }
  auto enter = [&](uint32_t v, int i) {
    key[0][i] = v;
    val[0][i] = (uint16_t)i;
  };
  if (is64)
    each_key((const int64_t *)ids, n, rows, pad, enter);
  else
    each_key((const int32_t *)ids, n, rows, pad, enter);
  const int share = ((n + kSmallWaves - 1) / kSmallWaves + 63) & ~63;
  const int lo = wave * share, hi = lo + share < n ? lo + share : n;
  int from = 0;
  for (int p = 0; p < passes; ++p) {
    const int shift = p * bits;
    const uint32_t mask = (1u << bits) - 1u;
    for (int i = tid; i < kSmallWaves * kDigits; i += kSmallWaves * 64) (&cnt[0][0])[i] = 0u;
    __syncthreads();
    for (int i = lo + lane; i < hi; i += 64) atomicAdd(&cnt[wave][(key[from][i] >> shift) & mask], 1u);
    __syncthreads();
    // digit totals and their exclusive scan (512 digits in the first 8 waves)
    uint32_t mine = 0u;
    if (tid < kDigits) {
#pragma unroll
      for (int w = 0; w < kSmallWaves; ++w) mine += cnt[w][tid];
    }
    uint32_t base = scan_digits(mine, sums);
    if (tid < kDigits) {
#pragma unroll
      for (int w = 0; w < kSmallWaves; ++w) {
        const uint32_t c = cnt[w][tid];
        cnt[w][tid] = base;
        base += c;
      }
    }
    __syncthreads();
    for (int i0 = lo; i0 < hi; i0 += 64) {
      const int i = i0 + lane;
      const bool in = i < hi;
      const uint32_t k = in ? key[from][i] : 0u;
      const uint32_t d = (k >> shift) & mask;
      const uint64_t same = same_digit(d, in);
      if (in) {
        const int rank = __popcll(same & ((1ull << lane) - 1ull));
        const uint32_t at = cnt[wave][d] + rank;
        key[from ^ 1][at] = k;
        val[from ^ 1][at] = val[from][i];
      }
      wave_fence();
      if (in && (same >> lane) == 1ull) cnt[wave][d] += (uint32_t)__popcll(same);
      wave_fence();
    }
    from ^= 1;
    __syncthreads();
  }
  for (int i = tid; i < n; i += kSmallWaves * 64) {
    tok[i] = key[from][i];
    pos[i] = val[from][i];
  }
}

// Digit counts of one tile; the first pass makes the keys from the ids, and clears the
// marks of tokens that occur and the lists.  Workgroups from `tiles` on write rows of zeros (not in
// the first pass).
template <bool FIRST>
__global__ __launch_bounds__(kSortWaves * 64) void grad_count(
    const void *__restrict__ ids, int is64, const uint32_t *__restrict__ tok, int64_t n,
    int64_t tile, int tiles, int64_t rows, int64_t pad, int bits, int shift,
    uint32_t *__restrict__ hist, uint8_t *__restrict__ present, uint32_t *__restrict__ count,
    Zeros z) {
  __shared__ uint32_t cnt[kDigits];
  if ((int)blockIdx.x >= tiles) {
    zero_rows(z, present, (int64_t)blockIdx.x - tiles, (int64_t)gridDim.x - tiles);
    return;
  }
  if (FIRST) {
    if (blockIdx.x == 0 && threadIdx.x == 0) *count = 0u;
    for (int64_t i = (int64_t)blockIdx.x * kSortWaves * 64 + threadIdx.x; i < (rows + 3) / 4;
         i += (int64_t)tiles * kSortWaves * 64)
      ((uint32_t *)present)[i] = 0u;
  }
  if (threadIdx.x < kDigits) cnt[threadIdx.x] = 0u;
  __syncthreads();
  const int64_t lo = (int64_t)blockIdx.x * tile, hi = lo + tile < n ? lo + tile : n;
  const uint32_t mask = (1u << bits) - 1u;
  for (int64_t i = lo + threadIdx.x; i < hi; i += kSortWaves * 64) {
    const uint32_t k = FIRST ? token_key(ids, is64, i, rows, pad) : tok[i];
    atomicAdd(&cnt[(k >> shift) & mask], 1u);
  }
  __syncthreads();
  if (threadIdx.x < kDigits)
    hist[(int64_t)blockIdx.x * kDigits + threadIdx.x] = cnt[threadIdx.x];
}

// Stable scatter of one tile.  The tile's first place of each digit comes straight
// from the counts of all tiles: two threads per digit, 32 reads each at most, all in
// flight at once (with 128 tiles and 8 in flight they were most of the launch: 16 us for
// 262,144 positions).  The first pass also marks the tokens that occur; workgroups from
// `tiles` on write rows of zeros (not in the first pass).
template <bool FIRST>
__global__ __launch_bounds__(kSortWaves * 64) void grad_scatter(
    const void *__restrict__ ids, int is64, const uint32_t *__restrict__ tok,
    const uint32_t *__restrict__ pos, int64_t n, int64_t tile, int tiles, int64_t rows,
    int64_t pad, int bits, int shift, const uint32_t *__restrict__ hist,
    uint32_t *__restrict__ tok_out, uint32_t *__restrict__ pos_out,
    uint8_t *__restrict__ present, Zeros z) {
  __shared__ uint32_t cnt[kSortWaves][kDigits];
  __shared__ uint32_t other[2][kDigits];
  __shared__ uint32_t sums[kDigits / 64];
  if ((int)blockIdx.x >= tiles) {
    zero_rows(z, present, (int64_t)blockIdx.x - tiles, (int64_t)gridDim.x - tiles);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t mask = (1u << bits) - 1u;
  const int64_t lo = (int64_t)blockIdx.x * tile, hi = lo + tile < n ? lo + tile : n;
  const int64_t share = tile / kSortWaves;   // (a multiple of 64)
  const int64_t wlo = lo + wave * share < hi ? lo + wave * share : hi;
  const int64_t whi = wlo + share < hi ? wlo + share : hi;
  for (int i = tid; i < kSortWaves * kDigits; i += kSortWaves * 64) (&cnt[0][0])[i] = 0u;
  __syncthreads();
  // the wave's first kRounds x 64 keys stay in registers (all of them, up to 262,144
  // positions): their loads are in flight together, and with those of the counts
  uint32_t key[kRounds], val[kRounds];
  auto fetch = [&](int64_t i0) {
#pragma unroll
    for (int u = 0; u < kRounds; ++u) {
      const int64_t i = i0 + u * 64 + lane;
      key[u] = val[u] = 0u;
      if (i < whi) {
        key[u] = FIRST ? token_key(ids, is64, i, rows, pad) : tok[i];
        val[u] = FIRST ? (uint32_t)i : pos[i];
        if (FIRST && key[u] < (uint32_t)rows) present[key[u]] = 1;
      }
    }
  };
  fetch(wlo);
#pragma unroll
  for (int u = 0; u < kRounds; ++u)
    if (wlo + u * 64 + lane < whi) atomicAdd(&cnt[wave][(key[u] >> shift) & mask], 1u);
  for (int64_t i = wlo + kRounds * 64 + lane; i < whi; i += 64) {
    const uint32_t k = FIRST ? token_key(ids, is64, i, rows, pad) : tok[i];
    atomicAdd(&cnt[wave][(k >> shift) & mask], 1u);
  }
  const int digit = tid & (kDigits - 1), half = tid / kDigits;
  uint32_t before = 0u, all = 0u;
#pragma unroll
  for (int i = 0; i < kTilesMax / 2; ++i) {
    const int t = 2 * i + half;
    const uint32_t c = t < tiles ? hist[t * kDigits + digit] : 0u;
    before += t < (int)blockIdx.x ? c : 0u;
    all += c;
  }
  if (half == 1) {
    other[0][digit] = before;
    other[1][digit] = all;
  }
  __syncthreads();
  if (half == 0) {
    before += other[0][digit];
    all += other[1][digit];
  }
  uint32_t base = scan_digits(half == 0 ? all : 0u, sums) + before;
  if (half == 0) {
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t c = cnt[w][digit];
      cnt[w][digit] = base;
      base += c;
    }
  }
  __syncthreads();
  for (int64_t i0 = wlo; i0 < whi; i0 += kRounds * 64) {
    if (i0 > wlo) fetch(i0);
#pragma unroll
    for (int u = 0; u < kRounds; ++u) {
      const bool in = i0 + u * 64 + lane < whi;
      const uint32_t d = (key[u] >> shift) & mask;
      const uint64_t same = same_digit(d, in);
      if (in) {
        const uint32_t at = cnt[wave][d] + (uint32_t)__popcll(same & ((1ull << lane) - 1ull));
        tok_out[at] = key[u];
        pos_out[at] = val[u];
      }
      wave_fence();
      if (in && (same >> lane) == 1ull) cnt[wave][d] += (uint32_t)__popcll(same);
      wave_fence();
    }
  }
}

// ---------------------------------------------------------------- sums
//
// V consecutive columns per lane and slice.  A row's last lane takes the last V columns,
// some of them the lane before's too (of another wave, where it is the first lane of its
// slice): both get the same sums and store the same values, but where sums are added to what
// the table holds, one of them alone may do it (see write).
// Rows of less than V columns are one lane's.
template <int DT>
struct Slice {
  static constexpr int V = DT == HS_F32 ? 4 : 8;
  static constexpr int kCols = 64 * V;

  // The lane's first column; dim and above: none.
  __device__ static __forceinline__ int column(int slice, int lane, int dim) {
    const int c = slice * kCols + lane * V;
    return c < dim && c + V > dim && dim >= V ? dim - V : c;
  }

  __device__ static __forceinline__ void load(const uint8_t *row, int c, int dim, float *v) {
    if (dim >= V) {   // (the same for every lane; those without columns load the first)
      RawCols<DT, V> raw;
      raw.load(row, c < dim ? c : 0);
      raw.decode(v);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = c + j < dim ? load_col<DT>(row, c + j) : 0.0f;
    }
  }

  __device__ static __forceinline__ void part(float *row, int c, int dim, const float *v) {
    if (dim >= V) {
      if (c < dim) {
#pragma unroll
        for (int j = 0; j < V; j += 4)
          store_cols(row + c + j, round_cols<HS_F32, 4>(v + j));
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (c + j < dim) row[c + j] = v[j];
    }
  }

  // table[r] = (add: +=) scale * v
  template <int OT>
  __device__ static __forceinline__ void write(uint8_t *table, int64_t r, int c, int dim,
                                               float scale, int add, const float *v) {
    constexpr int OB = OT == HS_F32 ? 4 : 2;
    uint8_t *row = table + r * (int64_t)dim * OB;
    // (added to, columns below a multiple of V are the lane before's, which reads and writes
    // them by itself, in whatever wave it is)
    const int own = add ? (c + V - 1) / V * V : c;
    if (c + V <= dim && own == c) {
      float o[V];
#pragma unroll
      for (int j = 0; j < V; ++j) o[j] = v[j] * scale;
      if (add) {
        RawCols<OT, V> raw;
        float old[V];
        raw.load(row, c);
        raw.decode(old);
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] += old[j];
      }
      if constexpr (OT == HS_F32) {
#pragma unroll
        for (int j = 0; j < V; j += 4)
          stream_cols(row + (int64_t)(c + j) * 4, round_cols<HS_F32, 4>(o + j));
      } else if constexpr (V == 8) {
        stream_cols(row + (int64_t)c * 2, round_cols<HS_BF16, 8>(o));
      } else {
        *(WordsAt<2> *)(row + (int64_t)c * 2) =
            WordsAt<2>{{f32_to_bf16x2(o[0], o[1]), f32_to_bf16x2(o[2], o[3])}};
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (c + j < own || c + j >= dim) continue;
        const float o = v[j] * scale;
        store_col<OT>(row, c + j, add ? o + load_col<OT>(row, c + j) : o);
      }
    }
  }
};

// Lists token t, which begins in chunk c, if it goes on for many.  (With every token over
// two chunks in a list, the atomics took most of the launch: 60 us for 3,000 of them.)
__device__ __forceinline__ void list_many(const uint32_t *tok, int64_t n, int places, int64_t c,
                                          uint32_t t, uint32_t *count, uint32_t *many) {
  const int64_t far = (c + kSpanMany) * places;
  if (far < n && tok[far] == t) many[atomicAdd(count, 1u)] = (uint32_t)c;
}

template <int DT, int OT>
__global__ __launch_bounds__(256) void grad_sums(
    const uint8_t *__restrict__ grad, const uint32_t *__restrict__ tok,
    const uint32_t *__restrict__ pos, int64_t n, int64_t rows, int dim, int places,
    int64_t chunks, int slices, int64_t sum_blocks, float scale, int add,
    float *__restrict__ part, uint32_t *__restrict__ count, uint32_t *__restrict__ many,
    uint8_t *__restrict__ table,
    const uint8_t *__restrict__ present, Zeros z) {
  using S = Slice<DT>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if ((int64_t)blockIdx.x >= sum_blocks) {
    zero_rows(z, present, (int64_t)blockIdx.x - sum_blocks, (int64_t)gridDim.x - sum_blocks);
    return;
  }
  const int64_t task = (int64_t)blockIdx.x * 4 + wave;
  if (task >= chunks * slices) return;
  const int64_t c = task / slices;
  const int slice = (int)(task - c * slices), col = S::column(slice, lane, dim);
  const int64_t lo = c * places;
  const int m = (int)(n - lo < places ? n - lo : places);
  const uint32_t none = (uint32_t)rows;
  const uint32_t my_tok = lane < m ? tok[lo + lane] : none;
  const uint32_t my_pos = lane < m ? pos[lo + lane] : 0u;
  const uint32_t prev = lo > 0 ? tok[lo - 1] : none;
  const uint32_t next = lo + m < n ? tok[lo + m] : none;
  const int64_t gb = row_bytes<DT>(dim);
  float acc[S::V] = {};
  uint32_t cur = __builtin_amdgcn_readlane(my_tok, 0);
  bool head = cur == prev;   // the current token began in an earlier chunk
  constexpr int U = 8;
  for (int i0 = 0; i0 < m; i0 += U) {
    float v[U][S::V];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u < m ? i0 + u : m - 1;
      const int64_t at = (int64_t)(uint32_t)__builtin_amdgcn_readlane(my_pos, i);
      S::load(grad + at * gb, col, dim, v[u]);
    }
    const int end = i0 + U < m ? i0 + U : m;
#pragma unroll 1
    for (int i = i0; i < end; ++i) {   // (the next row moves into v[0])
      const uint32_t t = __builtin_amdgcn_readlane(my_tok, i);
      if (t != cur) {
        if (head) {
          S::part(part + (c * 2) * dim, col, dim, acc);
        } else {
          S::template write<OT>(table, cur, col, dim, scale, add, acc);
        }
#pragma unroll
        for (int j = 0; j < S::V; ++j) acc[j] = 0.0f;
        cur = t;
        head = false;
      }
      if (cur == none) return;   // (only positions without a token are left)
#pragma unroll
      for (int j = 0; j < S::V; ++j) {
        acc[j] += v[0][j];
#pragma unroll
        for (int u = 0; u + 1 < U; ++u) v[u][j] = v[u + 1][j];
      }
    }
  }
  if (cur == none) return;
  if (head) {
    S::part(part + (c * 2) * dim, col, dim, acc);
  } else if (cur == next) {
    S::part(part + (c * 2 + 1) * dim, col, dim, acc);
    if (slice == 0 && lane == 0) list_many(tok, n, places, c, cur, count, many);
  } else {
    S::template write<OT>(table, cur, col, dim, scale, add, acc);
  }
}

// The same for rows that half a wave or less takes: `lanes` lanes (a power of two) have a
// chunk each.  (200,000 bf16 rows of 64 columns with a wave for each chunk: 65 us.)
template <int DT, int OT>
__global__ __launch_bounds__(256) void grad_sums_narrow(
    const uint8_t *__restrict__ grad, const uint32_t *__restrict__ tok,
    const uint32_t *__restrict__ pos, int64_t n, int64_t rows, int dim, int places,
    int64_t chunks, int lanes, int64_t sum_blocks, float scale, int add,
    float *__restrict__ part, uint32_t *__restrict__ count, uint32_t *__restrict__ many,
    uint8_t *__restrict__ table,
    const uint8_t *__restrict__ present, Zeros z) {
  using S = Slice<DT>;
  if ((int64_t)blockIdx.x >= sum_blocks) {
    zero_rows(z, present, (int64_t)blockIdx.x - sum_blocks, (int64_t)gridDim.x - sum_blocks);
    return;
  }
  const int lane = threadIdx.x & (lanes - 1), col = S::column(0, lane, dim);
  const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) / lanes;
  if (c >= chunks) return;
  const int64_t lo = c * places;
  const int m = (int)(n - lo < places ? n - lo : places);
  const uint32_t none = (uint32_t)rows;
  const uint32_t prev = lo > 0 ? tok[lo - 1] : none;
  const uint32_t next = lo + m < n ? tok[lo + m] : none;
  const int64_t gb = row_bytes<DT>(dim);
  float acc[S::V] = {};
  uint32_t cur = tok[lo];
  bool head = cur == prev;
  constexpr int U = 8;
  for (int i0 = 0; i0 < m; i0 += U) {
    uint32_t t[U], p[U];
    float v[U][S::V];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = lo + (i0 + u < m ? i0 + u : m - 1);
      t[u] = tok[i];
      p[u] = pos[i];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) S::load(grad + (int64_t)p[u] * gb, col, dim, v[u]);
    const int end = i0 + U < m ? i0 + U : m;
#pragma unroll 1
    for (int i = i0; i < end; ++i) {   // (the next row moves into v[0])
      if (t[0] != cur) {
        if (head) {
          S::part(part + (c * 2) * dim, col, dim, acc);
        } else {
          S::template write<OT>(table, cur, col, dim, scale, add, acc);
        }
#pragma unroll
        for (int j = 0; j < S::V; ++j) acc[j] = 0.0f;
        cur = t[0];
        head = false;
      }
      if (cur == none) return;
#pragma unroll
      for (int u = 0; u + 1 < U; ++u) t[u] = t[u + 1];
#pragma unroll
      for (int j = 0; j < S::V; ++j) {
        acc[j] += v[0][j];
#pragma unroll
        for (int u = 0; u + 1 < U; ++u) v[u][j] = v[u + 1][j];
      }
    }
  }
  if (head) {
    S::part(part + (c * 2) * dim, col, dim, acc);
  } else if (cur == next) {
    S::part(part + (c * 2 + 1) * dim, col, dim, acc);
    if (lane == 0) list_many(tok, n, places, c, cur, count, many);
  } else {
    S::template write<OT>(table, cur, col, dim, scale, add, acc);
  }
}

// Tokens over several chunks: the sum at the end of the chunk where the token begins
// and those at the start of the following ones.  A wave joins a few chunks, 256 columns at
// a time, in order; a workgroup many, 64 columns at a time, in a contiguous share for each
// of its waves, whose sums are added in order.
template <int OT>
__device__ __forceinline__ void join_write(uint8_t *table, int64_t t, int c, int dim, float x,
                                           int add) {
  uint8_t *row = table + t * dim * (OT == HS_F32 ? 4 : 2);
  if (c < dim) store_col<OT>(row, c, add ? x + load_col<OT>(row, c) : x);
}

template <int OT>
__global__ __launch_bounds__(kJoinWaves * 64) void grad_join(
    const uint32_t *__restrict__ tok, int64_t n, int64_t rows, int dim, int places,
    int64_t chunks, int join_blocks, float scale, int add, const uint32_t *__restrict__ count,
    const uint32_t *__restrict__ many, const float *__restrict__ part,
    uint8_t *__restrict__ table, const uint8_t *__restrict__ present, Zeros z) {
  __shared__ float sums[kJoinWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if ((int)blockIdx.x >= join_blocks) {
    zero_rows(z, present, (int64_t)blockIdx.x - join_blocks, (int64_t)gridDim.x - join_blocks);
    return;
  }
  const int many_blocks = (dim + 63) / 64, few_blocks = (dim + 255) / 256;
  const int64_t n_many = (int64_t)*count * many_blocks, n_few = (chunks - 1) * few_blocks;
  for (int64_t task = blockIdx.x; task < n_many; task += join_blocks) {
    const int64_t e = task / many_blocks, c = many[e];
    const int col = (int)(task - e * many_blocks) * 64 + lane, cc = col < dim ? col : 0;
    const uint32_t t = tok[(c + 1) * places - 1];
    // its last chunk: between lo, whose first token it is, and hi, 64 tries at a time
    int64_t lo = c + kSpanMany, hi = chunks;
    while (hi - lo > 1) {
      const int64_t step = (hi - lo + 63) / 64, k = lo + (lane + 1) * step;
      lo += step * __popcll(__builtin_amdgcn_ballot_w64(k < hi && tok[k * places] == t));
      hi = hi < lo + step ? hi : lo + step;
    }
    const int64_t c1 = lo, share = (c1 - c + kJoinWaves - 1) / kJoinWaves;
    const int64_t a = c + 1 + wave * share, b = a + share < c1 + 1 ? a + share : c1 + 1;
    float v = wave == 0 ? part[(c * 2 + 1) * dim + cc] : 0.0f;
    // (16 in flight: with four, a token in 15,000 of 262,144 places took most of the launch)
#pragma unroll 16
    for (int64_t k = a; k < b; ++k) v += part[k * 2 * dim + cc];
    sums[wave][lane] = v;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int w = 1; w < kJoinWaves; ++w) v += sums[w][lane];
      join_write<OT>(table, t, col, dim, v * scale, add);
    }
    __syncthreads();
  }
  for (int64_t task = (int64_t)blockIdx.x * kJoinWaves + wave; task < n_few;
       task += (int64_t)join_blocks * kJoinWaves) {
    const int64_t c = task / few_blocks;
    const int col = (int)(task - c * few_blocks) * 256 + lane;
    const uint32_t t = tok[(c + 1) * places - 1];
    // whether it goes on in the next chunk, and began in this one
    const uint32_t first = tok[c * places], before = c > 0 ? tok[c * places - 1] : (uint32_t)rows;
    const int64_t k0 = c + 1 + lane < chunks ? c + 1 + lane : chunks - 1;
    const uint64_t same = __builtin_amdgcn_ballot_w64(tok[k0 * places] == t);
    if (t == (uint32_t)rows || !(same & 1u) || (first == t && before == t)) continue;
    // chunks that begin with it (past the last chunk, the last one is looked at again)
    const int more = ~same ? __builtin_ctzll(~same) : 64;
    const int left = (int)(chunks - 1 - c < 64 ? chunks - 1 - c : 64);
    const int64_t c1 = c + (more < left ? more : left);
    if (c1 - c >= kSpanMany) continue;   // (in the list)
    float v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      v[j] = part[(c * 2 + 1) * dim + (col + j * 64 < dim ? col + j * 64 : 0)];
#pragma unroll 4
    for (int64_t k = c + 1; k <= c1; ++k) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] += part[k * 2 * dim + (col + j * 64 < dim ? col + j * 64 : 0)];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) join_write<OT>(table, t, col + j * 64, dim, v[j] * scale, add);
  }
}

template <int DT, int OT>
hipError_t launch_sums(const GradWs &w, int side, const void *grad, int64_t n, int64_t rows,
                       int64_t dim, float scale, int add, void *table, Zeros z, hipStream_t st) {
  constexpr int V = DT == HS_F32 ? 4 : 8;
  const int places = chunk_places(n, dim);
  const int64_t chunks = (n + places - 1) / places;
  const int slices = (int)((dim + 64 * V - 1) / (64 * V));
  int lanes = 1;   // that a row takes
  while (lanes < 64 && lanes * V < dim) lanes *= 2;
  const bool narrow = lanes < 64;
  // the join's launch, short and far from the memory's rate, takes up to 24 MB of the zeros
  // (9,000 rows of 1,000 bf16 columns, 65,536 tokens, fp32 71 -> 68 us; 37 of 300 lost 1 us,
  // 262,144 of 1,024 2 us)
  Zeros last = z;
  if (n >= 512 && n <= kSmallMax) {
    const int64_t half = (z.last - z.first) / 2, fit = (24 << 20) / (dim * z.elem);
    z.last = z.first + (z.last - z.first - (half < fit ? half : fit)) / 4 * 4;
  }
  last.first = z.last;
  auto wgs_of = [](const Zeros &r, int waves, int most) {
    const int64_t wgs = (r.last - r.first + 4 * waves - 1) / (4 * waves);
    return (int)(wgs < most ? wgs : most);
  };
  const int zero_wgs = wgs_of(z, 4, 1024);
  const int64_t sum_blocks = narrow ? (chunks * lanes + 255) / 256 : (chunks * slices + 3) / 4;
  hipLaunchKernelGGL((narrow ? grad_sums_narrow<DT, OT> : grad_sums<DT, OT>),
                     dim3((unsigned)(sum_blocks + zero_wgs)), dim3(256), 0, st,
                     (const uint8_t *)grad, w.tok[side], w.pos[side], n, rows, (int)dim, places,
                     chunks, narrow ? lanes : slices, sum_blocks, scale, add, w.part, w.count,
                     w.many, (uint8_t *)table, w.present, z);
  if (chunks > 1) {
    // (as many tasks at most, in waves)
    const int64_t tasks = ((chunks - 1) * ((dim + 255) / 256) + kJoinWaves - 1) / kJoinWaves;
    const int join_blocks = (int)(tasks < 1024 ? tasks : 1024);
    hipLaunchKernelGGL(grad_join<OT>,
                       dim3((unsigned)(join_blocks + wgs_of(last, kJoinWaves, 512))),
                       dim3(kJoinWaves * 64), 0, st, w.tok[side], n, rows, (int)dim, places,
                       chunks, join_blocks, scale, add, w.count, w.many, w.part,
                       (uint8_t *)table, w.present, last);
  }
  return hipGetLastError();
}

}  // namespace

size_t embed_grad_workspace_bytes(int64_t n, int64_t rows, int64_t dim) {
  return layout(n, rows, dim, nullptr, nullptr);
}

hipError_t launch_embed_grad(const void *grad, int grad_dtype, const void *ids, int is64,
                             int64_t n, int64_t rows, int64_t dim, float scale, int64_t pad,
                             int add, void *table, int table_dtype, void *ws, hipStream_t st) {
  if (rows <= 0 || (n <= 0 && add)) return hipSuccess;
  GradWs w;
  layout(n, rows, dim, ws, &w);
  int key_bits = 1;   // of rows + 1 keys
  while (((int64_t)1 << key_bits) <= rows) ++key_bits;
  const int passes = (key_bits + kDigitBits - 1) / kDigitBits;
  const int bits = (key_bits + passes - 1) / passes;
  int side = 0;
  const int elem = table_dtype == HS_F32 ? 4 : 2;
  const int64_t stop = add ? 0 : rows;   // rows of zeros are written below it
  const Zeros all = {(uint8_t *)table, 0, stop, (int)dim, elem};
  Zeros part[3] = {all, all, all};       // of the second count and scatter, of the sums
  int zero_wgs[2] = {0, 0};
  if (n <= kSmallMax) {
    // the sort takes about 1.6 us per 1,024 positions, in which the other CUs write some
    // 10 KiB of zeros for each; the sums' launch, short too, gets the rest
    const int64_t fit = n * 10240 / (dim * elem) / 32 * 32;
    Zeros now = all;
    now.last = n == 0 || fit > stop ? stop : fit;
    part[2].first = now.last;
    const int64_t zeros = part[2].last - part[2].first;
    // slabs: one workgroup for each CU but the sort's; at most as many rows as the bitmaps
    // hold
    auto slab_of = [](int64_t r) {
      const int64_t slab = ((r + 254) / 255 + 31) / 32 * 32;
      return slab < 32 ? (int64_t)32 : slab > 32 * kSmallMax ? (int64_t)32 * kSmallMax : slab;
    };
    const int64_t slab = slab_of(now.last), noted = slab_of(zeros);
    int64_t wgs = (now.last + slab - 1) / slab;
    if (wgs < (zeros + noted - 1) / noted) wgs = (zeros + noted - 1) / noted;
    hipLaunchKernelGGL(grad_sort_small, dim3(1 + (unsigned)(wgs < 255 ? wgs : 255)),
                       dim3(kSmallWaves * 64), 0, st, ids, is64, (int)n, rows, pad, bits, passes,
                       w.tok[0], w.pos[0], w.count, now, stop, (int)slab, (int)noted, w.present);
  } else {
    int64_t tiles = (n + kTileMin - 1) / kTileMin;
    if (tiles > kTilesMax) tiles = kTilesMax;
    int64_t tile = (n + tiles - 1) / tiles;
    tile = (tile + kSortWaves * 64 - 1) / (kSortWaves * 64) * (kSortWaves * 64);
    tiles = (n + tile - 1) / tile;
    // the rows of zeros: most behind the second pass, whose launches take 5 and 11 us
    // without them (262,144 positions) and leave the memory idle
    if (passes > 1) {
      part[0].last = stop / 5 / 4 * 4;
      part[1].first = part[0].last;
      part[1].last = stop * 13 / 20 / 4 * 4;
      part[2].first = part[1].last;
    }
    for (int i = 0; i < 2 && passes > 1; ++i) {
      const int64_t wgs = (part[i].last - part[i].first + 4 * kSortWaves - 1) / (4 * kSortWaves);
      zero_wgs[i] = (int)(wgs < 1024 ? wgs : 1024);
    }
    const dim3 b(kSortWaves * 64);
    for (int p = 0; p < passes; ++p) {
      const int shift = p * bits;
      // (with more than two passes the later ones write no zeros)
      const int zc = p == 1 ? zero_wgs[0] : 0, zs = p == 1 ? zero_wgs[1] : 0;
      const dim3 gc((unsigned)(tiles + zc)), gs((unsigned)(tiles + zs));
      if (p == 0) {
        hipLaunchKernelGGL(grad_count<true>, gc, b, 0, st, ids, is64, nullptr, n, tile, (int)tiles,
                           rows, pad, bits, shift, w.hist, w.present, w.count, part[0]);
        hipLaunchKernelGGL(grad_scatter<true>, gs, b, 0, st, ids, is64, nullptr, nullptr, n, tile,
                           (int)tiles, rows, pad, bits, shift, w.hist, w.tok[0], w.pos[0],
                           w.present, part[1]);
      } else {
        hipLaunchKernelGGL(grad_count<false>, gc, b, 0, st, ids, is64, w.tok[side], n, tile,
                           (int)tiles, rows, pad, bits, shift, w.hist, w.present, w.count, part[0]);
        hipLaunchKernelGGL(grad_scatter<false>, gs, b, 0, st, ids, is64, w.tok[side], w.pos[side],
                           n, tile, (int)tiles, rows, pad, bits, shift, w.hist, w.tok[side ^ 1],
                           w.pos[side ^ 1], w.present, part[1]);
        side ^= 1;
      }
    }
  }
  if (n == 0) return hipGetLastError();
  if (grad_dtype == HS_F32)
    return table_dtype == HS_F32
               ? launch_sums<HS_F32, HS_F32>(w, side, grad, n, rows, dim, scale, add, table,
                                              part[2], st)
               : launch_sums<HS_F32, HS_BF16>(w, side, grad, n, rows, dim, scale, add, table,
                                              part[2], st);
  return table_dtype == HS_F32
             ? launch_sums<HS_BF16, HS_F32>(w, side, grad, n, rows, dim, scale, add, table,
                                              part[2], st)
             : launch_sums<HS_BF16, HS_BF16>(w, side, grad, n, rows, dim, scale, add, table,
                                              part[2], st);
}

}  // namespace hs
