// Products of a few rows with every row of a packed table (E2M1 codes, a scale per
// group of columns):
//   out[m][r] = sum_g scale[r][g] * sum_{c in g} x[m][c] * code[r][c].
//
// The codes become bf16 by the hardware's conversion (two a time, exact), so the
// products run on the bf16 matrix cores: mfma_f32_16x16x32_bf16 with 16 rows of x as
// the left and 16 table rows as the right operand.  The sums of one group are scaled
// and added in fp32.  fp32 rows of x are split into three bf16 parts (the top 8, the
// next 8 and the last 8 significant bits: exact from 2^-110 on; of smaller values the bits
// below bf16's least, 2^-133, are left out.  The matrix cores take subnormal parts as they
// are).
//
// A wave takes 256 columns of its table rows at a time: lane l has row l % 16 and the
// 32 bytes (64 columns) l / 16 of the 128, so each row's segment is a whole cache
// line.  (64-byte segments, 128 columns at a time, reached 3.3 TB/s without any
// arithmetic.)  One MFMA takes 8 columns from each of the four lane quarters, so
// without more it would mix the four pieces.  The pieces' words are exchanged between
// the quarters (swaps of halves, then of quarters; for groups of 128 columns halves
// alone), and x, staged in LDS, is read in the same order.
// Floor: the table, read once.  24 bf16 rows x 1M x 768, group 64 (504 MB): 105 us, 4.8
// TB/s; one row x 32,000 x 4,096, group 32 (74 MB): 16.5 us, 4.5 TB/s (a plain read of that
// size runs at 6); 48 bf16 rows x 100,000 x 4,096, group 128 (221 MB): 95 us, 0.4 PFLOP/s
// with x staged in parts.
#include "rows.h"

namespace hs {

int persistent_grid();

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int kBlock = 256;            // columns per step of a wave
// LDS bytes of staged x that leave room for three (MT = 1) or two workgroups a CU
template <int MT>
constexpr int kStageMax = (MT == 1 ? 48 : 56) * 1024;
constexpr int kLds = 158 * 1024;         // of a CU, for one

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

// Exchanges four words (8 columns each) of every quarter's piece.  Afterwards word j
// of quarter p is word sub_of(j, p) of the piece piece_of(j, p): one piece for all
// quarters (groups of 32 and 64 columns), or one of two neighbouring pieces (128).
template <int GROUP>
__device__ __forceinline__ void exchange(uint32_t *w) {
  swap_halves(w[0], w[1]);
  swap_halves(w[2], w[3]);
  if constexpr (GROUP < 128) {
    swap_quarters(w[0], w[2]);
    swap_quarters(w[1], w[3]);
  }
}

template <int GROUP>
__device__ __forceinline__ int piece_of(int j, int p) {
  return GROUP < 128 ? (j & 1) * 2 + (j >> 1) : (j & 1) * 2 + (p & 1);
}

template <int GROUP>
__device__ __forceinline__ int sub_of(int j, int p) {
  return GROUP < 128 ? (p & 1) * 2 + (p >> 1) : (j & 2) + (p >> 1);
}

// Group (of the block's 256 / GROUP) of word j in half h of the pieces.
template <int GROUP>
constexpr __host__ __device__ int group_of(int h, int j) {
  const int piece = (j & 1) * 2 + (GROUP < 128 ? j >> 1 : 0);
  return (piece * 64 + h * 32) / GROUP;
}

// How the scales are read: a block's at once (bf16), in the last block those of the
// row's last 256 columns, shifted into place, where the row has a part of a block left;
// or one by one.  Every load is unconditional, at a clamped place where it would lie
// outside: with loads under conditions the compiler cannot count those in flight, and
// waits for the next block's before it multiplies the present one.
enum ScaleMode { kWhole, kTail, kEach };

// The 256 columns of 16 NT table rows, as loaded.
template <int GROUP, int NT, int MODE>
struct Block {
  static constexpr int NG = kBlock / GROUP;
  uint32_t w[NT][2][4];                         // a lane's 64 codes of one row, in halves
  uint32_t s[NT][MODE == kEach ? NG : NG / 2];  // the row's scales; bf16 ones in pairs

  // kb: block; row, srow: the lane's table rows and their scales; p: its quarter
  __device__ __forceinline__ void load(int kb, int dim, int scale_bf16, const uint8_t *const *row,
                                       const uint8_t *const *srow, int p) {
    const int c0 = kb * kBlock;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        int c = c0 + p * 64 + h * 32;
        if (MODE != kWhole) c = c < dim ? c : 0;
        const u32x4v_t v = *(const u32x4v_t *)(row[t] + c / 2);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[t][h][j] = v[j];
      }
    int g0 = kb * NG;
    if constexpr (MODE == kEach) {
      if (scale_bf16) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int g = 0; g < NG; ++g)
            s[t][g] = (uint32_t)((const uint16_t *)srow[t])[c0 + g * GROUP < dim ? g0 + g : 0]
                      << 16;
      } else {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int g = 0; g < NG; ++g)
            s[t][g] = ((const uint32_t *)srow[t])[c0 + g * GROUP < dim ? g0 + g : 0];
      }
    } else {
      if (MODE == kTail && c0 + kBlock > dim) g0 = dim / GROUP - NG;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const WordsAt<NG / 2> v = *(const WordsAt<NG / 2> *)(srow[t] + g0 * 2);
#pragma unroll
        for (int i = 0; i < NG / 2; ++i) s[t][i] = v.w[i];
      }
    }
  }

  // In a row's last part of a block: codes past the last column become 0, scales move to
  // their places and become 0 past the last.
  __device__ __forceinline__ void trim(int kb, int dim, int p) {
    if (MODE == kWhole || (kb + 1) * kBlock <= dim) return;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool in = kb * kBlock + p * 64 + h * 32 < dim;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[t][h][j] = in ? w[t][h][j] : 0u;
      }
    if constexpr (MODE == kEach) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int g = 0; g < NG; ++g) s[t][g] = kb * kBlock + g * GROUP < dim ? s[t][g] : 0u;
    } else {
      for (int n = ((kb + 1) * kBlock - dim) / GROUP; n > 0; --n) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < NG / 2; ++i)
            s[t][i] = s[t][i] >> 16 | (i + 1 < NG / 2 ? s[t][i + 1 < NG / 2 ? i + 1 : i] << 16 : 0u);
      }
    }
  }

  __device__ __forceinline__ float scale(int t, int g) const {
    if constexpr (MODE == kEach) return __uint_as_float(s[t][g]);
    return __uint_as_float(g & 1 ? s[t][g / 2] & 0xFFFF0000u : s[t][g / 2] << 16);
  }

  // xs: the lane's MT rows of staged x at the block's first column; xq: bytes between
  // the parts.
  template <int MT, int PARTS>
  __device__ __forceinline__ void add(const uint8_t *const *xs, int xq, int p,
                                      f32x4_t (*tot)[MT]) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      exchange<GROUP>(w[t][0]);
      exchange<GROUP>(w[t][1]);
    }
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      f32x4_t acc[NT][MT];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[t][m] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (group_of<GROUP>(h, j) != g) continue;
          const int col = piece_of<GROUP>(j, p) * 64 + h * 32 + sub_of<GROUP>(j, p) * 8;
          bf16x8_t xa[MT][PARTS];
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int q = 0; q < PARTS; ++q)
              xa[m][q] = *(const bf16x8_t *)(xs[m] + q * xq + col * 2);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const bf16x8_t b = decode_codes(w[t][h][j]);
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
              for (int q = PARTS - 1; q >= 0; --q)   // (small parts first)
                acc[t][m] =
                    __builtin_amdgcn_mfma_f32_16x16x32_bf16(xa[m][q], b, acc[t][m], 0, 0, 0);
          }
        }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const float sc = scale(t, g);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int i = 0; i < 4; ++i) tot[t][m][i] = __builtin_fmaf(sc, acc[t][m][i], tot[t][m][i]);
      }
    }
  }
};

// Stages columns [c0, c0 + cols) of rows [m0, m0 + m) of x in LDS, zeros past the
// last column; fp32 as three bf16 parts (truncated, so that nothing overflows; each
// rest is exact, and 0 below 2^-133).  cols is a multiple of 8.
template <int XT>
__device__ __forceinline__ void stage_x(const uint8_t *x, int64_t m0, int m, int dim, int c0,
                                        int cols, int row_bytes, int part_bytes, uint8_t *lds) {
  const int vecs = cols / 8;
  for (int i = threadIdx.x; i < m * vecs; i += blockDim.x) {
    const int r = i / vecs, c = (i - r * vecs) * 8;
    uint8_t *to = lds + r * row_bytes + c * 2;
    const bool in = c0 + c < dim;
    const int64_t at = (m0 + r) * dim + c0 + c;
    if constexpr (XT == HS_BF16) {
      u32x4v_t v = {0u, 0u, 0u, 0u};
      if (in) v = *(const u32x4v_t *)(x + at * 2);
      *(u32x4v_t *)to = v;
    } else {
      uint32_t h[8] = {};
      if (in) {
        RawCols<HS_F32, 8> raw;
        raw.load(x, at);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = raw.w[e];
      }
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        u32x4v_t v;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t top = h[e] & 0xFFFF0000u;
          h[e] = __float_as_uint(__uint_as_float(h[e]) - __uint_as_float(top));
          if (e & 1)
            v[e / 2] |= top;
          else
            v[e / 2] = top >> 16;
        }
        *(u32x4v_t *)(to + q * part_bytes) = v;
      }
    }
  }
}

// Workgroups of four or kWaves<MT> waves that loop over items: ks of the waves share the
// columns (block kb goes to wave kb % ks; their sums are joined in LDS, in wave order), each
// ks of them have 16 NT table rows.  MT tiles of 16 rows of x, staged `chunk` columns at a
// time, once if that is all of them.  The next block's loads, also those of the next
// item's first, are in flight while a block is multiplied.
template <int MT>
constexpr int kWaves = MT == 1 ? 16 : 8;

template <int XT, int GROUP, int MT, int NT, int MODE>
__global__ __launch_bounds__(kWaves<MT> * 64, MT == 1 ? 4 : 2) void score_packed_kernel(
    const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, int scale_bf16,
    int64_t rows, int dim,
    const uint8_t *__restrict__ x, int64_t n_x, int ks, int chunk, int64_t row_blocks,
    int64_t items, void *__restrict__ out, int out_f32, int64_t out_stride) {
  constexpr int PARTS = XT == HS_F32 ? 3 : 1;
  extern __shared__ __align__(16) uint8_t lds[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int sets = (int)(blockDim.x >> 6) / ks;   // of 16 NT table rows
  f32x4_t *joined = (f32x4_t *)lds;   // [sets * (ks - 1)][NT * MT][64]
  uint8_t *xs = lds + sets * (ks - 1) * NT * MT * 64 * 16;
  const int i16 = lane & 15, p = lane >> 4;
  const int part_of = wave % ks;
  const int blocks = (dim + kBlock - 1) / kBlock;
  const int steps = (blocks + ks - 1) / ks, per_chunk = chunk / (ks * kBlock);
  const int row_bytes = chunk * 2 + 16;   // (16 rows' pieces fall on different banks)
  const int64_t cb = dim / 2, sb = (int64_t)(dim / GROUP) * (scale_bf16 ? 2 : 4);

  // loads run ahead of the sums: (l_item, l_step), with the lane's table rows
  const uint8_t *row[NT], *srow[NT];
  int64_t l_item = blockIdx.x;
  int l_step = 0;
  auto point = [&]() {
    const int64_t rb = l_item % row_blocks;
    const int64_t n0 = (rb * sets + wave / ks) * (16 * NT);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      // (rows past the last are stood in for by the last: their sums are not stored)
      int64_t r = n0 + t * 16 + i16;
      r = r < rows ? r : rows - 1;
      row[t] = codes + r * cb;
      srow[t] = scales + r * sb;
    }
  };
  using Blk = Block<GROUP, NT, MODE>;
  auto load = [&](Blk &blk) {
    const int kb = l_step * ks + part_of;
    blk.load(kb < blocks ? kb : blocks - 1, dim, scale_bf16, row, srow, p);
    if (++l_step == steps) {
      l_step = 0;
      if (l_item + gridDim.x < items) l_item += gridDim.x;   // (past the end: once more)
      point();
    }
  };

  f32x4_t tot[NT][MT];
  int64_t item = blockIdx.x;
  int step = 0;
  int64_t mb = 0, rb = 0, m0 = 0;
  int mrows = 0, part_bytes = 0;
  int64_t staged = -1;   // block of rows of x that is staged as a whole
  auto add = [&](Blk &blk) {
    if (step == 0) {
      mb = item / row_blocks;
      rb = item - mb * row_blocks;
      m0 = mb * (16 * MT);
      mrows = (int)(n_x - m0 < 16 * MT ? n_x - m0 : 16 * MT);
      part_bytes = mrows * row_bytes;
    }
    const int in_chunk = step % per_chunk;
    if (in_chunk == 0 && staged != mb) {
      const int left = (blocks - step * ks) * kBlock;
      __syncthreads();   // (the readers of what was staged are done)
      stage_x<XT>(x, m0, mrows, dim, step * ks * kBlock, left < chunk ? left : chunk, row_bytes,
                  part_bytes, xs);
      __syncthreads();
      if (per_chunk >= steps) staged = mb;
    }
    if (step == 0) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) tot[t][m] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const int kb = step * ks + part_of;
    if (kb < blocks) {
      const uint8_t *xc[MT];
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int r = m * 16 + i16;
        xc[m] = xs + (r < mrows ? r : mrows - 1) * row_bytes +
                (in_chunk * ks + part_of) * kBlock * 2;
      }
      blk.trim(kb, dim, p);
      blk.template add<MT, PARTS>(xc, part_bytes, p, tot);
    }
    if (++step < steps) return;
    step = 0;
    item += gridDim.x;
    // (into the first of the ks waves)
    if (ks > 1) {
      __syncthreads();   // (the last item's sums are read)
      if (part_of > 0) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int m = 0; m < MT; ++m)
            joined[((wave - wave / ks - 1) * NT * MT + t * MT + m) * 64 + lane] = tot[t][m];
      }
      __syncthreads();
      if (part_of > 0) return;
      for (int q = 1; q < ks; ++q) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const f32x4_t o =
                joined[((wave - wave / ks + q - 1) * NT * MT + t * MT + m) * 64 + lane];
#pragma unroll
            for (int i = 0; i < 4; ++i) tot[t][m][i] += o[i];
          }
      }
    }
    // lane l holds table row l % 16 of a tile and rows 4 (l / 16) .. + 3 of x
    const int64_t n0 = (rb * sets + wave / ks) * (16 * NT);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t r = m0 + m * 16 + p * 4 + i;
        if (r >= n_x) continue;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const int64_t n = n0 + t * 16 + i16;
          if (n >= rows) continue;
          if (out_f32)
            ((float *)out)[r * out_stride + n] = tot[t][m][i];
          else
            ((uint16_t *)out)[r * out_stride + n] = f32_to_bf16(tot[t][m][i]);
        }
      }
  };

  Blk a, b;
  point();
  load(a);
  while (item < items) {
    load(b);
    add(a);
    if (item >= items) break;
    load(a);
    add(b);
  }
}

template <int XT, int GROUP, int MT, int NT>
hipError_t launch_packed_t(const hs_row_table *t, const void *x, int64_t n_x, void *out,
                           int out_dtype, int64_t out_stride, hipStream_t st) {
  const int64_t mblocks = (n_x + 16 * MT - 1) / (16 * MT);
  const int64_t waves = (t->rows + 16 * NT - 1) / (16 * NT) * mblocks;
  // the columns shared by up to four waves while there are fewer than 4,096 (16 per CU)
  int ks = 1;
  while (ks < 4 && waves * ks < 4096 && t->dim > kBlock * ks) ks *= 2;
  // x is staged whole where that leaves room for more workgroups of four waves on a CU;
  // else one workgroup has as many waves, and stages it whole or a part at a time (with four
  // waves 5 fp32 rows x 66,088 x 3,712 took 90 us, 48 with 16)
  const int mrows = (int)(n_x < 16 * MT ? n_x : 16 * MT), parts = XT == HS_F32 ? 3 : 1;
  const int nb = (int)((t->dim + kBlock - 1) / kBlock), cus = persistent_grid();
  int wgs = MT == 1 ? 3 : 2, n_waves = 4;
  auto whole = [&](int k) { return (nb + k - 1) / k * k; };
  auto staged = [&](int blocks) { return (size_t)mrows * parts * (blocks * kBlock * 2 + 16); };
  auto joined = [&](int k) { return (size_t)(n_waves - n_waves / k) * NT * MT * 64 * 16; };
  int chunk = whole(ks);
  if (staged(chunk) > kStageMax<MT>) {
    wgs = 1;
    n_waves = kWaves<MT>;
    auto items = [&](int k) { return (waves + n_waves / k - 1) / (n_waves / k); };
    // (not whole, either, where the sums to be joined take the room that would let more CUs
    // have an item: see below)
    const bool few = nb > 1 && items(1) * 2 <= cus && staged(whole(2)) + joined(2) > kLds;
    if (staged(whole(1)) <= kLds && !few) {
      // the fewest steps one after another (ks = 4 against 1: 5 fp32 rows x 66,088 x 3,712 48
      // against 61 us, 30 bf16 rows x 150,000 x 1,280 52 against 31), and a join's time
      int64_t best = INT64_MAX;
      for (int k = 1; k <= 4 && staged(whole(k)) + joined(k) <= kLds; k *= 2) {
        const int64_t steps = 4 * (whole(k) / k) + (k > 1 ? 1 + NT * MT : 1);   // in quarters
        const int64_t cost = (items(k) + cus - 1) / cus * steps;
        if (cost < best) {
          best = cost;
          ks = k;
        }
      }
      chunk = whole(ks);
    } else {
      // every item stages x anew, so as many table rows share that as leave each CU one (48
      // bf16 rows x 100,000 x 4,096 147 -> 95 us; 35 x 15,726 x 2,048 26 us with ks = 1, 19
      // with 4)
      auto fit = [&](int k) {
        return (int)((kLds - joined(k)) / (mrows * parts) - 16) / (2 * kBlock);
      };
      for (ks = 1; ks < 4 && items(ks) * 2 <= cus && fit(2 * ks) >= 2 * ks;) ks *= 2;
      chunk = fit(ks) / ks * ks;
    }
  }
  const int64_t per = 16 * NT * (n_waves / ks), row_blocks = (t->rows + per - 1) / per;
  const int64_t items = row_blocks * mblocks;
  const size_t lds = staged(chunk) + joined(ks);
  const bool bf16 = t->scale_dtype == HS_BF16;
  auto kernel = !bf16 || t->dim < kBlock ? score_packed_kernel<XT, GROUP, MT, NT, kEach>
                : t->dim % kBlock        ? score_packed_kernel<XT, GROUP, MT, NT, kTail>
                                         : score_packed_kernel<XT, GROUP, MT, NT, kWhole>;
  // (workgroups per CU: 24 rows x 1M x 768 took 105 us with two, 114 with four; one row
  // x 32,000 x 4,096 18 us with three or four, 20 with two)
  const int64_t grid = wgs * (int64_t)cus;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(items < grid ? items : grid)),
                     dim3(n_waves * 64), lds, st,
                     (const uint8_t *)t->data, (const uint8_t *)t->scale, (int)bf16, t->rows,
                     (int)t->dim, (const uint8_t *)x, n_x, ks, chunk * kBlock, row_blocks, items,
                     out, (int)(out_dtype == HS_F32), out_stride);
  return hipGetLastError();
}

template <int XT, int GROUP>
hipError_t launch_packed_g(const hs_row_table *t, const void *x, int64_t n_x, void *out,
                           int out_dtype, int64_t out_stride, hipStream_t st) {
  if (n_x <= 16)
    return launch_packed_t<XT, GROUP, 1, 1>(t, x, n_x, out, out_dtype, out_stride, st);
  // (64 rows of fp32 parts do not fit in LDS)
  if (XT == HS_F32 || n_x <= 32)
    return launch_packed_t<XT, GROUP, 2, 2>(t, x, n_x, out, out_dtype, out_stride, st);
  return launch_packed_t<XT, GROUP, XT == HS_F32 ? 2 : 4, 2>(t, x, n_x, out, out_dtype,
                                                                  out_stride, st);
}

}  // namespace

hipError_t launch_score_packed(const hs_row_table *t, const void *x, int x_dtype, int64_t n_x,
                               void *out, int out_dtype, int64_t out_stride, hipStream_t st) {
  if (n_x <= 0 || t->rows <= 0) return hipSuccess;
#define HS_PACKED(G)                                                                        \
  (x_dtype == HS_F32 ? launch_packed_g<HS_F32, G>(t, x, n_x, out, out_dtype, out_stride, st) \
                     : launch_packed_g<HS_BF16, G>(t, x, n_x, out, out_dtype, out_stride, st))
  return t->group == 32 ? HS_PACKED(32) : t->group == 64 ? HS_PACKED(64) : HS_PACKED(128);
#undef HS_PACKED
}

}  // namespace hs
