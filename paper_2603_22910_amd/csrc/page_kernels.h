// The paged 8-bit cache: block tables, storing and reading back.
//
// A page holds 128 tokens of one sequence, for every KV head of a layer.  A (page, head) is a 128 x d matrix of keys and one of values, e4m3
// times one power of two each.  Both are stored in the order in which the matrix pipe takes them (see k_offset, v_offset), so that
// a wave of the attention kernels loads its operands with 16 bytes per lane, consecutive lanes at consecutive addresses, and the value
// matrix comes transposed without a transposition.  That is possible because only whole blocks are quantised: the tokens behind a sequence's
// last full block stay in bf16 rows (the tail) until their block is complete, which also makes the stored bytes a function
// of the block's rows alone, however they arrived.
#pragma once
#include "common.h"

namespace echokv {
namespace page {

constexpr int kTokens = 128;            // of a page
constexpr int kMaxBatch = 4096;         // sequences: their prefix sums fit LDS
constexpr int kMinExp = -100;           // least exponent of a scale: products of two of them and of a query stay normal numbers
// (query, query head) columns of a prefill workgroup: 384, 256 or 128; 32 of a sequence of up to kNarrow.
constexpr int kLCols = 384, kMCols = 256, kSCols = 128, kNCols = 32, kNarrow = 128;
// Large blocks at all: at least kPfMany of them over all KV heads, or kPfLong halves for each compute unit (kPfMany 512 or 900: 4001 queries 162 -> 188 us; kPfLong 25 and
// 60: 16 x 60 behind 4000 107 -> 124, 512 behind 16384 184 -> 216).  Few columns: kNarrow 64 and 256: 49 rows behind 34396 tokens 41 -> 52, 16 x 60 109 -> 115.
constexpr int kPfMany = 320, kPfLong = 40;
constexpr int kPfFill = 256;            // prefill workgroups that fill the chip, one to a compute unit: fewer are split over the keys

// ---- plan: what grow leaves for the other kernels, int32 words.  Words 16 on: row_start, then the arrays below, each of batch + 1 words.
// Prefill with a cap goes by a cut of its own (capped: 0 or 1), as its blocks are of other sizes: columns of a block, halves of a share, items.
enum { kStatus, kWideSeqs, kDecChunk, kDecItems, kCols, kPfChunk, kPfItems, kFree0, kCapped, kMaxRows = 11, kMagic, kNwChunk, kNwItems, kHeads, kHeadWords };
static_assert(kHeadWords == 16, "row_start's place is documented");
struct Blocks { int cols, chunk, items; };
constexpr int32_t kMagicWord = 0x45504732;
struct Plan {
  int32_t* w;
  int n;                                // batch
  __host__ __device__ int32_t* arr(int i) const { return w + kHeadWords + i * (n + 1); }
  __host__ __device__ int32_t* row_start() const { return arr(0); }      // prefix sums of the new rows
  __host__ __device__ int32_t* len() const { return arr(1); }            // lengths with the new tokens
  __host__ __device__ int32_t* app() const { return arr(2); }            // prefix sums of append's items
  __host__ __device__ int32_t* dec() const { return arr(3); }            // ... of decode's items
  __host__ __device__ int32_t* fresh() const { return arr(4); }          // ... of the new pages
  __host__ __device__ int32_t* nw() const { return arr(5); }             // ... of prefill's items of few columns
  __host__ __device__ int32_t* nws() const { return arr(6); }            // ... of those that leave partial results
  __host__ __device__ int32_t* order() const { return arr(7); }          // the sequences that have items of many columns, long ones first
  __host__ __device__ int32_t* pf(int capped) const { return arr(8 + 3 * capped); }          // prefix sums of those items, in that order
  __host__ __device__ int32_t* pf_of(int capped) const { return arr(9 + 3 * capped); }       // first of them, by sequence
  __host__ __device__ int32_t* split(int capped) const { return arr(10 + 3 * capped); }      // prefix sums of the columns whose keys are split
  static constexpr int kArrays = 14;
  __device__ __forceinline__ int32_t* blocks(int capped) const { return w + kCols + (kCapped - kCols) * capped; }      // cols, chunk, items
};

// What the attention kernels make of a plan: sizes of the call that made it (batch below 2^13, H_q up to 2^16, H_kv up to 2^12).
struct PlanKey { int batch, H_q, H_kv, max_rows; };
__device__ __forceinline__ int32_t mark(int batch) { return kMagicWord ^ batch; }
__device__ __forceinline__ int32_t heads_word(int H_q, int H_kv) { return H_q << 13 | H_kv; }
__device__ __forceinline__ bool made_for(const Plan& p, const PlanKey& k) {
  return p.w[kMagic] == mark(k.batch) && p.w[kHeads] == heads_word(k.H_q, k.H_kv) && p.w[kMaxRows] == k.max_rows;
}

// The sequence that item x belongs to, by all lanes of a wave: how many of start[1 .. n] are at most x.
__device__ __forceinline__ int find_item(const int32_t* start, int n, int x) {
  const int lane = threadIdx.x & 63;
  int at = 0;
  for (int base = 0; base < n; base += 64) {
    const bool below = base + lane < n && start[base + lane + 1] <= x;
    const int c = __popcll(__ballot(below));
    at += c;
    if (c < 64) break;
  }
  return __builtin_amdgcn_readfirstlane(at);
}

// A word that no kernel of this launch writes, at an address that all lanes share: through the scalar cache, so that it takes no vector register and
// no place among the vector loads that are waited for in order.
__device__ __forceinline__ int32_t scalar_word(const int32_t* p) { return *(const __attribute__((address_space(4))) int32_t*)(uintptr_t)p; }
// The same for a byte.
__device__ __forceinline__ int scalar_byte(const uint8_t* p) {
  const uintptr_t u = (uintptr_t)p;
  return (scalar_word((const int32_t*)(u & ~(uintptr_t)3)) >> (8 * (u & 3))) & 0xff;
}

// ---- page layout, byte offsets inside one head's 128 * d
// Keys: 16-byte chunk of a lane (r = token % 16, g) of the 16-token tile t: dims 8 g .. 8 g + 7 of two 32-dim steps of the product.
template <int HD> __device__ __forceinline__ int k_offset(int token, int dim) {
  const int t = token >> 4, r = token & 15, h = dim >> 6, half = (dim >> 5) & 1, g = (dim >> 3) & 3;
  return ((t * (HD / 64) + h) * 64 + g * 16 + r) * 16 + half * 8 + (dim & 7);
}
// Values: chunk of a lane (r = dim % 16, g) of the 16-dim tile u and the 64-token half: the tokens whose probabilities the same lane group
// holds after the product with the keys, 4 g .. 4 g + 3 of each of four 16-token tiles.
template <int HD> __device__ __forceinline__ int v_offset(int token, int dim) {
  const int h = token >> 6, tile = (token >> 4) & 3, g = (token >> 2) & 3, i = token & 3, u = dim >> 4, r = dim & 15;
  return ((h * (HD / 16) + u) * 64 + g * 16 + r) * 16 + tile * 4 + i;
}

__device__ __forceinline__ float exp_to_scale(int byte) { return __uint_as_float((uint32_t)byte << 23); }

// e4m3 pair -> bf16 pair times a power of two; exact (4 significant bits, exponents far inside bf16's).
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
template <bool HI> __device__ __forceinline__ uint32_t widen(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HI));
}
__device__ __forceinline__ uint4 widen8(uint32_t a, uint32_t b, float scale) {
  return make_uint4(widen<false>(a, scale), widen<true>(a, scale), widen<false>(b, scale), widen<true>(b, scale));
}

// A stored value: NaN as zero, what lies past 448 * 2^119 = 1.75 * 2^127 as that (the next number of a page would be 2^128, past bf16's).
__device__ __forceinline__ uint32_t finite_bits(uint32_t b) {        // b: 16 bits
  const uint32_t m = b & 0x7fffu;
  return m <= 0x7f60u ? b : m <= 0x7f80u ? (b & 0x8000u) | 0x7f60u : 0;
}
__device__ __forceinline__ uint32_t finite_pair(uint32_t w, bool& odd) {
  const uint32_t x = finite_bits(w & 0xffffu) | (finite_bits(w >> 16) << 16);
  odd |= x != w;
  return x;
}
__device__ __forceinline__ uint4 finite8(uint4 x, bool& odd) {
  return make_uint4(finite_pair(x.x, odd), finite_pair(x.y, odd), finite_pair(x.z, odd), finite_pair(x.w, odd));
}

// ---- lengths -> tables
struct GrowArgs {
  const int32_t *len0, *n_new, *free_list, *n_free0;
  int32_t *len1, *n_free1, *table, *slot, *pos;
  Plan plan;
  int max_pages, n_pages, max_rows, H_q, H_kv;
  int dec_items, pf_items, nw_items;    // items that share the work of a decode / prefill launch; pf_items = 0: blocks of queries suffice
  int rows_here;                        // the rows' slots are written by this launch, too
};

// One row's slot and, where the row completes a block, the block's table entry.
__device__ __forceinline__ void grow_row(const GrowArgs& a, int row, int b, int row0, int len1, int n, int fresh, int n_free0) {
  const int len0 = len1 - n, p = len0 + row - row0, blk = p / kTokens, full1 = len1 / kTokens;
  int slot = -1 - (b * kTokens + p % kTokens);
  if (blk < full1) {                                   // a block with a new row is a new page
    const int page = a.free_list[n_free0 - 1 - (fresh + blk - len0 / kTokens)];
    slot = page * kTokens + p % kTokens;
    if (p % kTokens == kTokens - 1) a.table[(int64_t)b * a.max_pages + blk] = page;
  }
  if (a.slot) a.slot[row] = slot;
  if (a.pos) a.pos[row] = p;
}

// Lane i gets the value of lane i - N of its row of 16, or with 0x142 / 0x143 rows 1 and 3 / 2 and 3 that of the last lane of row 0 and 2 / 1; else 0.
template <int CTRL, int ROWS> __device__ __forceinline__ int32_t from_lower(int32_t v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, CTRL < 0x140); }
template <int CTRL, int ROWS> __device__ __forceinline__ double from_lower(double v) {
  const int64_t b = __builtin_bit_cast(int64_t, v);
  const uint32_t lo = from_lower<CTRL, ROWS>((int32_t)b), hi = from_lower<CTRL, ROWS>((int32_t)(b >> 32));
  return __builtin_bit_cast(double, (int64_t)((uint64_t)hi << 32 | lo));
}
// Inclusive prefix sums over a wave; the last lane has the total.  (On the vector unit: through the LDS crossbar a step's scans took 4 us.)
template <typename T> __device__ __forceinline__ T wave_prefix(T v) {
  v += from_lower<0x111, 0xF>(v);
  v += from_lower<0x112, 0xF>(v);
  v += from_lower<0x114, 0xF>(v);
  v += from_lower<0x118, 0xF>(v);
  v += from_lower<0x142, 0xA>(v);
  v += from_lower<0x143, 0xC>(v);
  return v;
}
__device__ __forceinline__ double wave_total(double v) { return wave_prefix(v); }      // in lane 63

// Sums over the block's threads, in every thread.  (In double: exact far beyond what is compared with them.)
template <int N, int NT> __device__ __forceinline__ void block_sums(double (&v)[N], double (*lds)[NT / 64]) {
  constexpr int W = NT / 64;
  const int tid = threadIdx.x;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = wave_total(v[i]);
    if ((tid & 63) == 63) lds[i][tid >> 6] = v[i];
  }
  __syncthreads();
  static_assert(N * W <= NT && W <= 16, "a row of lanes per value");
  if (tid < N * W) {
    double x = lds[tid / W][tid % W];
    for (int o = W / 2; o > 0; o >>= 1) x += __shfl_xor(x, o, W);
    lds[tid / W][tid % W] = x;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = lds[i][0];
  __syncthreads();
}

// Inclusive prefix sums over the block's threads, on top of carry, which takes the totals.
template <int N, int NT> __device__ __forceinline__ void block_scan(int32_t (&v)[N], int32_t (&carry)[N], int32_t (*lds)[NT / 64]) {
  constexpr int W = NT / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = wave_prefix(v[i]);
    if (lane == 63) lds[i][wave] = v[i];
  }
  __syncthreads();
  if (tid < N * W) {
    int x = lds[tid / W][tid % W];
    for (int o = 1; o < W; o <<= 1) { const int y = __shfl_up(x, o, W); if (tid % W >= o) x += y; }
    lds[tid / W][tid % W] = x;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] += carry[i] + (wave ? lds[i][wave - 1] : 0);
    carry[i] += lds[i][W - 1];
  }
  __syncthreads();
}

// Columns of a sequence with n new rows, and the blocks of `many` columns, or of few, that prefill cuts them into.
struct Cut { bool narrow; int blocks; };
__device__ __forceinline__ Cut cut(int n, int G, int many) {       // n * G below 2^30
  const uint32_t cols = n * G;
  if (cols <= kNarrow) return {true, (int)((cols + kNCols - 1) / kNCols)};
  return {false, (int)(many == kLCols ? (cols + kLCols - 1) / kLCols : many == kMCols ? (cols + kMCols - 1) / kMCols : (cols + kSCols - 1) / kSCols)};
}

// A length's place among 256, eight to a factor of two.
__device__ __forceinline__ int bucket(int t) { return (int)(__float_as_uint((float)t) >> 20) - (127 << 3); }

// All or nothing: lengths, sums and chunk sizes by one workgroup, a thread per sequence.  Every later choice needs sums over all sequences, so it is a chain of
// loads, scans and barriers, 6 us for 32 sequences (8.6 a call) where an empty launch takes 3.9; 13 us for 512 prompts, and 5 for the 466 K slots and positions of
// their rows, which a launch of their own writes then (up to 4096 rows by this workgroup: no second launch for a step).
template <int NT>
__global__ __launch_bounds__(NT) void grow_kernel(GrowArgs a) {
  constexpr int S = 5, X = 8;
  __shared__ double red[X][NT / 64];
  __shared__ int32_t wsum[8][NT / 64], hist[256], longest;
  __shared__ int32_t rows[NT + 1], lens[NT], fresh[NT];      // row_start, len, fresh, where the rows are looked at here
  const int tid = threadIdx.x, B = a.plan.n, G = a.H_q / a.H_kv;
  const int64_t cap = (int64_t)a.max_pages * kTokens + kTokens - 1;
  const int n_free0 = *a.n_free0;
  int first_l = 0, first_n = 0;                        // of sequence tid
  if (tid < B) { first_l = a.len0[tid]; first_n = a.n_new[tid]; }
  const auto len_of = [&](int b) { return b == tid ? first_l : a.len0[b]; };
  const auto new_of = [&](int b) { return b == tid ? first_n : a.n_new[b]; };
  // the sums s of all sequences and x of those of many columns: blocks of 128, 256 and 384 columns, the halves they see at most and without a prefix
  enum { Rows, Pages, FullHalves, Wide, NarrowHalves }; enum { Small, Mid, Large, SmallHalves, MidHalves, LargeHalves, MidWork, LargeWork };
  double s[S] = {0, 0, 0, 0, 0}, x[X] = {0, 0, 0, 0, 0, 0, 0, 0};
  int wrong = 0, my_longest = 0;
  if (tid == 0) longest = 0;
  for (int b = tid; b < B; b += NT) {
    const int64_t l = len_of(b), n = new_of(b);
    if (l < 0 || l > cap || n < 0) { wrong |= 1; continue; }      // ECHOKV_PLAN_BAD_LENGTH
    if (l + n > cap) { wrong |= 2; continue; }                    // ECHOKV_PLAN_TABLE_FULL
    const int64_t t = l + n, seen = (t + 63) / 64;
    const int rows = (int)min(n, (int64_t)a.max_rows);       // (more than that: nothing comes of it)
    const Cut c = cut(rows, G, kSCols);
    s[Rows] += n; s[Pages] += t / kTokens - l / kTokens; s[FullHalves] += t / kTokens * 2;
    if (c.narrow) {
      s[NarrowHalves] += (double)c.blocks * seen;
    } else {
      const int blocks[3] = {c.blocks, cut(rows, G, kMCols).blocks, cut(rows, G, kLCols).blocks};
      for (int k = 0; k < 3; ++k) { x[Small + k] += blocks[k]; x[SmallHalves + k] += (double)blocks[k] * seen; }
      const double mean = 0.5 * (double)(l / 64 + seen);
      x[MidWork] += blocks[1] * mean; x[LargeWork] += blocks[2] * mean;
      s[Wide] += 1;
      my_longest = max(my_longest, (int)seen);
    }
  }
  block_sums<S, NT>(s, red);
  if (s[Wide] > 0) {                                   // (a step of single tokens: none)
    block_sums<X, NT>(x, red);
    const int top = (int)wave_max64((float)my_longest);      // (below 2^24; 64 lanes' maxima one by one took 2.5 us)
    if ((tid & 63) == 0) atomicMax(&longest, top);
  }
  int status = (__syncthreads_or(wrong & 1) ? 1 : 0) | (__syncthreads_or(wrong & 2) ? 2 : 0);
  if (n_free0 < 0 || n_free0 > a.n_pages) status |= 1;
  if (!status && s[Pages] > n_free0) status |= 4;      // ECHOKV_PLAN_NO_PAGES
  if (!status && s[Rows] > a.max_rows) status |= 8;    // ECHOKV_PLAN_TOO_MANY_ROWS
  const bool ok = status == 0;
  if (!ok) {                                           // nobody grows: the halves of the lengths as they were
    double h[1] = {0};
    for (int b = tid; b < B; b += NT) { const int64_t l = len_of(b); if (l >= 0 && l <= cap) h[0] += l / kTokens * 2; }
    block_sums<1, NT>(h, red);
    for (int i = 0; i < S; ++i) s[i] = 0;
    for (int i = 0; i < X; ++i) x[i] = 0;
    s[FullHalves] = h[0];
  }
  // halves per item: as many for each of its waves (decode, few columns); of a share of the keys.  (At most 2^26, more than a sequence has: sequences may share pages,
  // and the sum of their halves is bounded by nothing else.)
  // (The quotient is exact: whole numbers below 2^49 and 2^13.  A division of 64-bit integers would be some hundred instructions, fetched for this one use.)
  const auto chunk = [](double halves, int items, int waves) {
    return (int)fmin(fmax(ceil(halves / (double)(items * waves)), 1.0) * waves, 67108864.0);
  };
  const int dec_chunk = chunk(s[FullHalves], a.dec_items, 4);
  const int wide = (int)s[Wide], total = (int)s[Rows];
  // Large blocks have the rate, small ones fill the chip and end together.  A half of 64 tokens costs 384, 256 and 128 columns 3.1, 2.2 and 1.4 us with all compute
  // units busy, the longest blocks among them, which start first and run on alone, 2.5, 1.8 and 1.4; with a cap of 50 4.4, 2.65 and 1.7, so that 384 are never worth it.
  // In us, 32 query heads over 8 KV heads of 128, blocks of 384 | 256 | 128:
  // 8192 queries 532 | 558 | 714, with the cap 766 | 684 | 889; 6 x 257 .. 4001 192 | 201 | 259, with the cap 267 | 244 | 302; 4001 160 | 149 | 184; 2000 89 | 69 | 57;
  // 512 behind 16384 179 | 180 | 212; 12 heads over 2 of 64, 8192 435 | 381 | 505.
  Blocks blk[2];
  bool split[2];
  for (int capped = 0; capped < 2; ++capped) {
    int k = 0;                                         // 0, 1, 2: 128, 256, 384 columns
    if (capped) {
      if (x[Mid] * a.H_kv >= kPfMany || x[MidHalves] * a.H_kv >= kPfFill * kPfLong * 1.5) k = 1;
    } else if (x[Large] * a.H_kv >= kPfMany || x[LargeHalves] * a.H_kv >= kPfFill * kPfLong) {
      const double l = longest, mid = fmax(l * 1.8, x[MidWork] * a.H_kv * (2.2 / kPfFill)), large = fmax(l * 2.5, x[LargeWork] * a.H_kv * (3.1 / kPfFill));
      k = x[Mid] * a.H_kv >= kPfFill && mid < large ? 1 : 2;
    }
    blk[capped] = {k == 0 ? kSCols : k == 1 ? kMCols : kLCols, 0x7fffffff, 0};
    split[capped] = wide && x[Small + k] * a.H_kv < kPfFill;
    if (split[capped]) blk[capped].chunk = chunk(x[SmallHalves + k], a.pf_items, 8);      // the even share, for now
  }
  const bool alike = blk[0].cols == blk[1].cols;
  // A block's last share is short, and one workgroup more than the chip holds at a time doubles a launch's time: of 1, 5/4, 6/4 and 7/4 times the even share, a
  // wave each, the first that leaves no more items than that, else twice the even share.
  int nw_chunk = chunk(s[NarrowHalves], a.nw_items, 8);
  for (int which = 0; which < (alike ? 2 : 3); ++which) {
    const bool narrow = which == 0;
    const int capped = which == 2, unit = 8, slots = narrow ? a.nw_items : a.pf_items, even = narrow ? nw_chunk : blk[capped].chunk, many = blk[capped].cols;
    if (narrow ? even == unit : !split[capped]) continue;
    const auto candidate = [&](int k) { return (even * (4 + k) / 4 + unit - 1) / unit * unit; };
    const int wave = tid >> 6;
    if (wave < 4) {
      int64_t items = 0;
      for (int b = tid & 63; b < B; b += 64) {
        const int n = a.n_new[b];
        const Cut c = cut(n, G, many);
        if (c.narrow == narrow && n) items += c.blocks * (((a.len0[b] + n + 63) / 64 - 1) / candidate(wave) + 1);
      }
      for (int o = 32; o > 0; o >>= 1) items += __shfl_xor(items, o, 64);
      if ((tid & 63) == 0) red[0][wave] = items;
    }
    __syncthreads();
    int k = 0;
    while (k < 4 && red[0][k] > slots) ++k;
    (narrow ? nw_chunk : blk[capped].chunk) = candidate(k);
    __syncthreads();
  }
  if (alike) blk[1] = blk[0];
  const auto wide_items = [&](int b, const Blocks& x) {      // from what the plan got: the lengths may have been overwritten in place
    const bool here = b < NT;
    const int before = b == 0 ? 0 : here ? rows[b] : a.plan.row_start()[b], n = (here ? rows[b + 1] : a.plan.row_start()[b + 1]) - before;
    const int t = here ? lens[b] : a.plan.len()[b];
    const Cut c = cut(n, G, x.cols);
    return c.narrow ? 0 : c.blocks * (((t + 63) / 64 - 1) / x.chunk + 1);
  };
  int32_t carry[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int b0 = 0; b0 < B; b0 += NT) {
    const int b = b0 + tid;
    int l = 0, n = 0;
    if (b < B) {
      const int64_t ll = len_of(b);
      l = ll >= 0 && ll <= cap ? (int)ll : 0;
      n = ok ? new_of(b) : 0;
      a.len1[b] = ok ? l + n : (int)ll;
    }
    const int t = l + n, f0 = l / kTokens, f1 = t / kTokens, halves = f1 * 2, seen = (t + 63) / 64;
    const Cut c = cut(n, G, kSCols);
    const auto shares = [&](int chunk) { return n > 0 ? (seen - 1) / (c.narrow ? nw_chunk : chunk) + 1 : 0; };
    const int few = c.narrow ? c.blocks * shares(0) : 0;
    int32_t v[8];
    v[0] = n;
    v[1] = n > 0 ? max(1, f1 - f0) : 0;
    v[2] = (halves + dec_chunk - 1) / dec_chunk + (t % kTokens ? 1 : 0);
    v[3] = f1 - f0;
    v[4] = few;
    v[5] = c.narrow && shares(0) > 1 ? few : 0;
    v[6] = shares(blk[0].chunk) > 1 ? n * G : 0;
    v[7] = shares(blk[1].chunk) > 1 ? n * G : 0;
    block_scan<8, NT>(v, carry, wsum);
    if (b < B) {
      a.plan.row_start()[b + 1] = v[0]; a.plan.app()[b + 1] = v[1]; a.plan.dec()[b + 1] = v[2];
      a.plan.fresh()[b + 1] = v[3]; a.plan.nw()[b + 1] = v[4]; a.plan.nws()[b + 1] = v[5];
      a.plan.split(0)[b + 1] = v[6]; a.plan.split(1)[b + 1] = v[7];
      a.plan.len()[b] = t;
      if (b0 == 0) { rows[tid + 1] = v[0]; lens[tid] = t; fresh[tid] = v[3] - (f1 - f0); }
    }
  }
  int32_t items[2] = {0, 0};
  if (wide) {                                          // the longest sequences' blocks first: a long one that starts last would run on alone
    for (int i = tid; i < 256; i += NT) hist[i] = 0;
    __syncthreads();
    for (int b = tid; b < B; b += NT) if (wide_items(b, blk[0])) atomicAdd(&hist[bucket(a.plan.len()[b])], 1);
    __syncthreads();
    if (tid < 64) {                                    // places of the buckets, from the last one down
      int x[4], sum = 0;
      for (int i = 0; i < 4; ++i) { x[i] = sum; sum += hist[255 - 4 * tid - i]; }
      int before = sum;
      for (int o = 1; o < 64; o <<= 1) { const int y = __shfl_up(before, o, 64); if (tid >= o) before += y; }
      for (int i = 0; i < 4; ++i) hist[255 - 4 * tid - i] = before - sum + x[i];
    }
    __syncthreads();
    // (which of two of a bucket comes first is a matter of chance, and of none to any result)
    for (int b = tid; b < B; b += NT) if (wide_items(b, blk[0])) a.plan.order()[atomicAdd(&hist[bucket(a.plan.len()[b])], 1)] = b;
    __syncthreads();
    for (int r0 = 0; r0 < wide; r0 += NT) {
      const int r = r0 + tid;
      int32_t w[2] = {0, 0}, mine[2];
      const int b = r < wide ? a.plan.order()[r] : 0;
      for (int k = 0; k < 2; ++k) mine[k] = w[k] = r < wide ? wide_items(b, blk[k]) : 0;
      block_scan<2, NT>(w, items, wsum);
      for (int k = 0; k < 2; ++k) if (r < wide) { a.plan.pf(k)[r + 1] = w[k]; a.plan.pf_of(k)[b] = w[k] - mine[k]; }
    }
  }
  if (tid == 0) {
    int32_t* w = a.plan.w;
    for (int i : {0, 2, 3, 4, 5, 6, 8, 10, 11, 13}) a.plan.arr(i)[0] = 0;
    w[kStatus] = status; w[kWideSeqs] = wide; w[kDecChunk] = dec_chunk; w[kDecItems] = carry[2];
    w[kFree0] = n_free0; w[kNwChunk] = nw_chunk; w[kNwItems] = carry[4];
    for (int k = 0; k < 2; ++k) { int32_t* x = a.plan.blocks(k); x[0] = blk[k].cols; x[1] = blk[k].chunk; x[2] = items[k]; }
    w[kMaxRows] = a.max_rows; w[kHeads] = heads_word(a.H_q, a.H_kv); w[kMagic] = mark(B);
    *a.n_free1 = n_free0 - (int)s[Pages];
    rows[0] = 0;
  }
  if (!a.rows_here) return;
  __syncthreads();
  for (int row = tid; row < total; row += NT) {
    const int b = find_seq(rows, B, row);
    grow_row(a, row, b, rows[b], lens[b], rows[b + 1] - rows[b], fresh[b], n_free0);
  }
}

constexpr int kRowsPerBlock = 256;
__global__ __launch_bounds__(kRowsPerBlock) void grow_rows_kernel(GrowArgs a) {
  __shared__ int32_t starts[kMaxBatch + 1];
  const int32_t* rs = a.plan.row_start();
  const int row0 = blockIdx.x * kRowsPerBlock, B = a.plan.n, total = rs[B];
  if (row0 >= total) return;
  for (int i = threadIdx.x; i <= B; i += kRowsPerBlock) starts[i] = rs[i];
  __syncthreads();
  const int n_free0 = a.plan.w[kFree0];
  const int row = row0 + threadIdx.x;
  if (row >= total) return;
  const int b = find_seq(starts, B, row);
  grow_row(a, row, b, starts[b], a.plan.len()[b], starts[b + 1] - starts[b], a.plan.fresh()[b], n_free0);
}

// ---- slots of any cached tokens
struct SlotArgs {
  const int32_t *table, *len, *row_start, *first;
  int32_t* slot;
  int batch, max_pages, n_rows;
};
constexpr int32_t kNoSlot = (int32_t)0x80000000;
__global__ __launch_bounds__(256) void slots_kernel(SlotArgs a) {
  const int row = blockIdx.x * 256 + threadIdx.x;
  if (row >= a.n_rows || row < a.row_start[0] || row >= a.row_start[a.batch]) return;
  const int b = find_seq(a.row_start, a.batch, row);
  const int64_t p = (int64_t)a.first[b] + row - a.row_start[b], len = a.len[b];
  int32_t slot = kNoSlot;
  if (p >= 0 && p < len && len / kTokens <= a.max_pages) {
    if (p / kTokens < len / kTokens) {
      const int page = a.table[(int64_t)b * a.max_pages + p / kTokens];
      if (page >= 0) slot = (int32_t)((int64_t)page * kTokens + p % kTokens);
    } else {
      slot = -1 - (b * kTokens + (int)(p % kTokens));
    }
  }
  a.slot[row] = slot;
}

// ---- pages of finished sequences back onto the stack, in the order of sequences and blocks
struct ReleaseArgs {
  const int32_t* which;
  int32_t *table, *len, *free_list, *n_free;
  int batch, max_pages, n_pages;
};
template <int NT>
__global__ __launch_bounds__(NT) void release_kernel(ReleaseArgs a) {
  __shared__ int32_t start[kMaxBatch + 1];
  __shared__ int32_t wsum[NT / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, B = a.batch;
  const int n0 = *a.n_free;
  int64_t carry = 0;
  for (int b0 = 0; b0 < B; b0 += NT) {
    const int b = b0 + tid;
    int x = 0;
    if (b < B && a.which[b]) { const int l = a.len[b]; x = l < 0 ? 0 : min(l / kTokens, a.max_pages); }
    for (int o = 1; o < 64; o <<= 1) { const int y = __shfl_up(x, o, 64); if (lane >= o) x += y; }
    if (lane == 63) wsum[wave] = x;
    __syncthreads();
    int64_t before = carry;
    for (int k = 0; k < NT / 64; ++k) { if (k < wave) before += wsum[k]; carry += wsum[k]; }
    if (b < B) start[b + 1] = (int32_t)min(before + x, (int64_t)0x7fffffff);
    __syncthreads();
  }
  if (tid == 0) start[0] = 0;
  __syncthreads();
  if (n0 < 0 || carry > (int64_t)a.n_pages - n0) return;        // more pages than the pool has: released twice, nothing is touched
  for (int i = tid; i < (int)carry; i += NT) {
    const int b = find_seq(start, B, i);
    int32_t* e = a.table + (int64_t)b * a.max_pages + (i - start[b]);
    a.free_list[n0 + i] = *e;
    *e = -1;
  }
  for (int b = tid; b < B; b += NT) if (a.which[b]) a.len[b] = 0;
  if (tid == 0) *a.n_free = n0 + (int)carry;
}

// Larger one of either half, as unsigned numbers: of magnitudes of bf16 numbers.
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b) {
  typedef uint16_t pair_t __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(pair_t, a), __builtin_bit_cast(pair_t, b)));
}

__device__ __forceinline__ uint32_t magnitudes(uint4 x) {
  return max_pair(max_pair(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), max_pair(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu));
}
// Whether one of two magnitudes is one that finite_bits changes.
__device__ __forceinline__ bool beyond(uint32_t m) { return (m & 0xffffu) > 0x7f60u || (m >> 16) > 0x7f60u; }

// ---- rows into pages and tails
struct StoreArgs {
  uint8_t *k, *v, *ke, *ve;
  bf16_t *kt, *vt;
  const bf16_t *kn, *vn;
  const int32_t* table;
  Plan plan;
  PlanKey key;
  int max_pages, n_pages;
};

// Least power of two >= 2^kMinExp with amax <= 448 * 2^e, as its byte.  448 = 1.75 * 2^8; amax is a bf16 number.
__device__ __forceinline__ int scale_byte(float amax) {
  const uint32_t u = __float_as_uint(amax);
  return max((int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0), 127 + kMinExp);
}

// Bytes b of four words (0 .. 3: one token or dim each) to four words of their own.
__device__ __forceinline__ void transpose4(const uint32_t (&w)[4], uint32_t (&o)[4]) {
  const uint32_t a0 = __builtin_amdgcn_perm(w[1], w[0], 0x05010400), a1 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602);
  const uint32_t b0 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400), b1 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602);
  o[0] = __builtin_amdgcn_perm(b0, a0, 0x05040100); o[1] = __builtin_amdgcn_perm(b0, a0, 0x07060302);
  o[2] = __builtin_amdgcn_perm(b1, a1, 0x05040100); o[3] = __builtin_amdgcn_perm(b1, a1, 0x07060302);
}

// 16 bytes that are read once (non-temporal: 32 x 7808 tokens of decode 98 -> 85.7 us, 5.2 -> 6.0 TB/s).
__device__ __forceinline__ uint4 load_once(const uint4* p) {
  typedef uint32_t v4_t __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const v4_t*>(p)));
}

// One workgroup per (item, KV head, side).  A block's rows are read once, into registers; its codes go through LDS into the page's order, 1 KB of
// consecutive bytes per wave and store.  Memory bounds it: 20542 rows of 4096 dims, both sides, 85 - 97 us = 5.2 - 5.9 TB/s of 3 bytes for a number.  Item 0 of a sequence also moves the rows behind its last full block into the tail, after it has
// read the tail's old rows for the first block.
template <int HD>
__global__ __launch_bounds__(256, 4) void append_kernel(StoreArgs a) {
  constexpr int CPR = HD / 8, RPP = 256 / CPR, PASSES = kTokens / RPP;      // 16-byte chunks of a row, rows of a pass
  constexpr int ROW = HD + 8;                          // bytes of a row in LDS: rows that are read together lie in banks of their own
  __shared__ __attribute__((aligned(16))) uint8_t codes[kTokens * ROW];
  __shared__ float wmax[4];
  const int tid = threadIdx.x, wave = tid >> 6;
  const int side = blockIdx.x & 1, kvh = (blockIdx.x >> 1) % a.key.H_kv, item = (blockIdx.x >> 1) / a.key.H_kv;
  if (!made_for(a.plan, a.key) || item >= a.plan.app()[a.key.batch]) return;
  const int b = find_item(a.plan.app(), a.key.batch, item), j = item - a.plan.app()[b];
  const int row0 = a.plan.row_start()[b], n = a.plan.row_start()[b + 1] - row0, len1 = a.plan.len()[b], len0 = len1 - n;
  const int f0 = len0 / kTokens, f1 = len1 / kTokens;
  const int64_t D = (int64_t)a.key.H_kv * HD;
  const int rr = tid / CPR, cc = tid % CPR;
  bool odd = false;
  bf16_t* tail = (side ? a.vt : a.kt) + (int64_t)b * kTokens * D + kvh * HD;
  const bf16_t* rows = (side ? a.vn : a.kn) + (int64_t)row0 * D + kvh * HD;
  if (f1 > f0) {
    const int blk = f0 + j, page = a.table[(int64_t)b * a.max_pages + blk];
    uint4 x[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int tok = p * RPP + rr, at = blk * kTokens + tok;
      const bf16_t* from = at < len0 ? tail : rows + (int64_t)(blk * kTokens - len0) * D;
      x[p] = load_once(reinterpret_cast<const uint4*>(from + ((uint32_t)tok * (uint32_t)D + cc * 8)));
    }
    uint32_t m = 0;                                    // two largest magnitudes' bits, of the even and the odd dims
#pragma unroll
    for (int p = 0; p < PASSES; ++p) m = max_pair(m, magnitudes(x[p]));
    if (__any(beyond(m))) {                            // rare: not every row is looked at number by number
      m = 0;
#pragma unroll
      for (int p = 0; p < PASSES; ++p) { x[p] = finite8(x[p], odd); m = max_pair(m, magnitudes(x[p])); __builtin_amdgcn_sched_barrier(0); }
    }
    const float top = wave_max64(fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u)));
    if ((tid & 63) == 0) wmax[wave] = top;
    __syncthreads();
    const int e = scale_byte(fmaxf(fmaxf(wmax[0], wmax[1]), fmaxf(wmax[2], wmax[3])));
    const float down = exp_to_scale(254 - e);          // 2^-e: e is within +-120
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      float f[8];
      unpack_bf16x8(x[p], f);
      uint2 c;
      int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[0] * down, f[1] * down, 0, false);
      c.x = __builtin_amdgcn_cvt_pk_fp8_f32(f[2] * down, f[3] * down, w, true);
      w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4] * down, f[5] * down, 0, false);
      c.y = __builtin_amdgcn_cvt_pk_fp8_f32(f[6] * down, f[7] * down, w, true);
      *reinterpret_cast<uint2*>(codes + (p * RPP + rr) * ROW + cc * 8) = c;
      __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();
    if ((uint32_t)page < (uint32_t)a.n_pages) {
      const int64_t ph = (int64_t)page * a.key.H_kv + kvh;
      uint8_t* out = (side ? a.v : a.k) + ph * (kTokens * HD);
      if (!side) {
        for (int i = tid; i < kTokens * HD / 16; i += 256) {      // chunk of a lane (g, r), tile t and 64-dim part h
          const int r = i & 15, g = (i >> 4) & 3, h = (i >> 6) % (HD / 64), t = (i >> 6) / (HD / 64);
          const uint8_t* c = codes + (16 * t + r) * ROW + 64 * h + 8 * g;
          const uint2 lo = *reinterpret_cast<const uint2*>(c), hi = *reinterpret_cast<const uint2*>(c + 32);
          reinterpret_cast<uint4*>(out)[i] = make_uint4(lo.x, lo.y, hi.x, hi.y);
        }
      } else {
        // a thread: four dims of 16 tokens (those of one lane group and half), four chunks whose bytes are the tokens'
        for (int i = tid; i < HD / 4 * 8; i += 256) {
          const int dq = i % (HD / 4), g = i / (HD / 4) % 4, h = i / (HD / 4) / 4;
          uint32_t o[4][4];                            // [tile][dim]
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = *reinterpret_cast<const uint32_t*>(codes + (h * 64 + t * 16 + g * 4 + k) * ROW + dq * 4);
            transpose4(w, o[t]);
          }
#pragma unroll
          for (int d = 0; d < 4; ++d)
            *reinterpret_cast<uint4*>(out + v_offset<HD>(h * 64 + g * 4, dq * 4 + d)) = make_uint4(o[0][d], o[1][d], o[2][d], o[3][d]);
        }
      }
      if (tid == 0) (side ? a.ve : a.ke)[ph] = (uint8_t)e;
    }
  }
  if (j == 0) {                                        // (its reads of the tail's old rows are behind the barriers above)
    const int first = f1 > f0 ? f1 * kTokens : len0;
    for (int i = tid; i < (len1 - first) * CPR; i += 256) {
      const int p = first + i / CPR;
      uint4 x = load_once(reinterpret_cast<const uint4*>(rows + (int64_t)(p - len0) * D + i % CPR * 8));
      if (beyond(magnitudes(x))) x = finite8(x, odd);
      *reinterpret_cast<uint4*>(tail + (p % kTokens) * D + i % CPR * 8) = x;
    }
  }
  if (__any(odd) && (tid & 63) == 0) atomicOr(a.plan.w + kStatus, 16);            // ECHOKV_PLAN_NOT_FINITE
}

// ---- rows by their slots
template <typename TO> struct ReadArgs {
  const uint8_t *k, *v, *ke, *ve;
  const bf16_t *kt, *vt;
  const int32_t* slot;
  TO *ko, *vo;
  int n_rows, n_pages, batch, H_kv;
};

template <typename TO> __device__ __forceinline__ void put8(TO* p, uint4 b) {      // eight bf16 values
  if constexpr (sizeof(TO) == 2) {
    *reinterpret_cast<uint4*>(p) = b;
  } else {
    float f[8];
    unpack_bf16x8(b, f);
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
  }
}

template <typename TO> __device__ __forceinline__ void put4bf(TO* p, uint32_t a, uint32_t b) {      // four bf16 values
  if constexpr (sizeof(TO) == 2) *reinterpret_cast<uint2*>(p) = make_uint2(a, b);
  else *reinterpret_cast<float4*>(p) = make_float4(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u), __uint_as_float(b << 16), __uint_as_float(b & 0xffff0000u));
}

// 128 rows of one KV head per workgroup.  Runs of at least kLongRun consecutive rows of a page are read in the page's order, 16 bytes a lane, and written
// row by row; shorter ones, scattered rows and rows of tails are read where they are, all at once.  Memory bounds it: 20542 rows of 4096 dims 99 - 108 us = 4.7 - 5.1 TB/s.
// (Storing and reading them took 295 us together with codes stored and rows read where each lies in the page's order.)
constexpr int kLongRun = 16;
template <int HD, typename TO>
__global__ __launch_bounds__(256) void read_kernel(ReadArgs<TO> a) {
  constexpr int CPR = HD / 8, BYTES = kTokens * HD;
  __shared__ __attribute__((aligned(16))) uint8_t kb[BYTES];
  __shared__ int32_t slots[kTokens];
  const int tid = threadIdx.x, lane = tid & 63, kvh = blockIdx.x % a.H_kv, row0 = blockIdx.x / a.H_kv * kTokens, n = min(kTokens, a.n_rows - row0);
  const int64_t D = (int64_t)a.H_kv * HD;
  if (tid < n) slots[tid] = a.slot[row0 + tid];
  __syncthreads();
  // bit i: row i does not follow row i - 1 in one page; past the last row all bits are set
  const auto edge_at = [&](int i) { return i >= n || i == 0 || slots[i] < 0 || slots[i] != slots[i - 1] + 1 || (slots[i] & 127) == 0; };
  const uint64_t edge[2] = {__ballot(edge_at(lane)), __ballot(edge_at(64 + lane))};
  const auto run_end = [&](int i) {                       // first edge behind row i
    const uint64_t lo = i < 63 ? edge[0] >> (i + 1) << (i + 1) : 0, hi = i < 64 ? edge[1] : i < 127 ? edge[1] >> (i - 63) << (i - 63) : 0;
    return lo ? __ffsll((long long)lo) - 1 : hi ? 63 + __ffsll((long long)hi) : kTokens;
  };
  const auto run_start = [&](int i) {                     // last edge up to row i
    const uint64_t hi = i < 64 ? 0 : edge[1] << (127 - i), lo = i < 64 ? edge[0] << (63 - i) : edge[0];
    return hi ? i - __clzll((long long)hi) : (i < 64 ? i : 63) - __clzll((long long)lo);
  };
  for (int x = tid; x < n * CPR; x += 256) {
    const int i = x / CPR, c = x % CPR * 8, s = slots[i];
    const int64_t o = (row0 + i) * D + kvh * HD + c;
    if (s < 0) {
      const int64_t t = -1 - (int64_t)s;
      if (t >= (int64_t)a.batch * kTokens) continue;
      put8(a.ko + o, *reinterpret_cast<const uint4*>(a.kt + t * D + kvh * HD + c));
      put8(a.vo + o, *reinterpret_cast<const uint4*>(a.vt + t * D + kvh * HD + c));
    } else if ((s >> 7) < a.n_pages && run_end(i) - run_start(i) < kLongRun) {
      const int64_t ph = (int64_t)(s >> 7) * a.H_kv + kvh;
      const uint2 kk = *reinterpret_cast<const uint2*>(a.k + ph * BYTES + k_offset<HD>(s & 127, c));
      const uint8_t* vv = a.v + ph * BYTES + v_offset<HD>(s & 127, c);
      uint32_t w[2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
        w[h] = vv[64 * h] | (uint32_t)vv[64 * h + 16] << 8 | (uint32_t)vv[64 * h + 32] << 16 | (uint32_t)vv[64 * h + 48] << 24;
      put8(a.ko + o, widen8(kk.x, kk.y, exp_to_scale(a.ke[ph])));
      put8(a.vo + o, widen8(w[0], w[1], exp_to_scale(a.ve[ph])));
    }
  }
  const auto long_run = [&](int i) { return i < n && edge_at(i) && slots[i] >= 0 && (slots[i] >> 7) < a.n_pages && min(n, run_end(i)) - i >= kLongRun; };
  uint64_t starts[2] = {__ballot(long_run(lane)), __ballot(long_run(64 + lane))};
#pragma unroll 1
  for (int half = 0; half < 2; ++half)
    for (uint64_t left = starts[half]; left; left &= left - 1) {
      const int i = half * 64 + __ffsll((long long)left) - 1, end = __builtin_amdgcn_readfirstlane(min(n, run_end(i)));
      const int first = __builtin_amdgcn_readfirstlane(slots[i]), page = first >> 7;
      const int64_t ph = (int64_t)page * a.H_kv + kvh;
      const float ks = exp_to_scale(a.ke[ph]), vs = exp_to_scale(a.ve[ph]);
      const int t0 = first & 127, count = end - i;
      const int64_t out = (int64_t)(row0 + i - t0) * D + kvh * HD;      // of token 0 of the page
      __syncthreads();                                    // the keys of the page before are read
#pragma unroll
      for (int x = 0; x < BYTES / 16; x += 256) reinterpret_cast<uint4*>(kb)[x + tid] = reinterpret_cast<const uint4*>(a.k + ph * BYTES)[x + tid];
      __syncthreads();
#pragma unroll 4
      for (int x = tid; x < count * CPR; x += 256) {
        const int row = x / CPR, c = x % CPR * 8;
        const uint2 kk = *reinterpret_cast<const uint2*>(kb + k_offset<HD>(t0 + row, c));
        put8(a.ko + out + (int64_t)(t0 + row) * D + c, widen8(kk.x, kk.y, ks));
      }
      for (int x = tid; x < HD / 4 * 8; x += 256) {       // values: four dims of 16 tokens
        const int dq = x % (HD / 4), g = x / (HD / 4) % 4, h = x / (HD / 4) / 4, tok = h * 64 + g * 4;
        const uint4* p = reinterpret_cast<const uint4*>(a.v + ph * BYTES + v_offset<HD>(tok, dq * 4));
        uint4 c[4];
#pragma unroll
        for (int d = 0; d < 4; ++d) c[d] = p[d];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const auto word = [&](int d) { return t == 0 ? c[d].x : t == 1 ? c[d].y : t == 2 ? c[d].z : c[d].w; };
          const uint32_t w[4] = {word(0), word(1), word(2), word(3)};
          uint32_t o[4];
          transpose4(w, o);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if ((uint32_t)(tok + 16 * t + k - t0) < (uint32_t)count) put4bf(a.vo + out + (tok + 16 * t + k) * D + dq * 4, widen<false>(o[k], vs), widen<true>(o[k], vs));
        }
      }
    }
}

}  // namespace page
}  // namespace echokv
