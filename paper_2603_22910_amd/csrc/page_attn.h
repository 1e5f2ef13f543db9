// Attention over the paged 8-bit cache (page_kernels.h): decode, prefill and the merges of split sequences.
//
// Scores and value sums run on v_mfma_f32_16x16x32_bf16 with the cache as the row operand: S^T = K Q^T, O^T = V^T P^T.  A lane then
// holds one column, a (query, query head) pair, of scores and of outputs alike: the softmax' scaling is lane-local, its sums cross the
// four 16-lane rows once at the end, and the probabilities already lie where the second product wants them (the pages' token order
// is made for that).  The codes are widened to bf16 with their page's scale in one instruction for two values, exactly.  The matrix
// pipe takes e4m3 itself, too, at twice the rate, and bf16 queries are a sum of two e4m3 numbers; but its sums of e4m3
// products are cut off some 14 bits below the largest one (measured: up to 8e-5 of the sum of magnitudes, on average towards zero), where
// those of bf16 products are good to 4e-8.
#pragma once
#include "page_kernels.h"

namespace echokv {
namespace page {

typedef short frag_t __attribute__((ext_vector_type(8)));       // eight bf16
typedef __bf16 bf16x8v_t __attribute__((ext_vector_type(8)));
__device__ __forceinline__ floatx4_t mfma(uint4 a, uint4 b, floatx4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v_t, a), __builtin_bit_cast(bf16x8v_t, b), c, 0, 0, 0);
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNoScore = -1e30f;      // the maximum of no scores: finite, so that differences of two such are zero

struct AttnArgs {
  const uint8_t *k, *v, *ke, *ve;
  const bf16_t *kt, *vt, *q;
  const int32_t *table, *prefix;
  const float* slopes;
  void* out;
  float *lse, *part_o, *part_ml;        // partials: [item][H_q or H_kv * columns][d], then (maximum, sum) of each
  Plan plan;
  PlanKey key;
  float scale, cap;
  int max_pages, n_pages, G, col_tiles, n_items;
};

// Maximum / sum over the four 16-lane rows, in every lane.
template <class F> __device__ __forceinline__ float across_rows(float v, F f) {
  const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = f(__uint_as_float(p[0]), __uint_as_float(p[1]));
  const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f(__uint_as_float(h[0]), __uint_as_float(h[1]));
}
__device__ __forceinline__ float rows_max(float v) { return across_rows(v, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float rows_sum(float v) { return across_rows(v, [](float a, float b) { return a + b; }); }

// Raw products to scores in base 2.  cap: c tanh(s / c); where all of a wave's arguments are small by the odd series, of which the terms past
// x^9 are below 2^-25 of the first, else by 1 - 2 / (1 + e^2x), whose error is half a step of one, 2^-24 of the cap.
struct Mods { float scale2, cap2, to_arg, slope2; };
template <int N> __device__ __forceinline__ void score(float (&s)[N], const Mods& m, bool mods, float away0, const int (&step)[N]) {
  if (!mods) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] *= m.scale2;
    return;
  }
  if (m.cap2 > 0.f) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) { s[i] *= m.to_arg; top = fmaxf(top, fabsf(s[i])); }
    if (__any(!(top < 0.2f))) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float e = __builtin_amdgcn_exp2f(fabsf(s[i]) * (-2.f * kLog2e));          // (towards zero from either side: no overflow)
        s[i] = copysignf((1.f - e) * __builtin_amdgcn_rcpf(1.f + e), s[i]) * m.cap2;
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float x2 = s[i] * s[i];
        const float t = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
        s[i] = s[i] * t * m.cap2;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] *= m.scale2;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] = fmaf(m.slope2, away0 + (float)step[i], s[i]);
}
__device__ __forceinline__ Mods mods_of(const AttnArgs& a, float slope) {
  return {a.scale * kLog2e, a.cap * kLog2e, a.cap > 0.f ? a.scale / a.cap : 0.f, slope * kLog2e};
}

template <typename TO> __device__ __forceinline__ void put4(TO* p, float4 v) {
  if constexpr (sizeof(TO) == 2) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
  else *reinterpret_cast<float4*>(p) = v;
}

// ---- decode: one token of every sequence.  A workgroup takes an item (a run of 64-token halves of a sequence's full pages, or its tail) of one KV
// head and up to 16 of its query heads as columns.  Its four waves take the halves in turn, each with a softmax of its own; they are
// joined in LDS.  What bounds it is the reading of the pages.
constexpr int kDecodeItems = 1024;      // workgroups that the pages of a launch are shared out to

template <int HD, bool MODS, typename TO>
__global__ __launch_bounds__(256) void decode_kernel(AttnArgs a) {
  constexpr int KS = HD / 32, KC = HD / 64, U = HD / 16;
  __shared__ __attribute__((aligned(16))) float so[4][16][HD + 4];
  __shared__ float sm[4][16], sl[4][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
  if (!made_for(a.plan, a.key)) return;
  const int kvh = blockIdx.x % a.key.H_kv, rest = blockIdx.x / a.key.H_kv, ct = rest % a.col_tiles, item = rest / a.col_tiles;
  if (item >= a.plan.w[kDecItems]) return;
  const int B = a.key.batch, H_q = a.key.H_q;
  const int b = find_item(a.plan.dec(), B, item), item0 = a.plan.dec()[b], n_items = a.plan.dec()[b + 1] - item0, j = item - item0;
  const int len = a.plan.len()[b], halves = len / kTokens * 2, chunk = a.plan.w[kDecChunk], nc = min(16, a.G - ct * 16);
  const int head = kvh * a.G + ct * 16 + min(r, nc - 1);
  const bf16_t* qp = a.q + ((int64_t)b * H_q + head) * HD + 8 * g;
  uint4 qf[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const uint4*>(qp + 32 * s);
  const Mods md = mods_of(a, MODS && a.slopes ? a.slopes[head] : 0.f);

  floatx4_t o[U];
#pragma unroll
  for (int u = 0; u < U; ++u) o[u] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  float m = kNoScore, l = 0.f;

  const int begin = j * chunk, end = min(halves, begin + chunk);
  if (begin < halves) {
    const int32_t* pages = a.table + (int64_t)b * a.max_pages;
    for (int hf = begin + wave; hf < end; hf += 4) {
      const int page = pages[hf >> 1];
      if ((uint32_t)page >= (uint32_t)a.n_pages) continue;
      const int64_t ph = (int64_t)page * a.key.H_kv + kvh;
      const uint4* kp = reinterpret_cast<const uint4*>(a.k + ph * (kTokens * HD) + (hf & 1) * (64 * HD)) + lane;
      const uint4* vp = reinterpret_cast<const uint4*>(a.v + ph * (kTokens * HD) + (hf & 1) * (64 * HD)) + lane;
      uint4 kr[4][KC], vr[U];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int c = 0; c < KC; ++c) kr[t][c] = kp[(t * KC + c) * 64];
#pragma unroll
      for (int u = 0; u < U; ++u) vr[u] = vp[u * 64];
      const float ks = exp_to_scale(a.ke[ph]), vs = exp_to_scale(a.ve[ph]);
      float s[16];
      int step[16];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        floatx4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          acc = mfma(widen8(kr[t][c].x, kr[t][c].y, ks), qf[2 * c], acc);
          acc = mfma(widen8(kr[t][c].z, kr[t][c].w, ks), qf[2 * c + 1], acc);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) { s[4 * t + i] = acc[i]; step[4 * t + i] = 16 * t + i; }
      }
      score(s, md, MODS, (float)(hf * 64 + 4 * g - (len - 1)), step);
      float top = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
      top = rows_max(top);
      if (__any(top > m)) {
        const float up = fmaxf(m, top), f = __builtin_amdgcn_exp2f(m - up);
        m = up;
        l *= f;
#pragma unroll
        for (int u = 0; u < U; ++u) o[u] *= f;
      }
      uint32_t hi[8], lo[8];
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const float p0 = __builtin_amdgcn_exp2f(s[i] - m), p1 = __builtin_amdgcn_exp2f(s[i + 1] - m);
        l += p0 + p1;
        hi[i / 2] = pack_bf16(p0, p1);
        lo[i / 2] = pack_bf16(p0 - __uint_as_float(hi[i / 2] << 16), p1 - __uint_as_float(hi[i / 2] & 0xffff0000u));
      }
      const uint4 ph0 = make_uint4(hi[0], hi[1], hi[2], hi[3]), ph1 = make_uint4(hi[4], hi[5], hi[6], hi[7]);
      const uint4 pl0 = make_uint4(lo[0], lo[1], lo[2], lo[3]), pl1 = make_uint4(lo[4], lo[5], lo[6], lo[7]);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint4 v0 = widen8(vr[u].x, vr[u].y, vs), v1 = widen8(vr[u].z, vr[u].w, vs);
        o[u] = mfma(v0, ph0, o[u]);
        o[u] = mfma(v0, pl0, o[u]);
        o[u] = mfma(v1, ph1, o[u]);
        o[u] = mfma(v1, pl1, o[u]);
      }
    }
  } else {
    // the tail: 32 of its rows to a wave.  Rows past the last one may hold anything: they are read nowhere
    const int rows = len % kTokens, t0 = wave * 32;
    if (t0 < rows) {
      const int64_t D = (int64_t)a.key.H_kv * HD, base = (int64_t)b * kTokens * D + kvh * HD;
      float s[8];
      int step[8];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const bf16_t* kp = a.kt + base + (int64_t)min(t0 + 16 * t + r, rows - 1) * D + 8 * g;
        floatx4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KS; ++c) acc = mfma(*reinterpret_cast<const uint4*>(kp + 32 * c), qf[c], acc);
#pragma unroll
        for (int i = 0; i < 4; ++i) { s[4 * t + i] = acc[i]; step[4 * t + i] = 16 * t + i; }
      }
      score(s, md, MODS, (float)(t0 + 4 * g - (rows - 1)), step);
      float top = kNoScore;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (t0 + 4 * g + step[i] >= rows) s[i] = -INFINITY;
        top = fmaxf(top, s[i]);
      }
      m = rows_max(top);
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float p0 = __builtin_amdgcn_exp2f(s[i] - m), p1 = __builtin_amdgcn_exp2f(s[i + 1] - m);
        l += p0 + p1;
        hi[i / 2] = pack_bf16(p0, p1);
        lo[i / 2] = pack_bf16(p0 - __uint_as_float(hi[i / 2] << 16), p1 - __uint_as_float(hi[i / 2] & 0xffff0000u));
      }
      const uint4 ph = make_uint4(hi[0], hi[1], hi[2], hi[3]), pl = make_uint4(lo[0], lo[1], lo[2], lo[3]);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        uint32_t w[4];
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const int tok = t0 + 16 * (x / 4) + 4 * g + x % 4;
          const uint32_t e = a.vt[base + (int64_t)min(tok, rows - 1) * D + 16 * u + r];
          w[x / 2] = x % 2 ? w[x / 2] | e << 16 : e;
        }
        const uint4 v = make_uint4(w[0], w[1], w[2], w[3]);        // (past the last row: that row again, with probabilities of zero)
        o[u] = mfma(v, ph, o[u]);
        o[u] = mfma(v, pl, o[u]);
      }
    }
  }

  l = rows_sum(l);
  if (g == 0) { sm[wave][r] = m; sl[wave][r] = l; }
#pragma unroll
  for (int u = 0; u < U; ++u) *reinterpret_cast<floatx4_t*>(&so[wave][r][16 * u + 4 * g]) = o[u];
  __syncthreads();
  for (int x = tid; x < nc * (HD / 4); x += 256) {
    const int c = x / (HD / 4), d4 = x % (HD / 4) * 4;
    const float M = fmaxf(fmaxf(sm[0][c], sm[1][c]), fmaxf(sm[2][c], sm[3][c]));
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(sm[w][c] - M);
      const float4 y = *reinterpret_cast<const float4*>(&so[w][c][d4]);
      sum = fmaf(f, sl[w][c], sum);
      acc.x = fmaf(f, y.x, acc.x); acc.y = fmaf(f, y.y, acc.y); acc.z = fmaf(f, y.z, acc.z); acc.w = fmaf(f, y.w, acc.w);
    }
    const int h = kvh * a.G + ct * 16 + c;
    if (n_items == 1) {
      const int64_t row = (int64_t)b * H_q + h;
      const float inv = sum > 0.f ? 1.f / sum : 0.f;
      put4(reinterpret_cast<TO*>(a.out) + row * HD + d4, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
      if (a.lse && d4 == 0) a.lse[row] = sum > 0.f ? (M + __log2f(sum)) * kLn2 : -INFINITY;
    } else {
      const int64_t row = (int64_t)item * H_q + h;
      *reinterpret_cast<float4*>(a.part_o + row * HD + d4) = acc;
      if (d4 == 0) *reinterpret_cast<float2*>(a.part_ml + row * 2) = make_float2(M, sum);
    }
  }
}

// Joins `n` partials of one row, strided by `stride` rows, by a workgroup of 256 threads, in a fixed order.
template <int HD, typename TO>
__device__ __forceinline__ void join(const float* po, const float* pml, int n, int64_t stride, TO* out, float* lse) {
  constexpr int L = HD / 4, GR = 256 / L;
  __shared__ __attribute__((aligned(16))) float so[GR][HD];
  __shared__ float red[2][4];
  const int tid = threadIdx.x, d4 = tid % L * 4, gr = tid / L;
  float M = kNoScore;
  for (int i = tid; i < n; i += 256) M = fmaxf(M, pml[i * stride * 2]);
  M = wave_max64(M);
  if ((tid & 63) == 0) red[0][tid >> 6] = M;
  __syncthreads();
  M = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float sum = 0.f;
  for (int i = gr; i < n; i += GR) {
    const float2 ml = *reinterpret_cast<const float2*>(pml + i * stride * 2);
    const float4 y = *reinterpret_cast<const float4*>(po + i * stride * HD + d4);
    const float f = __builtin_amdgcn_exp2f(ml.x - M);
    sum = fmaf(f, ml.y, sum);
    acc.x = fmaf(f, y.x, acc.x); acc.y = fmaf(f, y.y, acc.y); acc.z = fmaf(f, y.z, acc.z); acc.w = fmaf(f, y.w, acc.w);
  }
  *reinterpret_cast<float4*>(&so[gr][d4]) = acc;
  __shared__ float ssum[GR];
  if (d4 == 0) ssum[gr] = sum;
  __syncthreads();
  if (tid < L) {
    sum = 0.f;
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k = 0; k < GR; ++k) {
      const float4 y = *reinterpret_cast<const float4*>(&so[k][d4]);
      sum += ssum[k];
      acc.x += y.x; acc.y += y.y; acc.z += y.z; acc.w += y.w;
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    put4(out + d4, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
    if (lse && tid == 0) *lse = sum > 0.f ? (M + __log2f(sum)) * kLn2 : -INFINITY;
  }
}

// One workgroup per (sequence, query head).  A sequence of one item is finished already; one of no tokens gets zeros and -inf.
template <int HD, typename TO>
__global__ __launch_bounds__(256) void decode_merge_kernel(AttnArgs a) {
  if (!made_for(a.plan, a.key)) return;
  const int H_q = a.key.H_q, b = blockIdx.x / H_q, h = blockIdx.x % H_q;
  const int item0 = a.plan.dec()[b], n = a.plan.dec()[b + 1] - item0;
  if (n == 1) return;
  const int64_t row = (int64_t)b * H_q + h, first = (int64_t)item0 * H_q + h;
  join<HD, TO>(a.part_o + first * HD, a.part_ml + first * 2, n, H_q, reinterpret_cast<TO*>(a.out) + row * HD, a.lse ? a.lse + row : nullptr);
}

// ---- prefill: the queries of the new tokens.  A workgroup of eight waves takes 384 columns (query, query head of the KV head) of one sequence,
// 48 to a wave, and walks the 64-token halves of the keys they see: codes to registers, widened to bf16 on their way into LDS
// (once for all eight waves), operands back in the order of the lanes.  Two buffers, one barrier per half.  Where few blocks of queries face
// long contexts the keys are split into shares, joined by a second launch.
constexpr int kPfWaves = 8, kPfThreads = 64 * kPfWaves, kColTiles = kQCols / kPfWaves / 16;
constexpr int kPfShares = 512;           // workgroups that too few blocks of queries are split into
constexpr float kRaise = 8.f;           // the reference of a softmax is raised once the maximum has passed it by 2^8: sums and outputs hold that

template <int HD, bool MODS, typename TO>
__global__ __launch_bounds__(kPfThreads, 2) void prefill_kernel(AttnArgs a) {
  constexpr int KS = HD / 32, KC = HD / 64, U = HD / 16, CT = kColTiles;
  constexpr int KFRAGS = 4 * KS, VFRAGS = 2 * U, NCH = HD / 64;      // 1 KB operands of a half; 16-byte chunks of codes a thread moves
  __shared__ __attribute__((aligned(16))) uint4 lds[2][(KFRAGS + VFRAGS) * 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
  if (!made_for(a.plan, a.key)) return;
  const int n_items = a.plan.w[kPfItems];
  const int kvh = blockIdx.x % a.key.H_kv, item = blockIdx.x / a.key.H_kv;
  if (item >= n_items) return;
  const int B = a.key.batch, H_q = a.key.H_q, G = a.G;
  const int b = find_item(a.plan.pf(), B, item), item0 = a.plan.pf()[b];
  const int row0 = a.plan.row_start()[b], n = a.plan.row_start()[b + 1] - row0, len = a.plan.len()[b], len0 = len - n;
  const int chunk = a.plan.w[kPfChunk], shares = ((len + 63) / 64 - 1) / chunk + 1;
  const int64_t cols = (int64_t)n * G;
  const int blocks = (int)((cols + kQCols - 1) / kQCols), j = item - item0, share = j % shares;
  const int64_t x0 = (int64_t)(blocks - 1 - j / shares) * kQCols;    // the longest ones first
  const int prefix = a.prefix ? min(max(a.prefix[b], 0), len) : 0;
  const int full_halves = len / kTokens * 2, tail_rows = len % kTokens;
  // what the block and the wave see: keys up to their last column's own, or the prefix
  const int64_t xl = min(x0 + kQCols, cols) - 1;
  const int seen = max(len0 + (int)(xl / G) + 1, prefix);
  const int h0 = share * min(chunk, 0x3fffffff), h1 = min((seen + 63) / 64, shares > 1 ? h0 + chunk : 0x7fffffff);
  const int64_t w0 = x0 + wave * (16 * CT);
  const bool active = w0 < cols;
  const int wave_first = len0 + (int)(min(w0, cols - 1) / G);         // position of the wave's first column
  const int wave_seen = active ? max(len0 + (int)(min(w0 + 16 * CT, cols) - 1) / G + 1, prefix) : 0;

  uint4 qf[CT][KS];
  int pos[CT];
  float m[CT], l[CT], slope[CT];
  floatx4_t o[CT][U];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int64_t x = min(w0 + 16 * c + r, cols - 1);
    const int qi = (int)(x / G), head = kvh * G + (int)(x - (int64_t)qi * G);
    pos[c] = len0 + qi;
    const bf16_t* qp = a.q + ((int64_t)(row0 + qi) * H_q + head) * HD + 8 * g;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[c][s] = *reinterpret_cast<const uint4*>(qp + 32 * s);
    slope[c] = MODS && a.slopes ? a.slopes[head] : 0.f;
    m[c] = kNoScore; l[c] = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) o[c][u] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  }
  Mods md = mods_of(a, 0.f);

  const int32_t* pages = a.table + (int64_t)b * a.max_pages;
  const int64_t D = (int64_t)a.key.H_kv * HD, tail = (int64_t)b * kTokens * D + kvh * HD;
  uint4 raw[NCH];
  float scale[2] = {0.f, 0.f};
  // a thread's 16-byte chunks: one of the keys and one of the values (HD = 128), or one of either by half of the threads
  const auto fetch = [&](int hf) {
    if (hf >= full_halves) return;
    const int page = pages[hf >> 1];
    const bool good = (uint32_t)page < (uint32_t)a.n_pages;
    const int64_t ph = (int64_t)(good ? page : 0) * a.key.H_kv + kvh;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const bool val = KC == 2 ? i == 1 : tid >= 256;
      raw[i] = reinterpret_cast<const uint4*>((val ? a.v : a.k) + ph * (kTokens * HD) + (hf & 1) * (64 * HD))[KC == 2 ? tid : tid & 255];
    }
    scale[0] = exp_to_scale(a.ke[ph]); scale[1] = exp_to_scale(a.ve[ph]);
  };
  const auto place = [&](int hf, uint4* buf) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const bool val = KC == 2 ? i == 1 : tid >= 256;
      const int id = KC == 2 ? tid : tid & 255, cl = id & 63, cf = id >> 6, cr = cl & 15, cg = cl >> 4;
      uint4 x0, x1;
      if (hf < full_halves) {
        const float sc = val ? scale[1] : scale[0];
        x0 = widen8(raw[i].x, raw[i].y, sc); x1 = widen8(raw[i].z, raw[i].w, sc);
      } else {
        const int first = (hf - full_halves) * 64;
        x0 = x1 = make_uint4(0, 0, 0, 0);
        if (!val) {
          const int tok = first + 16 * (cf / KC) + cr;
          if (tok < tail_rows) {
            const bf16_t* p = a.kt + tail + tok * D + 64 * (cf % KC) + 8 * cg;
            x0 = *reinterpret_cast<const uint4*>(p); x1 = *reinterpret_cast<const uint4*>(p + 32);
          }
        } else {
          uint32_t w[8];
#pragma unroll
          for (int y = 0; y < 16; ++y) {
            const int tok = first + 16 * (y / 4) + 4 * cg + y % 4;
            const uint32_t e = tok < tail_rows ? a.vt[tail + tok * D + 16 * cf + cr] : 0;
            w[y / 2] = y % 2 ? w[y / 2] | e << 16 : e;
          }
          x0 = make_uint4(w[0], w[1], w[2], w[3]); x1 = make_uint4(w[4], w[5], w[6], w[7]);
        }
      }
      uint4* f = buf + (val ? KFRAGS + 2 * cf : 2 * cf) * 64 + cl;
      f[0] = x0; f[64] = x1;
    }
  };

  if (h0 < h1) { fetch(h0); place(h0, lds[0]); }
  __syncthreads();
  for (int hf = h0; hf < h1; ++hf) {
    const uint4* buf = lds[(hf - h0) & 1];
    const bool more = hf + 1 < h1;
    if (more) fetch(hf + 1);
    const int first = hf * 64;
    // (a page outside the pool: its tokens are seen by nobody)
    if (first < wave_seen && (hf >= full_halves || (uint32_t)pages[hf >> 1] < (uint32_t)a.n_pages)) {
      floatx4_t s[CT][4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int c = 0; c < CT; ++c) s[c][t] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const uint4 f = buf[(t * KS + k) * 64 + lane];
#pragma unroll
          for (int c = 0; c < CT; ++c) s[c][t] = mfma(f, qf[c][k], s[c][t]);
        }
      }
      const bool masked = first + 63 > wave_first && first + 63 >= prefix;
      uint4 pf[CT][2];
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        float v[16];
        int step[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) { v[i] = s[c][i / 4][i % 4]; step[i] = 16 * (i / 4) + i % 4; }
        md.slope2 = slope[c] * kLog2e;
        score(v, md, MODS, (float)(first + 4 * g - pos[c]), step);
        if (masked) {
          const int lim = max(pos[c], prefix - 1) - first - 4 * g;      // (the last key seen, from this lane's first)
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = step[i] <= lim ? v[i] : -INFINITY;
        }
        float top = v[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, v[i]);
        top = rows_max(top);
        if (__any(top > m[c] + kRaise)) {
          const float up = fmaxf(m[c], top), f = __builtin_amdgcn_exp2f(m[c] - up);
          m[c] = up;
          l[c] *= f;
#pragma unroll
          for (int u = 0; u < U; ++u) o[c][u] *= f;
        }
        uint32_t p[8];
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          const float p0 = __builtin_amdgcn_exp2f(v[i] - m[c]), p1 = __builtin_amdgcn_exp2f(v[i + 1] - m[c]);
          l[c] += p0 + p1;
          p[i / 2] = pack_bf16(p0, p1);      // one rounding of the probabilities, the matrix pipe's operand: 2^-9 of each, of either sign
        }
        pf[c][0] = make_uint4(p[0], p[1], p[2], p[3]); pf[c][1] = make_uint4(p[4], p[5], p[6], p[7]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint4 f = buf[(KFRAGS + 2 * u + k) * 64 + lane];
#pragma unroll
          for (int c = 0; c < CT; ++c) o[c][u] = mfma(f, pf[c][k], o[c][u]);
        }
    }
    if (more) place(hf + 1, lds[(hf + 1 - h0) & 1]);
    __syncthreads();
  }

#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const float sum = rows_sum(l[c]);
    const int64_t x = w0 + 16 * c + r;
    if (x >= cols) continue;
    const int qi = (int)(x / G);
    const int64_t row = (int64_t)(row0 + qi) * H_q + kvh * G + (x - (int64_t)qi * G);
    if (shares == 1) {
      const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u)
        put4(reinterpret_cast<TO*>(a.out) + row * HD + 16 * u + 4 * g, make_float4(o[c][u][0] * inv, o[c][u][1] * inv, o[c][u][2] * inv, o[c][u][3] * inv));
      if (a.lse && g == 0) a.lse[row] = sum > 0.f ? (m[c] + __log2f(sum)) * kLn2 : -INFINITY;
    } else {
      const int64_t part = ((int64_t)item * a.key.H_kv + kvh) * kQCols + (x - x0);
#pragma unroll
      for (int u = 0; u < U; ++u) *reinterpret_cast<floatx4_t*>(a.part_o + part * HD + 16 * u + 4 * g) = o[c][u];
      if (g == 0) *reinterpret_cast<float2*>(a.part_ml + part * 2) = make_float2(m[c], sum);
    }
  }
}

// One workgroup per (item, KV head, 16 columns): joins the shares of the blocks whose first share the item is.
template <int HD, typename TO>
__global__ __launch_bounds__(256) void prefill_merge_kernel(AttnArgs a) {
  constexpr int L = HD / 4, ROWS = 256 / L;
  if (!made_for(a.plan, a.key)) return;
  const int kvh = blockIdx.x % a.key.H_kv, item = blockIdx.x / a.key.H_kv;
  if (item >= a.plan.w[kPfItems]) return;
  const int b = find_item(a.plan.pf(), a.key.batch, item), j = item - a.plan.pf()[b];
  const int row0 = a.plan.row_start()[b], n = a.plan.row_start()[b + 1] - row0, len = a.plan.len()[b];
  const int shares = ((len + 63) / 64 - 1) / a.plan.w[kPfChunk] + 1;
  if (shares == 1 || j % shares) return;
  const int64_t cols = (int64_t)n * a.G;
  const int64_t x0 = ((cols + kQCols - 1) / kQCols - 1 - j / shares) * kQCols;
  const int d4 = threadIdx.x % L * 4;
  for (int c = blockIdx.y * 16 + threadIdx.x / L; c < blockIdx.y * 16 + 16; c += ROWS) {
    const int64_t x = x0 + c;
    if (x >= cols) break;
    const int64_t part = ((int64_t)item * a.key.H_kv + kvh) * kQCols + c, stride = (int64_t)a.key.H_kv * kQCols;
    float M = kNoScore;
    for (int i = 0; i < shares; ++i) M = fmaxf(M, a.part_ml[(part + i * stride) * 2]);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
    for (int i = 0; i < shares; ++i) {
      const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + (part + i * stride) * 2);
      const float4 y = *reinterpret_cast<const float4*>(a.part_o + (part + i * stride) * HD + d4);
      const float f = __builtin_amdgcn_exp2f(ml.x - M);
      sum = fmaf(f, ml.y, sum);
      acc.x = fmaf(f, y.x, acc.x); acc.y = fmaf(f, y.y, acc.y); acc.z = fmaf(f, y.z, acc.z); acc.w = fmaf(f, y.w, acc.w);
    }
    const int qi = (int)(x / a.G);
    const int64_t row = (int64_t)(row0 + qi) * a.key.H_q + kvh * a.G + (x - (int64_t)qi * a.G);
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    put4(reinterpret_cast<TO*>(a.out) + row * HD + d4, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
    if (a.lse && d4 == 0) a.lse[row] = sum > 0.f ? (M + __log2f(sum)) * kLn2 : -INFINITY;
  }
}

}  // namespace page
}  // namespace echokv
