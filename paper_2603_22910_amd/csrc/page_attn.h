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
#include <type_traits>

#include "page_kernels.h"

namespace echokv {
namespace page {

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
  float *nw_o, *nw_ml;                  // the same of prefill's items of few columns
  Plan plan;
  PlanKey key;
  float scale, cap, to_arg, tanh_k[4];  // to_arg: scale / cap; tanh_k: see score
  int max_pages, n_pages, G, col_tiles, capped;
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

// What is done to the raw products q.k: nothing but a factor, which is left to the exponent's fused multiply-add; a bias by distance, which the sums
// start from; a cap; both, in which case the bias comes behind the cap.
enum { kPlain, kBias, kCap, kCapBias };
struct Mods { float scale2, cap2, to_arg, k0, k1, k2, k3; };
template <int MODE> __device__ __forceinline__ float factor(const Mods& m) { return MODE == kPlain || MODE == kBias ? m.scale2 : 1.f; }
__device__ __forceinline__ Mods mods_of(const AttnArgs& a) {
  return {a.scale * kLog2e, a.cap * kLog2e, a.to_arg, a.tanh_k[0], a.tanh_k[1], a.tanh_k[2], a.tanh_k[3]};
}
// The slope of a column's head in the units in which it is added.
template <int MODE> __device__ __forceinline__ float slope_of(const AttnArgs& a, int head) {
  return MODE == kBias ? a.slopes[head] / a.scale : MODE == kCapBias ? a.slopes[head] * kLog2e : 0.f;
}
// What the products' sums of a column start from: away keys between the query and the lane's first key of the tile.
template <int MODE> __device__ __forceinline__ floatx4_t start_of(float slope, float away) {
  if constexpr (MODE != kBias) return floatx4_t{0.f, 0.f, 0.f, 0.f};
  else return floatx4_t{slope * away, slope * (away + 1.f), slope * (away + 2.f), slope * (away + 3.f)};
}

// Sums of C columns to scores (see factor).  c tanh(s / c), by the largest argument of the wave's: below 0.34 and 0.75 odd polynomials, tanh(x) / x in x^2
// interpolated at the four or six Chebyshev nodes of the range, off by 3e-8 of the value at most; else (1 - e) / (1 + e), e = e^-2x, whose
// error is half a step of one, 2^-24 of the cap.  The shortest has the scale and the cap in its coefficients (tanh_k) and takes five operations where the
// last takes fourteen; the vector unit is what bounds prefill with a cap, and few scores come near one.
// away[c]: key minus query position at the lane's first key, at[i] keys before the i-th.
template <int MODE, int C, int N>
__device__ __forceinline__ void score(float (&s)[C][N], const Mods& m, const float (&slope)[C], const float (&away)[C], const int (&at)[N]) {
  if constexpr (MODE == kCap || MODE == kCapBias) {
    float top = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < N; ++i) top = fmaxf(top, fabsf(s[c][i]));
    if (!__any(!(top * m.to_arg < 0.34f)) && m.k0 != 0.f) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float u = s[c][i] * s[c][i];
          s[c][i] *= fmaf(u, fmaf(u, fmaf(u, m.k3, m.k2), m.k1), m.k0);
          if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);       // (four at a time: more take more registers than there are)
        }
      }
    } else if (__any(!(top * m.to_arg < 0.75f))) {
      const float arg2 = m.to_arg * (-2.f * kLog2e);
#pragma unroll
      for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float e = __builtin_amdgcn_exp2f(fabsf(s[c][i]) * arg2);        // (towards zero from either side: no overflow)
          s[c][i] = copysignf((m.cap2 - m.cap2 * e) * __builtin_amdgcn_rcpf(1.f + e), s[c][i]);
          if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
      }
    } else {
      constexpr float k[6] = {0.99999997f, -0.33332949f, 0.13325259f, -0.05333663f, 0.01956605f, -0.00470355f};
#pragma unroll
      for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float x = s[c][i] * m.to_arg, u = x * x;
          s[c][i] = x * m.cap2 * fmaf(u, fmaf(u, fmaf(u, fmaf(u, fmaf(u, k[5], k[4]), k[3]), k[2]), k[1]), k[0]);
          if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }
  if constexpr (MODE == kCapBias) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int i = 0; i < N; ++i) s[c][i] = fmaf(slope[c], away[c] + (float)at[i], s[c][i]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

template <typename TO> __device__ __forceinline__ void put4(TO* p, float4 v) {
  if constexpr (sizeof(TO) == 2) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
  else *reinterpret_cast<float4*>(p) = v;
}

// Four dims of a finished row, and with the first four its log-sum-exp; a row that sees nothing: zeros and -inf.
template <int HD, typename TO>
__device__ __forceinline__ void finish(const AttnArgs& a, int64_t row, int d4, float4 acc, float M, float sum) {
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  put4(reinterpret_cast<TO*>(a.out) + row * HD + d4, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
  if (a.lse && d4 == 0) a.lse[row] = sum == 0.f ? -INFINITY : (M + __log2f(sum)) * kLn2;
}

// Four dims of column c from the four waves' softmaxes of their own.
template <int HD>
__device__ __forceinline__ float4 join_waves(const float (&so)[4][16][HD + 4], const float (&sm)[4][16], const float (&sl)[4][16], int c, int d4,
                                             float& M, float& sum) {
  M = fmaxf(fmaxf(sm[0][c], sm[1][c]), fmaxf(sm[2][c], sm[3][c]));
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float f = __builtin_amdgcn_exp2f(sm[w][c] - M);
    const float4 y = *reinterpret_cast<const float4*>(&so[w][c][d4]);
    sum = fmaf(f, sl[w][c], sum);
    acc.x = fmaf(f, y.x, acc.x); acc.y = fmaf(f, y.y, acc.y); acc.z = fmaf(f, y.z, acc.z); acc.w = fmaf(f, y.w, acc.w);
  }
  return acc;
}

// The codes of a 64-token half of a page and KV head, as a lane takes them.
template <int HD, bool ONCE> struct Codes {
  static constexpr int KC = HD / 64, U = HD / 16;
  uint4 k[4][KC], v[U];
  __device__ __forceinline__ static uint4 load(const uint4* p) { if constexpr (ONCE) return load_once(p); else return *p; }
  __device__ __forceinline__ void fetch_k(const AttnArgs& a, int64_t ph, int half, int lane) {
    const uint4* p = reinterpret_cast<const uint4*>(a.k + ph * (kTokens * HD) + half * (64 * HD)) + lane;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int c = 0; c < KC; ++c) k[t][c] = load(p + (t * KC + c) * 64);
  }
  __device__ __forceinline__ void fetch_v(const AttnArgs& a, int64_t ph, int half, int lane) {
    const uint4* p = reinterpret_cast<const uint4*>(a.v + ph * (kTokens * HD) + half * (64 * HD)) + lane;
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load(p + u * 64);
  }
};

// A wave's way through every STEP-th half of a sequence's pages.  Pages outside the pool are passed over: their tokens are seen by nobody.
template <int STEP> struct PageWalk {
  const int32_t* pages;
  int n_pages, end, H_kv, kvh;
  // The first half from hf on, and its (page, head).
  __device__ __forceinline__ bool find(int& hf, int64_t& ph) const {
    for (; hf < end; hf += STEP) {
      const int page = scalar_word(pages + (hf >> 1));
      if ((uint32_t)page < (uint32_t)n_pages) { ph = (int64_t)page * H_kv + kvh; return true; }
    }
    return false;
  }
  __device__ __forceinline__ void scales(const AttnArgs& a, int64_t ph, float& ks, float& vs) const {
    ks = exp_to_scale(scalar_byte(a.ke + ph)); vs = exp_to_scale(scalar_byte(a.ve + ph));
  }
};

// ---- decode: one token of every sequence.  A workgroup takes an item (a run of 64-token halves of a sequence's full pages, or its tail) of one KV
// head and up to 16 of its query heads as columns.  Its four waves take the halves in turn, each with a softmax of its own; they are
// joined in LDS.  What bounds it is the reading of the pages: 8 x 4096 tokens of 32 KV heads 42 us, 131072 of 8 heads 43 us, both 6.3 TB/s (a plain streaming read: 6.2).
// The matrix pipe has room to spare, so the probabilities go in as two bf16 numbers, high and low part: an error of 2^-17 of each for two products more.
// Registers are the ring: 16 KB of codes in flight for a wave, eight waves to a compute unit.
// kDecodeItems: workgroups that the pages of a launch are shared out to.  1024, 2048, 4096: 32 sequences of 256 .. 36864 tokens 97, 96, 96 us,
// 2 x 131072 91, 96, 103; 512 is slower for the former.
constexpr int kDecodeItems = 1024;
constexpr int kNarrowItems = 256;       // the same of a prefill launch's few-column part: one round of its workgroups

template <int HD, int MODE, typename TO>
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
  const Mods md = mods_of(a);
  const float fac = factor<MODE>(md), slope[1] = {slope_of<MODE>(a, head)};

  floatx4_t o[U];
#pragma unroll
  for (int u = 0; u < U; ++u) o[u] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  float m = kNoScore, l = 0.f;

  const int begin = j * chunk, end = min(halves, begin + chunk);
  if (begin < halves) {
    // Codes of the next half are requested as soon as those of this one are used up: keys ahead of the softmax, values behind the second product.
    const int32_t* pages = a.table + (int64_t)b * a.max_pages;
    Codes<HD, true> x;
    const PageWalk<4> walk = {pages, a.n_pages, end, a.key.H_kv, kvh};
    int64_t ph = 0;
    float ks = 0.f, vs = 0.f;
    int hf = begin + wave;
    if (walk.find(hf, ph)) {
      x.fetch_k(a, ph, hf & 1, lane);
      x.fetch_v(a, ph, hf & 1, lane);
      walk.scales(a, ph, ks, vs);
    }
    while (hf < end) {
      int next = hf + 4;
      const bool more = walk.find(next, ph);
      float s1[1][16], (&s)[16] = s1[0];
      int step[16];
      const float away = (float)(hf * 64 + 4 * g - (len - 1));
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        floatx4_t acc = start_of<MODE>(slope[0], away + (float)(16 * t));
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          acc = mfma(widen8(x.k[t][c].x, x.k[t][c].y, ks), qf[2 * c], acc);
          acc = mfma(widen8(x.k[t][c].z, x.k[t][c].w, ks), qf[2 * c + 1], acc);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) { s[4 * t + i] = acc[i]; step[4 * t + i] = 16 * t + i; }
      }
      if (more) x.fetch_k(a, ph, next & 1, lane);
      score<MODE>(s1, md, slope, {away}, step);
      float top = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
      top = rows_max(top) * fac;
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
        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[i], fac, -m)), p1 = __builtin_amdgcn_exp2f(fmaf(s[i + 1], fac, -m));
        l += p0 + p1;
        hi[i / 2] = pack_bf16(p0, p1);
        lo[i / 2] = pack_bf16(p0 - __uint_as_float(hi[i / 2] << 16), p1 - __uint_as_float(hi[i / 2] & 0xffff0000u));
      }
      const uint4 ph0 = make_uint4(hi[0], hi[1], hi[2], hi[3]), ph1 = make_uint4(hi[4], hi[5], hi[6], hi[7]);
      const uint4 pl0 = make_uint4(lo[0], lo[1], lo[2], lo[3]), pl1 = make_uint4(lo[4], lo[5], lo[6], lo[7]);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint4 v0 = widen8(x.v[u].x, x.v[u].y, vs), v1 = widen8(x.v[u].z, x.v[u].w, vs);
        o[u] = mfma(v0, ph0, o[u]);
        o[u] = mfma(v0, pl0, o[u]);
        o[u] = mfma(v1, ph1, o[u]);
        o[u] = mfma(v1, pl1, o[u]);
      }
      if (more) { x.fetch_v(a, ph, next & 1, lane); walk.scales(a, ph, ks, vs); }
      hf = next;
    }
  } else {
    // the tail: 32 of its rows to a wave.  Rows past the last one may hold anything: they are read nowhere
    const int rows = len % kTokens, t0 = wave * 32;
    if (t0 < rows) {
      const int64_t D = (int64_t)a.key.H_kv * HD, base = (int64_t)b * kTokens * D + kvh * HD;
      float s1[1][8], (&s)[8] = s1[0];
      const float away = (float)(t0 + 4 * g - (rows - 1));
      int step[8];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const bf16_t* kp = a.kt + base + (int64_t)min(t0 + 16 * t + r, rows - 1) * D + 8 * g;
        floatx4_t acc = start_of<MODE>(slope[0], away + (float)(16 * t));
#pragma unroll
        for (int c = 0; c < KS; ++c) acc = mfma(*reinterpret_cast<const uint4*>(kp + 32 * c), qf[c], acc);
#pragma unroll
        for (int i = 0; i < 4; ++i) { s[4 * t + i] = acc[i]; step[4 * t + i] = 16 * t + i; }
      }
      score<MODE>(s1, md, slope, {away}, step);
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (t0 + 4 * g + step[i] >= rows) s[i] = -INFINITY;
        top = fmaxf(top, s[i]);
      }
      m = rows_max(top) * fac;
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[i], fac, -m)), p1 = __builtin_amdgcn_exp2f(fmaf(s[i + 1], fac, -m));
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
    float M, sum;
    const float4 acc = join_waves<HD>(so, sm, sl, c, d4, M, sum);
    const int h = kvh * a.G + ct * 16 + c;
    if (n_items == 1) {
      finish<HD, TO>(a, (int64_t)b * H_q + h, d4, acc, M, sum);
    } else {
      const int64_t row = (int64_t)item * H_q + h;
      *reinterpret_cast<float4*>(a.part_o + row * HD + d4) = acc;
      if (d4 == 0) *reinterpret_cast<float2*>(a.part_ml + row * 2) = make_float2(M, sum);
    }
  }
}

// Joins `n` partials of one row, strided by `stride` rows, by a workgroup of 256 threads, in a fixed order.
template <int HD, typename TO>
__device__ __forceinline__ void join(const AttnArgs& a, const float* po, const float* pml, int n, int64_t stride, int64_t row) {
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
#pragma unroll 8
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
    finish<HD, TO>(a, row, d4, acc, M, sum);
  }
}

// One workgroup per (sequence, query head): 4 - 5 us behind the other launch.  A sequence of one item is finished already; one of no tokens gets zeros and -inf.
// (Joined by the last workgroup of a row instead, no second launch: with fences at the GPU's scope 131072 tokens 49 -> 976 us, each of them writing back a whole L2; with
// loads and stores past the L2 and no fence 8 x 4096 47 -> 77, the counter of a row being one word for workgroups on all dies.)
template <int HD, typename TO>
__global__ __launch_bounds__(256) void decode_merge_kernel(AttnArgs a) {
  if (!made_for(a.plan, a.key)) return;
  const int H_q = a.key.H_q, b = blockIdx.x / H_q, h = blockIdx.x % H_q;
  const int item0 = a.plan.dec()[b], n = a.plan.dec()[b + 1] - item0;
  if (n == 1) return;
  const int64_t row = (int64_t)b * H_q + h, first = (int64_t)item0 * H_q + h;
  join<HD, TO>(a, a.part_o + first * HD, a.part_ml + first * 2, n, H_q, row);
}

// Shares of `chunk` halves that the first `tokens` of a sequence fill.
__device__ __forceinline__ int parts_of(int tokens, int chunk) { return ((tokens + 63) / 64 - 1) / chunk + 1; }

// ---- prefill: the queries of the new tokens.  A workgroup of eight waves takes 384 columns (query, query head of the KV head) of one sequence,
// 48 to a wave (256, 32 or 128, 16: see grow_kernel), and walks the 64-token halves of the keys they see: codes to registers, widened to bf16 on their way into LDS
// (once for all eight waves), operands back in the order of the lanes.  Two buffers, one barrier per half.  Where few blocks of queries face
// long contexts the keys are split into shares, joined by a second launch.
// The vector unit bounds it, beside the matrix pipe, with which it shares the SIMD's issue: per score an exponential of four slots, a multiply-add, a maximum, an addition,
// half a conversion.  So the running maximum is a reference that is raised by 2^8 at a time, a bias starts the products' sums instead of following
// them, masks cost nothing in halves that all columns see.  8192 causal queries, 32 heads of 128: 497 us = 1.11 PFLOP/s (a large library product: 1.21); 32
// heads over 8: 540, with slopes 604, with a cap of 50 686, of 10 809 (256 columns; of 384 765 and 903).  48 columns to a wave are what its 256 registers hold.
constexpr int kPfWaves = 8, kPfThreads = 64 * kPfWaves;
constexpr float kRaise = 8.f;           // the reference of a softmax is raised once the maximum has passed it by 2^8: sums and outputs hold that

// The same number, of which the compiler knows nothing: what depends on it stays where it is used (out of a loop's registers).
__device__ __forceinline__ int opaque(int x) { asm volatile("" : "+v"(x)); return x; }

// Products with N operands that lie in LDS one KB apart, in order; operand n is requested four products' operands ahead (its latency is that of three
// to four groups of products, and what the compiler would choose is the order that takes the fewest registers).
template <int N, class F> __device__ __forceinline__ void with_operands(const uint4* p, F f) {
  constexpr int A = 4;
  uint4 x[A];
#pragma unroll
  for (int n = 0; n < A; ++n) x[n] = p[n * 64];
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    f(n, x[n % A]);
    if (n + A < N) x[n % A] = p[(n + A) * 64];
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Own LDS operations done, then the workgroup's barrier; loads from memory stay in flight.
__device__ __forceinline__ void barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);                                   // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <int HD, int MODE, typename TO, int CT>
__device__ __forceinline__ void many_columns(const AttnArgs& a, int item, int kvh, uint4* lds) {
  constexpr int KS = HD / 32, KC = HD / 64, U = HD / 16, QC = kPfWaves * 16 * CT;
  const auto kbuf = [&](int hf) { return lds + (hf & 1) * (4 * KS * 64); };                   // halves as operands of 1 KB
  const auto vbuf = [&](int hf) { return lds + (2 * 4 * KS + (hf & 1) * (2 * U)) * 64; };
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
  constexpr bool CAPPED = MODE == kCap || MODE == kCapBias;
  if (item >= a.plan.blocks(CAPPED)[2]) return;
  const int H_q = a.key.H_q, G = a.G;
  const int rank = find_item(a.plan.pf(CAPPED), a.plan.w[kWideSeqs], item), item0 = a.plan.pf(CAPPED)[rank], b = __builtin_amdgcn_readfirstlane(a.plan.order()[rank]);
  const int row0 = a.plan.row_start()[b], n = a.plan.row_start()[b + 1] - row0, len = a.plan.len()[b], len0 = len - n;
  const int chunk = a.plan.blocks(CAPPED)[1], shares = parts_of(len, chunk);
  const int cols = n * G;                   // (below 2^31: the host sees to it)
  const int blocks = (cols - 1) / QC + 1, j = item - item0, share = j % shares;
  const int x0 = (blocks - 1 - j / shares) * QC;    // the longest ones first
  const int prefix = a.prefix ? min(max(a.prefix[b], 0), len) : 0;
  const int full_halves = len / kTokens * 2, tail_rows = len % kTokens;
  // what the block and the wave see: keys up to their last column's own, or the prefix
  const int xl = min(x0, cols - QC) + QC - 1;
  const int seen = max(len0 + xl / G + 1, prefix), parts = parts_of(seen, chunk);
  if (share >= parts) return;
  const int h0 = share * min(chunk, 0x3fffffff), h1 = min((seen + 63) / 64, parts > 1 ? h0 + chunk : 0x7fffffff);
  const int w0 = min(x0 + wave * (16 * CT), cols);      // (cols: none of the wave's columns exists)
  const bool active = w0 < cols;
  const int wave_first = len0 + min(w0, cols - 1) / G;         // position of the wave's first column
  const int wave_seen = active ? max(len0 + (min(w0, cols - 16 * CT) + 16 * CT - 1) / G + 1, prefix) : 0;

  uint4 qf[CT][KS];
  int pos[CT];
  float m[CT], l[CT], slope[CT];
  floatx4_t o[CT][U];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int x = min(w0, cols - 1 - (16 * c + r)) + 16 * c + r;         // the last column again past the end
    const int qi = x / G, head = kvh * G + x - qi * G;
    pos[c] = len0 + qi;
    const bf16_t* qp = a.q + ((int64_t)(row0 + qi) * H_q + head) * HD + 8 * g;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[c][s] = *reinterpret_cast<const uint4*>(qp + 32 * s);
    slope[c] = slope_of<MODE>(a, head);
    m[c] = kNoScore; l[c] = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) o[c][u] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  }
  const Mods md = mods_of(a);
  const float fac = factor<MODE>(md);

  const int32_t* pages = a.table + (int64_t)b * a.max_pages;
  const int64_t D = (int64_t)a.key.H_kv * HD, tail = (int64_t)b * kTokens * D + kvh * HD;
  // What a thread moves of a half: chunks of codes, of the keys by all threads or half of them, of the values by all or the others.  The codes are
  // in registers a step before their place in LDS is free.
  constexpr int KTHREADS = 256 * KC, VOFF = KTHREADS % kPfThreads;
  const bool has_k = tid < KTHREADS, has_v = tid >= VOFF;
  const int vtid = tid - VOFF;
  uint4 kraw, vraw;
  float kscale = 0.f, vscale = 0.f;
  // Pages and scales come through the scalar cache during the softmax: in the products' phase they would be waited for together with the operands' LDS
  // reads, which then could not run ahead.  -1: no page, or none of the pool
  const auto page_of = [&](int hf) {
    if (hf >= min(h1, full_halves)) return -1;
    const int page = scalar_word(pages + (hf >> 1));
    return (uint32_t)page < (uint32_t)a.n_pages ? page : -1;
  };
  const auto head_of = [&](int page) { return (int64_t)max(page, 0) * a.key.H_kv + kvh; };
  const auto fetch_k = [&](int hf, int page) {
    if (hf < min(h1, full_halves) && has_k) kraw = reinterpret_cast<const uint4*>(a.k + head_of(page) * (kTokens * HD) + (hf & 1) * (64 * HD))[tid];
  };
  const auto fetch_v = [&](int hf, int page) {
    if (hf < min(h1, full_halves) && has_v) vraw = reinterpret_cast<const uint4*>(a.v + head_of(page) * (kTokens * HD) + (hf & 1) * (64 * HD))[vtid];
  };
  const auto place_k = [&](int hf) {
    if (hf >= h1 || !has_k) return;
    uint4 x0, x1;
    int id = tid;
    if (hf < full_halves) {
      x0 = widen8(kraw.x, kraw.y, kscale); x1 = widen8(kraw.z, kraw.w, kscale);
    } else {
      id = opaque(tid);
      const int cl = id & 63, cf = id >> 6;
      const int tok = (hf - full_halves) * 64 + 16 * (cf / KC) + (cl & 15);
      x0 = x1 = make_uint4(0, 0, 0, 0);
      if (tok < tail_rows) {
        const bf16_t* p = a.kt + tail + tok * D + 64 * (cf % KC) + 8 * (cl >> 4);
        x0 = *reinterpret_cast<const uint4*>(p); x1 = *reinterpret_cast<const uint4*>(p + 32);
      }
    }
    uint4* f = kbuf(hf - h0) + (id & ~63) + id;      // operands 2 cf and 2 cf + 1 of 64 lanes
    f[0] = x0; f[64] = x1;
  };
  const auto place_v = [&](int hf) {
    if (hf >= h1 || !has_v) return;
    if (hf < full_halves) {
      uint4* f = vbuf(hf - h0) + (vtid & ~63) + vtid;
      f[0] = widen8(vraw.x, vraw.y, vscale); f[64] = widen8(vraw.z, vraw.w, vscale);
    } else {
      const int id = opaque(vtid), cl = id & 63, cf = id >> 6;
      uint16_t* f = reinterpret_cast<uint16_t*>(vbuf(hf - h0) + 2 * cf * 64 + cl);
      const int tok0 = (hf - full_halves) * 64 + 4 * (cl >> 4);
#pragma unroll 1
      for (int y = 0; y < 16; ++y) {
        const int tok = tok0 + 16 * (y / 4) + y % 4;
        f[(y / 8) * 512 + y % 8] = tok < tail_rows ? a.vt[tail + tok * D + 16 * cf + (cl & 15)] : 0;
      }
    }
  };

  uint4 pf[CT][2];
  int page0 = page_of(h0), page1 = page_of(h0 + 1), page2 = page_of(h0 + 2);      // of this half and the next two
  bool have = false;                      // probabilities of the half before
  // A step: products (values of the half before, keys of this one) and softmax.  Waves 0 .. 3 meet the barrier behind the softmax, waves 4 .. 7, which share
  // their SIMDs, behind the products: between two barriers the ones have the matrix pipe first and the others the vector unit.  The wave whose phase is the
  // longer one goes first where both could issue (8192 queries, 32 heads: 515 us, without priorities 570, the other way round 564; with a cap, in blocks of 384, 338, 358, 356).
  const bool lag = wave >= 4;
  const auto step = [&](int hf) {
    __builtin_amdgcn_s_setprio(CAPPED ? 0 : 1);
    const auto stage = [&](int part) {
      if (part == 0) { place_k(hf + 1); fetch_k(hf + 2, page2); }
      if (part == 1) { place_v(hf); fetch_v(hf + 1, page1); }
    };
    if (have) {
      with_operands<2 * U>(vbuf(hf - 1 - h0) + lane, [&](int n, const uint4& f) {
#pragma unroll
        for (int c = 0; c < CT; ++c) o[c][n / 2] = mfma(f, pf[c][n % 2], o[c][n / 2]);
        if (n == 1) stage(0);                          // (in the shadow of the products)
        if (n == 4) stage(1);
      });
    } else {
      stage(0);
      stage(1);
    }
    const int first = hf * 64;
    // (a page outside the pool: its tokens are seen by nobody)
    have = hf < h1 && first < wave_seen && (hf >= full_halves || page0 >= 0);
    floatx4_t s[CT][4];
    if (have)
      with_operands<4 * KS>(kbuf(hf - h0) + lane, [&](int n, const uint4& f) {
#pragma unroll
        for (int c = 0; c < CT; ++c) s[c][n / KS] = mfma(f, qf[c][n % KS], n % KS ? s[c][n / KS] : start_of<MODE>(slope[c], (float)(first + 16 * (n / KS) + 4 * g - pos[c])));
      });
    if (lag) barrier();
    __builtin_amdgcn_s_setprio(CAPPED ? 1 : 0);
    kscale = exp_to_scale(scalar_byte(a.ke + head_of(page2)));
    vscale = exp_to_scale(scalar_byte(a.ve + head_of(page1)));
    const int next = scalar_word(pages + (max(min(hf + 3, full_halves - 1), 0) >> 1));
    if (have) {
      const bool masked = first + 63 > wave_first && first + 63 >= prefix;
      float v[CT][16], top[CT];
      int at[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) at[i] = 16 * (i / 4) + i % 4;
      float away[CT];
#pragma unroll
      for (int c = 0; c < CT; ++c) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[c][i] = s[c][i / 4][i % 4];
        away[c] = (float)(first + 4 * g - pos[c]);
      }
      score<MODE>(v, md, slope, away, at);
      bool higher = false;
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        if (masked) {
          const int lim = max(pos[c], prefix - 1) - first - 4 * g;      // (the last key seen, from this lane's first)
#pragma unroll
          for (int i = 0; i < 16; ++i) v[c][i] = at[i] <= lim ? v[c][i] : -INFINITY;
        }
        top[c] = v[c][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top[c] = fmaxf(top[c], v[c][i]);
        top[c] = rows_max(top[c]) * fac;
        higher |= top[c] > m[c] + kRaise;
      }
      if (__any(higher)) {
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          const float up = fmaxf(m[c], top[c]), f = __builtin_amdgcn_exp2f(m[c] - up);
          m[c] = up;
          l[c] *= f;
#pragma unroll
          for (int u = 0; u < U; ++u) o[c][u] *= f;
        }
      }
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        uint32_t p[8];
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(v[c][i], fac, -m[c])), p1 = __builtin_amdgcn_exp2f(fmaf(v[c][i + 1], fac, -m[c]));
          l[c] += p0 + p1;
          p[i / 2] = pack_bf16(p0, p1);      // one rounding of the probabilities, the matrix pipe's operand: 2^-9 of each, of either sign
        }
        pf[c][0] = make_uint4(p[0], p[1], p[2], p[3]); pf[c][1] = make_uint4(p[4], p[5], p[6], p[7]);
      }
    } else {                              // (they do not live on through the products with the keys)
#pragma unroll
      for (int c = 0; c < CT; ++c) pf[c][0] = pf[c][1] = make_uint4(0, 0, 0, 0);
    }
    page0 = page1; page1 = page2;
    page2 = hf + 3 < min(h1, full_halves) && (uint32_t)next < (uint32_t)a.n_pages ? next : -1;
    if (!lag) barrier();
  };
  if (h0 < h1) {
    fetch_k(h0, page0);
    fetch_v(h0, page0);
    kscale = exp_to_scale(scalar_byte(a.ke + head_of(page0)));
    vscale = exp_to_scale(scalar_byte(a.ve + head_of(page0)));
    place_k(h0);
    fetch_k(h0 + 1, page1);
    kscale = exp_to_scale(scalar_byte(a.ke + head_of(page1)));
    __builtin_amdgcn_s_waitcnt(0x0F70);                                 // vmcnt(0): no load of the queries is waited for inside the loop
    barrier();
    for (int hf = h0; hf <= h1; ++hf) step(hf);       // (the last step adds the last half's values and nothing else)
  }

#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const float sum = rows_sum(l[c]);
    const int off = 16 * c + opaque(r);
    if (off >= cols - w0) continue;
    const int x = w0 + off, qi = x / G;
    const int64_t row = (int64_t)(row0 + qi) * H_q + kvh * G + (x - qi * G);
    if (parts == 1) {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
      for (int u = 0; u < U; ++u)
        put4(reinterpret_cast<TO*>(a.out) + row * HD + 16 * u + 4 * g, make_float4(o[c][u][0] * inv, o[c][u][1] * inv, o[c][u][2] * inv, o[c][u][3] * inv));
      if (a.lse && g == 0) a.lse[row] = sum == 0.f ? -INFINITY : (m[c] + __log2f(sum)) * kLn2;
    } else {
      const int64_t part = ((int64_t)item * a.key.H_kv + kvh) * QC + (x - x0);
#pragma unroll
      for (int u = 0; u < U; ++u) *reinterpret_cast<floatx4_t*>(a.part_o + part * HD + 16 * u + 4 * g) = o[c][u];
      if (g == 0) *reinterpret_cast<float2*>(a.part_ml + part * 2) = make_float2(m[c], sum);
    }
  }
}

// Few columns: a workgroup takes up to 32 columns of one sequence and KV head and a run of halves, which its eight waves take in turn,
// straight from memory to registers as in decode.  Waves that share halves instead of columns have work however few columns there are.
// 49 rows behind 34396 tokens of 8 KV heads, four sequences: 34 us + the join's 5, where the bytes would take 12: a chain of four dependent loads to the first
// half (plan, table, scale, codes), widening once per 32 columns, one round of workgroups.
template <int HD, int MODE, typename TO>
__device__ __forceinline__ void few_columns(const AttnArgs& a, int item, int kvh, uint4* lds) {
  constexpr int KS = HD / 32, KC = HD / 64, U = HD / 16, CT = kNCols / 16;
  struct Join { float so[4][16][HD + 4], sm[4][16], sl[4][16]; };
  static_assert(sizeof(Join) <= (2 * 4 * KS + 2 * 2 * U) * 1024, "in the other form's LDS");
  Join& jn = *reinterpret_cast<Join*>(lds);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
  if (item >= a.plan.w[kNwItems]) return;
  const int H_q = a.key.H_q, G = a.G, b = find_item(a.plan.nw(), a.key.batch, item), j = item - a.plan.nw()[b];
  const int row0 = a.plan.row_start()[b], n = a.plan.row_start()[b + 1] - row0, len = a.plan.len()[b], len0 = len - n;
  const int chunk = a.plan.w[kNwChunk], shares = parts_of(len, chunk), share = j % shares;
  const int cols = n * G, x0 = j / shares * kNCols, nc = min(kNCols, cols - x0);
  const int prefix = a.prefix ? min(max(a.prefix[b], 0), len) : 0;
  const int full_halves = len / kTokens * 2, tail_rows = len % kTokens;
  const int block_first = len0 + x0 / G, seen = max(len0 + (x0 + nc - 1) / G + 1, prefix);
  const int begin = share * chunk, end = min(begin + chunk, (seen + 63) / 64), parts = parts_of(seen, chunk);
  if (share >= parts) return;

  uint4 qf[CT][KS];
  int pos[CT];
  float m[CT], l[CT], slope[CT];
  floatx4_t o[CT][U];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int x = x0 + min(16 * c + r, nc - 1), qi = x / G, head = kvh * G + x - qi * G;
    pos[c] = len0 + qi;
    const bf16_t* qp = a.q + ((int64_t)(row0 + qi) * H_q + head) * HD + 8 * g;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[c][s] = *reinterpret_cast<const uint4*>(qp + 32 * s);
    slope[c] = slope_of<MODE>(a, head);
    m[c] = kNoScore; l[c] = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) o[c][u] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  }
  const Mods md = mods_of(a);
  const float fac = factor<MODE>(md);
  const int32_t* pages = a.table + (int64_t)b * a.max_pages;
  const int64_t D = (int64_t)a.key.H_kv * HD, tail = (int64_t)b * kTokens * D + kvh * HD;

  // Codes of the next half are requested as soon as those of this one are used up, as in decode; other blocks of the sequence read them, too.
  const PageWalk<kPfWaves> walk = {pages, a.n_pages, min(end, full_halves), a.key.H_kv, kvh};
  Codes<HD, false> codes;
  int64_t ph = 0;
  float ks = 0.f, vs = 0.f;
  const auto half = [&](int hf, int next, bool more, auto paged) {
    constexpr bool PAGE = decltype(paged)::value;
    const int first = hf * 64;
    floatx4_t s[CT][4];
    if constexpr (PAGE) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int k = 0; k < KC; ++k) {
          const uint4 f0 = widen8(codes.k[t][k].x, codes.k[t][k].y, ks), f1 = widen8(codes.k[t][k].z, codes.k[t][k].w, ks);
#pragma unroll
          for (int c = 0; c < CT; ++c) {
            s[c][t] = mfma(f0, qf[c][2 * k], k ? s[c][t] : start_of<MODE>(slope[c], (float)(first + 16 * t + 4 * g - pos[c])));
            s[c][t] = mfma(f1, qf[c][2 * k + 1], s[c][t]);
          }
        }
        __builtin_amdgcn_sched_barrier(0);             // (a tile's codes are widened at a time)
      }
      if (more) codes.fetch_k(a, ph, next & 1, lane);
    } else {
      const int t0 = first - full_halves * 64;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const uint32_t at32 = (uint32_t)min(t0 + 16 * t + r, tail_rows - 1) * (uint32_t)D + 8 * g;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const uint4 f = *reinterpret_cast<const uint4*>(a.kt + tail + (at32 + 32 * k));
#pragma unroll
          for (int c = 0; c < CT; ++c) s[c][t] = mfma(f, qf[c][k], k ? s[c][t] : start_of<MODE>(slope[c], (float)(first + 16 * t + 4 * g - pos[c])));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    const bool masked = first + 63 > block_first && first + 63 >= prefix;
    float v[CT][16], away[CT];
    int at[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) at[i] = 16 * (i / 4) + i % 4;
#pragma unroll
    for (int c = 0; c < CT; ++c) {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[c][i] = s[c][i / 4][i % 4];
      away[c] = (float)(first + 4 * g - pos[c]);
    }
    score<MODE>(v, md, slope, away, at);
    uint4 pf[CT][2];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      if (masked) {
        const int lim = max(pos[c], prefix - 1) - first - 4 * g;
#pragma unroll
        for (int i = 0; i < 16; ++i) v[c][i] = at[i] <= lim ? v[c][i] : -INFINITY;
      }
      float top = v[c][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, v[c][i]);
      top = rows_max(top) * fac;
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
        const float p0 = __builtin_amdgcn_exp2f(fmaf(v[c][i], fac, -m[c])), p1 = __builtin_amdgcn_exp2f(fmaf(v[c][i + 1], fac, -m[c]));
        l[c] += p0 + p1;
        p[i / 2] = pack_bf16(p0, p1);        // (rounded once, as in the kernel for many columns)
      }
      pf[c][0] = make_uint4(p[0], p[1], p[2], p[3]); pf[c][1] = make_uint4(p[4], p[5], p[6], p[7]);
    }
    if constexpr (PAGE) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint4 v0 = widen8(codes.v[u].x, codes.v[u].y, vs), v1 = widen8(codes.v[u].z, codes.v[u].w, vs);
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          o[c][u] = mfma(v0, pf[c][0], o[c][u]);
          o[c][u] = mfma(v1, pf[c][1], o[c][u]);
        }
        if (u % 2) __builtin_amdgcn_sched_barrier(0);
      }
      if (more) { codes.fetch_v(a, ph, next & 1, lane); walk.scales(a, ph, ks, vs); }
    } else {
      const int t0 = first - full_halves * 64 + 4 * g;
      const bf16_t* vp = a.vt + tail;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint32_t at32[8];                 // (past the last row: that row again, with probabilities of zero)
#pragma unroll
        for (int x = 0; x < 8; ++x) at32[x] = (uint32_t)min(t0 + 32 * k + 16 * (x / 4) + x % 4, tail_rows - 1) * (uint32_t)D + r;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          uint32_t w[4];
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            const uint32_t e = vp[at32[x] + 16 * u];
            w[x / 2] = x % 2 ? w[x / 2] | e << 16 : e;
          }
          const uint4 f = make_uint4(w[0], w[1], w[2], w[3]);
#pragma unroll
          for (int c = 0; c < CT; ++c) o[c][u] = mfma(f, pf[c][k], o[c][u]);
          if (u % 4 == 3) __builtin_amdgcn_sched_barrier(0);       // (32 loads at a time: more take more registers than there are)
        }
      }
    }
  };
  int hf = begin + wave;
  if (walk.find(hf, ph)) {
    codes.fetch_k(a, ph, hf & 1, lane);
    codes.fetch_v(a, ph, hf & 1, lane);
    walk.scales(a, ph, ks, vs);
  }
  while (hf < walk.end) {
    int next = hf + kPfWaves;
    const bool more = walk.find(next, ph);
    half(hf, next, more, std::true_type{});
    hf = next;
  }
  for (; hf < end; hf += kPfWaves) half(hf, 0, false, std::false_type{});

  const int slot = parts > 1 ? a.plan.nws()[b] + j : 0;
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const float sum1 = rows_sum(l[c]);
    const auto leave = [&] {
      if (g == 0) { jn.sm[wave & 3][r] = m[c]; jn.sl[wave & 3][r] = l[c]; }
#pragma unroll
      for (int u = 0; u < U; ++u) *reinterpret_cast<floatx4_t*>(&jn.so[wave & 3][r][16 * u + 4 * g]) = o[c][u];
    };
    l[c] = sum1;
    __syncthreads();
    if (wave >= 4) leave();
    __syncthreads();
    if (wave < 4) {                                    // each of the first four waves takes one of the others in
      const float m2 = jn.sm[wave][r], up = fmaxf(m[c], m2), f1 = __builtin_amdgcn_exp2f(m[c] - up), f2 = __builtin_amdgcn_exp2f(m2 - up);
      l[c] = l[c] * f1 + jn.sl[wave][r] * f2;
      m[c] = up;
#pragma unroll
      for (int u = 0; u < U; ++u) o[c][u] = o[c][u] * f1 + *reinterpret_cast<floatx4_t*>(&jn.so[wave][r][16 * u + 4 * g]) * f2;
      leave();
    }
    __syncthreads();
    for (int x = tid; x < min(16, nc - 16 * c) * (HD / 4); x += kPfThreads) {
      const int k = x / (HD / 4), d4 = x % (HD / 4) * 4;
      float M, sum;
      const float4 acc = join_waves<HD>(jn.so, jn.sm, jn.sl, k, d4, M, sum);
      if (parts == 1) {
        const int col = x0 + 16 * c + k, qi = col / G;
        const int64_t row = (int64_t)(row0 + qi) * H_q + kvh * G + (col - qi * G);
        finish<HD, TO>(a, row, d4, acc, M, sum);
      } else {
        const int64_t part = ((int64_t)slot * a.key.H_kv + kvh) * kNCols + 16 * c + k;
        *reinterpret_cast<float4*>(a.nw_o + part * HD + d4) = acc;
        if (d4 == 0) *reinterpret_cast<float2*>(a.nw_ml + part * 2) = make_float2(M, sum);
      }
    }
  }
}

template <int HD, int MODE, typename TO>
__global__ __launch_bounds__(kPfThreads, 2) void prefill_kernel(AttnArgs a, int wide_items) {
  __shared__ __attribute__((aligned(16))) uint4 lds[(2 * 4 * (HD / 32) + 2 * 2 * (HD / 16)) * 64];
  if (!made_for(a.plan, a.key)) return;
  const int kvh = blockIdx.x % a.key.H_kv, item = blockIdx.x / a.key.H_kv;
  constexpr bool CAPPED = MODE == kCap || MODE == kCapBias;
  const int cols = a.plan.blocks(CAPPED)[0];
  if constexpr (!CAPPED) {
    if (item < wide_items && cols == kLCols) return many_columns<HD, MODE, TO, 3>(a, item, kvh, lds);
  }
  if (item < wide_items && cols == kMCols) many_columns<HD, MODE, TO, 2>(a, item, kvh, lds);
  else if (item < wide_items) many_columns<HD, MODE, TO, 1>(a, item, kvh, lds);
  else few_columns<HD, MODE, TO>(a, item - wide_items, kvh, lds);
}

// Joins the shares of the columns whose keys are split: a wave per column and KV head, or where those are few a workgroup.
constexpr int kMergeBlocks = 1024;
template <int HD, typename TO>
__global__ __launch_bounds__(256) void prefill_merge_kernel(AttnArgs a) {
  constexpr int L = HD / 4, GR = 64 / L;               // lanes of a row, rows at a time
  if (!made_for(a.plan, a.key)) return;
  const int B = a.key.batch, H_kv = a.key.H_kv, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t units = (int64_t)a.plan.split(a.capped)[B] * H_kv;
  const bool whole = units <= kMergeBlocks;
  for (int64_t i = whole ? blockIdx.x : blockIdx.x * 4 + wave; i < units; i += whole ? gridDim.x : gridDim.x * 4) {
    const int kvh = (int)(i % H_kv), at = (int)(i / H_kv), b = find_item(a.plan.split(a.capped), B, at), x = at - a.plan.split(a.capped)[b];
    const int row0 = a.plan.row_start()[b], cols = a.plan.split(a.capped)[b + 1] - a.plan.split(a.capped)[b], len = a.plan.len()[b];
    const bool narrow = cols <= kNarrow;
    const int chunk = narrow ? a.plan.w[kNwChunk] : a.plan.blocks(a.capped)[1], shares = parts_of(len, chunk), bc = narrow ? kNCols : a.plan.blocks(a.capped)[0];
    // what the column's block sees, hence its parts: a block of one is finished already
    const int last = min(x / bc * bc, cols - bc) + bc - 1, seen = max(len - cols / a.G + last / a.G + 1, a.prefix ? min(a.prefix[b], len) : 0);
    const int parts = parts_of(seen, chunk);
    if (parts == 1) continue;
    const int first = narrow ? a.plan.nws()[b] + x / bc * shares : a.plan.pf_of(a.capped)[b] + ((cols - 1) / bc - x / bc) * shares;
    const int64_t part = ((int64_t)first * H_kv + kvh) * bc + x % bc, stride = (int64_t)H_kv * bc;
    const float* po = (narrow ? a.nw_o : a.part_o) + part * HD;
    const float* pml = (narrow ? a.nw_ml : a.part_ml) + part * 2;
    const int64_t row = (int64_t)(row0 + x / a.G) * a.key.H_q + kvh * a.G + x % a.G;
    if (whole) {
      join<HD, TO>(a, po, pml, parts, stride, row);
      __syncthreads();
      continue;
    }
    const int d4 = lane % L * 4, gr = lane / L;
    float M = kNoScore;
    for (int k = lane; k < parts; k += 64) M = fmaxf(M, pml[k * stride * 2]);
    M = wave_max64(M);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
#pragma unroll 4
    for (int k = gr; k < parts; k += GR) {
      const float2 ml = *reinterpret_cast<const float2*>(pml + k * stride * 2);
      const float4 y = *reinterpret_cast<const float4*>(po + k * stride * HD + d4);
      const float f = __builtin_amdgcn_exp2f(ml.x - M);
      sum = fmaf(f, ml.y, sum);
      acc.x = fmaf(f, y.x, acc.x); acc.y = fmaf(f, y.y, acc.y); acc.z = fmaf(f, y.z, acc.z); acc.w = fmaf(f, y.w, acc.w);
    }
#pragma unroll
    for (int w = L; w < 64; w *= 2) {
      sum += __shfl_xor(sum, w, 64);
      acc.x += __shfl_xor(acc.x, w, 64); acc.y += __shfl_xor(acc.y, w, 64); acc.z += __shfl_xor(acc.z, w, 64); acc.w += __shfl_xor(acc.w, w, 64);
    }
    if (gr == 0) finish<HD, TO>(a, row, d4, acc, M, sum);
  }
}

}  // namespace page
}  // namespace echokv
