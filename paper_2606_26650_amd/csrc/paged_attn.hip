// Attention of new tokens over the paged 8-bit cache (gfx950).
//
// Rows.  The queries of one kv head of a sequence form rows r = i * G + g (new token i,
// query head g of the G = n_q / n_kv that share the kv head); a workgroup takes a tile of
// 16 NR rows and a span of the context, and its four waves take 32-token steps of the span
// in turn, each with a running maximum, sum and output of its own, joined through LDS at the
// end.  Nothing passes through LDS in the loop and no wave waits for another.
//
// Products.  Both are v_mfma_f32_16x16x32_f16.  The scores are formed transposed,
// S^T = K Q^T, so a lane holds one query (column lane % 16) and the tokens 4 g .. 4 g + 3
// (g = lane / 16) of each 16-token unit: exactly the four tokens of a word of the v
// layout, so the probabilities go from the score accumulators into the second product
// O^T = V^T P^T as its operand without leaving the lane, and a row's statistics are per lane.
//   k operand: lane (g, m) holds 16 bytes of token m, values 64 hh + 16 g .. + 15, which are two
//              k-slices of the contraction; the q operand is loaded in the same order.
//   v operand: lane (g, m) holds 16 bytes, the words of values 64 hh + 4 m .. + 3 of tokens
//              4 g .. + 3; the word of value 4 m + e is row m of output tile 4 hh + e.
//
// Codes to fp16: the byte c + 128 under the exponent of 1024 is 1152 + c exactly, minus
// 1152 (one exclusive or per four codes, one byte permute and one packed addition per two).
// Scales: a k scale multiplies the scores, with the softmax scale and the row's q scale. A v
// scale moves into the exponent, p' = 2^(s + log2 v_scale - m), which keeps p' within 2^8
// whatever the scales are (fp16 operands); the denominator adds p' / v_scale.  p' underflows
// at 2^-126, so a token is lost from the denominator where its scale is 2^91 below the
// scale behind the maximum and its weight is not yet under 2^-35: scales are
// therefore held to [2^-61, 2^30], where that cannot be.
// p' is rounded to fp16 for the second product, 2^-11 of each term and an eighth of the half step that the
// bf16 output loses (the sum l adds it in fp32, unrounded); a second product for its lower bits would be
// half as many again. exp2, log2 and the reciprocal are the hardware's, off by one unit of fp32
// each, below the d roundings of a score: the library's add instructions for denormals and the last
// bit, which neither the output nor a score holds.
// The running maximum is only raised when a score exceeds it by 2^8 (p' <= 256 is as good
// in fp16 as p' <= 1), so the rescaling of the output is rare.
//
// What bounds it: the codes from HBM where the context is long (64 sequences of up to 8192 tokens, 8 kv
// heads of 128: 131 us, 4.5 TB/s; vector ALU 32%, matrix cores 6%), and where it is
// short one chain of latencies (lengths, page, codes, join): 7.5 us at 300 tokens. One
// sequence of 131072 tokens: 46 us and 4 for the join of its 64 spans a head (58 us together with the gap).
#include <algorithm>
#include <type_traits>

#include "kv_common.h"

namespace catq {
namespace {

typedef _Float16 f16;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

struct PaArgs {
  KvGeom g;
  const int8_t* K;
  const int8_t* V;
  const float* KS;
  const float* VS;
  const bf16* Q;
  bf16* O;
  float* lse;
  float* part_o;     // [span][token][head][D], where the context is split
  float* part_ml;    // [span][token][head][2]
  int32_t G;         // query heads per kv head
  int32_t row_tiles; // of a sequence and kv head
  int32_t tile_rows; // of a workgroup
  int32_t spans;
  int32_t span;      // tokens of a span: a multiple of 128
  int32_t limit;     // no position from here on is read: the pages' and the spans' end
  float c;           // softmax scale * log2(e)
};

constexpr float kNone = -3.0e38f;    // running maximum before any token
constexpr float kRaise = 8.0f;       // log2 units a score may exceed it by
constexpr float kTinyScale = 8.673617379884035e-19f;   // 2^-60: a smaller v scale counts as 0
constexpr float kHugeScale = 1073741824.0f;            // 2^30: a larger one as NaN

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// four codes of a word as fp16
__device__ __forceinline__ void codes_f16(unsigned int w, unsigned int& lo, unsigned int& hi) {
  const unsigned int u = w ^ 0x80808080u;
  const unsigned int a = __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u);   // 0x64 u1 0x64 u0
  const unsigned int b = __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u);
  const f16x2 bias = {(f16)-1152.0f, (f16)-1152.0f};
  lo = __builtin_bit_cast(unsigned int, __builtin_bit_cast(f16x2, a) + bias);
  hi = __builtin_bit_cast(unsigned int, __builtin_bit_cast(f16x2, b) + bias);
}
__device__ __forceinline__ f16x8 codes8(unsigned int w0, unsigned int w1) {
  u32x4 r;
  unsigned int a, b;
  codes_f16(w0, a, b);
  r[0] = a; r[1] = b;
  codes_f16(w1, a, b);
  r[2] = a; r[3] = b;
  return __builtin_bit_cast(f16x8, r);
}
__device__ __forceinline__ f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
// the larger, or NaN if either is
__device__ __forceinline__ float nan_max(float a, float b) { return __builtin_elementwise_maximum(a, b); }
// over the four lanes that hold a query's tokens
__device__ __forceinline__ float col_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float col_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// tokens that new token i of sequence q sees
__device__ __forceinline__ int visible(const PaArgs& a, const KvSeq& q, int i) {
  const int64_t v = min((int64_t)q.ctx + i + 1, (int64_t)a.limit);
  return v < 0 ? 0 : (int)v;
}

template <int D, int NR, bool PER_TOKEN>
__global__ __launch_bounds__(256) void paged_attn_kernel(PaArgs a) {
  constexpr int HH = D / 64;          // 64-value halves of a head
  constexpr int NT = D / 16;          // output tiles
  constexpr int PITCH = D + 4;
  __shared__ __align__(16) float s_o[4][16 * PITCH];
  __shared__ float s_m[4][16], s_l[4][16];
  const KvGeom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lg = lane >> 4, lm = lane & 15;
  // kv heads fastest: the tiles of a head then share an L2 where n_kv is a multiple of 8
  unsigned b = blockIdx.x;
  const int h = b % g.n_kv;
  b /= g.n_kv;
  const int rt = a.row_tiles - 1 - (int)(b % a.row_tiles);   // the longest rows first
  const int sp = b / a.row_tiles, s = blockIdx.y;
  const KvSeq q = kv_seq(g, s);
  const int rows = q.n * a.G, r0 = rt * 16 * NR;
  if (r0 >= rows) return;
  const int last = min(r0 + 16 * NR, rows) - 1;
  const int vmax = visible(a, q, last / a.G);
  const int c0 = sp * a.span;
  if (sp > 0 && c0 >= vmax) return;      // the join knows which spans are there
  const int c1 = min(vmax, c0 + a.span);
  const int vmin = visible(a, q, r0 / a.G);   // every row of the tile sees that much

  // queries: fp16 of q over the power of two at its row's largest magnitude. A row with a NaN or an
  // infinity in it (or a magnitude that passes fp32 times the softmax scale) is taken as zeros and made
  // NaN at the end if it has seen a token.
  f16x8 qf[NR][2 * HH];
  float qc[NR];        // that power times the softmax scale, in log2 units
  int vis[NR];
  bool odd[NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const int row = min(r0 + 16 * r + lm, rows - 1);
    const int i = row / a.G, hq = h * a.G + (row - i * a.G);
    vis[r] = visible(a, q, i);
    const bf16* qp = a.Q + ((q.row0 + i) * g.n_q + hq) * D + 16 * lg;
    float v[HH][16];
    float m = 0.f;
#pragma unroll
    for (int hh = 0; hh < HH; ++hh) {
      float t[8];
      load8<bf16>(qp + 64 * hh, t);
#pragma unroll
      for (int j = 0; j < 8; ++j) { v[hh][j] = t[j]; m = nan_max(m, fabsf(t[j])); }
      load8<bf16>(qp + 64 * hh + 8, t);
#pragma unroll
      for (int j = 0; j < 8; ++j) { v[hh][8 + j] = t[j]; m = nan_max(m, fabsf(t[j])); }
    }
    m = nan_max(m, __shfl_xor(m, 16, 64));
    m = nan_max(m, __shfl_xor(m, 32, 64));
    const int e = min(max((int)(__float_as_uint(m) >> 23) - 127, -100), 126);
    const float down = __uint_as_float((unsigned)(127 - e) << 23);
    qc[r] = __uint_as_float((unsigned)(127 + e) << 23) * a.c;
    odd[r] = !(m < INFINITY) || !(qc[r] < INFINITY);
    if (odd[r]) {
      qc[r] = 0.f;
#pragma unroll
      for (int hh = 0; hh < HH; ++hh)
#pragma unroll
        for (int j = 0; j < 16; ++j) v[hh][j] = 0.f;
    }
#pragma unroll
    for (int hh = 0; hh < HH; ++hh)
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) qf[r][2 * hh + k][j] = (f16)(v[hh][8 * k + j] * down);
  }

  f32x4 o[NR][NT];
  float m[NR], l[NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    m[r] = kNone;
    l[r] = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t) o[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const int32_t* table = g.table + (int64_t)s * g.max_pages;
  const int ps_mask = (1 << g.ps_log2) - 1;
  // page of each 16-token unit of 1024 tokens, one per lane
  auto pages_at = [&](int tok) {
    const int t = tok + 16 * lane;
    return t < vmax ? table[t >> g.ps_log2] : -1;
  };
  u32x4 kc[2][HH], vc[2][HH];
  float ks[2][PER_TOKEN ? 4 : 1], vs[2][PER_TOKEN ? 4 : 1];
  bool bad[2];
  int held = 0;            // first token of the pages in `pg`
  int pg = 0;
  auto fetch = [&](int tok) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int t = tok + 16 * u;
      const int page = __builtin_amdgcn_readlane(pg, (t - held) >> 4);
      bad[u] = page < 0 || page >= g.n_pages;
      const int pid = bad[u] ? 0 : page, ti = t & ps_mask;
      const int64_t base = kv_code_base(g, pid, h, ti);
      const int8_t* kp = a.K + base + lm * D + 16 * lg;
      const int8_t* vp = a.V + base + lg * 4 * D + 16 * lm;
#pragma unroll
      for (int hh = 0; hh < HH; ++hh) {
        kc[u][hh] = *reinterpret_cast<const u32x4*>(kp + 64 * hh);
        vc[u][hh] = *reinterpret_cast<const u32x4*>(vp + 256 * hh);
      }
      const int64_t si = kv_scale_index(g, pid, h, ti);
      if constexpr (PER_TOKEN) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(a.KS + si + 4 * lg);
        const f32x4 y = *reinterpret_cast<const f32x4*>(a.VS + si + 4 * lg);
#pragma unroll
        for (int i = 0; i < 4; ++i) { ks[u][i] = x[i]; vs[u][i] = y[i]; }
      } else {
        ks[u][0] = a.KS[si];
        vs[u][0] = a.VS[si];
      }
    }
  };

  const int t0 = c0 + 32 * wave;
  if (t0 < c1) {
    held = c0;
    pg = pages_at(held);
    fetch(t0);
  }
  for (int tok = t0; tok < c1; tok += 128) {
    // operands of this step, then the loads of the next
    f16x8 kf[2][2 * HH], vf[NT];
    constexpr int NS = PER_TOKEN ? 4 : 1;
    float ksc[2][NS], lv[2][NS], rv[2][NS];
    bool masked[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int hh = 0; hh < HH; ++hh) {
        kf[u][2 * hh] = codes8(kc[u][hh][0], kc[u][hh][1]);
        kf[u][2 * hh + 1] = codes8(kc[u][hh][2], kc[u][hh][3]);
      }
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        ksc[u][i] = ks[u][i];
        const float y = vs[u][i] < kTinyScale    ? kTinyScale
                        : vs[u][i] <= kHugeScale ? vs[u][i]
                                                 : __builtin_nanf("");
        lv[u][i] = __builtin_amdgcn_logf(y);
        rv[u][i] = __builtin_amdgcn_rcpf(y);
      }
      masked[u] = bad[u];
    }
#pragma unroll
    for (int hh = 0; hh < HH; ++hh)
#pragma unroll
      for (int e = 0; e < 4; ++e) vf[4 * hh + e] = codes8(vc[0][hh][e], vc[1][hh][e]);
    bool zero[2][NS];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < NS; ++i) zero[u][i] = vs[u][i] < kTinyScale;
    if (tok + 128 < c1) {
      if (tok + 128 - held >= 1024) {
        held += 1024;
        pg = pages_at(held);
      }
      fetch(tok + 128);
    }
    const bool edge = tok + 32 > vmin || masked[0] || masked[1];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      float x[2][4];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 2 * HH; ++k) acc = mfma(kf[u][k], qf[r][k], acc);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int si = PER_TOKEN ? i : 0;
          x[u][i] = fmaf(acc[i], ksc[u][si] * qc[r], lv[u][si]);
        }
        if (edge) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (masked[u] || tok + 16 * u + 4 * lg + i >= vis[r]) x[u][i] = -INFINITY;
        }
      }
      float mx = x[0][0];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, x[u][i]);
      if (__any(mx > m[r] + kRaise)) {
        const float mn = col_max(fmaxf(m[r], mx));
        const float f = exp2_fast(m[r] - mn);
        m[r] = mn;
        l[r] *= f;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[r][t][i] *= f;
      }
      f16x8 p;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int si = PER_TOKEN ? i : 0;
          const float w = exp2_fast(x[u][i] - m[r]);
          if (edge)
            l[r] += x[u][i] == -INFINITY ? 0.f : w * rv[u][si];   // (a masked scale may be anything)
          else
            l[r] = fmaf(w, rv[u][si], l[r]);
          p[4 * u + i] = zero[u][si] ? (f16)0.f : (f16)w;
        }
#pragma unroll
      for (int t = 0; t < NT; ++t) o[r][t] = mfma(vf[t], p, o[r][t]);
    }
  }

  // join the four waves, one row tile at a time
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    if (r0 + 16 * r >= rows) break;
    float lr = col_sum(l[r]);
    if (odd[r] && lr != 0.f) lr = __builtin_nanf("");
    if (lg == 0) {
      s_m[wave][lm] = m[r];
      s_l[wave][lm] = lr;
    }
    __syncthreads();
    float M = s_m[0][lm];
#pragma unroll
    for (int w = 1; w < 4; ++w) M = fmaxf(M, s_m[w][lm]);
    const float f = exp2_fast(m[r] - M);
    // lane (g, column): values 64 hh + 16 g + 4 i + e of output tile 4 hh + e, register i
#pragma unroll
    for (int hh = 0; hh < HH; ++hh)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = o[r][4 * hh + e][i] * f;
        *reinterpret_cast<f32x4*>(&s_o[wave][lm * PITCH + 64 * hh + 16 * lg + 4 * i]) = y;
      }
    __syncthreads();
    for (int c = tid; c < 16 * (D / 8); c += 256) {
      const int col = c / (D / 8), d8 = (c % (D / 8)) * 8, row = r0 + 16 * r + col;
      if (row >= rows) continue;
      float Mc = s_m[0][col];
#pragma unroll
      for (int w = 1; w < 4; ++w) Mc = fmaxf(Mc, s_m[w][col]);
      float L = 0.f, y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        L = fmaf(s_l[w][col], exp2_fast(s_m[w][col] - Mc), L);
        float z[8];
        load8<float>(&s_o[w][col * PITCH + d8], z);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] += z[j];
      }
      const int i = row / a.G, hq = h * a.G + (row - i * a.G);
      const int64_t at = (q.row0 + i) * g.n_q + hq;
      if (a.spans > 1) {
        const int64_t pa = (int64_t)sp * g.n_tokens * g.n_q + at;
        store8<float>(a.part_o + pa * D + d8, y);
        if (d8 == 0) {
          a.part_ml[2 * pa] = Mc;
          a.part_ml[2 * pa + 1] = L;
        }
        continue;
      }
      const float inv = L > 0.f ? 1.0f / L : (L == 0.f ? 0.f : L);   // (a NaN stays)
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] *= inv;
      store8<bf16>(a.O + at * D + d8, y);
      if (a.lse && d8 == 0)
        a.lse[at] = L == 0.f ? -INFINITY : (Mc + __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ many rows
//
// A workgroup takes 32 NW rows (128 or 256), 32 per wave, and 64-token tiles of the span: the NW
// waves convert a tile's codes once, into LDS as fp16 operands, and each forms S^T = K Q^T and
// O^T = V^T P^T of its rows with v_mfma_f32_32x32x16_f16. As above a lane holds one query
// (column lane % 32), its scores of a 32-token block are the tokens 8 qd + 4 h + e (h = lane / 32)
// in register 4 qd + e, and those are, in order, the contraction slots of the second
// product when the v operand takes the four-token words 4 T + h and 4 T + 2 + h of each 16 tokens.
//   s_k [slice ks][h][token], 65 tokens apart: values 16 ks + 8 h .. + 7 of the token, 16 bytes
//   s_v [T][h][d]: the eight tokens of those two words at value d, 16 bytes
// (16 lanes read, and write k, in 16 different 16-byte banks; one lane address for all reads).
// LDS is double-buffered, one barrier per tile; the codes of the next tile are loaded while
// this one is multiplied.
//
// Three prompt chunks of 2000, 792 and 1184 tokens behind up to 4000, 40 + 8 heads of 128: 401 us,
// 825 TFLOP/s. Per wave and tile 248 vector instructions (32 of them exponentials at a quarter rate)
// and 32 products, 1380 and 1024 cycles, which do not overlap: the matrix cores are busy
// 34% of the time, the vector ALU 50%, and 16% of the units wait at the end. Giving the two
// waves of a SIMD turns (one multiplies, one exponentiates, a barrier between) brought nothing
// (420 us), nor did half tiles interleaved inside a wave (they spill).
// A tile's v scale is in lv (log2, NaN outside its range, -inf on a page that does not
// exist) and rv (its reciprocal, always finite, so that a masked token adds 0). One that counts as 0
// has the lv and rv of 2^-61, which no scale that counts has.
constexpr int kTile = 64, kPitch = kTile + 1;
constexpr float kTinyLog = -61.0f;

template <int D, int NW, bool PER_TOKEN>
__global__ __launch_bounds__(NW * 64, 2) void paged_tile_kernel(PaArgs a) {
  constexpr int KS = D / 16;            // contraction slices of the scores
  constexpr int DB = D / 32;            // output blocks
  constexpr int NT = NW * 64, kRows = NW * 32;
  constexpr int KP = (4 * D + NT - 1) / NT;   // 16-byte pieces of k per thread
  __shared__ __align__(16) u32x4 s_k[2][KS * 2 * kPitch];
  __shared__ __align__(16) u32x4 s_v[2][8 * D];
  __shared__ __align__(16) float s_ks[2][kTile], s_lv[2][kTile], s_rv[2][kTile];
  __shared__ int s_tiny[2];
  const KvGeom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5, l32 = lane & 31;
  unsigned b = blockIdx.x;
  const int h = b % g.n_kv;
  b /= g.n_kv;
  const int rt = a.row_tiles - 1 - (int)(b % a.row_tiles);   // the longest rows first
  const int sp = b / a.row_tiles, s = blockIdx.y;
  const KvSeq q = kv_seq(g, s);
  const int rows = q.n * a.G, r0 = rt * kRows;
  if (r0 >= rows) return;
  const int vmax = visible(a, q, (min(r0 + kRows, rows) - 1) / a.G);
  const int c0 = sp * a.span;
  if (sp > 0 && c0 >= vmax) return;      // the join knows which spans are there
  const int c1 = min(vmax, c0 + a.span);
  // this wave's rows
  const int w0 = r0 + 32 * wave;
  const bool has_rows = w0 < rows;
  const int row = min(w0 + l32, rows - 1), qi = row / a.G, hq = h * a.G + (row - qi * a.G);
  const int vis = visible(a, q, qi);
  const int wmin = visible(a, q, min(w0, rows - 1) / a.G);
  const int wmax = has_rows ? visible(a, q, min(w0 + 31, rows - 1) / a.G) : 0;

  // queries as above; the score of a token on a missing page is then -inf whatever the query is.
  // (Setting those scores in the loop took 396 us for the prompt chunks above where this takes 386.)
  f16x8 qf[KS];
  float qc;
  bool odd;
  {
    const bf16* qp = a.Q + ((q.row0 + qi) * g.n_q + hq) * D + 8 * hh;
    float m = 0.f;
    u32x4 raw[KS];
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      raw[k] = *reinterpret_cast<const u32x4*>(qp + 16 * k);
#pragma unroll
      for (int j = 0; j < 4; ++j) m = nan_max(m, nan_max(fabsf(bf16_lo(raw[k][j])), fabsf(bf16_hi(raw[k][j]))));
    }
    m = nan_max(m, __shfl_xor(m, 32, 64));
    const int e = min(max((int)(__float_as_uint(m) >> 23) - 127, -100), 126);
    const float down = __uint_as_float((unsigned)(127 - e) << 23);
    qc = __uint_as_float((unsigned)(127 + e) << 23) * a.c;
    odd = !(m < INFINITY) || !(qc < INFINITY);
    if (odd) {
      qc = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) raw[k] = u32x4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        qf[k][2 * j] = (f16)(bf16_lo(raw[k][j]) * down);
        qf[k][2 * j + 1] = (f16)(bf16_hi(raw[k][j]) * down);
      }
  }

  const int32_t* table = g.table + (int64_t)s * g.max_pages;
  const int ps_mask = (1 << g.ps_log2) - 1;
  auto page_of = [&](int tok) {
    const int pg = tok < vmax ? table[tok >> g.ps_log2] : -1;
    return pg < 0 || pg >= g.n_pages ? -1 : pg;
  };
  // staging: k piece p = tid + NT i is values 16 (p % KS) .. + 15 of token p / KS; v: thread tid
  // takes values VD dv .. + VD - 1 of word rows 4 T + vh and 4 T + 2 + vh
  constexpr int VD = 8 * D >= NT * 4 ? 4 : 8 * D >= NT * 2 ? 2 : 1;
  constexpr int VT = D / VD;               // threads per (T, vh)
  constexpr bool kAllK = 4 * D >= NT, kAllV = VT * 8 >= NT;   // (else some threads have none)
  const int dv = VD * (tid % VT), vt = tid / VT, vT = (vt >> 1) & 3, vh = vt & 1;
  const bool k_mine = kAllK || tid < 4 * D, v_mine = kAllV || vt < 8;
  static_assert(VT * 8 <= NT, "one v task per thread");
  typedef __attribute__((ext_vector_type(VD))) unsigned int vwords;
  u32x4 kc[KP];
  vwords vc[2];
  float ksr, vsr;
  bool none;
  // a page's bytes in either code array, and its scales, with the head's place in them
  const unsigned page_codes = (unsigned)(g.n_kv << g.ps_log2) * D, head_codes = (unsigned)(h << g.ps_log2) * D;
  const unsigned page_scales = (unsigned)g.n_kv << (g.ps_log2 - g.bt_log2),
                 head_scales = (unsigned)h << (g.ps_log2 - g.bt_log2);
  // places inside the tile
  const int kt = (tid % (4 * D)) / KS, vtok = 16 * vT + 4 * vh;
  const unsigned koff = 16 * (tid % KS), voff = 4 * dv;
  // the next tile's pages: one for all of it where a page holds whole tiles, one per lane's part
  // of it (each k piece, its v words, token `lane`) elsewhere
  const bool one_page = g.ps_log2 >= 6;
  int pk[KP], pv, pp;
  auto pages = [&](int t0) __attribute__((always_inline)) {
    if (one_page) {
      pp = page_of(__builtin_amdgcn_readfirstlane(t0));
      return;
    }
#pragma unroll
    for (int i = 0; i < KP; ++i) pk[i] = page_of(t0 + kt + i * (NT / KS));
    pv = page_of(t0 + vtok);
    pp = page_of(t0 + lane);
  };
  auto fetch = [&](int t0) __attribute__((always_inline)) {
    if (one_page) {
      const int pg = __builtin_amdgcn_readfirstlane(pp), t = t0 & ps_mask;
      const uint64_t base = (uint64_t)(unsigned)max(pg, 0) * page_codes + (head_codes + (unsigned)t * D);
      const int8_t *kb = a.K + base, *vb = a.V + base;
#pragma unroll
      for (int i = 0; i < KP; ++i)
        kc[i] = *reinterpret_cast<const u32x4*>(kb + ((unsigned)(kt + i * (NT / KS)) * D + koff));
      vc[0] = *reinterpret_cast<const vwords*>(vb + ((unsigned)vtok * D + voff));
      vc[1] = *reinterpret_cast<const vwords*>(vb + ((unsigned)(vtok + 8) * D + voff));
      const uint64_t sb = (uint64_t)(unsigned)max(pg, 0) * page_scales + (head_scales + ((unsigned)t >> g.bt_log2));
      ksr = a.KS[sb + ((unsigned)lane >> g.bt_log2)];
      vsr = a.VS[sb + ((unsigned)lane >> g.bt_log2)];
      none = pg < 0;
      return;
    }
#pragma unroll
    for (int i = 0; i < KP; ++i) {
      const unsigned off = head_codes + (unsigned)((t0 + kt + i * (NT / KS)) & ps_mask) * D + koff;
      kc[i] = *reinterpret_cast<const u32x4*>(a.K + ((uint64_t)(unsigned)max(pk[i], 0) * page_codes + off));
    }
    const unsigned off = head_codes + (unsigned)((t0 + vtok) & ps_mask) * D + voff;
    const int8_t* vp = a.V + ((uint64_t)(unsigned)max(pv, 0) * page_codes + off);
    vc[0] = *reinterpret_cast<const vwords*>(vp);
    vc[1] = *reinterpret_cast<const vwords*>(vp + 8 * D);
    const uint64_t si = (uint64_t)(unsigned)max(pp, 0) * page_scales +
                        (head_scales + ((unsigned)((t0 + lane) & ps_mask) >> g.bt_log2));
    ksr = a.KS[si];
    vsr = a.VS[si];
    none = pp < 0;
  };
  auto stage = [&](int buf) __attribute__((always_inline)) {
    if (k_mine) {
#pragma unroll
      for (int i = 0; i < KP; ++i) {
        const int tok = kt + i * (NT / KS), ks = tid % KS;
        s_k[buf][(2 * ks) * kPitch + tok] = __builtin_bit_cast(u32x4, codes8(kc[i][0], kc[i][1]));
        s_k[buf][(2 * ks + 1) * kPitch + tok] =
            __builtin_bit_cast(u32x4, codes8(kc[i][2], kc[i][3]));
      }
    }
    if (v_mine) {
#pragma unroll
      for (int e = 0; e < VD; ++e) {
        const int d = dv + e;
        s_v[buf][(2 * vT + vh) * D + d] =
            __builtin_bit_cast(u32x4, codes8(vc[0][e], vc[1][e]));
      }
    }
    if (wave == 0) {
      const bool tiny = vsr < kTinyScale, fine = vsr <= kHugeScale && !tiny;
      s_ks[buf][lane] = none ? 0.f : ksr;
      s_lv[buf][lane] = none ? -INFINITY : fine ? __builtin_amdgcn_logf(vsr) : tiny ? kTinyLog : __builtin_nanf("");
      s_rv[buf][lane] = none || !(fine || tiny) ? 1.f : __builtin_amdgcn_rcpf(fine ? vsr : 0.5f * kTinyScale);
      s_tiny[buf] = __any(tiny && !none);
    }
  };

  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  // m: the running maximum, 0 until the row has seen a token; limit: what a score may exceed it by
  float m = 0.f, l = 0.f, limit = -INFINITY;

  if (c0 < c1) {
    pages(c0);
    fetch(c0);
    pages(c0 + kTile);
  }
  int buf = 0;
  for (int t0 = c0; t0 < c1; t0 += kTile, buf ^= 1) {
    stage(buf);
    __syncthreads();
    if (t0 + kTile < c1) {
      fetch(t0 + kTile);
      pages(t0 + 2 * kTile);
    }
    if (t0 >= wmax) continue;   // (the wave still stages what the others need)
    f32x16 x[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[u][i] = 0.f;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int u = 0; u < 2; ++u)
        x[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
            __builtin_bit_cast(f16x8, s_k[buf][(2 * k + hh) * kPitch + 32 * u + l32]), qf[k], x[u],
            0, 0, 0);
    // scores over the running maximum: one scale per 16 tokens (two groups of four registers), or per token
    float mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int qd = 0; qd < 4; ++qd) {
        if constexpr (PER_TOKEN) {
          const f32x4 k4 = *reinterpret_cast<const f32x4*>(&s_ks[buf][32 * u + 8 * qd + 4 * hh]);
          const f32x4 l4 = *reinterpret_cast<const f32x4*>(&s_lv[buf][32 * u + 8 * qd + 4 * hh]);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[u][4 * qd + e] = fmaf(x[u][4 * qd + e], k4[e] * qc, l4[e] - m);
        } else {
          const float kq = s_ks[buf][32 * u + 16 * (qd >> 1)] * qc, lm = s_lv[buf][32 * u + 16 * (qd >> 1)] - m;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[u][4 * qd + e] = fmaf(x[u][4 * qd + e], kq, lm);
        }
      }
    if (t0 + kTile > wmin) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (t0 + 32 * u + 8 * (i >> 2) + 4 * hh + (i & 3) >= vis) x[u][i] = -INFINITY;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, x[u][i]);
    if (__any(mx > limit)) {
      // raise the maximum to the largest score of the row (of both halves' tokens); the first
      // one seen sets it, also below 0
      const float rm = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const bool first = limit != kRaise, any = rm > -INFINITY;
      const float up = first ? (any ? rm : 0.f) : fmaxf(rm, 0.f);
      const float f = first ? 1.0f : exp2_fast(-up);
      limit = any ? kRaise : limit;
      m += up;
      l *= f;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= f;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[u][i] -= up;
    }
    f16x8 p[2][2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int qd = 0; qd < 4; ++qd) {
        float w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w[e] = exp2_fast(x[u][4 * qd + e]);
          p[u][qd >> 1][4 * (qd & 1) + e] = (f16)w[e];
        }
        if constexpr (PER_TOKEN) {
          const f32x4 r4 = *reinterpret_cast<const f32x4*>(&s_rv[buf][32 * u + 8 * qd + 4 * hh]);
#pragma unroll
          for (int e = 0; e < 4; ++e) l = fmaf(w[e], r4[e], l);
        } else {
          l = fmaf((w[0] + w[1]) + (w[2] + w[3]), s_rv[buf][32 * u + 16 * (qd >> 1)], l);
        }
      }
    if (__builtin_amdgcn_readfirstlane(s_tiny[buf])) {   // some scales count as 0: their tokens' terms are 0
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (s_lv[buf][32 * u + 8 * (i >> 2) + 4 * hh + (i & 3)] == kTinyLog) p[u][i >> 3][i & 7] = (f16)0.f;
    }
#pragma unroll
    for (int T = 0; T < 4; ++T)
#pragma unroll
      for (int d = 0; d < DB; ++d)
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
            __builtin_bit_cast(f16x8, s_v[buf][(2 * T + hh) * D + 32 * d + l32]), p[T >> 1][T & 1], o[d], 0,
            0, 0);
  }
  if (!has_rows || w0 + l32 >= rows) return;
  float L = l + __shfl_xor(l, 32, 64);
  if (odd && L != 0.f) L = __builtin_nanf("");
  const int64_t at = (q.row0 + qi) * g.n_q + hq;
  // register 4 qd + e of block d: value 32 d + 8 qd + 4 hh + e
  if (a.spans > 1) {
    const int64_t pa = (int64_t)sp * g.n_tokens * g.n_q + at;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int qd = 0; qd < 4; ++qd)
        *reinterpret_cast<f32x4*>(a.part_o + pa * D + 32 * d + 8 * qd + 4 * hh) =
            f32x4{o[d][4 * qd], o[d][4 * qd + 1], o[d][4 * qd + 2], o[d][4 * qd + 3]};
    if (hh == 0) {
      a.part_ml[2 * pa] = limit == kRaise || L != 0.f ? m : kNone;
      a.part_ml[2 * pa + 1] = L;
    }
    return;
  }
  const float inv = L > 0.f ? 1.0f / L : (L == 0.f ? 0.f : L);   // (a NaN stays)
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int qd = 0; qd < 4; ++qd)
      *reinterpret_cast<uint2*>(a.O + at * D + 32 * d + 8 * qd + 4 * hh) =
          make_uint2(pack_bf16x2(o[d][4 * qd] * inv, o[d][4 * qd + 1] * inv),
                     pack_bf16x2(o[d][4 * qd + 2] * inv, o[d][4 * qd + 3] * inv));
  if (a.lse && hh == 0)
    a.lse[at] = L == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
}

// The spans of a row joined: one workgroup per (token, query head). Every span's weight
// first, 2^(its maximum - the row's), all of them at once into LDS; then the weighted sum of the
// partial outputs, D / 4 lanes of four values by 1024 / D spans, loads that wait for nothing.
// (With a running maximum over the spans instead, 256 spans took 12 us.)
constexpr int kMaxSpans = 512;

template <int D>
__global__ __launch_bounds__(256) void paged_join_kernel(PaArgs a) {
  constexpr int LN = D / 4, GR = 256 / LN;
  __shared__ __align__(16) float s_o[GR][D];
  __shared__ float s_w[kMaxSpans], s_red[4];
  const KvGeom& g = a.g;
  const int tid = threadIdx.x, wave = tid >> 6;
  const int64_t t = blockIdx.x / g.n_q;
  const int hq = blockIdx.x % g.n_q;
  int lo = 0, hi = g.n_seqs;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (g.cu[mid] <= t) lo = mid; else hi = mid;
  }
  const KvSeq q = kv_seq(g, lo);
  if (t < q.row0 || t >= q.row0 + q.n) return;
  const int i = (int)(t - q.row0);
  const int r0 = (i * a.G + hq % a.G) / a.tile_rows * a.tile_rows;
  const int vmax = visible(a, q, (min(r0 + a.tile_rows, q.n * a.G) - 1) / a.G);
  const int live = max((vmax + a.span - 1) / a.span, 1);
  const int64_t at = t * g.n_q + hq, step = g.n_tokens * g.n_q;
  float M = kNone;
  for (int sp = tid; sp < live; sp += 256) {
    const float pm = a.part_ml[2 * (sp * step + at)];
    s_w[sp] = pm;
    M = fmaxf(M, pm);
  }
  M = wave_max(M);
  if ((tid & 63) == 0) s_red[wave] = M;
  __syncthreads();
  M = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
  __syncthreads();
  float L = 0.f;
  for (int sp = tid; sp < live; sp += 256) {
    const float w = exp2_fast(s_w[sp] - M);
    L = fmaf(a.part_ml[2 * (sp * step + at) + 1], w, L);
    s_w[sp] = w;
  }
  L = wave_sum(L);
  if ((tid & 63) == 0) s_red[wave] = L;
  __syncthreads();
  L = (s_red[0] + s_red[1]) + (s_red[2] + s_red[3]);
  const int gr = tid / LN, d4 = (tid % LN) * 4;
  const float* po = a.part_o + at * D + d4;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int sp = gr; sp < live; sp += GR) {
    const float w = s_w[sp];
    const f32x4 v = *reinterpret_cast<const f32x4*>(po + sp * step * D);
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = fmaf(v[j], w, y[j]);
  }
  *reinterpret_cast<f32x4*>(&s_o[gr][d4]) = y;
  __syncthreads();
  if (gr != 0) return;
  f32x4 z = y;
#pragma unroll
  for (int k = 1; k < GR; ++k) {
    const f32x4 w = *reinterpret_cast<const f32x4*>(&s_o[k][d4]);
#pragma unroll
    for (int j = 0; j < 4; ++j) z[j] += w[j];
  }
  const float inv = L > 0.f ? 1.0f / L : (L == 0.f ? 0.f : L);
  uint2 out;
  out.x = pack_bf16x2(z[0] * inv, z[1] * inv);
  out.y = pack_bf16x2(z[2] * inv, z[3] * inv);
  *reinterpret_cast<uint2*>(a.O + at * D + d4) = out;
  if (a.lse && d4 == 0)
    a.lse[at] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
}

// How a call is split: rows per workgroup (16 or 32: the waves split the context; 128 or 256: the
// waves split the rows; 256 rows share a tile's conversion, 404 us for three prompt chunks where
// 128 take 421) and spans of the context. Both are chosen once for the batch, from max_new and
// max_len: one sequence of 131072 tokens among 63 of 500 is walked in one span (1391 us; 50 and 17
// in calls of their own), and 63 single tokens after 4000 beside a chunk of 2000 take its tiles
// (904 us; 94 and 81). Heads of 256 have tiles of at most 32 rows: 256 values a row do not fit the
// registers of the other kernel, and those of this one spill 13-18 (1000 tokens after 1000, 16 + 4
// heads: 105 us, where a kernel at the rate of the products would take 17).
struct Plan {
  int tile_rows, row_tiles, spans, span;
};

Plan plan(const catq_kv_desc* d, const catq_kv_batch* b) {
  const int64_t rows = (int64_t)b->max_new * (d->n_q / d->n_kv);
  Plan p;
  p.tile_rows = rows <= 16 ? 16 : rows <= 32 || d->head_dim == 256 ? 32 : rows <= 128 ? 128 : 256;
  p.row_tiles = (int)((rows + p.tile_rows - 1) / p.tile_rows);
  // Spans so that the chip has 512 workgroups where the context allows (131072 tokens of one sequence:
  // 58 us; 62 with 1024, 67 with 2048), none under 256 tokens (1000 tokens of one sequence: 9.9 us; 12.4
  // where none is under 512), and one up to 512, where the join costs more than it gives (300 tokens:
  // 7.8 us, 10.2 in two spans).
  const int64_t base = (int64_t)p.row_tiles * d->n_kv * b->n_seqs;
  const int64_t len = b->max_len > 0 ? b->max_len : 1;
  const int64_t want = len <= 512 ? 1 : std::max<int64_t>(1, 512 / std::max<int64_t>(base, 1));
  int64_t span = (len + want - 1) / want;
  span = std::max<int64_t>(256, (span + 127) / 128 * 128);
  p.spans = (int)((len + span - 1) / span);
  p.span = (int)span;
  return p;
}

template <int D>
catq_status launch_paged(const PaArgs& a, bool per_token, double flops, double bytes, hipStream_t stream) {
  const dim3 grid((unsigned)((int64_t)a.row_tiles * a.spans * a.g.n_kv), (unsigned)a.g.n_seqs);
  char tag[64];
  trace_tag(tag, sizeof tag, "paged_attn<%d rows, head_dim %d>", a.tile_rows, D);
  auto go = [&](auto kernel) {
    CATQ_TRACED(stream, tag, flops, bytes, a.g.n_tokens, a.g.n_q, D,
                hipLaunchKernelGGL(kernel, grid, dim3(a.tile_rows == 256 ? 512 : 256), 0, stream, a));
  };
  if (a.tile_rows == 16) per_token ? go(paged_attn_kernel<D, 1, true>) : go(paged_attn_kernel<D, 1, false>);
  else if (a.tile_rows == 32) per_token ? go(paged_attn_kernel<D, 2, true>) : go(paged_attn_kernel<D, 2, false>);
  else if constexpr (D <= 128) {
    if (a.tile_rows == 128) per_token ? go(paged_tile_kernel<D, 4, true>) : go(paged_tile_kernel<D, 4, false>);
    else per_token ? go(paged_tile_kernel<D, 8, true>) : go(paged_tile_kernel<D, 8, false>);
  }
  CATQ_CHECK_LAUNCH("paged attention");
  if (a.spans > 1) {
    CATQ_TRACED(stream, "paged_join_kernel", 0.0, (double)a.g.n_tokens * a.g.n_q * D * (4.0 * a.spans + 2.0),
                a.g.n_tokens, a.g.n_q, D,
                hipLaunchKernelGGL((paged_join_kernel<D>), dim3((unsigned)(a.g.n_tokens * a.g.n_q)), dim3(256), 0,
                                   stream, a));
    CATQ_CHECK_LAUNCH("paged attention join");
  }
  return CATQ_OK;
}

size_t plan_bytes(const catq_kv_desc* d, const catq_kv_batch* b, const Plan& p) {
  if (p.spans <= 1) return 0;
  const size_t rows = (size_t)b->n_tokens * (size_t)d->n_q * (size_t)p.spans;
  return round_up(rows * (size_t)d->head_dim * 4, 256) + round_up(rows * 8, 256);
}

}  // namespace
}  // namespace catq

using namespace catq;

extern "C" size_t catq_paged_attention_workspace_bytes(const catq_kv_desc* d, const catq_kv_batch* b) {
  if (kv_check_sizes(d, b) != CATQ_OK || b->n_seqs == 0 || b->n_tokens == 0 || b->max_new == 0) return 0;
  return plan_bytes(d, b, plan(d, b));
}

extern "C" catq_status catq_aux_paged_attention(const catq_kv_desc* d, const catq_kv_cache* cache,
                                                const catq_kv_batch* batch, const void* q, float scale,
                                                void* o, float* lse, void* workspace,
                                                size_t workspace_bytes, hipStream_t stream) {
  clear_error();
  CATQ_TRY(kv_check(d, cache, batch));
  CATQ_REQUIRE(scale >= 0.f && scale < 3.0e38f, CATQ_ERR_VALUE, "scale must be finite and >= 0");
  if (batch->n_seqs == 0 || batch->n_tokens == 0 || batch->max_new == 0) return CATQ_OK;
  CATQ_REQUIRE(q && o, CATQ_ERR_NULL, "q and o must not be NULL");
  CATQ_REQUIRE(aligned16(q) && aligned16(o) && aligned16(workspace) &&
                   (reinterpret_cast<uintptr_t>(lse) & 3) == 0,
               CATQ_ERR_ALIGN, "misaligned");
  const Plan p = plan(d, batch);
  // (a launch has fewer than 2^32 threads along x)
  CATQ_REQUIRE((int64_t)p.row_tiles * p.spans * d->n_kv < (1 << 23) &&
                   (p.spans == 1 || batch->n_tokens * d->n_q < (1 << 24)) &&
                   (int64_t)batch->max_new * (d->n_q / d->n_kv) <= INT32_MAX / 2 &&
                   (int64_t)d->max_pages * d->page_size <= INT32_MAX / 2,
               CATQ_ERR_SHAPE, "too many rows or too long a context for one launch");
  const size_t need = plan_bytes(d, batch, p);
  CATQ_REQUIRE(need == 0 || (workspace && workspace_bytes >= need), CATQ_ERR_WORKSPACE,
               "workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
  PaArgs a{};
  a.g = kv_geom(d, batch);
  a.K = cache->k;
  a.V = cache->v;
  a.KS = cache->k_scale;
  a.VS = cache->v_scale;
  a.Q = static_cast<const bf16*>(q);
  a.O = static_cast<bf16*>(o);
  a.lse = lse;
  if (need) {
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float*>(
        static_cast<char*>(workspace) +
        round_up((size_t)batch->n_tokens * d->n_q * p.spans * d->head_dim * 4, 256));
  }
  a.G = d->n_q / d->n_kv;
  a.row_tiles = p.row_tiles;
  a.tile_rows = p.tile_rows;
  a.spans = p.spans;
  a.span = p.span;
  a.limit = (int32_t)std::min<int64_t>((int64_t)d->max_pages * d->page_size, (int64_t)p.spans * p.span);
  a.c = scale * 1.44269504088896341f;
  const bool per_token = d->scale_block == 1;
  const double flops = 4.0 * (double)batch->n_tokens * batch->max_len * d->n_q * d->head_dim;
  const double bytes = 2.0 * (double)batch->n_seqs * batch->max_len * d->n_kv * d->head_dim;
  switch (d->head_dim) {
    case 64: return launch_paged<64>(a, per_token, flops, bytes, stream);
    case 128: return launch_paged<128>(a, per_token, flops, bytes, stream);
    default: return launch_paged<256>(a, per_token, flops, bytes, stream);
  }
}
