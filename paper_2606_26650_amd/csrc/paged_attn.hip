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
// at 2^-126, so a token is lost from the denominator where its scale is 2^90 below the
// scale behind the maximum and its weight is not yet under 2^-36: scales are
// therefore held to [2^-60, 2^30], where that cannot be.
// The running maximum is only raised when a score exceeds it by 2^8 (p' <= 256 is as good
// in fp16 as p' <= 1), so the rescaling of the output is rare.
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

  // queries: fp16 of q over the power of two at its row's largest magnitude
  f16x8 qf[NR][2 * HH];
  float qc[NR];        // that power times the softmax scale, in log2 units
  int vis[NR];
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
      for (int j = 0; j < 8; ++j) { v[hh][j] = t[j]; m = fmaxf(m, fabsf(t[j])); }
      load8<bf16>(qp + 64 * hh + 8, t);
#pragma unroll
      for (int j = 0; j < 8; ++j) { v[hh][8 + j] = t[j]; m = fmaxf(m, fabsf(t[j])); }
    }
    m = col_max(m);
    const int e = min(max((int)(__float_as_uint(m) >> 23) - 127, -100), 126);
    const float down = __uint_as_float((unsigned)(127 - e) << 23);
    qc[r] = __uint_as_float((unsigned)(127 + e) << 23) * a.c;
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
    const float lr = col_sum(l[r]);
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

// The spans of a row joined: one workgroup per (token, query head); its D / 4 lanes of
// four values each take every (1024 / D)-th span.
template <int D, int NR>
__global__ __launch_bounds__(256) void paged_join_kernel(PaArgs a) {
  constexpr int LN = D / 4, GR = 256 / LN;
  __shared__ __align__(16) float s_o[GR][D];
  __shared__ float s_m[GR], s_l[GR];
  const KvGeom& g = a.g;
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
  const int r0 = (i * a.G + hq % a.G) / (16 * NR) * (16 * NR);
  const int vmax = visible(a, q, (min(r0 + 16 * NR, q.n * a.G) - 1) / a.G);
  const int live = max((vmax + a.span - 1) / a.span, 1);
  const int gr = threadIdx.x / LN, d4 = (threadIdx.x % LN) * 4;
  const int64_t at = t * g.n_q + hq, step = g.n_tokens * g.n_q;
  float m = kNone, l = 0.f;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  for (int sp = gr; sp < live; sp += GR) {
    const int64_t pa = sp * step + at;
    const float pm = a.part_ml[2 * pa], pl = a.part_ml[2 * pa + 1];
    const f32x4 po = *reinterpret_cast<const f32x4*>(a.part_o + pa * D + d4);
    const float mn = fmaxf(m, pm);
    const float f = exp2_fast(m - mn), fp = exp2_fast(pm - mn);
    m = mn;
    l = l * f + pl * fp;
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = y[j] * f + po[j] * fp;
  }
  *reinterpret_cast<f32x4*>(&s_o[gr][d4]) = y;
  if (d4 == 0) {
    s_m[gr] = m;
    s_l[gr] = l;
  }
  __syncthreads();
  if (gr != 0) return;
  float M = s_m[0];
#pragma unroll
  for (int k = 1; k < GR; ++k) M = fmaxf(M, s_m[k]);
  float L = 0.f;
  f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < GR; ++k) {
    const float f = exp2_fast(s_m[k] - M);
    L += s_l[k] * f;
    const f32x4 w = *reinterpret_cast<const f32x4*>(&s_o[k][d4]);
#pragma unroll
    for (int j = 0; j < 4; ++j) z[j] += w[j] * f;
  }
  const float inv = L > 0.f ? 1.0f / L : (L == 0.f ? 0.f : L);
  uint2 out;
  out.x = pack_bf16x2(z[0] * inv, z[1] * inv);
  out.y = pack_bf16x2(z[2] * inv, z[3] * inv);
  *reinterpret_cast<uint2*>(a.O + at * D + d4) = out;
  if (a.lse && d4 == 0)
    a.lse[at] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
}

// How a call is split: rows per workgroup and spans of the context.
struct Plan {
  int nr, row_tiles, spans, span;
};
Plan plan(const catq_kv_desc* d, const catq_kv_batch* b) {
  const int64_t rows = (int64_t)b->max_new * (d->n_q / d->n_kv);
  Plan p;
  p.nr = rows <= 16 ? 1 : rows <= 32 || d->head_dim == 256 ? 2 : 4;
  p.row_tiles = (int)((rows + 16 * p.nr - 1) / (16 * p.nr));
  // spans so that the chip has 2048 workgroups where the context allows, none under 256 tokens
  const int64_t base = (int64_t)p.row_tiles * d->n_kv * b->n_seqs;
  const int64_t len = b->max_len > 0 ? b->max_len : 1;
  const int64_t want = std::max<int64_t>(1, 2048 / std::max<int64_t>(base, 1));
  int64_t span = (len + want - 1) / want;
  span = std::max<int64_t>(256, (span + 127) / 128 * 128);
  p.spans = (int)((len + span - 1) / span);
  p.span = (int)span;
  return p;
}

template <int D>
catq_status launch_paged(const PaArgs& a, const Plan& p, bool per_token, double flops, double bytes,
                         hipStream_t stream) {
  const dim3 grid((unsigned)((int64_t)p.row_tiles * p.spans * a.g.n_kv), (unsigned)a.g.n_seqs);
  auto with = [&](auto nr, auto pt) {
    constexpr int NR = decltype(nr)::value;
    constexpr bool PT = decltype(pt)::value;
    CATQ_TRACED(stream, "paged_attn_kernel", flops, bytes, a.g.n_tokens, a.g.n_q, D,
                hipLaunchKernelGGL((paged_attn_kernel<D, NR, PT>), grid, dim3(256), 0, stream, a));
    if (p.spans > 1)
      CATQ_TRACED(stream, "paged_join_kernel", 0.0,
                  (double)a.g.n_tokens * a.g.n_q * D * (4.0 * p.spans + 2.0), a.g.n_tokens, a.g.n_q, D,
                  hipLaunchKernelGGL((paged_join_kernel<D, NR>), dim3((unsigned)(a.g.n_tokens * a.g.n_q)),
                                     dim3(256), 0, stream, a));
  };
  auto rows = [&](auto nr) {
    if (per_token) with(nr, std::true_type{});
    else with(nr, std::false_type{});
  };
  using std::integral_constant;
  if (p.nr == 1) rows(integral_constant<int, 1>{});
  else if (p.nr == 2) rows(integral_constant<int, 2>{});
  else if constexpr (D <= 128) rows(integral_constant<int, 4>{});
  CATQ_CHECK_LAUNCH("paged attention");
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
  CATQ_REQUIRE((int64_t)p.row_tiles * p.spans * d->n_kv <= INT32_MAX &&
                   (p.spans == 1 || batch->n_tokens * d->n_q <= INT32_MAX) &&
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
  a.spans = p.spans;
  a.span = p.span;
  a.limit = (int32_t)std::min<int64_t>((int64_t)d->max_pages * d->page_size, (int64_t)p.spans * p.span);
  a.c = scale * 1.44269504088896341f;
  const bool per_token = d->scale_block == 1;
  const double flops = 4.0 * (double)batch->n_tokens * batch->max_len * d->n_q * d->head_dim;
  const double bytes = 2.0 * (double)batch->n_seqs * batch->max_len * d->n_kv * d->head_dim;
  switch (d->head_dim) {
    case 64: return launch_paged<64>(a, p, per_token, flops, bytes, stream);
    case 128: return launch_paged<128>(a, p, per_token, flops, bytes, stream);
    default: return launch_paged<256>(a, p, per_token, flops, bytes, stream);
  }
}
