// The paged 8-bit key/value cache (gfx950): new tokens in, with the head norms and
// the rotation on the way, and values back out.
//
// Append.  One launch, two kinds of workgroups:
//  * q: a workgroup takes one token and as many query heads as 256 threads cover at
//    sixteen values each; the rotation angles are formed once in LDS.
//  * k and v: a workgroup takes a window of W tokens of one kv head of K or V, W the
//    larger of a scale block and what 256 threads cover (32 tokens of 128), so it
//    owns whole scale blocks and whole four-token words of the v layout: no other
//    workgroup reads or writes them.  It keeps the window's values in registers
//    (sixteen per thread and pass of 256 threads), reduces their magnitudes to the blocks'
//    scales through LDS, and writes codes (v through a transposed LDS tile, so that
//    four tokens make one word).  Where a block holds older tokens and its scale
//    grows, their codes are read, rescaled and written with the new ones.
// A few new tokens cost a launch and three memory latencies in a row (lengths, page, scale; 64
// single tokens: 7.5 us). Many: 9400 tokens of 32 + 8 + 8 heads of 128 take 55 us, 3.9 TB/s; the rotation and
// the quantizer's vector instructions are what the rest is (72 us with one value in
// each lane's pairs and the angles in float64).
#include <type_traits>

#include "kv_common.h"
#include "quant8.h"

namespace catq {

catq_status kv_check_sizes(const catq_kv_desc* d, const catq_kv_batch* b) {
  CATQ_REQUIRE(d && b, CATQ_ERR_NULL, "descriptor and batch must not be NULL");
  CATQ_REQUIRE(d->n_q > 0 && d->n_kv > 0 && d->n_q % d->n_kv == 0 && d->n_q <= 1024,
               CATQ_ERR_SHAPE, "n_q must be a multiple of n_kv and at most 1024");
  CATQ_REQUIRE(d->head_dim == 64 || d->head_dim == 128 || d->head_dim == 256, CATQ_ERR_SHAPE,
               "head_dim must be 64, 128 or 256");
  const int ps = d->page_size, bt = d->scale_block;
  CATQ_REQUIRE(ps >= 16 && ps <= 256 && (ps & (ps - 1)) == 0, CATQ_ERR_SHAPE,
               "page_size must be 16, 32, 64, 128 or 256");
  CATQ_REQUIRE(bt == 1 || (bt >= 16 && bt <= 128 && bt <= ps && (bt & (bt - 1)) == 0),
               CATQ_ERR_SHAPE, "scale_block must be 1, or 16, 32, 64 or 128 and at most page_size");
  CATQ_REQUIRE(d->n_pages > 0 && d->max_pages > 0 &&
                   count_ok((int64_t)d->n_pages * ps, d->n_kv, d->head_dim),
               CATQ_ERR_SHAPE, "n_pages and max_pages must be > 0, the pool within 2^38 elements");
  CATQ_REQUIRE(b->n_seqs >= 0 && b->n_tokens >= 0 && b->max_new >= 0 && b->max_len >= 0,
               CATQ_ERR_SHAPE, "batch sizes must be >= 0");
  CATQ_REQUIRE(b->n_tokens <= INT32_MAX && b->n_seqs <= 65535 && b->max_new <= (1 << 24),
               CATQ_ERR_SHAPE, "at most 2^31 - 1 tokens, 65535 sequences and 2^24 new tokens in one");
  CATQ_REQUIRE(b->max_len <= (int64_t)d->max_pages * ps, CATQ_ERR_SHAPE,
               "max_len exceeds what max_pages pages hold");
  CATQ_REQUIRE(b->n_tokens == 0 ||
                   count_ok(b->n_tokens, d->n_q + 2 * (int64_t)d->n_kv, d->head_dim),
               CATQ_ERR_SHAPE, "too many tokens (more than 2^38 elements)");
  return CATQ_OK;
}

catq_status kv_check(const catq_kv_desc* d, const catq_kv_cache* c, const catq_kv_batch* b) {
  CATQ_TRY(kv_check_sizes(d, b));
  CATQ_REQUIRE(c && c->k && c->v && c->k_scale && c->v_scale, CATQ_ERR_NULL, "cache arrays must not be NULL");
  CATQ_REQUIRE(b->n_seqs == 0 || (b->page_table && b->cu_new && b->ctx_len), CATQ_ERR_NULL,
               "batch arrays must not be NULL");
  CATQ_REQUIRE(aligned16(c->k) && aligned16(c->v) && aligned16(c->k_scale) && aligned16(c->v_scale),
               CATQ_ERR_ALIGN, "cache arrays must be 16-byte aligned");
  CATQ_REQUIRE(((reinterpret_cast<uintptr_t>(b->page_table) | reinterpret_cast<uintptr_t>(b->cu_new) |
                 reinterpret_cast<uintptr_t>(b->ctx_len)) & 3) == 0,
               CATQ_ERR_ALIGN, "batch arrays must be 4-byte aligned");
  return CATQ_OK;
}

KvGeom kv_geom(const catq_kv_desc* d, const catq_kv_batch* b) {
  return KvGeom{b->page_table, b->cu_new, b->ctx_len, b->n_tokens, d->n_q, d->n_kv, d->head_dim,
                __builtin_ctz((unsigned)d->page_size), __builtin_ctz((unsigned)d->scale_block),
                d->n_pages, d->max_pages, b->n_seqs, b->max_new};
}

namespace {

struct AppendArgs {
  KvGeom g;
  catq_kv_cache c;
  const float* inv_freq;
  const bf16* q_w;
  const bf16* k_w;
  const bf16* qkv;
  bf16* q_out;
  int32_t rot, inter, qk_norm, act_quant;
  float rope_scale, eps;
  int32_t win;          // windows a sequence can reach
  int32_t w_log2;       // tokens of a window
  int64_t kv_blocks;    // n_seqs * win * n_kv * 2 workgroups come first
  int32_t q_parts;      // workgroups per token for the query heads
};

// The turns of one position, inv_freq / 2 pi, as a 64-bit fraction of a turn (whole turns are left
// out, which is what makes it exact for far positions: an integer times it, modulo 2^64, is
// the fraction for that position).  1 / 2 pi is taken in two float64, of 2^-108 together, and the
// product as a float64 and its error, so with |f| < 2^20 the fraction is off by less than 2^-63.
__device__ __forceinline__ uint64_t turn_fraction(float f) {
#pragma clang fp contract(off)   // (hi is the rounded product, also where it is subtracted from)
  const double x = f, h = 0x1.45f306dc9c883p-3, l = -0x1.6b01ec5417056p-57;
  const double hi = x * h, lo = fma(x, l, fma(x, h, -hi));
  double frac = hi - rint(hi);                 // exact, within a half
  if (frac >= 0.5) frac -= 1.0;
  return (uint64_t)(int64_t)(frac * 0x1p64) + (uint64_t)(int64_t)(int)rint(lo * 0x1p64);
}

// cos and sin of `n` positions from pos0 on, times the scale, at cs[t][rot/2]: by one wave, a
// lane per frequency.  The fraction's upper 32 bits round to fp32 by 2^-26 of a turn, all
// else is below 2^-31.  (Two floats with the whole turns taken off in an fma take the same time, 56 us
// for the prompts above with their read back, and were off by 2^-24, more at frequencies above 1.)
// Frequencies of 2^20 and above, infinite and NaN ones give NaN.
__device__ __forceinline__ void angles(const AppendArgs& a, int64_t pos0, int n, float2* cs) {
  const int half = a.rot >> 1;
  for (int f = threadIdx.x & 63; f < half; f += 64) {
    const float freq = a.inv_freq[f];
    const bool fine = fabsf(freq) < 0x1p20f;
    const float scale = fine ? a.rope_scale : __builtin_nanf("");
    const uint64_t turn = turn_fraction(fine ? freq : 0.f);
    uint64_t at = turn * (uint64_t)pos0;
    for (int t = 0; t < n; ++t, at += turn) {
      float s, c;
      sincospif((float)(int32_t)(at >> 32) * 0x1p-31f, &s, &c);   // (of twice the fraction, in [-1, 1])
      cs[t * half + f] = make_float2(c * scale, s * scale);
    }
  }
}

// A head is held by LPH lanes of sixteen values each, in two runs of eight at `a` and `b`: a lane
// has both sides of its pairs, value 8 sub + j and the one rot/2 further on (or, interleaved and
// where nothing rotates, sixteen neighbours), and needs the angles 8 sub .. + 7.
struct HeadPart {
  int a, b;
  bool turn;
};
__device__ __forceinline__ HeadPart head_part(const AppendArgs& a, int sub) {
  const int lanes = a.rot >> 4;
  if (a.inter) return {16 * sub, 16 * sub + 8, sub < lanes};
  if (sub < lanes) return {8 * sub, (a.rot >> 1) + 8 * sub, true};
  return {16 * sub, 16 * sub + 8, false};
}
__device__ __forceinline__ void load16(const bf16* p, HeadPart h, float (&v)[16]) {
  float x[8], y[8];
  load8<bf16>(p + h.a, x);
  load8<bf16>(p + h.b, y);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    v[j] = x[j];
    v[8 + j] = y[j];
  }
}
__device__ __forceinline__ unsigned int mag16(const float (&v)[16]) {
  unsigned int m = 0u;
#pragma unroll
  for (int j = 0; j < 16; ++j) m = max(m, mag_bits(v[j]));
  return m;
}

// norm (with its gain) and rotation
template <int LPH>
__device__ __forceinline__ void prep_head(const AppendArgs& a, float (&v)[16], int sub, HeadPart h, const bf16* w,
                                          const float2* cs) {
  constexpr int D = LPH * 16;
  if (a.qk_norm) {
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) ss = fmaf(v[j], v[j], ss);
#pragma unroll
    for (int m = LPH >> 1; m >= 1; m >>= 1) ss += __shfl_xor(ss, m, 64);
    const float r = 1.0f / sqrtf(ss / (float)D + a.eps);
    if (w) {
      float g[16];
      load16(w, h, g);
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = v[j] * r * g[j];
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] *= r;
    }
  }
  if (!h.turn) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float2 t = cs[8 * sub + j];
    if (a.inter) {
      const float p = v[2 * j], q = v[2 * j + 1];
      v[2 * j] = p * t.x - q * t.y;
      v[2 * j + 1] = q * t.x + p * t.y;
    } else {
      const float p = v[j], q = v[8 + j];
      v[j] = p * t.x - q * t.y;
      v[8 + j] = q * t.x + p * t.y;
    }
  }
}

// One token and as many heads as fit the workgroup. (Four tokens a workgroup were slower, 62 us
// against 55 for the prompts above.)
template <int LPH>
__device__ __forceinline__ void append_q(const AppendArgs& a, int64_t block, float2* cs, int64_t* s_pos) {
  constexpr int D = LPH * 16, HP = 256 / LPH;   // heads per workgroup
  const int64_t t = block / a.q_parts;
  const int part = (int)(block % a.q_parts);
  const int sub = threadIdx.x & (LPH - 1), h = part * HP + threadIdx.x / LPH;
  const bool live = h < a.g.n_q;
  const HeadPart hp = head_part(a, sub);
  float v[16];
  if (live)
    load16(a.qkv + t * (a.g.n_q + 2 * (int64_t)a.g.n_kv) * D + (int64_t)h * D, hp, v);
  else
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = 0.f;
  // the token's sequence: the last one that starts at or before it (empty ones before it start
  // there too)
  if (threadIdx.x == 0) {
    int lo = 0, hi = a.g.n_seqs;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.g.cu[mid] <= t) lo = mid; else hi = mid;
    }
    const KvSeq q = kv_seq(a.g, lo);
    // (a row of no sequence)
    *s_pos = t < q.row0 || t >= q.row0 + q.n ? INT64_MIN : q.ctx + (t - q.row0);
  }
  __syncthreads();
  const int64_t pos = *s_pos;
  if (pos == INT64_MIN) return;
  if (threadIdx.x < 64) angles(a, pos, 1, cs);
  __syncthreads();
  prep_head<LPH>(a, v, sub, hp, a.q_w, cs);
  if (a.act_quant) {
    unsigned int m = mag16(v);
#pragma unroll
    for (int k = LPH >> 1; k >= 1; k >>= 1) m = max(m, (unsigned)__shfl_xor((int)m, k, 64));
    const float s = quant8_scale(m);
    quant8_n(v, s);
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] *= s;
  }
  if (live) {
    bf16* o = a.q_out + (t * a.g.n_q + h) * D;
    float x[8], y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] = v[j];
      y[j] = v[8 + j];
    }
    store8<bf16>(o + hp.a, x);
    store8<bf16>(o + hp.b, y);
  }
}

// byte b of a word as a signed code
__device__ __forceinline__ float code_of(unsigned int w, int b) {
  return (float)(int)(signed char)(w >> (8 * b));
}

// LPH lanes per head, NP passes of TP = 256 / LPH tokens (or one of fewer)
template <int LPH, int NP>
__device__ __forceinline__ void append_kv(const AppendArgs& a, int64_t block, float2* cs,
                                          unsigned int* s_mag, float* s_scale, float* s_ratio,
                                          unsigned char* s_tile) {
  constexpr int D = LPH * 16, TP = 256 / LPH;
  const KvGeom& g = a.g;
  const int is_v = (int)(block & 1);
  block >>= 1;
  const int h = (int)(block % g.n_kv);
  block /= g.n_kv;
  const int wi = (int)(block % a.win), s = (int)(block / a.win);
  const KvSeq q = kv_seq(g, s);
  const int W = 1 << a.w_log2;
  // positions first <= p < first + W of the window, of which lo <= p < hi are new
  const int64_t begin = q.ctx < 0 ? 0 : q.ctx;
  const int64_t first = ((begin >> a.w_log2) + wi) << a.w_log2;
  const int64_t end = min((int64_t)q.ctx + q.n, kv_capacity(g));
  if (first >= end || begin >= end) return;
  const int tok0 = (int)(first & ((1 << g.ps_log2) - 1));   // of the page
  const int lo = (int)max(begin - first, (int64_t)0), hi = (int)min(end - first, (int64_t)W);
  const int bt = 1 << g.bt_log2;
  // the block with older tokens, if there is one: [lo & ~(bt-1), lo) hold them
  const int old0 = lo & ~(bt - 1);
  const bool has_old = first + lo == begin && old0 < lo;

  const int sub = threadIdx.x & (LPH - 1), tl = threadIdx.x / LPH;
  const int64_t ld = (g.n_q + 2 * (int64_t)g.n_kv) * D;
  const HeadPart hp = is_v ? HeadPart{16 * sub, 16 * sub + 8, false} : head_part(a, sub);
  const bf16* src = a.qkv + (int64_t)(g.n_q + (is_v ? g.n_kv : 0) + h) * D;
  // (the values are on their way while the page is looked up)
  const int page = g.table[(int64_t)s * g.max_pages + (first >> g.ps_log2)];
  float v[NP][16];
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int t = p * TP + tl;
    if (t >= lo && t < hi) {
      load16(src + (q.row0 + (first + t - q.ctx)) * ld, hp, v[p]);
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j) v[p][j] = 0.f;
    }
  }
  if (page < 0 || page >= g.n_pages) return;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int t = p * TP + tl;
    if (!is_v) {
      if (p > 0) __syncthreads();   // the table of the pass before is read
      // of the pass's new tokens, a quarter by each wave
      const int ta = max(lo - p * TP, 0), n = min(hi - p * TP, TP) - ta, w = threadIdx.x >> 6;
      const int w0 = n * w >> 2, w1 = n * (w + 1) >> 2;
      if (n > 0) angles(a, first + p * TP + ta + w0, w1 - w0, cs + (ta + w0) * (a.rot >> 1));
      __syncthreads();
      prep_head<LPH>(a, v[p], sub, hp, a.k_w, cs + tl * (a.rot >> 1));
      if (t < lo || t >= hi)        // (a norm turns zeros into zeros, an angle may be anything)
#pragma unroll
        for (int j = 0; j < 16; ++j) v[p][j] = 0.f;
    }
    unsigned int m = mag16(v[p]);
#pragma unroll
    for (int k = LPH >> 1; k >= 1; k >>= 1) m = max(m, (unsigned)__shfl_xor((int)m, k, 64));
    if (sub == 0 && t < W) s_mag[t] = m;
  }
  __syncthreads();
  float* scales = is_v ? a.c.v_scale : a.c.k_scale;
  int8_t* codes = is_v ? a.c.v : a.c.k;
  const int64_t cbase = kv_code_base(g, page, h, tok0);
  const int64_t sbase = kv_scale_index(g, page, h, tok0);
  for (int b = threadIdx.x; b < (W >> g.bt_log2); b += 256) {
    const int t0 = b << g.bt_log2;
    if (t0 >= hi || t0 + bt <= lo) continue;
    unsigned int m = 0u;
    for (int i = 0; i < bt; ++i) m = max(m, s_mag[t0 + i]);
    float sc = quant8_scale(m), ratio = 1.0f;
    if (has_old && t0 == old0) {
      const float was = scales[sbase + b];
      if (sc > was) ratio = was / sc;
      else if (!(sc != sc)) sc = was;    // the larger; a NaN in either stays
      if (sc != sc) ratio = 1.0f;
      s_ratio[0] = ratio;
    }
    scales[sbase + b] = sc;
    s_scale[b] = sc;
  }
  __syncthreads();
  const bool grew = has_old && s_ratio[0] != 1.0f;
  const int wlo = grew ? old0 : lo;   // tokens wlo .. hi - 1 are written
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int t = p * TP + tl;
    if (t < wlo || t >= hi) continue;
    if (t < lo) {   // an older token of the block whose scale grew
      const float r = s_ratio[0];
      if (is_v) {
        const int8_t* vp = codes + cbase + (int64_t)(t >> 2) * (4 * D) + 4 * hp.a + (t & 3);
#pragma unroll
        for (int j = 0; j < 16; ++j) v[p][j] = rintf((float)vp[4 * j] * r);
      } else {
        const int8_t* kp = codes + cbase + (int64_t)t * D;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[p][j] = rintf((float)kp[hp.a + j] * r);
          v[p][8 + j] = rintf((float)kp[hp.b + j] * r);
        }
      }
    } else {
      quant8_n(v[p], s_scale[t >> g.bt_log2]);
    }
    const uint2 c0 = make_uint2(pack_codes(v[p][0], v[p][1], v[p][2], v[p][3]),
                                pack_codes(v[p][4], v[p][5], v[p][6], v[p][7]));
    const uint2 c1 = make_uint2(pack_codes(v[p][8], v[p][9], v[p][10], v[p][11]),
                                pack_codes(v[p][12], v[p][13], v[p][14], v[p][15]));
    if (is_v) {
      *reinterpret_cast<uint2*>(s_tile + t * D + hp.a) = c0;
      *reinterpret_cast<uint2*>(s_tile + t * D + hp.b) = c1;
    } else {
      *reinterpret_cast<uint2*>(codes + cbase + (int64_t)t * D + hp.a) = c0;
      *reinterpret_cast<uint2*>(codes + cbase + (int64_t)t * D + hp.b) = c1;
    }
  }
  if (!is_v) return;
  __syncthreads();
  // words of four tokens at one d, whole ones at once and the others by bytes
  for (int i = threadIdx.x; i < (W >> 2) * D; i += 256) {
    const int t4 = (i / D) * 4, dd = i % D;
    if (t4 + 4 <= wlo || t4 >= hi) continue;
    int8_t* dst = codes + cbase + (int64_t)t4 * D + dd * 4;
    if (t4 >= wlo && t4 + 4 <= hi) {
      *reinterpret_cast<unsigned int*>(dst) =
          (unsigned)s_tile[t4 * D + dd] | ((unsigned)s_tile[(t4 + 1) * D + dd] << 8) |
          ((unsigned)s_tile[(t4 + 2) * D + dd] << 16) | ((unsigned)s_tile[(t4 + 3) * D + dd] << 24);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (t4 + k >= wlo && t4 + k < hi) dst[k] = (int8_t)s_tile[(t4 + k) * D + dd];
    }
  }
}

template <int LPH, int NP>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a) {
  constexpr int D = LPH * 16, TP = 256 / LPH;
  __shared__ float2 cs[TP * D / 2];
  __shared__ unsigned int s_mag[TP * NP];
  __shared__ float s_scale[TP * NP];
  __shared__ float s_ratio[1];
  __shared__ int64_t s_pos;
  __shared__ __align__(16) unsigned char s_tile[TP * NP * D];
  const int64_t b = blockIdx.x;
  if (b < a.kv_blocks)
    append_kv<LPH, NP>(a, b, cs, s_mag, s_scale, s_ratio, s_tile);
  else
    append_q<LPH>(a, b - a.kv_blocks, cs, &s_pos);
}

// Eight values of one (token, head) per thread.  A v word holds four tokens: the
// thread reads the 32 bytes of its eight words and takes its token's (the other three
// tokens' threads find them in the cache).
__global__ __launch_bounds__(256) void kv_read_kernel(KvGeom g, catq_kv_cache c, bf16* ko, bf16* vo) {
  const int lph = g.d >> 3;
  const int s = blockIdx.y;
  const KvSeq q = kv_seq(g, s);
  const int64_t per = (int64_t)g.n_kv * lph;
  const int64_t total = (int64_t)q.n * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t t = i / per;
    const int hs = (int)(i - t * per), h = hs / lph, sub = hs % lph;
    const int64_t pos = q.ctx + t;
    float k[8], v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) k[j] = v[j] = 0.f;
    const int page = pos >= 0 && pos < kv_capacity(g)
                         ? g.table[(int64_t)s * g.max_pages + (pos >> g.ps_log2)] : -1;
    if (page >= 0 && page < g.n_pages) {
      const int tok = (int)(pos & ((1 << g.ps_log2) - 1));
      const int64_t si = kv_scale_index(g, page, h, tok);
      if (ko) {
        const uint2 w = *reinterpret_cast<const uint2*>(c.k + kv_code_base(g, page, h, tok) + sub * 8);
        const float sc = c.k_scale[si];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          k[j] = code_of(w.x, j) * sc;
          k[4 + j] = code_of(w.y, j) * sc;
        }
      }
      if (vo) {
        const u32x4* p = reinterpret_cast<const u32x4*>(c.v + kv_code_base(g, page, h, tok & ~3) + sub * 32);
        const u32x4 a0 = p[0], a1 = p[1];
        const float sc = c.v_scale[si];
        const int sh = 8 * (tok & 3);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[j] = code_of(a0[j] >> sh, 0) * sc;
          v[4 + j] = code_of(a1[j] >> sh, 0) * sc;
        }
      }
    }
    const int64_t o = ((q.row0 + t) * g.n_kv + h) * g.d + sub * 8;
    if (ko) store8<bf16>(ko + o, k);
    if (vo) store8<bf16>(vo + o, v);
  }
}

template <int LPH>
catq_status launch_append(const AppendArgs& a, int64_t blocks, double bytes, hipStream_t stream) {
  constexpr int TP = 256 / LPH;
  auto go = [&](auto np) {
    constexpr int NP = decltype(np)::value;
    CATQ_TRACED(stream, "kv_append_kernel", 0.0, bytes, a.g.n_tokens, a.g.n_q + 2 * a.g.n_kv, a.g.d,
                hipLaunchKernelGGL((kv_append_kernel<LPH, NP>), dim3((unsigned)blocks), dim3(256), 0,
                                   stream, a));
  };
  using std::integral_constant;
  const int passes = ((1 << a.w_log2) + TP - 1) / TP;   // a power of two
  switch (passes) {
    case 1: go(integral_constant<int, 1>{}); break;
    case 2: go(integral_constant<int, 2>{}); break;
    case 4:
      if constexpr (TP <= 32) go(integral_constant<int, 4>{});
      break;
    // a window has at most 128 tokens: more passes only where fewer fit one
    case 8:
      if constexpr (TP <= 16) go(integral_constant<int, 8>{});
      break;
    default:
      break;
  }
  CATQ_CHECK_LAUNCH("kv append");
  return CATQ_OK;
}

}  // namespace
}  // namespace catq

using namespace catq;

extern "C" catq_status catq_aux_kv_append(const catq_kv_desc* d, const catq_kv_cache* cache,
                                          const catq_kv_batch* batch, const catq_kv_prep* prep,
                                          const void* qkv, void* q_out, hipStream_t stream) {
  clear_error();
  CATQ_TRY(kv_check(d, cache, batch));
  CATQ_REQUIRE(prep, CATQ_ERR_NULL, "prep must not be NULL");
  CATQ_REQUIRE(prep->rot_dim >= 0 && prep->rot_dim <= d->head_dim && prep->rot_dim % 16 == 0,
               CATQ_ERR_SHAPE, "rot_dim must be a multiple of 16, at most head_dim");
  CATQ_REQUIRE(prep->rot_dim == 0 || prep->inv_freq, CATQ_ERR_NULL, "inv_freq must not be NULL");
  CATQ_REQUIRE((prep->interleaved | prep->qk_norm | prep->act_quant) >> 1 == 0, CATQ_ERR_VALUE,
               "interleaved, qk_norm and act_quant must be 0 or 1");
  CATQ_REQUIRE(prep->eps >= 0.0f, CATQ_ERR_VALUE, "eps must be >= 0");
  if (batch->n_seqs == 0 || batch->n_tokens == 0 || batch->max_new == 0) return CATQ_OK;
  CATQ_REQUIRE(qkv && q_out, CATQ_ERR_NULL, "qkv and q_out must not be NULL");
  CATQ_REQUIRE(aligned16(qkv) && aligned16(q_out) && aligned16(prep->q_weight) &&
                   aligned16(prep->k_weight) && aligned16(prep->inv_freq),
               CATQ_ERR_ALIGN, "misaligned");
  AppendArgs a{};
  a.g = kv_geom(d, batch);
  a.c = *cache;
  a.inv_freq = prep->inv_freq;
  a.q_w = static_cast<const bf16*>(prep->q_weight);
  a.k_w = static_cast<const bf16*>(prep->k_weight);
  a.qkv = static_cast<const bf16*>(qkv);
  a.q_out = static_cast<bf16*>(q_out);
  a.rot = prep->rot_dim;
  a.inter = prep->interleaved;
  a.qk_norm = prep->qk_norm;
  a.act_quant = prep->act_quant;
  a.rope_scale = prep->rope_scale;
  a.eps = prep->eps;
  const int lph = d->head_dim / 16, tp = 256 / lph;
  // a window lies in one page
  const int w = d->scale_block > tp ? d->scale_block : (tp < d->page_size ? tp : d->page_size);
  a.w_log2 = __builtin_ctz((unsigned)w);
  a.win = (batch->max_new + w - 2) / w + 1;
  a.q_parts = (d->n_q + tp - 1) / tp;
  const int64_t max_blocks = (1 << 24) - 1;   // (a launch has fewer than 2^32 threads along x)
  CATQ_REQUIRE((int64_t)a.win * batch->n_seqs <= max_blocks / (2 * d->n_kv), CATQ_ERR_SHAPE,
               "too many sequences and new tokens for one launch");
  a.kv_blocks = (int64_t)a.win * batch->n_seqs * d->n_kv * 2;
  const int64_t blocks = a.kv_blocks + batch->n_tokens * a.q_parts;
  CATQ_REQUIRE(blocks <= max_blocks, CATQ_ERR_SHAPE, "too many tokens for one launch");
  const double e = (double)batch->n_tokens * d->head_dim;
  const double bytes = e * (4.0 * d->n_q + 6.0 * d->n_kv);
  switch (lph) {
    case 4: return launch_append<4>(a, blocks, bytes, stream);
    case 8: return launch_append<8>(a, blocks, bytes, stream);
    default: return launch_append<16>(a, blocks, bytes, stream);
  }
}

extern "C" catq_status catq_aux_kv_read(const catq_kv_desc* d, const catq_kv_cache* cache,
                                        const catq_kv_batch* batch, void* k_out, void* v_out,
                                        hipStream_t stream) {
  clear_error();
  CATQ_TRY(kv_check(d, cache, batch));
  CATQ_REQUIRE(aligned16(k_out) && aligned16(v_out), CATQ_ERR_ALIGN, "misaligned");
  if (batch->n_seqs == 0 || batch->n_tokens == 0 || batch->max_new == 0) return CATQ_OK;
  CATQ_REQUIRE(k_out || v_out, CATQ_ERR_NULL, "one of k_out and v_out must be given");
  const int64_t per_seq = (int64_t)batch->max_new * d->n_kv * (d->head_dim / 8);
  const unsigned gx = (unsigned)((per_seq + 255) / 256 < (1 << 20) ? (per_seq + 255) / 256 : (1 << 20));
  const double bytes = (double)batch->n_tokens * d->n_kv * d->head_dim * ((k_out ? 3.0 : 0) + (v_out ? 3.0 : 0));
  CATQ_TRACED(stream, "kv_read_kernel", 0.0, bytes, batch->n_tokens, d->n_kv, d->head_dim,
              hipLaunchKernelGGL(kv_read_kernel, dim3(gx, (unsigned)batch->n_seqs), dim3(256), 0, stream,
                                 kv_geom(d, batch), *cache, (bf16*)k_out, (bf16*)v_out));
  CATQ_CHECK_LAUNCH("kv read");
  return CATQ_OK;
}
