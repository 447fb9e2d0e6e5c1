// Pages of the 8-bit cache copied, and accepted tokens moved to the front of the drafted ones (gfx950).
//
// Copy.  A page is three or four runs of consecutive bytes: its codes of k and of v, and its scales. A workgroup
// copies 16 KB of one code array, four 16-byte loads in flight per lane, or all scales of a page. 625 pages of 64
// tokens, 8 heads of 128: 37 us, 4.5 TB/s read and written; four pages: the launch, 3.1 us.
//
// Compact.  Token i of a sequence's accepted ones moves from position ctx + keep[i] to ctx + i.  keep rises, so
// keep[i] >= i: a token moves down or stays, and what is read for one scale block lies in that block or behind
// it.  A workgroup takes K or V of one kv head of a sequence and goes through its blocks in order: it reads a
// window of tokens into registers, waits for all its waves, and writes them; nothing that it writes is read later
// by it, so the next window's reads are under way meanwhile, and no other workgroup reads or writes these blocks.
// A block's scale becomes the largest of the scales that its tokens (the older ones too) come with, and codes that
// come with another are rounded again: rne(code * (their scale / the block's)), half a step of the block's scale
// at most.  With a scale per token (scale_block 1) nothing is rounded.
// Up to 8 of 60 drafted tokens in each of 64 sequences, 8 heads of 128: 10 us, 1024 workgroups that each wait for
// lengths, list, page, source page and codes in turn; one sequence: 4.5.  20000 of 30000 tokens in each of 4: 766 us,
// 64 workgroups that each take 5 us for a window of 128 (with a window's loads not ahead and 32 tokens a window 3.5 us,
// 2220 in all).
#include <algorithm>

#include "kv_common.h"
#include "quant8.h"

namespace catq {
namespace {

struct CopyArgs {
  catq_kv_cache c;
  const int32_t* src;
  const int32_t* dst;
  int32_t n_pages;
  int64_t code_bytes;     // of a page in one of the arrays
  int64_t scales;         // of a page in one of the arrays
  int32_t pieces;         // workgroups of a page and code array
};

constexpr int kCopy = 4;   // 16-byte loads in flight per lane

__global__ __launch_bounds__(256) void kv_copy_kernel(CopyArgs a) {
  const int per = 2 * a.pieces + 1;
  const int64_t pair = blockIdx.x / per;
  const int part = (int)(blockIdx.x % per);
  const int s = a.src[pair], d = a.dst[pair];
  if (s < 0 || s >= a.n_pages || d < 0 || d >= a.n_pages || s == d) return;
  if (part == 2 * a.pieces) {
    for (int64_t i = threadIdx.x; i < a.scales; i += 256) {
      a.c.k_scale[d * a.scales + i] = a.c.k_scale[s * a.scales + i];
      a.c.v_scale[d * a.scales + i] = a.c.v_scale[s * a.scales + i];
    }
    return;
  }
  const bool is_v = part >= a.pieces;
  int8_t* codes = is_v ? a.c.v : a.c.k;
  const u32x4* from = reinterpret_cast<const u32x4*>(codes + s * a.code_bytes);
  u32x4* to = reinterpret_cast<u32x4*>(codes + d * a.code_bytes);
  const int64_t n = a.code_bytes / 16, i0 = (int64_t)(part - (is_v ? a.pieces : 0)) * (256 * kCopy) + threadIdx.x;
  u32x4 v[kCopy];
#pragma unroll
  for (int j = 0; j < kCopy; ++j)
    if (i0 + 256 * j < n) v[j] = from[i0 + 256 * j];
#pragma unroll
  for (int j = 0; j < kCopy; ++j)
    if (i0 + 256 * j < n) to[i0 + 256 * j] = v[j];
}

struct CompactArgs {
  KvGeom g;
  catq_kv_cache c;
  const int32_t* keep;
  const int32_t* n_keep;
  int32_t w_log2;       // tokens of a window
};

// Sixteen codes of a token out of the array's words: of k as they stand, of v a byte of each of sixteen words
__device__ __forceinline__ u32x4 token_codes(const u32x4 (&w)[4], int tok, bool is_v) {
  if (!is_v) return w[0];
  const unsigned pair = 0x0c0c0400u + 0x0101u * (unsigned)(tok & 3), high = (pair << 16) | 0x0c0cu;
  u32x4 r;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    r[j] = __builtin_amdgcn_perm(w[j][1], w[j][0], pair) | __builtin_amdgcn_perm(w[j][3], w[j][2], high);
  return r;
}

// The codes times a ratio of scales, rounded
__device__ __forceinline__ u32x4 rescale(u32x4 c, float r) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float f[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) f[b] = rintf((float)(int)(signed char)(c[j] >> (8 * b)) * r);
    c[j] = pack_codes(f[0], f[1], f[2], f[3]);
  }
  return c;
}

// LPH lanes per head, NP passes of TP = 256 / LPH tokens make a window
template <int LPH, int NP>
__global__ __launch_bounds__(256) void kv_compact_kernel(CompactArgs a) {
  constexpr int D = LPH * 16, TP = 256 / LPH;
  __shared__ int s_end;
  __shared__ unsigned int s_mag[3][TP * NP];   // the blocks' largest scales: a window's, the next one's, cleared ones
  __shared__ __align__(16) unsigned char s_tile[TP * NP * D];
  const KvGeom& g = a.g;
  const int tid = threadIdx.x, sub = tid & (LPH - 1), tl = tid / LPH;
  const int is_v = blockIdx.x & 1, h = blockIdx.x >> 1, s = blockIdx.y;
  const KvSeq q = kv_seq(g, s);
  const int want = min(max(a.n_keep[s], 0), q.n);
  if (want == 0) return;
  const int32_t* keep = a.keep + q.row0;
  // the list ends before the first entry that does not rise or is no new token of the sequence
  if (tid == 0) s_end = want;
  for (int i = tid; i < 3 * TP * NP; i += 256) s_mag[0][i] = 0u;
  __syncthreads();
  for (int i = tid; i < want; i += 256) {
    const int k = keep[i];
    if (k < 0 || k >= q.n || (i > 0 && k <= keep[i - 1])) atomicMin(&s_end, i);
  }
  __syncthreads();
  const int n = s_end;
  if (n == 0) return;
  const int W = 1 << a.w_log2, bt = 1 << g.bt_log2, ps_mask = (1 << g.ps_log2) - 1;
  const int64_t begin = q.ctx < 0 ? 0 : q.ctx;
  const int64_t end = min((int64_t)q.ctx + n, kv_capacity(g));   // positions begin .. end - 1 are written
  int8_t* codes = is_v ? a.c.v : a.c.k;
  float* scales = is_v ? a.c.v_scale : a.c.k_scale;
  const int32_t* table = g.table + (int64_t)s * g.max_pages;
  const int64_t begin_w = begin >> a.w_log2 << a.w_log2;
  if (begin_w >= end) return;
  // A window's tokens come through three loads in a row: their place in the list, its page, the codes.  Each is under way
  // while the window before is written, from clamped addresses, and what does not count is dropped when it has come: no
  // earlier window writes what a later one reads.
  auto places = [&](int64_t first, int (&k)[NP]) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < NP; ++p)
      k[p] = keep[min(max(first + p * TP + tl - q.ctx, (int64_t)0), (int64_t)want - 1)];
  };
  auto page_at = [&](int64_t pos) __attribute__((always_inline)) {
    return table[min(max(pos >> g.ps_log2, (int64_t)0), (int64_t)g.max_pages - 1)];
  };
  auto pages = [&](int64_t first, const int (&k)[NP], int64_t (&pos)[NP], int (&id)[NP]) __attribute__((always_inline)) {
    const int lo = (int)max(begin - first, (int64_t)0), hi = (int)max(min(end - first, (int64_t)W), (int64_t)0);
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int t = p * TP + tl;
      pos[p] = t < lo ? first + t : (int64_t)q.ctx + k[p];
      if (t < (lo & ~(bt - 1)) || t >= hi || pos[p] >= kv_capacity(g)) pos[p] = -1;
      id[p] = page_at(pos[p]);
    }
  };
  auto load = [&](const int64_t (&pos)[NP], const int (&id)[NP], u32x4 (&w)[NP][4], float (&sc)[NP], int (&at)[NP])
      __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const bool ok = pos[p] >= 0 && id[p] >= 0 && id[p] < g.n_pages;
      const int page = ok ? id[p] : 0, tok = ok ? (int)(pos[p] & ps_mask) : 0;
      at[p] = ok ? tok : -1;
      const u32x4* from = reinterpret_cast<const u32x4*>(codes + kv_code_base(g, page, h, is_v ? tok & ~3 : tok)) +
                          (is_v ? 4 * sub : sub);
      w[p][0] = from[0];
      if (is_v) {
#pragma unroll
        for (int j = 1; j < 4; ++j) w[p][j] = from[j];
      }
      sc[p] = scales[kv_scale_index(g, page, h, tok)];
    }
  };
  int k[NP], id[NP], at[NP];
  int lane0 = 0;       // (so that the window's own page is held a lane, not waited for to be held once)
  asm volatile("" : "+v"(lane0));
  int64_t pos[NP];
  u32x4 w[NP][4];
  float came[NP];
  int page_next = page_at(begin_w + lane0);
  places(begin_w, k);
  pages(begin_w, k, pos, id);
  places(begin_w + W, k);
  load(pos, id, w, came, at);
  pages(begin_w + W, k, pos, id);
  places(begin_w + 2 * W, k);
  int mine = 0;
  for (int64_t first = begin_w; first < end; first += W, mine = mine == 2 ? 0 : mine + 1) {
    const int tok0 = (int)(first & ps_mask);
    const int lo = (int)max(begin - first, (int64_t)0), hi = (int)min(end - first, (int64_t)W);
    const int old0 = lo & ~(bt - 1);      // tokens old0 .. lo - 1 of the window are the older ones of a block
    const int page = __builtin_amdgcn_readfirstlane(page_next);
    const bool there = page >= 0 && page < g.n_pages;
    u32x4 v[NP];
    float sc[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) {        // (a token without a page counts as zeros)
      v[p] = at[p] < 0 ? u32x4{0u, 0u, 0u, 0u} : token_codes(w[p], at[p], is_v);
      sc[p] = at[p] < 0 ? 0.f : came[p];
      const int t = p * TP + tl;
      // (on the bits: a NaN is above all)
      if (sub == 0 && t < W) atomicMax(&s_mag[mine][t >> g.bt_log2], mag_bits(sc[p]));
    }
    wait_vmem();       // everything that this window's writes could change has been read
#pragma unroll
    for (int p = 0; p < NP; ++p) asm volatile("" : "+v"(id[p]), "+v"(k[p]));
    load(pos, id, w, came, at);
    pages(first + 2 * W, k, pos, id);
    places(first + 3 * W, k);
    page_next = page_at(first + W + lane0);
    __syncthreads();
    const int64_t cbase = kv_code_base(g, there ? page : 0, h, tok0);
    const int64_t sbase = kv_scale_index(g, there ? page : 0, h, tok0);
    for (int b = tid; b < (W >> g.bt_log2); b += 256) {
      const int t0 = b << g.bt_log2;
      s_mag[mine == 0 ? 2 : mine - 1][b] = 0u;   // the window before has read them, the one after the next fills them
      if (there && t0 < hi && t0 + bt > lo) scales[sbase + b] = __uint_as_float(s_mag[mine][b]);
    }
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int t = p * TP + tl;
      if (!there || t < old0 || t >= hi) continue;
      const float now = __uint_as_float(s_mag[mine][t >> g.bt_log2]);
      if (now > sc[p]) v[p] = rescale(v[p], sc[p] / now);
      if (is_v) *reinterpret_cast<u32x4*>(s_tile + t * D + 16 * sub) = v[p];
      else *reinterpret_cast<u32x4*>(codes + cbase + (int64_t)t * D + 16 * sub) = v[p];
    }
    if (is_v) {
      __syncthreads();
      // words of four tokens at one d, whole ones at once and the others by bytes
      for (int i = tid; there && i < (W >> 2) * D; i += 256) {
        const int t4 = (i / D) * 4, dd = i % D;
        if (t4 + 4 <= old0 || t4 >= hi) continue;
        int8_t* dst = codes + cbase + (int64_t)t4 * D + dd * 4;
        if (t4 >= old0 && t4 + 4 <= hi) {
          *reinterpret_cast<unsigned int*>(dst) =
              (unsigned)s_tile[t4 * D + dd] | ((unsigned)s_tile[(t4 + 1) * D + dd] << 8) |
              ((unsigned)s_tile[(t4 + 2) * D + dd] << 16) | ((unsigned)s_tile[(t4 + 3) * D + dd] << 24);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (t4 + k >= old0 && t4 + k < hi) dst[k] = (int8_t)s_tile[(t4 + k) * D + dd];
        }
      }
    }
  }
}

template <int LPH>
catq_status launch_compact(const CompactArgs& a, hipStream_t stream) {
  constexpr int TP = 256 / LPH;
  const double bytes = 4.0 * (double)a.g.n_tokens * a.g.n_kv * a.g.d;
  auto go = [&](auto np) {
    constexpr int NP = decltype(np)::value;
    CATQ_TRACED(stream, "kv_compact_kernel", 0.0, bytes, a.g.n_tokens, a.g.n_kv, a.g.d,
                hipLaunchKernelGGL((kv_compact_kernel<LPH, NP>), dim3(2u * a.g.n_kv, (unsigned)a.g.n_seqs),
                                   dim3(256), 0, stream, a));
  };
  using std::integral_constant;
  // a window has at most 128 tokens (a page of 16 at least a quarter of a pass)
  switch (((1 << a.w_log2) + TP - 1) / TP) {
    case 1: go(integral_constant<int, 1>{}); break;
    case 2: go(integral_constant<int, 2>{}); break;
    case 4:
      if constexpr (TP <= 32) go(integral_constant<int, 4>{});
      break;
    case 8:
      if constexpr (TP <= 16) go(integral_constant<int, 8>{});
      break;
    default: break;
  }
  CATQ_CHECK_LAUNCH("kv compact");
  return CATQ_OK;
}

}  // namespace
}  // namespace catq

using namespace catq;

extern "C" catq_status catq_aux_kv_copy_pages(const catq_kv_desc* d, const catq_kv_cache* cache, const int32_t* src,
                                              const int32_t* dst, int64_t n, hipStream_t stream) {
  clear_error();
  CATQ_TRY(kv_check_pool(d, cache));
  CATQ_REQUIRE(n >= 0, CATQ_ERR_SHAPE, "n must be >= 0");
  if (n == 0) return CATQ_OK;
  CATQ_REQUIRE(src && dst, CATQ_ERR_NULL, "src and dst must not be NULL");
  CATQ_REQUIRE(((reinterpret_cast<uintptr_t>(src) | reinterpret_cast<uintptr_t>(dst)) & 3) == 0, CATQ_ERR_ALIGN,
               "src and dst must be 4-byte aligned");
  CopyArgs a{};
  a.c = *cache;
  a.src = src;
  a.dst = dst;
  a.n_pages = d->n_pages;
  a.code_bytes = (int64_t)d->n_kv * d->page_size * d->head_dim;
  a.scales = (int64_t)d->n_kv * (d->page_size / d->scale_block);
  a.pieces = (int)((a.code_bytes / 16 + 256 * kCopy - 1) / (256 * kCopy));
  // (a launch has fewer than 2^32 threads along x)
  CATQ_REQUIRE(n < (1 << 24) / (2 * a.pieces + 1), CATQ_ERR_SHAPE, "too many pages for one launch");
  CATQ_TRACED(stream, "kv_copy_kernel", 0.0, 4.0 * (double)n * (a.code_bytes + 4 * a.scales), n, d->n_kv, d->head_dim,
              hipLaunchKernelGGL(kv_copy_kernel, dim3((unsigned)(n * (2 * a.pieces + 1))), dim3(256), 0, stream, a));
  CATQ_CHECK_LAUNCH("kv copy pages");
  return CATQ_OK;
}

extern "C" catq_status catq_aux_kv_compact(const catq_kv_desc* d, const catq_kv_cache* cache,
                                           const catq_kv_batch* batch, const int32_t* keep, const int32_t* n_keep,
                                           hipStream_t stream) {
  clear_error();
  CATQ_TRY(kv_check(d, cache, batch));
  if (batch->n_seqs == 0 || batch->n_tokens == 0 || batch->max_new == 0) return CATQ_OK;
  CATQ_REQUIRE(keep && n_keep, CATQ_ERR_NULL, "keep and n_keep must not be NULL");
  CATQ_REQUIRE(((reinterpret_cast<uintptr_t>(keep) | reinterpret_cast<uintptr_t>(n_keep)) & 3) == 0, CATQ_ERR_ALIGN,
               "keep and n_keep must be 4-byte aligned");
  CompactArgs a{};
  a.g = kv_geom(d, batch);
  a.c = *cache;
  a.keep = keep;
  a.n_keep = n_keep;
  // A window lies in one page and holds whole scale blocks; up to four passes of the threads (one pass: 984 us where
  // four take 766, and the same for a few tokens).
  const int w = std::max(d->scale_block, std::min(std::min(4 * 256 / (d->head_dim / 16), 128), d->page_size));
  a.w_log2 = __builtin_ctz((unsigned)w);
  switch (d->head_dim) {
    case 64: return launch_compact<4>(a, stream);
    case 128: return launch_compact<8>(a, stream);
    default: return launch_compact<16>(a, stream);
  }
}
