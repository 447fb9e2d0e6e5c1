// Routed experts on packed-ternary weights and 8-bit activations, for few tokens (gfx950):
//   ids, w = the top_k largest logits of a token and their softmax
//   a      = silu(gate) * up,  [gate | up] = x_scale * q (alpha T)^T of the slot's expert
//   y      = res + sum_j w_j * s_j * qa_j (alpha T)^T,  qa, s the 8-bit codes and scale of slot j's a
//
// What a few tokens cost is the weights of the experts that they hit, read once: 2 bits each and a scale per group.
// A wave takes rows of 16 weights and a run of 128-code chunks, and brings up to eight or twelve chunks of their codes
// into LDS of its own at once by direct copies, so that a unit has some 100 KB in flight without a wait between waves;
// the matrix products take 16 slots, of which a few are used.
//
// Launches.  One token: every wave of the first kernel finds its experts itself, every workgroup of the second forms the
// codes of a: two launches.  More tokens: the experts and their slots are laid out by a kernel of their own (in the first
// kernel, two tokens took as long, four 54 us instead of 49.5).  Where the codes are more than LDS takes (24 KB, and
// from 9 tokens on), a kernel forms them, for one token too.
//
// What bounds it, 128 experts of 4096 x 1536, 8 a token: at one token (21 us, 42 MB) chains of latencies, routing 4 of the first
// kernel's 12 us, codes 2 of the second's 10. At 32 tokens (147 us, 111 experts, 594 MB, 4.0 TB/s) HBM and the vector ALU
// (54% of the issue in the first kernel, 42 in the second): of the instructions of a chunk of 16 rows 22 decode, 4 scale, 12 read
// and address; with the activations as columns, in plain order and loaded for all of them, it took 221 us.
// From 64 tokens on (215 us, where the weights read once take 130) the down kernel's weights, read again for every 32
// tokens: 322 us at 128 tokens, 2095 at 1024.
#include <type_traits>

#include "kernels.h"
#include "moe_topk.h"
#include "quant8.h"
#include "ternary8.h"

namespace catq {
namespace {

struct MoeArgs {
  const float* logits;
  const int8_t* X;
  const float* xs;
  int64_t ldx;
  const uint8_t* P1;      // [E][2 F][h/4]
  const float* A1;
  const uint8_t* P2;      // [E][h][F/4]
  const float* A2;
  const void* res;
  void* Y;
  int32_t* ids;           // [T][k]
  float* w;               // [T][k]
  float* act;             // [T][k][F]
  int8_t* qa;             // [T][k][F], in the order of matrix operands
  float* sa;              // [T][k]
  int8_t* xt;             // [T][h]: q in the order of matrix operands
  int32_t* hits;          // experts that are hit, from hits[1] on their ids, first slots and numbers of slots
  int32_t* slots;         // [T][k], by expert
  int32_t T, E, k, h, F;
  int32_t shift;          // log2(g / 128)
};

// A wave's tile of 16 weight rows
struct Tile {
  i32x4_rsrc codes;
  __amdgpu_buffer_rsrc_t alpha;
};
__device__ __forceinline__ Tile tile_at(const uint8_t* P, const float* A, int64_t row, int n, int shift) {
  Tile t;
  const int64_t row_bytes = n >> 2;
  const int ng = n >> (7 + shift);
  t.codes = buf_rsrc(P + row * row_bytes, (uint32_t)(16 * row_bytes));
  t.alpha = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(A + row * ng), 0, 16 * ng * 4, 0x00020000);
  return t;
}

// LDS of a wave: for each of R tiles NB / 2 copies of 1 KB ([16 rows][4 pieces of 16 bytes], piece p of row t at
// p ^ (t / 4): two chunks) and the scales of the groups of NB chunks
constexpr int scale_slots(int NB) { return NB <= 8 ? 8 : 16; }
template <int R, int NB>
constexpr int own_bytes() {
  return R * (NB / 2 * 1024 + scale_slots(NB) * 64);
}

// Up to 16 slots' activations are the rows of a product, a tile's 16 weight rows its columns. Slot i is row
// 4 (i % 4) + i / 4, so that its sums are element i / 4 of the lanes of group i % 4: with up to four slots only the first
// element of every lane is converted and scaled.
__device__ __forceinline__ int slot_of_row(int row) { return 4 * (row & 3) + (row >> 2); }

// The copies of nb <= NB chunks' codes from chunk b0 on into a wave's LDS.
template <int R, int NB>
__device__ __forceinline__ void copy_codes(const Tile (&tile)[R], int b0, int nb, int n, char* own) {
  const int lane = threadIdx.x & 63;
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)own;
  const uint32_t woff = (uint32_t)((lane >> 2) * (n >> 2) + ((lane & 3) ^ (lane >> 4)) * 16);
#pragma unroll
  for (int p = 0; p < NB / 2; ++p) {
    if (2 * p >= nb) continue;
#pragma unroll
    for (int r = 0; r < R; ++r)    // (past a row's end: the next row, or zeros; never used)
      dma16_lds(tile[r].codes, woff + (uint32_t)(b0 + 2 * p) * 32u, 0u, lds + (r * (NB / 2) + p) * 1024);
  }
}

// out[r][e] += sum over chunks c0 .. c1 - 1 of alpha * (codes . x) of weight row lane % 16 of tile r and slot
// 4 e + lane / 16, e < ne. x: the activations of this lane's row, if it has a slot. n: codes of a row. NB chunks at a
// time. ORDERED: the activations are in the order of the operands.
template <int R, int NB, bool ORDERED>
__device__ __forceinline__ void rows_product(const Tile (&tile)[R], const int8_t* x, bool used, int ne, int c0, int c1,
                                             int n, int shift, char* own, f32x4 (&out)[R]) {
  constexpr int G = scale_slots(NB), AU = 16 * G / 64;
  const int lane = threadIdx.x & 63, q = lane >> 4, c16 = lane & 15;
  const int ng = n >> (7 + shift);
  float* s_al = reinterpret_cast<float*>(own + R * (NB / 2 * 1024));
  for (int b0 = c0; b0 < c1; b0 += NB) {
    const int nb = min(c1 - b0, NB), g0 = b0 >> shift;
    wait_lds();     // what the last burst read may be written over
    copy_codes<R, NB>(tile, b0, nb, n, own);
    float av[R][AU];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int u = 0; u < AU; ++u) {
        const int i = lane + 64 * u, g = min(g0 + i % G, ng - 1);
        av[r][u] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(tile[r].alpha, (i / G * ng + g) * 4, 0, 0));
      }
    // activations, some chunks ahead (only where a column is used: a load takes the L1 as long as it has lanes)
    constexpr int PF = NB <= 8 ? NB : 6;
    u32x4 xr[PF][2];
    auto load_x = [&](int c, u32x4 (&v)[2]) __attribute__((always_inline)) {
      const int at = min(b0 + c, c1 - 1) * 128 + 32 * q;
      v[0] = *reinterpret_cast<const u32x4*>(x + at);
      v[1] = *reinterpret_cast<const u32x4*>(x + at + 16);
    };
    if (used) {
#pragma unroll
      for (int c = 0; c < PF; ++c) load_x(c, xr[c]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int u = 0; u < AU; ++u) {
        const int i = lane + 64 * u;
        s_al[(r * G + i % G) * 16 + i / G] = av[r][u];
      }
    wait_vmem();
    wait_lds();
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      if (c >= nb) continue;
      const u32x4 x0 = ORDERED ? xr[c % PF][0] : transpose16(xr[c % PF][0]);
      const u32x4 x1 = ORDERED ? xr[c % PF][1] : transpose16(xr[c % PF][1]);
      if (c + PF < NB && used) load_x(c + PF, xr[c % PF]);
      const int g = ((b0 + c) >> shift) - g0;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const uint2 w = *reinterpret_cast<const uint2*>(own + (r * (NB / 2) + c / 2) * 1024 + c16 * 64 +
                                                        ((2 * (c & 1) + (q >> 1)) ^ (c16 >> 2)) * 16 + 8 * (q & 1));
        const float sc = s_al[(r * G + g) * 16 + c16];
        i32x4 acc = {0, 0, 0, 0};
        acc = mfma_i8(x0, decode16_i8(w.x), acc);
        acc = mfma_i8(x1, decode16_i8(w.y), acc);
        out[r][0] = fmaf(sc, (float)acc[0], out[r][0]);
        if (ne > 1) {
#pragma unroll
          for (int e = 1; e < 4; ++e) out[r][e] = fmaf(sc, (float)acc[e], out[r][e]);
        }
      }
    }
  }
}

__device__ __forceinline__ void topk_any(const MoeArgs& a, int t, int lane, int& id, float& w) {
  const float* row = a.logits + (int64_t)t * a.E;
  if (a.E <= 64) topk_token<1>(row, a.E, a.k, lane, id, w);
  else if (a.E <= 128) topk_token<2>(row, a.E, a.k, lane, id, w);
  else if (a.E <= 256) topk_token<4>(row, a.E, a.k, lane, id, w);
  else topk_token<16>(row, a.E, a.k, lane, id, w);
}

// The first workgroup: the experts of every token, and the slots of every expert that is hit. (The order of an
// expert's slots is that of LDS atomics: it decides in which row a slot is computed, and nothing else.)
// The others: the activations in the order of the operands.
constexpr int kListed = 4096;    // slots whose experts are kept in LDS
__global__ __launch_bounds__(1024) void moe_experts_kernel(MoeArgs a) {
  __shared__ int s_count[1024], s_first[1024];
  __shared__ int s_wave[16], s_wave_hits[16];
  __shared__ short s_ids[kListed];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.T * a.k;
  if (blockIdx.x > 0) {
    const int i = (blockIdx.x - 1) * 1024 + tid, per = a.h >> 4;
    if (i >= a.T * per) return;
    const int t = i / per, p = i - t * per;
    *reinterpret_cast<u32x4*>(a.xt + (int64_t)t * a.h + 16 * p) =
        transpose16(*reinterpret_cast<const u32x4*>(a.X + t * a.ldx + 16 * p));
    return;
  }
  s_count[tid] = 0;
  __syncthreads();
  for (int t = wave; t < a.T; t += 16) {
    int id;
    float w;
    topk_any(a, t, lane, id, w);
    if (lane < a.k) {
      const int i = t * a.k + lane;
      a.ids[i] = id;
      a.w[i] = w;
      if (i < kListed) s_ids[i] = (short)id;
      atomicAdd(&s_count[id], 1);
    }
  }
  __syncthreads();
  const int c = s_count[tid];           // (thread e: expert e)
  const unsigned long long m = __ballot(c > 0);
  int at = c;                           // inclusive sum over the wave
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(at, d, 64);
    if (lane >= d) at += o;
  }
  if (lane == 63) {
    s_wave[wave] = at;
    s_wave_hits[wave] = __popcll(m);
  }
  __syncthreads();
  int before = 0, hit = 0, hits = 0;
  for (int w = 0; w < 16; ++w) {
    if (w < wave) {
      before += s_wave[w];
      hit += s_wave_hits[w];
    }
    hits += s_wave_hits[w];
  }
  const int first = before + at - c;
  s_first[tid] = first;
  if (c > 0) {
    int32_t* h = a.hits + 1 + 3 * (hit + __popcll(m & ((1ull << lane) - 1)));
    h[0] = tid;
    h[1] = first;
    h[2] = c;
  }
  if (tid == 0) a.hits[0] = hits;
  __syncthreads();
  for (int i = tid; i < n; i += 1024) {
    const int id = i < kListed ? (int)s_ids[i] : a.ids[i];      // (this workgroup's own writes)
    a.slots[atomicAdd(&s_first[id], 1)] = i;
  }
}

// Values f .. f + 15 of a slot's a: their largest magnitude (as bits), and their codes in the order of the operands.
__device__ __forceinline__ unsigned int mag_16(const float* p) {
  unsigned int m = 0u;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(p + 4 * j);
    m = max(max(m, max(mag_bits(v[0]), mag_bits(v[1]))), max(mag_bits(v[2]), mag_bits(v[3])));
  }
  return m;
}
__device__ __forceinline__ u32x4 codes_16(const float* p, float s) {
  u32x4 c;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(p + 4 * j);
    float v[4] = {x[0], x[1], x[2], x[3]};
    quant8_n(v, s);
    c[j] = pack_codes(v[0], v[1], v[2], v[3]);
  }
  return transpose16(c);
}
// The codes and scales of a, a wave a slot, as the quantizer forms them.
__global__ __launch_bounds__(256) void moe_codes_kernel(MoeArgs a) {
  const int slot = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (slot >= a.T * a.k) return;
  const float* p = a.act + (int64_t)slot * a.F;
  unsigned int m = 0u;
  for (int f = 16 * lane; f < a.F; f += 1024) m = max(m, mag_16(p + f));
  const float s = quant8_scale(wave_umax(m));
  if (lane == 0) a.sa[slot] = s;
  for (int f = 16 * lane; f < a.F; f += 1024)
    *reinterpret_cast<u32x4*>(a.qa + (int64_t)slot * a.F + f) = codes_16(p + f, s);
}

// Gate, up and their product: 16 values of a for all slots of an expert.
// FUSED (one token): every wave finds the token's experts, item i is that of slot i. Otherwise item i is the i-th expert
// that is hit.
constexpr int kUpWaves = 4, kUpBurst = 8;
template <bool FUSED>
__global__ __launch_bounds__(kUpWaves * 64) void moe_up_kernel(MoeArgs a) {
  constexpr int OWN = own_bytes<2, kUpBurst>();
  __shared__ __align__(16) char s_own[kUpWaves][OWN];
  __shared__ int s_slot[16];
  static_assert(OWN >= 2 * 16 * 17 * 4, "the waves' sums fit their place");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int item = blockIdx.y;
  int e, slots;
  const int32_t* list = nullptr;
  if constexpr (FUSED) {
    int id;
    float w;
    topk_any(a, 0, lane, id, w);
    if (blockIdx.x == 0 && item == 0 && tid < a.k) {
      a.ids[tid] = id;
      a.w[tid] = w;
    }
    e = __builtin_amdgcn_readlane(id, item);
    slots = 1;
  } else {
    if (item >= a.hits[0]) return;
    const int32_t* h = a.hits + 1 + 3 * item;
    e = __builtin_amdgcn_readfirstlane(h[0]);
    list = a.slots + h[1];
    slots = __builtin_amdgcn_readfirstlane(h[2]);
  }
  const int f0 = blockIdx.x * 16, nch = a.h >> 7;
  const int64_t row = (int64_t)e * 2 * a.F + f0;
  const Tile tile[2] = {tile_at(a.P1, a.A1, row, a.h, a.shift), tile_at(a.P1, a.A1, row + a.F, a.h, a.shift)};
  for (int s0 = 0; s0 < slots; s0 += 16) {
    const int here = min(slots - s0, 16), mine = slot_of_row(lane & 15);
    if (tid < here) s_slot[tid] = FUSED ? item : list[s0 + tid];
    const bool used = mine < here;
    const int slot = !used ? 0 : FUSED ? item : list[s0 + mine];
    const int t = slot / a.k;
    f32x4 out[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    rows_product<2, kUpBurst, !FUSED>(tile, FUSED ? a.X + t * a.ldx : a.xt + (int64_t)t * a.h, used, (here + 3) >> 2,
                                      wave * nch / kUpWaves, (wave + 1) * nch / kUpWaves, a.h, a.shift, s_own[wave], out);
    float* red = reinterpret_cast<float*>(s_own[wave]);
    wait_lds();
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) red[(r * 16 + 4 * i + (lane >> 4)) * 17 + (lane & 15)] = out[r][i];
    __syncthreads();
    if (tid < 16 * here) {
      const int c = tid >> 4, f = tid & 15;
      float g = 0.f, u = 0.f;
#pragma unroll
      for (int w = 0; w < kUpWaves; ++w) {
        const float* p = reinterpret_cast<const float*>(s_own[w]);
        g += p[c * 17 + f];
        u += p[(16 + c) * 17 + f];
      }
      const int sl = s_slot[c];
      const float xs = a.xs[sl / a.k];
      a.act[(int64_t)sl * a.F + f0 + f] = swiglu1(g * xs, u * xs);
    }
    __syncthreads();
  }
}

// Down and the sum over a token's experts: 16 outputs of TG tokens. The waves take the experts that these hit in turn,
// or runs of their chunks where they are few, 16 of an expert's slots at a time, and add to sums of their own in LDS.
// FUSED: the codes of a, kFusedCodes at most, are formed here, in LDS.
constexpr int kDownWaves = 16, kDownBurst = 12, kFusedCodes = 24 * 1024;
template <typename T, int TG, bool FUSED>
__global__ __launch_bounds__(kDownWaves * 64) void moe_down_kernel(MoeArgs a) {
  constexpr int OWN = own_bytes<1, kDownBurst>(), SLOTS = 16 * TG;
  __shared__ __align__(16) char s_own[kDownWaves][OWN];
  __shared__ __align__(16) int8_t s_qa[FUSED ? kFusedCodes : 16];
  __shared__ float s_sum[kDownWaves][TG][17];
  __shared__ int s_ids[SLOTS];
  __shared__ float s_w[SLOTS];
  __shared__ short s_col[kDownWaves][TG];
  __shared__ unsigned int s_bits[32];
  __shared__ short s_list[SLOTS];
  static_assert(SLOTS <= kDownWaves * 64, "a slot per thread");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t0 = blockIdx.y * TG, toks = min(a.T - t0, TG), n = toks * a.k;
  if (tid < 32) s_bits[tid] = 0u;
  for (int i = lane; i < TG * 17; i += 64) s_sum[wave][0][i] = 0.f;
  __syncthreads();
  if (tid < n) {
    const int e = a.ids[t0 * a.k + tid];
    s_ids[tid] = e;
    s_w[tid] = FUSED ? a.w[t0 * a.k + tid] : a.w[t0 * a.k + tid] * a.sa[t0 * a.k + tid];
    atomicOr(&s_bits[e >> 5], 1u << (e & 31));
  }
  __syncthreads();
  int hit = 0;
  for (int w = 0; w < (a.E + 31) / 32; ++w) hit += __popc(s_bits[w]);
  if (tid < a.E) {
    const unsigned int bits = s_bits[tid >> 5];
    if ((bits >> (tid & 31)) & 1u) {
      int at = __popc(bits & ((1u << (tid & 31)) - 1u));
      for (int w = 0; w < (tid >> 5); ++w) at += __popc(s_bits[w]);
      s_list[at] = (short)tid;
    }
  }
  __syncthreads();
  const int r0 = blockIdx.x * 16, c16 = lane & 15, nch = a.F >> 7;
  int parts = 1;
  while (hit * parts < kDownWaves && 2 * parts <= nch) parts *= 2;
  if constexpr (FUSED) {
    for (int i = wave; i < n; i += kDownWaves) {
      const float* p = a.act + (int64_t)(t0 * a.k + i) * a.F;
      unsigned int m = 0u;
      for (int f = 16 * lane; f < a.F; f += 1024) m = max(m, mag_16(p + f));
      const float s = quant8_scale(wave_umax(m));
      if (lane == 0) s_w[i] *= s;
      for (int f = 16 * lane; f < a.F; f += 1024) *reinterpret_cast<u32x4*>(s_qa + i * a.F + f) = codes_16(p + f, s);
    }
    __syncthreads();
  }
  for (int i = wave; i < hit * parts; i += kDownWaves) {
    const int e = __builtin_amdgcn_readfirstlane((int)s_list[i / parts]), part = i % parts;
    int slots = 0;
    for (int b = 0; b < n; b += 64) {
      const bool mine = b + lane < n && s_ids[b + lane] == e;
      const unsigned long long m = __ballot(mine);
      if (mine) s_col[wave][slots + __popcll(m & ((1ull << lane) - 1))] = (short)(b + lane);
      slots += __popcll(m);
    }
    const Tile tile[1] = {tile_at(a.P2, a.A2, (int64_t)e * a.h + r0, a.F, a.shift)};
    for (int c0 = 0; c0 < slots; c0 += 16) {
      const bool used = c0 + slot_of_row(c16) < slots;
      const int slot = used ? (int)s_col[wave][c0 + slot_of_row(c16)] : 0, here = min(slots - c0, 16);
      f32x4 out[1] = {{0.f, 0.f, 0.f, 0.f}};
      rows_product<1, kDownBurst, true>(tile, FUSED ? s_qa + slot * a.F : a.qa + (int64_t)(t0 * a.k + slot) * a.F, used,
                                        (here + 3) >> 2, part * nch / parts, (part + 1) * nch / parts, a.F, a.shift,
                                        s_own[wave], out);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int j = 4 * v + (lane >> 4);
        if (j >= here) continue;
        const int sl = s_col[wave][c0 + j];
        float* p = &s_sum[wave][sl / a.k][c16];
        *p = fmaf(s_w[sl], out[0][v], *p);
      }
    }
  }
  __syncthreads();
  if (tid < 16 * toks) {
    const int col = tid >> 4, r = tid & 15;
    const int64_t at = (int64_t)(t0 + col) * a.h + r0 + r;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kDownWaves; ++w) v += s_sum[w][col][r];
    if (a.res) v += to_f(static_cast<const T*>(a.res)[at]);
    static_cast<T*>(a.Y)[at] = (T)v;
  }
}

catq_status moe_check(const catq_moe_desc* d, int64_t T) {
  CATQ_REQUIRE(d, CATQ_ERR_NULL, "descriptor must not be NULL");
  const int g = d->group_size;
  CATQ_REQUIRE(g >= 128 && g % 128 == 0 && ((g / 128) & (g / 128 - 1)) == 0, CATQ_ERR_VALUE,
               "group_size must be 128 times a power of two");
  CATQ_REQUIRE(d->n_experts > 0 && d->n_experts <= 1024 && d->top_k > 0 && d->top_k <= 16 &&
                   d->top_k <= d->n_experts,
               CATQ_ERR_SHAPE, "need 1 <= top_k <= min(16, n_experts), n_experts <= 1024");
  CATQ_REQUIRE(d->hidden > 0 && d->ffn > 0 && d->hidden % g == 0 && d->ffn % g == 0 && d->hidden <= 32768 &&
                   d->ffn <= 32768,
               CATQ_ERR_SHAPE, "hidden and ffn must be multiples of group_size, at most 32768");
  CATQ_REQUIRE(T >= 0 && T <= 1024, CATQ_ERR_SHAPE, "T must be 0 .. 1024");
  return CATQ_OK;
}

struct MoeSpace {
  size_t ids, w, sa, hits, slots, xt, qa, act, end;
};
MoeSpace moe_space(const catq_moe_desc* d, int64_t T) {
  const size_t n = (size_t)T * d->top_k;
  MoeSpace s;
  s.ids = 0;
  s.w = round_up(n * 4, 256);
  s.sa = s.w + round_up(n * 4, 256);
  s.hits = s.sa + round_up(n * 4, 256);
  s.slots = s.hits + round_up((1 + 3 * (size_t)d->n_experts) * 4, 256);
  s.xt = s.slots + round_up(n * 4, 256);
  s.qa = s.xt + round_up((size_t)T * d->hidden, 256);
  s.act = s.qa + round_up(n * d->ffn, 256);
  s.end = s.act + round_up(n * d->ffn * 4, 256);
  return s;
}

}  // namespace
}  // namespace catq

using namespace catq;

extern "C" size_t catq_ternary_moe_a8_workspace_bytes(const catq_moe_desc* d, int64_t T) {
  if (moe_check(d, T) != CATQ_OK || T == 0) return 0;
  return moe_space(d, T).end;
}

extern "C" catq_status catq_ternary_moe_a8(const catq_moe_desc* d, const float* logits, const int8_t* q, int64_t T,
                                           int64_t ldq, const float* x_scale, const uint8_t* gu_packed,
                                           const float* gu_alpha, const uint8_t* down_packed,
                                           const float* down_alpha, const void* res, void* y, catq_dtype y_dtype,
                                           void* workspace, size_t workspace_bytes, hipStream_t stream) {
  clear_error();
  CATQ_TRY(moe_check(d, T));
  if (T == 0) return CATQ_OK;
  CATQ_REQUIRE(logits && q && x_scale && gu_packed && gu_alpha && down_packed && down_alpha && y, CATQ_ERR_NULL,
               "only res may be NULL");
  CATQ_REQUIRE(dtype_ok(y_dtype), CATQ_ERR_DTYPE, "y must be fp32 or bf16");
  CATQ_REQUIRE(ldq >= d->hidden && ldq % 16 == 0 && ldq <= (1 << 24), CATQ_ERR_SHAPE,
               "ldq must be >= hidden, a multiple of 16 and <= 2^24");
  auto at4 = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; };
  CATQ_REQUIRE(aligned16(q) && aligned16(gu_packed) && aligned16(gu_alpha) && aligned16(down_packed) &&
                   aligned16(down_alpha) && aligned16(res) && aligned16(y) && aligned16(workspace) && at4(logits) &&
                   at4(x_scale),
               CATQ_ERR_ALIGN, "logits and x_scale must be 4-byte aligned, the others 16-byte");
  const MoeSpace sp = moe_space(d, T);
  CATQ_REQUIRE(workspace && workspace_bytes >= sp.end, CATQ_ERR_WORKSPACE,
               "workspace of %zu bytes needed, %zu given", sp.end, workspace ? workspace_bytes : (size_t)0);
  char* ws = static_cast<char*>(workspace);
  MoeArgs a{logits, q, x_scale, ldq, gu_packed, gu_alpha, down_packed, down_alpha, res, y,
            reinterpret_cast<int32_t*>(ws + sp.ids), reinterpret_cast<float*>(ws + sp.w),
            reinterpret_cast<float*>(ws + sp.act), reinterpret_cast<int8_t*>(ws + sp.qa),
            reinterpret_cast<float*>(ws + sp.sa), reinterpret_cast<int8_t*>(ws + sp.xt),
            reinterpret_cast<int32_t*>(ws + sp.hits), reinterpret_cast<int32_t*>(ws + sp.slots), (int32_t)T, d->n_experts, d->top_k, d->hidden, d->ffn,
            __builtin_ctz((unsigned)d->group_size / 128)};
  const int n = (int)T * a.k, hit = n < a.E ? n : a.E;
  const double wt = (double)hit * a.h * a.F * (0.25 + 4.0 / d->group_size);
  const bool fused = T == 1, codes_here = T <= 8 && (int64_t)n * a.F <= kFusedCodes;
  if (!fused) {
    CATQ_TRACED(stream, "moe_experts_kernel", 0.0, 4.0 * T * a.E, T, a.E, a.k,
                hipLaunchKernelGGL(moe_experts_kernel, dim3(1 + (unsigned)((T * (a.h >> 4) + 1023) / 1024)), dim3(1024), 0,
                                   stream, a));
    CATQ_CHECK_LAUNCH("moe experts");
  }
  auto up = fused ? moe_up_kernel<true> : moe_up_kernel<false>;
  CATQ_TRACED(stream, fused ? "moe_up_kernel<fused>" : "moe_up_kernel", 4.0 * n * a.h * a.F, 2.0 * wt, n, 2 * a.F, a.h,
              hipLaunchKernelGGL(up, dim3((unsigned)(a.F / 16), (unsigned)hit), dim3(kUpWaves * 64), 0, stream, a));
  CATQ_CHECK_LAUNCH("moe gate and up");
  if (!codes_here) {
    CATQ_TRACED(stream, "moe_codes_kernel", 0.0, 5.0 * n * a.F, n, a.F, 1,
                hipLaunchKernelGGL(moe_codes_kernel, dim3((unsigned)((n + 3) / 4)), dim3(256), 0, stream, a));
    CATQ_CHECK_LAUNCH("moe codes");
  }
  const int cols = T > 16 ? 32 : 16;
  auto down = [&](auto out) {
    using Out = decltype(out);
    auto kernel = codes_here ? moe_down_kernel<Out, 8, true> : cols == 16 ? moe_down_kernel<Out, 16, false>
                                                                          : moe_down_kernel<Out, 32, false>;
    CATQ_TRACED(stream, "moe_down_kernel", 2.0 * n * a.h * a.F, wt, n, a.h, a.F,
                hipLaunchKernelGGL(kernel, dim3((unsigned)(a.h / 16), (unsigned)((T + cols - 1) / cols)),
                                   dim3(kDownWaves * 64), 0, stream, a));
  };
  if (y_dtype == CATQ_F32) down(float{});
  else down(bf16{});
  CATQ_CHECK_LAUNCH("moe down");
  return CATQ_OK;
}
