// Routed experts on packed-ternary weights and 8-bit activations, for few tokens (gfx950):
//   ids, w = the top_k largest logits of a token and their softmax
//   a      = silu(gate) * up,  [gate | up] = x_scale * q (alpha T)^T of the slot's expert
//   y      = res + sum_j w_j * s_j * qa_j (alpha T)^T,  qa, s the 8-bit codes and scale of slot j's a
//
// What a few tokens cost is the weights of the experts that they hit, read once: 2 bits each and a scale per group.
// A wave takes rows of 16 weights and a run of 128-code chunks (or of experts), and brings up to eight chunks of their
// codes into LDS of its own at once by direct copies, so that a unit has some 100 KB in flight without a wait between
// waves; the matrix products take 16 token columns, of which a few are used.
#include <type_traits>

#include "kernels.h"
#include "moe_topk.h"
#include "ternary8.h"

namespace catq {
namespace {

constexpr int kBurst = 8;        // chunks of 128 codes copied at once
constexpr int kPitch = 20;       // floats between groups of a tile's scales in LDS

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
  int8_t* qa;             // [T][k][F]
  float* sa;              // [T][k]
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

// LDS of a wave: for each of R tiles four copies of 1 KB ([16 rows][4 pieces of 16 bytes], piece p of row t at
// p ^ (t / 4): two chunks) and the scales of up to eight groups
template <int R>
constexpr int own_bytes() {
  return R * (kBurst / 2 * 1024 + 8 * kPitch * 4);
}

// out[r][e] += sum over chunks c0 .. c1 - 1 of alpha * (codes . x): row 4 (lane / 16) + e of tile r, the column of x
// that this lane points to. n: codes of a row.
template <int R>
__device__ __forceinline__ void rows_product(const Tile (&tile)[R], const int8_t* x, int c0, int c1, int n, int shift,
                                             char* own, f32x4 (&out)[R]) {
  const int lane = threadIdx.x & 63, q = lane >> 4, c16 = lane & 15;
  const int row_bytes = n >> 2, ng = n >> (7 + shift);
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)own;
  float* s_al = reinterpret_cast<float*>(own + R * (kBurst / 2 * 1024));
  const uint32_t woff = (uint32_t)((lane >> 2) * row_bytes + ((lane & 3) ^ (lane >> 4)) * 16);
  for (int b0 = c0; b0 < c1; b0 += kBurst) {
    const int nb = min(c1 - b0, kBurst), g0 = b0 >> shift;
    wait_lds();     // what the last burst read may be written over
#pragma unroll
    for (int p = 0; p < kBurst / 2; ++p) {
      if (2 * p >= nb) break;
#pragma unroll
      for (int r = 0; r < R; ++r)    // (past a row's end: the next row, or zeros; never used)
        dma16_lds(tile[r].codes, woff + (uint32_t)(b0 + 2 * p) * 32u, 0u, lds + (r * (kBurst / 2) + p) * 1024);
    }
    float av[R][2];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int i = lane + 64 * u, g = min(g0 + (i & 7), ng - 1);
        av[r][u] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(tile[r].alpha, ((i >> 3) * ng + g) * 4, 0, 0));
      }
    u32x4 xr[kBurst][2];
#pragma unroll
    for (int c = 0; c < kBurst; ++c) {
      const int at = min(b0 + c, c1 - 1) * 128 + 32 * q;
      xr[c][0] = *reinterpret_cast<const u32x4*>(x + at);
      xr[c][1] = *reinterpret_cast<const u32x4*>(x + at + 16);
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int i = lane + 64 * u;
        s_al[(r * 8 + (i & 7)) * kPitch + (i >> 3)] = av[r][u];
      }
    wait_vmem();
    wait_lds();
#pragma unroll
    for (int c = 0; c < kBurst; ++c) {
      if (c >= nb) break;
      const u32x4 x0 = transpose16(xr[c][0]), x1 = transpose16(xr[c][1]);
      const int g = ((b0 + c) >> shift) - g0;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const uint2 w = *reinterpret_cast<const uint2*>(own + (r * (kBurst / 2) + c / 2) * 1024 + c16 * 64 +
                                                        ((2 * (c & 1) + (q >> 1)) ^ (c16 >> 2)) * 16 + 8 * (q & 1));
        const f32x4 sc = *reinterpret_cast<const f32x4*>(&s_al[(r * 8 + g) * kPitch + 4 * q]);
        i32x4 acc = {0, 0, 0, 0};
        acc = mfma_i8(decode16_i8(w.x), x0, acc);
        acc = mfma_i8(decode16_i8(w.y), x1, acc);
#pragma unroll
        for (int e = 0; e < 4; ++e) out[r][e] = fmaf(sc[e], (float)acc[e], out[r][e]);
      }
    }
  }
}

// The experts of every token, a wave each.
template <int PER>
__global__ __launch_bounds__(256) void moe_experts_kernel(MoeArgs a) {
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (t >= a.T) return;
  int id;
  float w;
  topk_token<PER>(a.logits + (int64_t)t * a.E, a.E, a.k, lane, id, w);
  if (lane < a.k) {
    a.ids[t * a.k + lane] = id;
    a.w[t * a.k + lane] = w;
  }
}

// Gate, up and their product: 16 values of a for all slots of an expert. Item i is the expert of slot i, if none
// before it has the same, or, where there are more slots than experts, expert i if any slot has it.
constexpr int kUpWaves = 4;
__global__ __launch_bounds__(kUpWaves * 64) void moe_up_kernel(MoeArgs a) {
  constexpr int OWN = own_bytes<2>();
  __shared__ __align__(16) char s_own[kUpWaves][OWN];
  __shared__ int s_slot[1024];
  __shared__ int s_n, s_e;
  static_assert(OWN >= 2 * 16 * 17 * 4, "the waves' sums fit their place");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = a.T * a.k, item = blockIdx.y;
  if (wave == 0) {
    const int e = n <= a.E ? a.ids[item] : item;
    int have = 0;
    bool first = true;
    for (int b = 0; b < n; b += 64) {
      const bool mine = b + lane < n && a.ids[b + lane] == e;
      const unsigned long long m = __ballot(mine);
      if (n <= a.E && have == 0 && m && b + __builtin_ctzll(m) < item) {
        first = false;
        break;
      }
      if (mine) s_slot[have + __popcll(m & ((1ull << lane) - 1))] = b + lane;
      have += __popcll(m);
    }
    if (lane == 0) {
      s_n = first ? have : 0;
      s_e = e;
    }
  }
  __syncthreads();
  const int slots = __builtin_amdgcn_readfirstlane(s_n), e = __builtin_amdgcn_readfirstlane(s_e);
  if (slots == 0) return;
  const int f0 = blockIdx.x * 16, nch = a.h >> 7;
  const int64_t row = (int64_t)e * 2 * a.F + f0;
  const Tile tile[2] = {tile_at(a.P1, a.A1, row, a.h, a.shift), tile_at(a.P1, a.A1, row + a.F, a.h, a.shift)};
  for (int s0 = 0; s0 < slots; s0 += 16) {
    const int here = min(slots - s0, 16);
    const int token = s_slot[s0 + min(lane & 15, here - 1)] / a.k;
    f32x4 out[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    rows_product<2>(tile, a.X + token * a.ldx, wave * nch / kUpWaves, (wave + 1) * nch / kUpWaves, a.h, a.shift,
                    s_own[wave], out);
    float* red = reinterpret_cast<float*>(s_own[wave]);
    wait_lds();
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) red[(r * 16 + (lane & 15)) * 17 + 4 * (lane >> 4) + i] = out[r][i];
    __syncthreads();
    for (int i = tid; i < 16 * here; i += kUpWaves * 64) {
      const int col = i >> 4, f = i & 15;
      float g = 0.f, u = 0.f;
#pragma unroll
      for (int w = 0; w < kUpWaves; ++w) {
        const float* p = reinterpret_cast<const float*>(s_own[w]);
        g += p[col * 17 + f];
        u += p[(16 + col) * 17 + f];
      }
      const int slot = s_slot[s0 + col];
      const float xs = a.xs[slot / a.k];
      a.act[(int64_t)slot * a.F + f0 + f] = swiglu1(g * xs, u * xs);
    }
    __syncthreads();
  }
}

// Down and the sum over a token's experts: 16 outputs of 16 tokens; the waves take the experts that these hit in turn.
constexpr int kDownWaves = 8;
template <typename T>
__global__ __launch_bounds__(kDownWaves * 64) void moe_down_kernel(MoeArgs a) {
  constexpr int OWN = own_bytes<1>();
  __shared__ __align__(16) char s_own[kDownWaves][OWN];
  __shared__ int s_ids[256];
  __shared__ float s_w[256];
  __shared__ unsigned int s_bits[32];
  __shared__ short s_list[256];
  __shared__ int s_n;
  static_assert(OWN >= 16 * 17 * 4, "the waves' sums fit their place");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t0 = blockIdx.y * 16, toks = min(a.T - t0, 16), n = toks * a.k;
  if (tid < 32) s_bits[tid] = 0u;
  __syncthreads();
  if (tid < n) {
    const int e = a.ids[t0 * a.k + tid];
    s_ids[tid] = e;
    s_w[tid] = a.w[t0 * a.k + tid] * a.sa[t0 * a.k + tid];
    atomicOr(&s_bits[e >> 5], 1u << (e & 31));
  }
  __syncthreads();
  for (int e = tid; e < a.E; e += kDownWaves * 64) {
    const unsigned int bits = s_bits[e >> 5];
    if (!((bits >> (e & 31)) & 1u)) continue;
    int at = __popc(bits & ((1u << (e & 31)) - 1u));
    for (int w = 0; w < (e >> 5); ++w) at += __popc(s_bits[w]);
    s_list[at] = (short)e;
  }
  if (tid == 0) {
    int c = 0;
    for (int w = 0; w < (a.E + 31) / 32; ++w) c += __popc(s_bits[w]);
    s_n = c;
  }
  __syncthreads();
  const int r0 = blockIdx.x * 16, c16 = lane & 15, hit = s_n;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int i = wave; i < hit; i += kDownWaves) {
    const int e = __builtin_amdgcn_readfirstlane((int)s_list[i]);
    int slot = -1, any = 0;
    for (int j = 0; j < a.k; ++j)
      if (c16 < toks && s_ids[c16 * a.k + j] == e) slot = c16 * a.k + j;
    const unsigned long long m = __ballot(slot >= 0);
    any = __shfl(slot, __builtin_ctzll(m), 64);      // (the other columns repeat one that is used)
    const float f = slot >= 0 ? s_w[slot] : 0.f;
    const Tile tile[1] = {tile_at(a.P2, a.A2, (int64_t)e * a.h + r0, a.F, a.shift)};
    f32x4 out[1] = {{0.f, 0.f, 0.f, 0.f}};
    rows_product<1>(tile, a.qa + (int64_t)(t0 * a.k + (slot >= 0 ? slot : any)) * a.F, 0, a.F >> 7, a.F, a.shift,
                    s_own[wave], out);
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] = slot >= 0 ? fmaf(f, out[0][j], sum[j]) : sum[j];
  }
  wait_lds();
  float* red = reinterpret_cast<float*>(s_own[wave]);
#pragma unroll
  for (int j = 0; j < 4; ++j) red[c16 * 17 + 4 * (lane >> 4) + j] = sum[j];
  __syncthreads();
  for (int i = tid; i < 16 * toks; i += kDownWaves * 64) {
    const int col = i >> 4, r = i & 15;
    const int64_t at = (int64_t)(t0 + col) * a.h + r0 + r;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kDownWaves; ++w) v += reinterpret_cast<const float*>(s_own[w])[col * 17 + r];
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
  size_t ids, w, sa, qa, act, end;
};
MoeSpace moe_space(const catq_moe_desc* d, int64_t T) {
  const size_t n = (size_t)T * d->top_k;
  MoeSpace s;
  s.ids = 0;
  s.w = round_up(n * 4, 256);
  s.sa = s.w + round_up(n * 4, 256);
  s.qa = s.sa + round_up(n * 4, 256);
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
            reinterpret_cast<float*>(ws + sp.sa), (int32_t)T, d->n_experts, d->top_k, d->hidden, d->ffn,
            __builtin_ctz((unsigned)d->group_size / 128)};
  const int n = (int)T * a.k, hit = n < a.E ? n : a.E;
  const double wt = (double)hit * a.h * a.F * (0.25 + 4.0 / d->group_size);
  auto experts = [&](auto kernel) {
    CATQ_TRACED(stream, "moe_experts_kernel", 0.0, 4.0 * T * a.E, T, a.E, a.k,
                hipLaunchKernelGGL(kernel, dim3((unsigned)((T + 3) / 4)), dim3(256), 0, stream, a));
  };
  if (a.E <= 64) experts(moe_experts_kernel<1>);
  else if (a.E <= 128) experts(moe_experts_kernel<2>);
  else if (a.E <= 256) experts(moe_experts_kernel<4>);
  else experts(moe_experts_kernel<16>);
  CATQ_TRACED(stream, "moe_up_kernel", 4.0 * n * a.h * a.F, 2.0 * wt, n, 2 * a.F, a.h,
              hipLaunchKernelGGL(moe_up_kernel, dim3((unsigned)(a.F / 16), (unsigned)hit), dim3(kUpWaves * 64), 0,
                                 stream, a));
  CATQ_CHECK_LAUNCH("moe gate and up");
  CATQ_TRY(catq_aux_act_quant8(a.act, CATQ_F32, n, a.F, a.F, a.qa, a.sa, stream));
  auto down = y_dtype == CATQ_F32 ? moe_down_kernel<float> : moe_down_kernel<bf16>;
  CATQ_TRACED(stream, "moe_down_kernel", 2.0 * n * a.h * a.F, wt, n, a.h, a.F,
              hipLaunchKernelGGL(down, dim3((unsigned)(a.h / 16), (unsigned)((T + 15) / 16)), dim3(kDownWaves * 64), 0,
                                 stream, a));
  CATQ_CHECK_LAUNCH("moe down");
  return CATQ_OK;
}
