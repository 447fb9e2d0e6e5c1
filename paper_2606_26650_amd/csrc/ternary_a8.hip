// Packed-ternary linear on 8-bit activations (gfx950): Y[m][n] = x_scale[m] *
// sum_j alpha[n][j] * sum_{k in group j} q[m][k] T[n][k], read straight from the 2-bit
// storage.  The products of a 128-code chunk are integers (v_mfma_i32_16x16x64_i8, sums
// below 127 * 128), converted to fp32 exactly and added with the chunk's scale.
//
// Codes to operands.  Word w of 16 codes (code i in bits 2i) gives four operand words:
// the codes j, 4 + j, 8 + j, 12 + j are the bytes of (w >> 2j) & 0x03030303, and one byte
// permute looks their values T up (0 -> -1, 1 -> 0, 2 -> 1, 3 -> 0): 11 instructions for
// 16 codes, where bf16 operands take 22.  The contraction order inside 16 values is thus
// 0 4 8 12 1 5 9 13 ..., and the activations are brought into the same order, a 4 x 4
// transposition of bytes.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kernels.h"

namespace catq {
namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(16))) int i32x16;

struct A8Args {
  const int8_t* X;
  const float* xs;
  int64_t ldx, M;
  const uint8_t* P;
  const float* A;
  int64_t d_out, d_in, ldy;
  int32_t n_chunks;   // d_in / 128
  int32_t cpg_shift;  // log2(g / 128)
  void* Y;
};

constexpr uint32_t kTernTab = 0x000100FFu;   // bytes by code: -1, 0, 1, 0

__device__ __forceinline__ u32x4 decode16_i8(uint32_t w) {
  u32x4 r;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    r[j] = __builtin_amdgcn_perm(0u, kTernTab, (w >> (2 * j)) & 0x03030303u);
  return r;
}

// 16 bytes x0 .. x15 -> words {x0 x4 x8 x12} {x1 x5 x9 x13} ...
__device__ __forceinline__ u32x4 transpose16(u32x4 x) {
  const uint32_t a = __builtin_amdgcn_perm(x[1], x[0], 0x05010400u);   // x0 x4 x1 x5
  const uint32_t b = __builtin_amdgcn_perm(x[1], x[0], 0x07030602u);   // x2 x6 x3 x7
  const uint32_t c = __builtin_amdgcn_perm(x[3], x[2], 0x05010400u);   // x8 x12 x9 x13
  const uint32_t d = __builtin_amdgcn_perm(x[3], x[2], 0x07030602u);
  u32x4 r;
  r[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
  r[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  r[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
  r[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
  return r;
}

__device__ __forceinline__ i32x4 mfma_i8(u32x4 a, u32x4 b, i32x4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c,
                                               0, 0, 0);
}

template <typename OutT>
__device__ __forceinline__ void store1(OutT* p, float v) {
  *p = (OutT)v;
}

// f(integral constant I) for I = 0 .. N-1, expanded at compile time
template <int I, int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    static_for<I + 1, N>(f);
  }
}

constexpr int kBufferFlags = 0x00020000;  // raw buffer resource word 3 (gfx9 family)
constexpr int kOutOfRange = 0x40000000;   // offset past every slice this kernel builds

// Few tokens.  One workgroup = R tiles of 16 output rows x NT tiles of 16 tokens; its NW
// waves take the 128-code chunks in turn and are added through LDS in a fixed order.  A
// code is decoded once for all token tiles, a token's activations are brought into order once
// for all row tiles.  A ring of D + 1 register slots keeps D chunks of every wave in flight;
// the scales are staged in LDS once, loaded before the ring's first chunks and stored
// after them.  XL (at most four tokens): the activations lie in LDS, in operand order.
// Dynamic LDS: groups * (RT + 4) floats, then with XL tokens * d_in bytes.
template <int NW, int R, int NT, int D, bool XL, typename OutT>
__global__ __launch_bounds__(NW * 64) void ternary_a8_gemv_kernel(A8Args a) {
  constexpr int RT = 16 * R, AP = RT + 4, S = D + 1, T = NW * 64, AMAX = 16;
  extern __shared__ __align__(16) float s_alpha[];
  __shared__ float s_red[NW][16][RT + 1];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int q = lane >> 4, c16 = lane & 15;
  const int64_t n0 = (int64_t)blockIdx.x * RT, m0 = (int64_t)blockIdx.y * (16 * NT);
  const int nch = a.n_chunks, ng = nch >> a.cpg_shift;
  const int64_t row_bytes = a.d_in >> 2;
  const int rows_here = (int)min<int64_t>(RT, a.d_out - n0);
  const int toks_here = (int)min<int64_t>(16 * NT, a.M - m0);

  // scales of the tile: index u T + tid = row * ng + group; past the tile zero
  const __amdgpu_buffer_rsrc_t ar = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<float*>(a.A + n0 * ng), 0, rows_here * ng * 4, kBufferFlags);
  float av[AMAX];
#pragma unroll
  for (int u = 0; u < AMAX; ++u)
    av[u] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(ar, (tid + T * u) * 4, 0, 0));
  u32x4* s_x = reinterpret_cast<u32x4*>(s_alpha + ng * AP);
  if constexpr (XL) {
    const int slots = nch * 8;   // 16-byte pieces per token
    for (int i = tid; i < toks_here * slots; i += T) {
      const int t = i / slots, sl = i - t * slots;
      s_x[i] = transpose16(*reinterpret_cast<const u32x4*>(a.X + (m0 + t) * a.ldx + sl * 16));
    }
  }
  const __amdgpu_buffer_rsrc_t pr = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint8_t*>(a.P + n0 * row_bytes), 0, (int)(rows_here * row_bytes), kBufferFlags);
  int poff[R];
#pragma unroll
  for (int r = 0; r < R; ++r)
    poff[r] = 16 * r + c16 < rows_here ? (int)((16 * r + c16) * row_bytes + 8 * q) : kOutOfRange;
  const int8_t* xp[NT];   // (a token past the last reads the last's: its results are not stored)
#pragma unroll
  for (int t = 0; t < NT; ++t) xp[t] = a.X + min(m0 + 16 * t + c16, a.M - 1) * a.ldx + 32 * q;

  const int my = wave < nch ? (nch - wave + NW - 1) / NW : 0;
  const int last = my > 0 ? wave + NW * (my - 1) : 0;
  uint2 cw[S][R];
  [[maybe_unused]] u32x4 xv[S][NT][2];
  auto issue = [&](int k, auto slot_c) __attribute__((always_inline)) {
    constexpr int s = decltype(slot_c)::value;
    const int ch = min(wave + NW * k, last);   // (past the end: re-read, never multiplied)
    if constexpr (!XL) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          xv[s][t][j] = *reinterpret_cast<const u32x4*>(xp[t] + (int64_t)ch * 128 + 16 * j);
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
      cw[s][r] = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(pr, poff[r], ch * 32, 0));
  };
  static_for<0, D>([&](auto I) {
    issue(I(), I);
    __builtin_amdgcn_sched_barrier(0);
  });
#pragma unroll
  for (int u = 0; u < AMAX; ++u) {
    const int idx = tid + T * u, r = idx / ng;
    if (r < RT) s_alpha[(idx - r * ng) * AP + r] = av[u];
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");

  f32x4 out[NT][R];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < R; ++r) out[t][r] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto compute = [&](int k, auto slot_c) __attribute__((always_inline)) {
    constexpr int i = decltype(slot_c)::value;
    const int ch = wave + NW * k;
    u32x4 xf[NT][2];
    if constexpr (XL) {
      const u32x4* p = s_x + (min(c16, toks_here - 1) * nch + ch) * 8 + 2 * q;
      xf[0][0] = p[0];
      xf[0][1] = p[1];
    } else {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < 2; ++j) xf[t][j] = transpose16(xv[i][t][j]);
    }
    const float* al = &s_alpha[(ch >> a.cpg_shift) * AP + 4 * q];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const u32x4 w0 = decode16_i8(cw[i][r].x), w1 = decode16_i8(cw[i][r].y);
      const f32x4 sc = *reinterpret_cast<const f32x4*>(al + 16 * r);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        i32x4 acc = {0, 0, 0, 0};
        acc = mfma_i8(w0, xf[t][0], acc);
        acc = mfma_i8(w1, xf[t][1], acc);
#pragma unroll
        for (int e = 0; e < 4; ++e) out[t][r][e] = fmaf(sc[e], (float)acc[e], out[t][r][e]);
      }
    }
  };
  const int full = my / S * S;
  for (int k0 = 0; k0 < full; k0 += S) {
    static_for<0, S>([&](auto I) {
      constexpr int i = I();
      issue(k0 + i + D, std::integral_constant<int, (i + D) % S>{});
      __builtin_amdgcn_sched_barrier(0);
      compute(k0 + i, I);
    });
  }
  static_for<0, S - 1>([&](auto I) {
    if (full + I() < my) compute(full + I(), I);
  });

#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (t > 0) __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int e = 0; e < 4; ++e) s_red[wave][c16][16 * r + 4 * q + e] = out[t][r][e];
    __syncthreads();
    for (int i = tid; i < 16 * RT; i += T) {
      const int tk = 16 * t + i / RT, r = i % RT;
      if (tk >= toks_here || r >= rows_here) continue;
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) sum += s_red[w][i / RT][r];
      store1(static_cast<OutT*>(a.Y) + (m0 + tk) * a.ldy + n0 + r, sum * a.xs[m0 + tk]);
    }
  }
}

// Many tokens.  One workgroup = 32 NWV weight rows x 32 CB tokens (128 x 64); each of its NWV
// waves takes 32 rows and all the tokens, so a code is decoded once per workgroup.  Per 128-code
// chunk the tokens' activations go through registers (where they are brought into operand order;
// loaded two chunks ahead) into a double-buffered LDS tile [token][8 slots of 16 bytes], slot s of
// token t at s ^ ((t >> 1) & 7): 16 lanes then read 16 different 16-byte banks.  The codes come
// two chunks of a row (64 bytes) at a time by direct copies into a tile of the same kind, and the
// scales eight groups of a row at a time: read where they are used, 32 bytes and 4 bytes a row and
// chunk, they took most of the L1's accesses (1265 per workgroup and chunk; 315 -> 286 us at 1000
// tokens x 34816 x 5120 once they came in whole pieces).  Lane half h takes the
// chunk's values 64 h .. 64 h + 63, in four contraction steps of v_mfma_i32_32x32x32_i8.  The sums of
// a chunk are converted and added with the rows' scales; with larger groups only once a group.
//
// 1000 x 34816 x 5120: 284 us, 1.26 PFLOP/s.  What bounds it is the sum of what one compute
// unit does per chunk: the LDS reads of the operands (50% of its bandwidth), 37% of the vector
// issue (decode, conversion, scaling) and 21% of the matrix cores, four waves per SIMD overlapping
// them; leaving out any one of them gains 5-15%, the activations' staging 18%.
template <int NWV, int CB, bool G128, typename OutT>
__global__ __launch_bounds__(NWV * 64, 4) void ternary_a8_gemm_kernel(A8Args a) {
  constexpr int T = NWV * 64, RT = 32 * NWV, TT = 32 * CB;
  constexpr int NX = TT * 8 / T;      // 16-byte pieces of a chunk per thread
  static_assert(NX >= 1 && TT * 8 % T == 0, "whole pieces per thread");
  __shared__ __align__(16) u32x4 s_x[2][TT * 8];
  __shared__ __align__(16) u32x4 s_w[2][RT * 4];
  __shared__ __align__(16) float s_al[2][8][RT];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, l32 = lane & 31;
  const int64_t n0 = (int64_t)blockIdx.x * RT, m0 = (int64_t)blockIdx.y * TT;
  const int nch = a.n_chunks, ng = nch >> a.cpg_shift, cpg_mask = (1 << a.cpg_shift) - 1;
  const int64_t row_bytes = a.d_in >> 2;
  const int rows_here = (int)min<int64_t>(RT, a.d_out - n0);
  const int toks_here = (int)min<int64_t>(TT, a.M - m0);

  const int8_t* xg[NX];
  int xs[NX];
#pragma unroll
  for (int i = 0; i < NX; ++i) {
    const int p = tid + T * i, t = p >> 3, sl = p & 7;
    xg[i] = a.X + (m0 + min(t, toks_here - 1)) * a.ldx + sl * 16;
    xs[i] = t * 8 + (sl ^ ((t >> 1) & 7));
  }
  // codes: instruction i of a wave copies rows 32 wave + 16 i .. + 15, lane's row lane / 4
  const i32x4_rsrc wr = buf_rsrc(a.P + n0 * row_bytes, (uint32_t)(rows_here * row_bytes));
  uint32_t woff[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = 32 * wave + 16 * i + (lane >> 2);
    woff[i] = (uint32_t)(r * row_bytes) + (uint32_t)(((lane & 3) ^ ((r >> 2) & 3)) * 16);
  }
  const uint32_t wlds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) u32x4*)&s_w[0][0];
  // scales: piece p = tid: row p / 2, groups 4 (p % 2) .. + 3 of eight
  const __amdgpu_buffer_rsrc_t ar = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<float*>(a.A + n0 * ng), 0, rows_here * ng * 4, kBufferFlags);

  u32x4 xn[2][NX];   // chunk c in slot c & 1, two chunks ahead
  f32x4 an;
  auto fetch_x = [&](int chunk, auto slot_c) __attribute__((always_inline)) {
    constexpr int sl = decltype(slot_c)::value;
    const int c = min(chunk, nch - 1);    // (past the end: re-read, never used)
#pragma unroll
    for (int i = 0; i < NX; ++i) xn[sl][i] = *reinterpret_cast<const u32x4*>(xg[i] + (int64_t)c * 128);
  };
  auto copy_w = [&](int chunk, int buf) __attribute__((always_inline)) {   // (past a row's end: the next row, or zeros; never used)
#pragma unroll
    for (int i = 0; i < 2; ++i)
      dma16_lds(wr, woff[i] + (uint32_t)chunk * 32u, 0u,
                wlds + (uint32_t)(buf * RT * 4 + (32 * wave + 16 * i) * 4) * 16u);
  };
  auto fetch_a = [&](int group) __attribute__((always_inline)) {
    an = __builtin_bit_cast(
        f32x4, __builtin_amdgcn_raw_buffer_load_b128(ar, ((tid >> 1) * ng + 4 * (tid & 1) + group) * 4, 0, 0));
  };
  auto stage_x = [&](auto slot_c) __attribute__((always_inline)) {
    constexpr int sl = decltype(slot_c)::value;   // (its slot is its LDS buffer)
#pragma unroll
    for (int i = 0; i < NX; ++i) s_x[sl][xs[i]] = transpose16(xn[sl][i]);
  };
  auto stage_a = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 4; ++e) s_al[buf][4 * (tid & 1) + e][tid >> 1] = an[e];
  };
  const int amask = (8 << a.cpg_shift) - 1;   // chunks of 8 groups, less one
  copy_w(0, 0);
  fetch_a(0);
  using S0 = std::integral_constant<int, 0>;
  using S1 = std::integral_constant<int, 1>;
  fetch_x(0, S0());
  fetch_x(1, S1());
  stage_x(S0());
  stage_a(0);
  wait_vmem();
  __syncthreads();
  f32x16 out[CB];
  i32x16 acc[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      out[cb][r] = 0.f;
      acc[cb][r] = 0;
    }
  auto step = [&](int c, auto par_c) __attribute__((always_inline)) {
    constexpr int par = decltype(par_c)::value;   // c & 1
    const int gi = c >> a.cpg_shift;
    if (par == 0) {
      if ((c & amask) == 0) fetch_a(gi + 8);
      if (c + 2 < nch) copy_w(c + 2, ((c >> 1) & 1) ^ 1);
    }
    fetch_x(c + 2, par_c);
    const u32x4* xt = s_x[par];
    const u32x4 cw = s_w[(c >> 1) & 1][(32 * wave + l32) * 4 + ((2 * par + h) ^ ((l32 >> 2) & 3))];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const i32x4 w = __builtin_bit_cast(i32x4, decode16_i8(cw[s]));
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        const int t = 32 * cb + l32;
        const i32x4 x = __builtin_bit_cast(i32x4, xt[t * 8 + ((4 * h + s) ^ ((t >> 1) & 7))]);
        acc[cb] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w, x, G128 && s == 0 ? i32x16{} : acc[cb], 0, 0, 0);
      }
    }
    if (G128 || (c & cpg_mask) == cpg_mask) {
#pragma unroll
      for (int qd = 0; qd < 4; ++qd) {   // register r: row 8 (r / 4) + 4 h + r % 4
        const f32x4 sc = *reinterpret_cast<const f32x4*>(&s_al[(gi >> 3) & 1][gi & 7][32 * wave + 8 * qd + 4 * h]);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            out[cb][4 * qd + e] = fmaf(sc[e], (float)acc[cb][4 * qd + e], out[cb][4 * qd + e]);
            if (!G128) acc[cb][4 * qd + e] = 0;
          }
      }
      // (here: the two steps would otherwise leave their sums to the end)
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) asm volatile("" : "+v"(out[cb]));
    }
    stage_x(std::integral_constant<int, par ^ 1>());
    if (par == 1) {
      if ((c & amask) == amask) stage_a(((gi >> 3) & 1) ^ 1);
      // the codes of the next two chunks: older than the activations of chunks c + 1 and c + 2
      wait_vmem_n<NX>();
    }
    __syncthreads();
  };
  int c = 0;
  for (; c + 1 < nch; c += 2) {
    step(c, S0());
    step(c + 1, S1());
  }
  if (c < nch) step(c, S0());
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    const int tok = 32 * cb + l32;
    if (tok >= toks_here) continue;
    OutT* y = static_cast<OutT*>(a.Y) + (m0 + tok) * a.ldy + n0;
    const float xsc = a.xs[m0 + tok];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = 32 * wave + 8 * (r >> 2) + 4 * h + (r & 3);
      if (row < rows_here) store1(y + row, out[cb][r] * xsc);
    }
  }
}

template <typename T>
struct OutTag {
  using type = T;
};

struct A8Work {
  double flops, bytes;
};

template <int NW, int R, int NT, int D>
catq_status launch_gemv(const A8Args& a, catq_dtype y_dtype, const A8Work& w, hipStream_t stream) {
  constexpr int RT = 16 * R;
  const int ng = a.n_chunks >> a.cpg_shift;
  const dim3 grid((unsigned)((a.d_out + RT - 1) / RT), (unsigned)((a.M + 16 * NT - 1) / (16 * NT)));
  size_t lds = (size_t)ng * (RT + 4) * sizeof(float);
  // every scale of a tile has a register, and the LDS stays within 64 KB
  CATQ_REQUIRE(ng * RT <= 16 * NW * 64 && lds + sizeof(float) * NW * 16 * (RT + 1) <= 65536, CATQ_ERR_SHAPE,
               "ternary_linear_a8: no launch shape for d_in = %lld", (long long)a.d_in);
  const size_t lds_x = (size_t)a.M * (size_t)a.d_in;
  const bool xl = NT == 1 && a.M <= 4 && lds + lds_x + sizeof(float) * NW * 16 * (RT + 1) <= 65536;
  if (xl) lds += lds_x;
  static char tag[64];
  trace_tag(tag, sizeof tag, "ternary_a8_gemv_kernel<%d, %d, %d%s>", NW, R, NT, xl ? ", x in lds" : "");
  auto launch = [&](auto xl_c, auto out_c) {
    using OutT = typename decltype(out_c)::type;
    CATQ_TRACED(stream, tag, w.flops, w.bytes, a.M, a.d_out, a.d_in,
                hipLaunchKernelGGL((ternary_a8_gemv_kernel<NW, R, NT, D, decltype(xl_c)::value, OutT>), grid,
                                   dim3(NW * 64), lds, stream, a));
  };
  auto with = [&](auto out_c) {
    if constexpr (NT == 1) {
      if (xl) return launch(std::true_type{}, out_c);
    }
    launch(std::false_type{}, out_c);
  };
  if (y_dtype == CATQ_F32) with(OutTag<float>{});
  else with(OutTag<bf16>{});
  CATQ_CHECK_LAUNCH("ternary_linear_a8");
  return CATQ_OK;
}

template <int NWV, int CB>
catq_status launch_gemm(const A8Args& a, catq_dtype y_dtype, const A8Work& w, hipStream_t stream) {
  const dim3 grid((unsigned)((a.d_out + 32 * NWV - 1) / (32 * NWV)), (unsigned)((a.M + 32 * CB - 1) / (32 * CB)));
  static char tag[64];
  trace_tag(tag, sizeof tag, "ternary_a8_gemm_kernel<%d, %d>", NWV, CB);
  auto launch = [&](auto g128, auto out_c) {
    using OutT = typename decltype(out_c)::type;
    CATQ_TRACED(stream, tag, w.flops, w.bytes, a.M, a.d_out, a.d_in,
                hipLaunchKernelGGL((ternary_a8_gemm_kernel<NWV, CB, decltype(g128)::value, OutT>), grid,
                                   dim3(NWV * 64), 0, stream, a));
  };
  auto with = [&](auto out_c) {
    if (a.cpg_shift == 0) launch(std::true_type{}, out_c);
    else launch(std::false_type{}, out_c);
  };
  if (y_dtype == CATQ_F32) with(OutTag<float>{});
  else with(OutTag<bf16>{});
  CATQ_CHECK_LAUNCH("ternary_linear_a8");
  return CATQ_OK;
}

}  // namespace
}  // namespace catq

extern "C" catq_status catq_ternary_linear_a8(const int8_t* q, int64_t M, int64_t ldq,
                                              const float* x_scale, const uint8_t* packed,
                                              const float* alpha, int64_t d_out, int64_t d_in,
                                              int32_t g, void* Y, catq_dtype y_dtype, int64_t ldy,
                                              hipStream_t stream) {
  using namespace catq;
  clear_error();
  CATQ_REQUIRE(M >= 0, CATQ_ERR_SHAPE, "M must be >= 0");
  if (M == 0) return CATQ_OK;
  CATQ_REQUIRE(q && x_scale && packed && alpha && Y, CATQ_ERR_NULL,
               "q, x_scale, packed, alpha and Y must not be NULL");
  CATQ_REQUIRE(count_ok(d_out, d_in), CATQ_ERR_SHAPE,
               "d_out and d_in must be > 0 with d_out*d_in <= 2^38");
  CATQ_REQUIRE(g >= 128 && g % 128 == 0 && ((g / 128) & (g / 128 - 1)) == 0, CATQ_ERR_VALUE,
               "g must be 128 times a power of two");
  CATQ_REQUIRE(d_in % g == 0, CATQ_ERR_SHAPE, "d_in (%lld) must be a multiple of g (%d)",
               (long long)d_in, g);
  CATQ_REQUIRE(d_in <= 65536, CATQ_ERR_SHAPE, "d_in must be <= 65536");
  // (a launch has fewer than 2^32 threads along x: 512 per 16 rows at least)
  CATQ_REQUIRE((d_out + 15) / 16 < (1 << 23) && (M + 15) / 16 <= 65535, CATQ_ERR_SHAPE,
               "d_out or M too large for one launch");
  CATQ_REQUIRE(ldq >= d_in && ldq % 16 == 0 && ldq <= (1 << 24), CATQ_ERR_SHAPE,
               "ldq must be >= d_in, a multiple of 16 and <= 2^24");
  CATQ_REQUIRE(ldy >= d_out, CATQ_ERR_SHAPE, "ldy must be >= d_out");
  CATQ_REQUIRE(y_dtype == CATQ_F32 || y_dtype == CATQ_BF16, CATQ_ERR_DTYPE, "Y must be fp32 or bf16");
  CATQ_REQUIRE(aligned16(q) && aligned16(alpha) && (reinterpret_cast<uintptr_t>(packed) & 7) == 0 &&
                   (reinterpret_cast<uintptr_t>(Y) & 3) == 0 && (reinterpret_cast<uintptr_t>(x_scale) & 3) == 0,
               CATQ_ERR_ALIGN, "q and alpha must be 16-byte aligned, packed 8-byte, x_scale and Y 4-byte");
  const A8Args a{q, x_scale, ldq, M, packed, alpha, d_out, d_in, ldy, (int32_t)(d_in / 128),
                 (int32_t)__builtin_ctz((unsigned)(g / 128)), Y};
  const A8Work w{2.0 * (double)M * (double)d_out * (double)d_in,
                 (double)d_out * (double)d_in / 4.0 + 4.0 * (double)d_out * (double)(d_in / g) +
                     (double)M * (double)d_in + (double)M * (double)d_out * (double)dtype_size(y_dtype)};
  // Which kernel: the least of a cost model in microseconds, fitted on MI355X.  A workgroup of
  // the kernel for few tokens takes as long per eight chunks as the table says
  // (rows and tokens in tiles of 16; at most four tokens lie in LDS), a compute unit takes
  // its workgroups one after the other, and a launch costs 3.  The tiled kernel's workgroups (128
  // rows x 64 tokens) take 0.42 per chunk, a lone one 0.72.  34816 x 5120: R = 3 at one
  // token (14.7 us; 19.8 for R = 2), 16 (21.4; 34.5) and 32 (28.3 for 32 tokens at once; 39.3 for 16),
  // tiled from 48 (38.4; 43.9).  5120 x 17408: R = 2 to 16 tokens (11.8, 18.9), R = 3 on 32 tokens
  // at once at 48 (30.4; 33.1 for R = 2 on 48), on 64 at 100 (46.9; tiled 85.9).
  const int ng = a.n_chunks >> a.cpg_shift;
  if (ng > 256) return launch_gemv<8, 1, 1, 3>(a, y_dtype, w, stream);   // (scales: one per thread register)
  const bool few = M <= 4;
  const double t21 = few ? 0.60 : 0.95, t31 = few ? 0.78 : 1.2;
  auto gemv = [&](int r, int nt, double t) {
    const double wgs = std::ceil((double)d_out / (16 * r)) * std::ceil((double)M / (16 * nt));
    return r == 3 && ng > 170 ? 1e300 : 3.0 + a.n_chunks / 8.0 * std::ceil(wgs / 256.0) * t;
  };
  const double cost[6] = {gemv(2, 1, t21), gemv(3, 1, t31), gemv(2, 2, 1.31), gemv(3, 2, 1.65), gemv(3, 4, 2.7),
                          4.0 + a.n_chunks * std::max(0.72, 0.42 * std::ceil(std::ceil(d_out / 128.0) *
                                                                             std::ceil(M / 64.0) / 256.0))};
  switch (std::min_element(cost, cost + 6) - cost) {
    case 0: return launch_gemv<8, 2, 1, 3>(a, y_dtype, w, stream);
    case 1: return launch_gemv<8, 3, 1, 2>(a, y_dtype, w, stream);
    case 2: return launch_gemv<8, 2, 2, 2>(a, y_dtype, w, stream);
    case 3: return launch_gemv<8, 3, 2, 1>(a, y_dtype, w, stream);
    case 4: return launch_gemv<8, 3, 4, 1>(a, y_dtype, w, stream);
    default: return launch_gemm<4, 2>(a, y_dtype, w, stream);
  }
}
