// Packed-ternary linear on 8-bit activations (gfx950): Y[m][n] = x_scale[m] *
// sum_j alpha[n][j] * sum_{k in group j} q[m][k] T[n][k], read straight from the 2-bit
// storage.  The products of a 128-code chunk are integers (v_mfma_i32_16x16x64_i8, sums
// below 127 * 128), converted to fp32 exactly and added with the chunk's scale.
// The operands are those of ternary8.h.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kernels.h"
#include "ternary8.h"

namespace catq {
namespace {

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

// Few tokens.  One workgroup = R tiles of 16 output rows x NT tiles of 16 tokens; each of its NW
// waves takes a run of 128-code chunks, and they are added through LDS in a fixed order.  A code is
// decoded once for all token tiles, a token's activations are brought into order once for all row
// tiles.  Codes (two chunks at a time) and activations come by direct copies into LDS of each
// wave's own (no barriers); their operands are read at once, and the next copies are issued into
// the same place before the products.  A matrix operand has 16 neighbouring lanes in
// 16 different rows, and loading it so, straight into registers, cost the L1 64 cycles an
// instruction whatever its width; a copy's neighbouring lanes take 64 bytes of a row of codes, 128 of
// a token, and LDS does the exchange (5120 x 17408: 19.0 -> 13 us at 16 tokens, 30.3 -> 18.4 at 48).
// Within a row the 16-byte pieces are permuted, so that the operands' reads use all banks.
//   codes of a row tile  [16 rows][4 pieces], piece p of row t at p ^ (t / 4)
//   activations          [16 NT tokens][8 pieces], piece p of token t at p ^ (t / 2 % 8)
// XL (at most four tokens): the activations lie in LDS as a whole, in operand order.
//
// What bounds it: at one token (34816 x 5120: 13.2 us) the codes, 10.5 us from HBM, behind 3 of
// launch and first loads; with more the vector instructions (per chunk 16 a token tile, 22 a row tile,
// 8 a pair of them: 7 of the 18 us at 48 tokens x 5120 x 17408 if all units had the same
// share, but its 160 workgroups leave 96 of 256 idle).  A ring of two or three slots brought nothing,
// and its LDS costs workgroups per unit (34816 x 5120 at 16: 20.3 us with two, 18.4 with one).
// Dynamic LDS: groups * (RT + 4) floats, then with XL tokens * d_in bytes.
template <int NW, int R, int NT, bool XL, typename OutT>
__global__ __launch_bounds__(NW * 64) void ternary_a8_gemv_kernel(A8Args a) {
  constexpr int RT = 16 * R, AP = RT + 4, T = NW * 64, AMAX = 128 / NW;
  constexpr int WB = R * 1024, OWN = WB + (XL ? 0 : NT * 2048), RED = NW * 16 * (RT + 1) * 4;   // bytes
  __shared__ __align__(16) char s_own[NW * OWN > RED ? NW * OWN : RED];
  extern __shared__ __align__(16) float s_alpha[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int q = lane >> 4, c16 = lane & 15;
  const int64_t n0 = (int64_t)blockIdx.x * RT, m0 = (int64_t)blockIdx.y * (16 * NT);
  const int nch = a.n_chunks, ng = nch >> a.cpg_shift;
  const int64_t row_bytes = a.d_in >> 2;
  const int rows_here = (int)min<int64_t>(RT, a.d_out - n0);
  const int toks_here = (int)min<int64_t>(16 * NT, a.M - m0);
  const int ch0 = wave * nch / NW, my = (wave + 1) * nch / NW - ch0;

  // codes: a lane copies to piece lane % 4 of row lane / 4 of a tile; past the tile zeros
  const i32x4_rsrc wr = buf_rsrc(a.P + n0 * row_bytes, (uint32_t)(rows_here * row_bytes));
  uint32_t woff[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = 16 * r + (lane >> 2);
    woff[r] = row < rows_here ? (uint32_t)(row * row_bytes) + ((lane & 3) ^ (lane >> 4)) * 16 + ch0 * 32 : kOutOfRange;
  }
  // activations: to piece lane % 8 of token lane / 8 of eight; past the last token zeros
  const i32x4_rsrc xr = buf_rsrc(a.X + m0 * a.ldx, (uint32_t)((toks_here - 1) * a.ldx + a.d_in));
  uint32_t xoff[2 * NT];
#pragma unroll
  for (int i = 0; i < 2 * NT; ++i) {
    const int t = 8 * i + (lane >> 3);
    xoff[i] = t < toks_here ? (uint32_t)(t * a.ldx) + ((lane & 7) ^ ((t >> 1) & 7)) * 16 : kOutOfRange;
  }
  const char* own = s_own + wave * OWN;
  const uint32_t olds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)s_own + wave * OWN;
  auto copy_w = [&](int k) __attribute__((always_inline)) {   // (past a row's end: the next row, or zeros; never used)
#pragma unroll
    for (int r = 0; r < R; ++r) dma16_lds(wr, woff[r] + (uint32_t)k * 32u, 0u, olds + r * 1024);
  };
  auto copy_x = [&](int k) __attribute__((always_inline)) {
    if constexpr (!XL) {
      const uint32_t ch = min(ch0 + k, nch - 1);   // (past the end: re-read, never used)
#pragma unroll
      for (int i = 0; i < 2 * NT; ++i) dma16_lds(xr, xoff[i] + ch * 128u, 0u, olds + WB + i * 1024);
    }
  };
  copy_w(0);
  copy_x(0);

  // scales of the tile: index u T + tid = row * ng + group; past the tile zero
  const __amdgpu_buffer_rsrc_t ar = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<float*>(a.A + n0 * ng), 0, rows_here * ng * 4, kBufferFlags);
  float av[AMAX];
#pragma unroll
  for (int u = 0; u < AMAX; ++u)
    if (T * u < RT * ng)
      av[u] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(ar, (tid + T * u) * 4, 0, 0));
  u32x4* s_x = reinterpret_cast<u32x4*>(s_alpha + ng * AP);
  if constexpr (XL) {
    const int slots = nch * 8;   // 16-byte pieces per token
    for (int i = tid; i < toks_here * slots; i += T) {
      const int t = (i >= slots) + (i >= 2 * slots) + (i >= 3 * slots), sl = i - t * slots;
      s_x[i] = transpose16(*reinterpret_cast<const u32x4*>(a.X + (m0 + t) * a.ldx + sl * 16));
    }
  }
  // (the division in fp32: a quotient of at most 8192 / ng is a half / ng or more from an integer.  As an
  // integer division, and for all of AMAX, this took 3 us)
  const float inv_ng = 1.0f / (float)ng;
#pragma unroll
  for (int u = 0; u < AMAX; ++u) {
    if (T * u >= RT * ng) break;
    const int idx = tid + T * u, r = (int)(((float)idx + 0.5f) * inv_ng);
    if (r < RT) s_alpha[(idx - r * ng) * AP + r] = av[u];
  }
  wait_vmem();
  __syncthreads();

  f32x4 out[NT][R];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < R; ++r) out[t][r] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int wrd = c16 * 64 + 8 * (q & 1), wsw = c16 >> 2;
  const int xrd = WB + c16 * 128, xsw = (c16 >> 1) & 7;
  uint2 cw[2][R];
  auto step = [&](int k, auto par_c) __attribute__((always_inline)) {
    constexpr int par = decltype(par_c)::value;   // k & 1
    const int ch = ch0 + k;
    // (in order of their issue: activations of k, then with odd k the codes of k + 1 and k + 2)
    if constexpr (par == 0) wait_vmem();
    else if constexpr (!XL) wait_vmem_n<R>();
    if constexpr (par == 0) {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int p = 0; p < 2; ++p)
          cw[p][r] = *reinterpret_cast<const uint2*>(own + r * 1024 + wrd + ((2 * p + (q >> 1)) ^ wsw) * 16);
    }
    u32x4 xf[NT][2];
    if constexpr (XL) {
      const u32x4* p = s_x + (min(c16, toks_here - 1) * nch + ch) * 8 + 2 * q;
      xf[0][0] = p[0];
      xf[0][1] = p[1];
    } else {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          xf[t][j] = *reinterpret_cast<const u32x4*>(own + t * 2048 + xrd + ((2 * q + j) ^ xsw) * 16);
    }
    const float* al = &s_alpha[(ch >> a.cpg_shift) * AP + 4 * q];
    f32x4 sc[R];
#pragma unroll
    for (int r = 0; r < R; ++r) sc[r] = *reinterpret_cast<const f32x4*>(al + 16 * r);
    if (!XL || par == 0) wait_lds();   // what was read may be written over
    copy_x(k + 1);
    if constexpr (par == 0) copy_w(k + 2);
    if constexpr (!XL) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < 2; ++j) xf[t][j] = transpose16(xf[t][j]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const u32x4 w0 = decode16_i8(cw[par][r].x), w1 = decode16_i8(cw[par][r].y);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        i32x4 acc = {0, 0, 0, 0};
        acc = mfma_i8(w0, xf[t][0], acc);
        acc = mfma_i8(w1, xf[t][1], acc);
#pragma unroll
        for (int e = 0; e < 4; ++e) out[t][r][e] = fmaf(sc[r][e], (float)acc[e], out[t][r][e]);
      }
    }
  };
  for (int k = 0; k < my; k += 2) {
    step(k, std::integral_constant<int, 0>{});
    if (k + 1 < my) step(k + 1, std::integral_constant<int, 1>{});
  }
  wait_vmem();     // (the last copies, never read: their place takes the sums)
  __syncthreads();

  auto s_red = reinterpret_cast<float (*)[16][RT + 1]>(s_own);
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

// Many tokens.  One workgroup = 32 NWV weight rows x 32 CB tokens (128 or 256 x 64); each of its NWV
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
// 1000 x 34816 x 5120 with eight waves: 275 us, 1.3 PFLOP/s, at a clock of 1.9 GHz.  What bounds it is the
// vector instructions: 136 per wave and chunk (64 convert and scale the sums, 44 decode, 8 bring
// activations into order; 145 with four waves, 16 of them for the order) take 65% of the issue cycles (72% with
// four), beside matrix cores at 30% and the LDS reads of the operands at half of its bandwidth, four waves per SIMD
// overlapping them.  With four waves, leaving out any one of them gained 5-15%, the activations' staging 18%.
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

// LDS of a unit; a launch's scales, the waves' own places (or the reduction's)
constexpr size_t kLds = 160 * 1024;
template <int NW, int R, int NT>
constexpr size_t gemv_lds(int ng, bool xl) {
  const size_t own = NW * 1024 * (R + (xl ? 0 : 2 * NT)), red = sizeof(float) * NW * 16 * (16 * R + 1);
  return (size_t)ng * (16 * R + 4) * sizeof(float) + std::max(own, red);
}
// every scale of a tile has a register of some thread, and the LDS suffices
template <int NW, int R, int NT>
constexpr bool gemv_fits(int ng) {
  return ng * 16 * R <= 8192 && gemv_lds<NW, R, NT>(ng, false) <= kLds;
}

template <int NW, int R, int NT>
catq_status launch_gemv(const A8Args& a, catq_dtype y_dtype, const A8Work& w, hipStream_t stream) {
  constexpr int RT = 16 * R;
  const int ng = a.n_chunks >> a.cpg_shift;
  const dim3 grid((unsigned)((a.d_out + RT - 1) / RT), (unsigned)((a.M + 16 * NT - 1) / (16 * NT)));
  size_t lds = (size_t)ng * (RT + 4) * sizeof(float);   // (dynamic; the rest is static)
  const size_t lds_x = (size_t)a.M * (size_t)a.d_in;
  const bool xl = NT == 1 && a.M <= 4 && gemv_lds<NW, R, NT>(ng, true) + lds_x <= kLds;
  if (xl) lds += lds_x;
  char tag[64];
  trace_tag(tag, sizeof tag, "ternary_a8_gemv_kernel<%d, %d, %d%s>", NW, R, NT, xl ? ", x in lds" : "");
  auto launch = [&](auto xl_c, auto out_c) {
    using OutT = typename decltype(out_c)::type;
    CATQ_TRACED(stream, tag, w.flops, w.bytes, a.M, a.d_out, a.d_in,
                hipLaunchKernelGGL((ternary_a8_gemv_kernel<NW, R, NT, decltype(xl_c)::value, OutT>), grid,
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
  char tag[64];
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
  // Which kernel: the least of a cost model in microseconds, fitted on MI355X over 56 sizes (1024 x 5120
  // to 100000 x 2048, one token to 100; its choice is 3% behind the best of 15 on average, 14% at
  // worst).  It is fitted for the choice: the times themselves are too long where a last round of
  // workgroups is nearly empty (5120 x 17408 at one token: 14.4, measured 9.1).  A launch costs base;
  // then per chunk a workgroup alone on its compute unit takes alone, and several of them each
  // apiece.  Measured with the fit, 5120 x 17408: R = 1 at one token (9.1 us; 13.7 for R = 2), R = 2
  // with three token tiles at 48 (19.9, 18.4 as the kernel is now; 21.3 with one, 24.6 with two).  34816 x 5120: R = 2 on four waves at one
  // token (13.3; 14.4 for R = 1), R = 3 on four waves with two token tiles at 48 (32.2; tiled 38.2), tiled from 64.
  // 8192 x 8192 at 16: R = 1 (8.4; 9.9 for R = 2 with two token tiles).
  const int ng = a.n_chunks >> a.cpg_shift;
  struct Choice {
    int rows, tokens;
    double base, alone, each;
    bool fits;
  };
  const Choice choices[6] = {{16, 16, 3.2, 0.049, 0.041, gemv_fits<8, 1, 1>(ng)},
                             {32, 16, 3.2, 0.091, 0.060, gemv_fits<4, 2, 1>(ng)},
                             {32, 32, 3.3, 0.094, 0.100, gemv_fits<8, 2, 2>(ng)},
                             {32, 48, 3.8, 0.115, 0.131, gemv_fits<8, 2, 3>(ng)},
                             {48, 32, 4.0, 0.148, 0.122, gemv_fits<4, 3, 2>(ng)},
                             {128, 64, 5.7, 0.58, 0.39, true}};
  int best = 5;
  double least = 1e300;
  for (int i = 0; i < 6; ++i) {
    const Choice& c = choices[i];
    if (!c.fits) continue;
    const double wgs = std::ceil((double)d_out / c.rows) * std::ceil((double)M / c.tokens);
    const double cost = c.base + a.n_chunks * (wgs <= 256 ? c.alone : c.each * std::ceil(wgs / 256.0));
    if (cost < least) {
      least = cost;
      best = i;
    }
  }
  switch (best) {
    case 0: return launch_gemv<8, 1, 1>(a, y_dtype, w, stream);
    case 1: return launch_gemv<4, 2, 1>(a, y_dtype, w, stream);
    case 2: return launch_gemv<8, 2, 2>(a, y_dtype, w, stream);
    case 3: return launch_gemv<8, 2, 3>(a, y_dtype, w, stream);
    case 4: return launch_gemv<4, 3, 2>(a, y_dtype, w, stream);
    default:
      // Eight waves share the activations of a tile where 1024 workgroups or more are left, four to a
      // unit (1000 x 34816 x 5120: 275 us, 288 with four waves; 4000 x 5120 x 5120: 163, 170; but 1000 x 5120
      // x 17408, 320 workgroups: 170, 157).
      if (std::ceil(d_out / 256.0) * std::ceil(M / 64.0) >= 1024) return launch_gemm<8, 2>(a, y_dtype, w, stream);
      return launch_gemm<4, 2>(a, y_dtype, w, stream);
  }
}
