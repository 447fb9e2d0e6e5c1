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
#include <type_traits>

#include "kernels.h"

namespace catq {
namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4;

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

// One workgroup = R tiles of 16 rows x up to 16 tokens; its NW waves take the 128-code
// chunks in turn and are added through LDS in a fixed order.
template <int NW, int R, typename OutT>
__global__ __launch_bounds__(NW * 64) void ternary_a8_gemv_kernel(A8Args a) {
  constexpr int RT = 16 * R;
  __shared__ float s_red[NW][16][RT + 1];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int q = lane >> 4, c16 = lane & 15;
  const int64_t n0 = (int64_t)blockIdx.x * RT, m0 = (int64_t)blockIdx.y * 16;
  const int64_t row_bytes = a.d_in >> 2;
  const int ng = a.n_chunks >> a.cpg_shift;
  const int64_t tok = m0 + c16;
  const bool live = tok < a.M;
  const int8_t* xp = a.X + (live ? tok : a.M - 1) * a.ldx + 32 * q;
  const uint8_t* pp[R];
#pragma unroll
  for (int r = 0; r < R; ++r) pp[r] = a.P + min(n0 + 16 * r + c16, a.d_out - 1) * row_bytes + 8 * q;
  float out[R][4];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int e = 0; e < 4; ++e) out[r][e] = 0.f;
  for (int ch = wave; ch < a.n_chunks; ch += NW) {
    const u32x4 x0 = transpose16(*reinterpret_cast<const u32x4*>(xp + ch * 128));
    const u32x4 x1 = transpose16(*reinterpret_cast<const u32x4*>(xp + ch * 128 + 16));
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint2 w = *reinterpret_cast<const uint2*>(pp[r] + ch * 32);
      i32x4 acc = {0, 0, 0, 0};
      acc = mfma_i8(decode16_i8(w.x), x0, acc);
      acc = mfma_i8(decode16_i8(w.y), x1, acc);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int64_t row = min(n0 + 16 * r + 4 * q + e, a.d_out - 1);
        out[r][e] = fmaf(a.A[row * ng + (ch >> a.cpg_shift)], (float)acc[e], out[r][e]);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int e = 0; e < 4; ++e) s_red[wave][c16][16 * r + 4 * q + e] = out[r][e];
  __syncthreads();
  for (int i = tid; i < 16 * RT; i += NW * 64) {
    const int t = i / RT, r = i % RT;
    if (m0 + t >= a.M || n0 + r >= a.d_out) continue;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) sum += s_red[w][t][r];
    store1(static_cast<OutT*>(a.Y) + (m0 + t) * a.ldy + n0 + r, sum * a.xs[m0 + t]);
  }
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
  CATQ_REQUIRE((d_out + 15) / 16 <= INT32_MAX && (M + 15) / 16 <= 65535, CATQ_ERR_SHAPE,
               "d_out or M too large for one launch");
  CATQ_REQUIRE(ldq >= d_in && ldq % 16 == 0 && ldq <= (1 << 24), CATQ_ERR_SHAPE,
               "ldq must be >= d_in, a multiple of 16 and <= 2^24");
  CATQ_REQUIRE(ldy >= d_out, CATQ_ERR_SHAPE, "ldy must be >= d_out");
  CATQ_REQUIRE(y_dtype == CATQ_F32 || y_dtype == CATQ_BF16, CATQ_ERR_DTYPE, "Y must be fp32 or bf16");
  CATQ_REQUIRE(aligned16(q) && aligned16(alpha) && (reinterpret_cast<uintptr_t>(packed) & 7) == 0 &&
                   (reinterpret_cast<uintptr_t>(Y) & 3) == 0 && (reinterpret_cast<uintptr_t>(x_scale) & 3) == 0,
               CATQ_ERR_ALIGN, "q and alpha must be 16-byte aligned, packed 8-byte, x_scale and Y 4-byte");
  A8Args a{q, x_scale, ldq, M, packed, alpha, d_out, d_in, ldy, (int32_t)(d_in / 128),
           (int32_t)__builtin_ctz((unsigned)(g / 128)), Y};
  constexpr int NW = 4, R = 2;
  const dim3 grid((unsigned)((d_out + 16 * R - 1) / (16 * R)), (unsigned)((M + 15) / 16));
  const double flops = 2.0 * (double)M * (double)d_out * (double)d_in;
  const double bytes = (double)d_out * (double)d_in / 4.0 + 4.0 * (double)d_out * (double)(d_in / g) +
                       (double)M * (double)d_in + (double)M * (double)d_out * (double)dtype_size(y_dtype);
  if (y_dtype == CATQ_F32)
    CATQ_TRACED(stream, "ternary_a8_gemv_kernel", flops, bytes, M, d_out, d_in,
                hipLaunchKernelGGL((ternary_a8_gemv_kernel<NW, R, float>), grid, dim3(NW * 64), 0, stream, a));
  else
    CATQ_TRACED(stream, "ternary_a8_gemv_kernel", flops, bytes, M, d_out, d_in,
                hipLaunchKernelGGL((ternary_a8_gemv_kernel<NW, R, bf16>), grid, dim3(NW * 64), 0, stream, a));
  CATQ_CHECK_LAUNCH("ternary_linear_a8");
  return CATQ_OK;
}
