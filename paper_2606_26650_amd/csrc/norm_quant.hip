// Residual addition, RMSNorm and 8-bit output in one pass (gfx950): the input of
// a W1.58A8 linear layer as codes and scales.  Also the quantizer alone.
//
// One workgroup per row.  A thread holds its chunks of eight values (at most four,
// chunk c = thread + NT i) in registers between the pass over memory, the sum of
// squares, the group maxima and the store, so every operand is read once and
// every output written once: HBM bound for many rows (8192 x 5120, bf16 + fp32 stream: 102 us,
// 5.3 TB/s; a copy reaches 4.8), one memory latency and two block reductions for few
// (one row of 5120: 4 us).
#include <type_traits>

#include "kernels.h"
#include "quant8.h"

namespace catq {
namespace {

struct NormQuantArgs {
  const void* x;
  const void* res;
  const bf16* w;
  void* sum;
  bf16* y;
  int8_t* q;
  float* scale;
  int n;          // <= 32768
  int cpg;        // chunks of 8 per group
  int groups;     // per row
  float eps;
};

template <typename T>
__device__ __forceinline__ T block_reduce_sum(T v, T* red, int nw) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  T s = red[0];
  for (int i = 1; i < nw; ++i) s += red[i];
  return s;
}

template <int NT, int CH, bool NORM, typename XT, typename RT>
__global__ __launch_bounds__(NT) void norm_quant_kernel(NormQuantArgs a) {
  constexpr int NW = NT / 64;
  __shared__ float red_f[NW];
  __shared__ unsigned int red_u[NW];
  __shared__ unsigned int s_mag[NT * CH];   // chunk maxima, where a group is no power of two
  const int64_t row = blockIdx.x;
  const int nc = a.n >> 3, tid = threadIdx.x;
  const XT* x = static_cast<const XT*>(a.x) + row * a.n;
  float v[CH][8];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = tid + NT * i;
    if (c < nc) {
      load8<XT>(x + c * 8, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    }
  }
  u32x4 w8[NORM ? CH : 1];   // the gains, in flight with the rest
  if constexpr (NORM) {
#pragma unroll
    for (int i = 0; i < CH; ++i)
      if (a.w && tid + NT * i < nc) w8[i] = *reinterpret_cast<const u32x4*>(a.w + (tid + NT * i) * 8);
    if (a.res) {
      const RT* r = static_cast<const RT*>(a.res) + row * a.n;
      RT* sum = static_cast<RT*>(a.sum);
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int c = tid + NT * i;
        if (c >= nc) continue;
        float b[8];
        load8<RT>(r + c * 8, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[i][j] += b[j];
          // the norm is of the stream as stored
          if constexpr (std::is_same<RT, bf16>::value) v[i][j] = bf16_round_f(v[i][j]);
        }
        if (sum) store8<RT>(sum + row * a.n + c * 8, v[i]);
      }
    }
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) ss = fmaf(v[i][j], v[i][j], ss);
    ss = block_reduce_sum<float>(ss, red_f, NW);
    const float r = 1.0f / sqrtf(ss / (float)a.n + a.eps);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = tid + NT * i;
      if (a.w && c < nc) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[i][2 * j] = v[i][2 * j] * r * bf16_lo(w8[i][j]);
          v[i][2 * j + 1] = v[i][2 * j + 1] * r * bf16_hi(w8[i][j]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] *= r;
      }
    }
  }
  unsigned int mag[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    mag[i] = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j) mag[i] = max(mag[i], mag_bits(v[i][j]));
  }
  const int cpg = a.cpg;
  if (cpg == nc) {          // one group: the row
    unsigned int m = mag[0];
#pragma unroll
    for (int i = 1; i < CH; ++i) m = max(m, mag[i]);
#pragma unroll
    for (int k = 32; k >= 1; k >>= 1) m = max(m, (unsigned)__shfl_xor((int)m, k, 64));
    if ((tid & 63) == 0) red_u[tid >> 6] = m;
    __syncthreads();
    m = red_u[0];
#pragma unroll
    for (int i = 1; i < NW; ++i) m = max(m, red_u[i]);
#pragma unroll
    for (int i = 0; i < CH; ++i) mag[i] = m;
  } else if (cpg <= 64 && (cpg & (cpg - 1)) == 0) {   // consecutive lanes of one wave
    for (int k = cpg >> 1; k >= 1; k >>= 1)
#pragma unroll
      for (int i = 0; i < CH; ++i) mag[i] = max(mag[i], (unsigned)__shfl_xor((int)mag[i], k, 64));
  } else {   // (any other group: one value after the other, as many as a group has chunks)
#pragma unroll
    for (int i = 0; i < CH; ++i) s_mag[tid + NT * i] = mag[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = tid + NT * i, g0 = c / cpg * cpg;
      if (c < nc)
        for (int k = 0; k < cpg; ++k) mag[i] = max(mag[i], s_mag[g0 + k]);
    }
  }
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = tid + NT * i;
    if (c >= nc) continue;
    const float s = quant8_scale(mag[i]);
    quant8_n(v[i], s);
    if (a.q) {
      uint2 p;
      p.x = pack_codes(v[i][0], v[i][1], v[i][2], v[i][3]);
      p.y = pack_codes(v[i][4], v[i][5], v[i][6], v[i][7]);
      *reinterpret_cast<uint2*>(a.q + row * a.n + c * 8) = p;
      if (c % cpg == 0) a.scale[row * a.groups + c / cpg] = s;
    }
    if (a.y) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= s;
      store8<bf16>(a.y + row * a.n + c * 8, v[i]);
    }
  }
}

template <bool NORM, typename XT, typename RT>
void launch_norm_quant(const NormQuantArgs& a, int64_t rows, hipStream_t stream) {
  const dim3 grid((unsigned)rows);
  const int nc = a.n / 8;
  auto go = [&](auto nt, auto ch) {
    constexpr int NT = decltype(nt)::value, CH = decltype(ch)::value;
    hipLaunchKernelGGL((norm_quant_kernel<NT, CH, NORM, XT, RT>), grid, dim3(NT), 0, stream, a);
  };
  using std::integral_constant;
  // few rows: more threads to each (5120 values in one row: 3.6 us, 4.7 on 256 threads)
  if (rows <= 256 && nc > 256) {
    if (nc <= 512) go(integral_constant<int, 512>{}, integral_constant<int, 1>{});
    else if (nc <= 1024) go(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
    else if (nc <= 2048) go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
    else go(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
    return;
  }
  if (nc <= 256) go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  else if (nc <= 512) go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  else if (nc <= 1024) go(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  else if (nc <= 2048) go(integral_constant<int, 512>{}, integral_constant<int, 4>{});
  else go(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}

inline bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

catq_status check_quant(int64_t rows, int64_t n, int64_t group) {
  CATQ_REQUIRE(n > 0 && group > 0 && n % group == 0 && group % 8 == 0, CATQ_ERR_SHAPE,
               "group must be a multiple of 8 dividing n");
  CATQ_REQUIRE(n <= 32768, CATQ_ERR_SHAPE, "n must be <= 32768");
  // (a launch has fewer than 2^32 threads along x, and a row at most 1024)
  CATQ_REQUIRE(rows < (1 << (n <= 8192 ? 24 : 22)) && count_ok(rows, n), CATQ_ERR_SHAPE, "too many rows");
  return CATQ_OK;
}

}  // namespace
}  // namespace catq

using namespace catq;

extern "C" catq_status catq_aux_rmsnorm_quant(const void* x, catq_dtype x_dtype, const void* res,
                                              catq_dtype r_dtype, const void* weight, int64_t rows,
                                              int64_t n, int64_t group, float eps, void* sum,
                                              void* y, int8_t* q, float* scale,
                                              hipStream_t stream) {
  clear_error();
  CATQ_REQUIRE(rows >= 0, CATQ_ERR_SHAPE, "rows must be >= 0");
  if (rows == 0) return CATQ_OK;
  CATQ_REQUIRE(x, CATQ_ERR_NULL, "x must not be NULL");
  CATQ_REQUIRE((q != nullptr) == (scale != nullptr) && (q || y), CATQ_ERR_NULL,
               "q and scale go together, and one of q and y must be given");
  CATQ_REQUIRE(res || !sum, CATQ_ERR_NULL, "sum needs res");
  CATQ_REQUIRE(dtype_ok(x_dtype) && (!res || dtype_ok(r_dtype)), CATQ_ERR_DTYPE,
               "x and res must be bf16 or fp32");
  CATQ_TRY(check_quant(rows, n, group));
  CATQ_REQUIRE(eps >= 0, CATQ_ERR_VALUE, "eps must be >= 0");
  CATQ_REQUIRE(aligned16(x) && aligned16(res) && aligned16(weight) && aligned16(sum) &&
                   aligned16(y) && aligned(q, 8) && aligned(scale, 4),
               CATQ_ERR_ALIGN, "misaligned");
  CATQ_REQUIRE(!sum || sum != x || x_dtype == r_dtype, CATQ_ERR_VALUE,
               "sum can be x only where the types agree");
  const NormQuantArgs a{x, res, (const bf16*)weight, sum, (bf16*)y, q, scale, (int)n,
                        (int)(group / 8), (int)(n / group), eps};
  const double e = (double)rows * (double)n;
  const double rs = res ? (double)dtype_size(r_dtype) * (sum ? 2.0 : 1.0) : 0.0;
  const double bytes = e * (dtype_size(x_dtype) + rs + (q ? 1.0 : 0.0) + (y ? 2.0 : 0.0)) +
                       (q ? 4.0 * rows * (double)(n / group) : 0.0);
  auto go = [&](auto xt, auto rt) {
    launch_norm_quant<true, decltype(xt), decltype(rt)>(a, rows, stream);
  };
  const bool rf = res && r_dtype == CATQ_F32;
  auto launch = [&] {
    if (x_dtype == CATQ_BF16) {
      if (rf) go(bf16(), 0.f);
      else go(bf16(), bf16());
    } else {
      if (rf) go(0.f, 0.f);
      else go(0.f, bf16());
    }
  };
  CATQ_TRACED(stream, "norm_quant_kernel", 0.0, bytes, rows, n, group, launch());
  CATQ_CHECK_LAUNCH("rmsnorm quant");
  return CATQ_OK;
}

extern "C" catq_status catq_aux_act_quant8(const void* x, catq_dtype x_dtype, int64_t rows,
                                           int64_t n, int64_t group, int8_t* q, float* scale,
                                           hipStream_t stream) {
  clear_error();
  CATQ_REQUIRE(rows >= 0, CATQ_ERR_SHAPE, "rows must be >= 0");
  if (rows == 0) return CATQ_OK;
  CATQ_REQUIRE(x && q && scale, CATQ_ERR_NULL, "NULL argument");
  CATQ_REQUIRE(dtype_ok(x_dtype), CATQ_ERR_DTYPE, "x must be bf16 or fp32");
  CATQ_TRY(check_quant(rows, n, group));
  CATQ_REQUIRE(aligned16(x) && aligned(q, 8) && aligned(scale, 4), CATQ_ERR_ALIGN, "misaligned");
  const NormQuantArgs a{x, nullptr, nullptr, nullptr, nullptr, q, scale, (int)n,
                        (int)(group / 8), (int)(n / group), 0.f};
  const double bytes = (double)rows * (double)n * (dtype_size(x_dtype) + 1.0) +
                       4.0 * rows * (double)(n / group);
  auto launch = [&] {
    if (x_dtype == CATQ_BF16) launch_norm_quant<false, bf16, bf16>(a, rows, stream);
    else launch_norm_quant<false, float, bf16>(a, rows, stream);
  };
  CATQ_TRACED(stream, "norm_quant_kernel<quant only>", 0.0, bytes, rows, n, group, launch());
  CATQ_CHECK_LAUNCH("act quant 8");
  return CATQ_OK;
}
