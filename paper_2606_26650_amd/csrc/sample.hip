// A token per row of logits (gfx950): temperature, top-k, top-p, min-p, and the inverse of the cumulative
// distribution at a given number.
//
// Order.  Tokens are ordered by logit, the largest first, equal ones by index: by the composite
// c = (~key << 20) | index, key the logit's bits as an ordered integer; a smaller c comes first.  Each filter keeps a
// prefix of that order, so what is kept are the tokens with c up to one bound.
//
// Weights.  w = exp((logit - largest) / temperature) as an integer multiple of 2^-43: the exponent is taken in fp64
// (far tokens and small temperatures lose nothing), its fraction through the hardware's exp2 in fp32, off by one unit
// of 2^-23.  Sums of at most 2^20 weights of at most 1 are exact in 64 bits and do not depend on their order, so
// atomics in LDS give the same result every time.
#include <type_traits>

#include "kernels.h"

namespace catq {
namespace {

typedef unsigned long long u64;

constexpr int kT = 1024;              // threads of a workgroup
constexpr int kBins = 2048;
constexpr int kList = 2048;           // composites that are sorted in LDS
constexpr int kOne = 43;              // a weight of 1 is 2^43

struct SampleArgs {
  const void* logits;
  int64_t ld;
  int32_t V;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* u;
  int32_t* token;
  float* prob;
};

__device__ __forceinline__ unsigned int key_of(float x) {
  const unsigned int u = x == 0.0f ? 0u : __float_as_uint(x);   // (-0 as 0)
  return (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ u64 composite(float x, int i) { return ((u64)(~key_of(x)) << 20) | (unsigned)i; }
__device__ __forceinline__ float logit_of(u64 c) {
  const unsigned int key = ~(unsigned int)(c >> 20);
  return __uint_as_float((key >> 31) ? key & 0x7fffffffu : ~key);
}

// What a row's weights and bins are made of
struct Row {
  float top;       // its largest logit
  double scale;    // log2(e) / temperature
  float bins;      // bins per unit of logit
};
// (logit - largest) log2(e) / temperature; equal ones give 0 also where both are infinite
__device__ __forceinline__ double exponent(const Row& r, float x) {
  return x == r.top ? 0.0 : ((double)x - (double)r.top) * r.scale;
}
__device__ __forceinline__ u64 weight(const Row& r, float x) {
  const double z = exponent(r, x);
  if (z < -60.0) return 0;
  const double n = rint(z);
  const u64 m = (u64)(unsigned int)(__builtin_amdgcn_exp2f((float)(z - n)) * 0x1p24f);
  const int s = kOne - 24 + (int)n;      // n <= 0
  return s >= 0 ? m << s : m >> -s;
}
// Bins of the distance from the largest logit: 64 per unit of exp's argument, the last for all that is far
__device__ __forceinline__ int bin_of(const Row& r, float x) {
  return x == r.top ? 0 : (int)fminf((r.top - x) * r.bins, (float)(kBins - 1));
}

// f(logit, index) for the row's elements i0 .. i1 - 1, `lanes` lanes taking 16-byte pieces in turn, U loads in flight.
// A row may start at any element: the pieces are aligned in memory.
template <typename T, int U = 4, typename F>
__device__ __forceinline__ void for_range(const T* row, int V, int i0, int i1, int lane, int lanes, F&& f) {
  constexpr int E = 16 / sizeof(T);
  if (i0 >= i1) return;
  const int off = (int)(((uintptr_t)row & 15u) / sizeof(T));
  const int v1 = (i1 - 1 + off) / E;
  for (int v = (i0 + off) / E + lane; v <= v1; v += U * lanes) {
    u32x4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e0 = (v + u * lanes) * E - off;
      if (v + u * lanes > v1) continue;
      if (e0 >= 0 && e0 + E <= V) {
        raw[u] = *reinterpret_cast<const u32x4*>(row + e0);
      } else {                         // the first or last piece of the row
        raw[u] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int j = 0; j < E; ++j) {
          if (e0 + j < 0 || e0 + j >= V) continue;
          if constexpr (sizeof(T) == 4) raw[u][j] = __builtin_bit_cast(unsigned int, row[e0 + j]);
          else raw[u][j / 2] |= (unsigned)__builtin_bit_cast(u16, row[e0 + j]) << (16 * (j & 1));
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e0 = (v + u * lanes) * E - off;
      if (v + u * lanes > v1) continue;
#pragma unroll
      for (int j = 0; j < E; ++j) {
        const int i = e0 + j;
        if (i < i0 || i >= i1) continue;
        float x;
        if constexpr (sizeof(T) == 4) x = __uint_as_float(raw[u][j]);
        else x = (j & 1) ? bf16_hi(raw[u][j / 2]) : bf16_lo(raw[u][j / 2]);
        if (x > -INFINITY) f(x, i);    // (not -inf, no NaN)
      }
    }
  }
}

__device__ __forceinline__ u64 shfl_up64(u64 v, int d) { return __shfl_up(v, d, 64); }

// Inclusive prefix sum over the workgroup; `total` is the whole.  s: one value per wave.
__device__ __forceinline__ u64 block_scan(u64 v, u64* s, u64& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const u64 o = shfl_up64(v, d);
    if (lane >= d) v += o;
  }
  __syncthreads();
  if (lane == 63) s[wave] = v;
  __syncthreads();
  u64 before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kT / 64; ++w) {
    const u64 t = s[w];
    if (w < wave) before += t;
    total += t;
  }
  return v + before;
}
template <typename F>
__device__ __forceinline__ u64 block_reduce(u64 v, u64* s, F&& f) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v = f(v, (u64)__shfl_xor(v, d, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
#pragma unroll
  for (int w = 1; w < kT / 64; ++w) v = f(v, s[w]);
  return v;
}

struct Shared {
  u64 list[kList];
  u64 mass[kBins];
  unsigned int count[kBins];
  u64 wave[kT / 64];
  u64 at[4];
  unsigned int n;
};

// s.list[0 .. n) in ascending order (n <= kList)
__device__ __forceinline__ void sort_list(Shared& s, int n) {
  int size = 2;
  while (size < n) size <<= 1;
  for (int i = n + threadIdx.x; i < size; i += kT) s.list[i] = ~0ull;
  __syncthreads();
  for (int k = 2; k <= size; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      for (int p = threadIdx.x; p < size / 2; p += kT) {
        const int a = 2 * (p & ~(j - 1)) + (p & (j - 1)), b = a + j;
        const u64 x = s.list[a], y = s.list[b];
        if ((x > y) == ((a & k) == 0)) {
          s.list[a] = y;
          s.list[b] = x;
        }
      }
      __syncthreads();
    }
}

// Of the row's tokens in bin b (n of them): the composite of the last one that is kept, and their mass up to it.
// By count: the first `want` of them are kept.  By mass: those before which the mass (with `base`) is below `target`,
// of the ones with c <= most.
struct Bound {
  u64 c, mass;
};
template <typename T>
__device__ Bound resolve(Shared& s, const T* row, int V, const Row& r, int b, int n, bool by_mass, u64 want, u64 base,
                         double target, u64 most) {
  u64 lo = 0, hi = most, before = 0;      // composites lo .. hi are in question; the mass of those below lo
  // more than the list takes: the interval is cut to one of up to 2048 parts, again and again
  while (n > kList) {
    u64 least = ~0ull, last = 0;
    for_range<T>(row, V, 0, V, threadIdx.x, kT, [&](float x, int i) {
      const u64 c = composite(x, i);
      if (bin_of(r, x) != b || c < lo || c > hi) return;
      least = min(least, c);
      last = max(last, c);
    });
    lo = block_reduce(least, s.wave, [](u64 p, u64 q) { return min(p, q); });
    hi = block_reduce(last, s.wave, [](u64 p, u64 q) { return max(p, q); });
    const int bits = 64 - __builtin_clzll((hi - lo) | 1);
    const int shift = bits > 11 ? bits - 11 : 0;
    for (int i = threadIdx.x; i < kBins; i += kT) {
      s.count[i] = 0;
      s.mass[i] = 0;
    }
    __syncthreads();
    for_range<T>(row, V, 0, V, threadIdx.x, kT, [&](float x, int i) {
      const u64 c = composite(x, i);
      if (bin_of(r, x) != b || c < lo || c > hi) return;
      atomicAdd(&s.count[(c - lo) >> shift], 1u);
      atomicAdd(&s.mass[(c - lo) >> shift], weight(r, x));
    });
    __syncthreads();
    const int t = 2 * threadIdx.x;
    u64 all;
    const u64 c0 = s.count[t], c1 = s.count[t + 1], m0 = s.mass[t], m1 = s.mass[t + 1];
    const u64 pc = block_scan(c0 + c1, s.wave, all) - c0 - c1, pm = block_scan(m0 + m1, s.wave, all) - m0 - m1;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const u64 ec = pc + (k ? c0 : 0), em = pm + (k ? m0 : 0), c = k ? c1 : c0, m = k ? m1 : m0;
      const bool here = by_mass ? (double)(base + before + em) < target && target <= (double)(base + before + em + m)
                                : ec < want && want <= ec + c;
      if (here) {
        s.at[0] = t + k;
        s.at[1] = ec;
        s.at[2] = em;
        s.at[3] = c;
      }
    }
    __syncthreads();
    const u64 part = s.at[0];
    before += s.at[2];
    want -= by_mass ? 0 : s.at[1];
    n = (int)s.at[3];
    lo += part << shift;
    hi = min(hi, lo + ((1ull << shift) - 1));
    __syncthreads();
  }
  if (threadIdx.x == 0) s.n = 0;
  __syncthreads();
  for_range<T>(row, V, 0, V, threadIdx.x, kT, [&](float x, int i) {
    const u64 c = composite(x, i);
    if (bin_of(r, x) != b || c < lo || c > hi) return;
    const unsigned int at = atomicAdd(&s.n, 1u);
    if (at < kList) s.list[at] = c;
  });
  __syncthreads();
  n = (int)min(s.n, (unsigned)kList);
  sort_list(s, n);
  // two neighbours a thread
  const int t = 2 * threadIdx.x;
  const u64 m0 = t < n ? weight(r, logit_of(s.list[t])) : 0, m1 = t + 1 < n ? weight(r, logit_of(s.list[t + 1])) : 0;
  u64 all;
  const u64 pm = block_scan(m0 + m1, s.wave, all) - m0 - m1;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const u64 em = before + pm + (k ? m0 : 0), m = k ? m1 : m0;
    const bool here = t + k < n && (by_mass ? (double)(base + em) < target && target <= (double)(base + em + m)
                                            : (u64)(t + k + 1) == want);
    if (here) {
      s.at[0] = s.list[t + k];
      s.at[1] = em + m;
    }
  }
  __syncthreads();
  const Bound out = {s.at[0], s.at[1]};
  __syncthreads();
  return out;
}

// One workgroup per row.
template <typename T>
__global__ __launch_bounds__(kT) void sample_kernel(SampleArgs a) {
  __shared__ Shared s;
  const int64_t r0 = blockIdx.x;
  const T* row = static_cast<const T*>(a.logits) + r0 * a.ld;
  const int tid = threadIdx.x, V = a.V;
  const float temp = a.temperature ? a.temperature[r0] : 1.0f;
  const float top_p = a.top_p ? a.top_p[r0] : 1.0f, min_p = a.min_p ? a.min_p[r0] : 0.0f;
  const int top_k = a.top_k ? a.top_k[r0] : 0;
  // the largest
  u64 first = ~0ull;
  for_range<T>(row, V, 0, V, tid, kT, [&](float x, int i) { first = min(first, composite(x, i)); });
  first = block_reduce(first, s.wave, [](u64 p, u64 q) { return min(p, q); });
  if (first == ~0ull || !(temp > 0.0f) || top_k == 1 || top_p <= 0.0f) {
    if (tid == 0) {
      a.token[r0] = first == ~0ull ? -1 : (int)(first & 0xfffffu);
      if (a.prob) a.prob[r0] = first == ~0ull ? 0.f : 1.f;
    }
    return;
  }
  Row r;
  r.top = logit_of(first);
  r.scale = 1.4426950408889634 / (double)temp;
  r.bins = fminf(64.0f / temp, 1e30f);
  u64 bound = ~0ull;          // composites up to it are kept
  if (top_k > 0 || top_p < 1.0f) {
    for (int i = tid; i < kBins; i += kT) {
      s.count[i] = 0;
      s.mass[i] = 0;
    }
    __syncthreads();
    for_range<T>(row, V, 0, V, tid, kT, [&](float x, int) {
      const int b = bin_of(r, x);
      atomicAdd(&s.count[b], 1u);
      atomicAdd(&s.mass[b], weight(r, x));
    });
    __syncthreads();
    // two bins a thread
    const int t = 2 * tid;
    u64 n_all, m_all;
    const u64 c0 = s.count[t], c1 = s.count[t + 1], m0 = s.mass[t], m1 = s.mass[t + 1];
    const u64 pc = block_scan(c0 + c1, s.wave, n_all) - c0 - c1;
    const u64 pm = block_scan(m0 + m1, s.wave, m_all) - m0 - m1;
    u64 sum = m_all;          // of what top-k keeps
    int last_bin = kBins;     // the bin where top-k ends
    if (top_k > 0 && (u64)top_k < n_all) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const u64 e = pc + (k ? c0 : 0), c = k ? c1 : c0;
        if (e < (u64)top_k && (u64)top_k <= e + c) {
          s.at[0] = t + k;
          s.at[1] = top_k - e;
          s.at[2] = pm + (k ? m0 : 0);
          s.at[3] = c;
        }
      }
      __syncthreads();
      last_bin = (int)s.at[0];
      const u64 want = s.at[1], base = s.at[2];
      const int n = (int)s.at[3];
      __syncthreads();
      const Bound k = resolve(s, row, V, r, last_bin, n, false, want, base, 0.0, ~0ull);
      bound = k.c;
      sum = base + k.mass;
    }
    if (top_p < 1.0f) {
      const double target = (double)top_p * (double)sum;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const u64 e = pm + (k ? m0 : 0), m = t + k == last_bin ? sum - e : k ? m1 : m0;
        if (t + k <= last_bin && (double)e < target && target <= (double)(e + m)) {
          s.at[0] = t + k;
          s.at[2] = e;
          s.at[3] = k ? c1 : c0;
        }
      }
      __syncthreads();
      const int b = (int)s.at[0], n = (int)s.at[3];
      const u64 base = s.at[2];
      __syncthreads();
      bound = min(bound, resolve(s, row, V, r, b, n, true, 0, base, target, bound).c);
    }
  }
  const double least = min_p > 0.0f ? fmin(log2((double)min_p), 0.0) : -INFINITY;
  auto kept = [&](float x, int i) { return composite(x, i) <= bound && exponent(r, x) >= least; };
  // the segment of the row in which the distribution passes u, cut in 16 by the waves' sums until a lane has one token
  float u = a.u[r0];
  u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
  int i0 = 0, i1 = V;
  u64 base = 0;
  double all = 0.0, target = 0.0;
  const int wave = tid >> 6, lane = tid & 63;
  for (bool whole = true; whole || i1 - i0 > kT; whole = false) {
    const int seg = (i1 - i0 + 15) / 16, a0 = min(i0 + wave * seg, i1), a1 = min(a0 + seg, i1);
    u64 m = 0;
    for_range<T>(row, V, a0, a1, lane, 64, [&](float x, int i) {
      if (kept(x, i)) m += weight(r, x);
    });
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) m += __shfl_xor(m, d, 64);
    __syncthreads();
    if (lane == 0) s.wave[wave] = m;
    __syncthreads();
    if (whole) {
      u64 sum = 0;
#pragma unroll
      for (int w = 0; w < 16; ++w) sum += s.wave[w];
      all = (double)sum;
      target = (double)u * all;
    }
    int w = 0;
    while (w < 15 && !((double)(base + s.wave[w]) > target)) base += s.wave[w++];
    i0 = min(i0 + w * seg, i1);
    i1 = min(i0 + seg, i1);
  }
  const int i = i0 + tid;
  u64 m = 0;
  if (i < i1) {
    const float x = to_f(row[i]);
    if (x > -INFINITY && kept(x, i)) m = weight(r, x);
  }
  u64 sum;
  const u64 upto = base + block_scan(m, s.wave, sum);
  if ((double)upto > target && !((double)(upto - m) > target)) {
    a.token[r0] = i;
    if (a.prob) a.prob[r0] = (float)((double)m / all);
  }
}

}  // namespace
}  // namespace catq

using namespace catq;

extern "C" size_t catq_aux_sample_workspace_bytes(int64_t rows, int64_t V) {
  if (rows <= 0 || V <= 0) return 0;
  return 0;
}

extern "C" catq_status catq_aux_sample(const void* logits, catq_dtype dtype, int64_t rows, int64_t V, int64_t ld,
                                       const float* temperature, const int32_t* top_k, const float* top_p,
                                       const float* min_p, const float* u, int32_t* token, float* prob,
                                       void* workspace, size_t workspace_bytes, hipStream_t stream) {
  clear_error();
  CATQ_REQUIRE(rows >= 0, CATQ_ERR_SHAPE, "rows must be >= 0");
  if (rows == 0) return CATQ_OK;
  CATQ_REQUIRE(logits && u && token, CATQ_ERR_NULL, "logits, u and token must not be NULL");
  CATQ_REQUIRE(dtype_ok(dtype), CATQ_ERR_DTYPE, "logits must be fp32 or bf16");
  CATQ_REQUIRE(V > 0 && V <= (1 << 20), CATQ_ERR_SHAPE, "V must be 1 .. 2^20");
  // (a launch has fewer than 2^32 threads along x)
  CATQ_REQUIRE(rows < (1 << 22) && ld >= V && count_ok(rows, ld), CATQ_ERR_SHAPE,
               "ld must be >= V, rows below 2^22 and rows * ld within 2^38");
  auto at4 = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; };
  CATQ_REQUIRE(aligned16(logits) && at4(temperature) && at4(top_k) && at4(top_p) && at4(min_p) && at4(u) &&
                   at4(token) && at4(prob) && aligned16(workspace),
               CATQ_ERR_ALIGN, "logits and workspace must be 16-byte aligned, the others 4-byte");
  const size_t need = catq_aux_sample_workspace_bytes(rows, V);
  CATQ_REQUIRE(need == 0 || (workspace && workspace_bytes >= need), CATQ_ERR_WORKSPACE,
               "workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
  const SampleArgs a{logits, ld, (int32_t)V, temperature, top_k, top_p, min_p, u, token, prob};
  const double bytes = (double)rows * (double)V * (double)dtype_size(dtype);
  auto kernel = dtype == CATQ_F32 ? sample_kernel<float> : sample_kernel<bf16>;
  CATQ_TRACED(stream, "sample_kernel", 0.0, bytes, rows, V, 1,
              hipLaunchKernelGGL(kernel, dim3((unsigned)rows), dim3(kT), 0, stream, a));
  CATQ_CHECK_LAUNCH("sample");
  return CATQ_OK;
}
