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
// atomics give the same result every time.
//
// Steps.  A row's tokens go into 2048 bins of 1/64 of exp's argument below the largest logit, with their number and
// their weight.  The bins tell where top-k (or, without it, top-p) ends.  Where the tokens up to that bin are few, they
// are gathered and the rest happens in LDS; where they are many, that bin's tokens are, and the weight before it is summed
// by slices of the row, of which the one where u falls is read again.  Only in the bins in which a filter ends are tokens compared.
// Without top-k and top-p no bins are needed, only the weight of every slice.
//
// Long rows are read by several workgroups each: the largest logit of every slice, then bins
// or weights of every slice, then the gathering, then one workgroup a row for what is left.
//
// What bounds it: for few rows the launches, 11 us for four, and the chains of latencies in them (150000 fp32 logits: greedy 12 us,
// no filter 13, top-50 22, top-p 0.9 28; 8192, alone: 7, 11, 16, 17.5). For many rows the loads, three times from the
// last-level cache, the LDS atomics of the bins (as many as tokens) and the weights' 20 instructions: 64 rows of 150000: 15, 32, 42,
// 64 us, where one read takes 7.5.
#include <algorithm>
#include <type_traits>

#include "kernels.h"

namespace catq {
namespace {

typedef unsigned long long u64;

constexpr int kAloneT = 1024;         // threads of a workgroup that has a row to itself
constexpr int kPickT = 512;           // of one that picks a row's token after others have read it
constexpr int kS = 512;               // threads of one that reads a slice
constexpr int kBins = 2048;
constexpr int kList = 4096;           // composites that are gathered
constexpr int kFew = 128;             // that are compared with each other, if they are at hand
constexpr int kOne = 43;              // a weight of 1 is 2^43
constexpr int kWide = 32;             // tokens that a thread reads in a row at most
constexpr int kMaxSlices = 256;

// What the workgroups of a row leave for those after them
struct RowSpace {
  u64 first[kMaxSlices];              // slice: its first composite
  u64 mass[kMaxSlices];               // slice: the weight that it keeps (rows without top-k and top-p)
  u64 bin_mass[kBins];
  u64 list[kList];
  unsigned int bin_count[kBins];
  unsigned int n;                     // composites in the list
  unsigned int pad[3];
};

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
  RowSpace* space;      // [rows], where a row has several workgroups
  int32_t slices;       // of a row
  int32_t slice;        // tokens of a slice
};

// A row's settings
struct Settings {
  float temp, top_p, min_p;
  int top_k;
  bool first_only;      // the first token is taken
  bool filtered;        // top-k or top-p
};
__device__ __forceinline__ Settings settings(const SampleArgs& a, int64_t row) {
  Settings p;
  p.temp = a.temperature ? a.temperature[row] : 1.0f;
  p.top_p = a.top_p ? a.top_p[row] : 1.0f;
  p.min_p = a.min_p ? a.min_p[row] : 0.0f;
  p.top_k = a.top_k ? a.top_k[row] : 0;
  p.first_only = !(p.temp > 0.0f) || p.top_k == 1 || p.top_p <= 0.0f || p.min_p > 1.0f;   // (no weight is above 1)
  p.filtered = p.top_k > 0 || p.top_p < 1.0f;
  return p;
}

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
  double offset;   // -top * scale
  float bins;      // bins per unit of logit
};
__device__ __forceinline__ Row row_of(u64 first, float temp) {
  Row r;
  r.top = logit_of(first);
  r.scale = 1.4426950408889634 / (double)temp;
  r.offset = -(double)r.top * r.scale;
  r.bins = fminf(64.0f / temp, 1e30f);
  return r;
}
// the least exponent that a min-p of at most 1 keeps
__device__ __forceinline__ double least_of(float min_p) {
  return min_p > 0.0f ? log2((double)min_p) : -INFINITY;
}
// (logit - largest) log2(e) / temperature, off by 2^-53 of the larger product; equal ones give 0 also where both
// are infinite
__device__ __forceinline__ double exponent(const Row& r, float x) {
  return x == r.top ? 0.0 : fma((double)x, r.scale, r.offset);
}
// 2^exponent in units of 2^-43; 0 for what is below 2^-43, -inf and NaN among it (without a branch)
__device__ __forceinline__ u64 weight_of(double exponent) {
  const double z = fmax(exponent, -62.0), n = rint(z);
  const u64 m = (unsigned int)(__builtin_amdgcn_exp2f((float)(z - n)) * 0x1p24f);
  return (m << (kOne - 24)) >> -(int)n;      // n <= 0
}
__device__ __forceinline__ u64 weight(const Row& r, float x) { return weight_of(exponent(r, x)); }
// Bins of the distance from the largest logit: 64 per unit of exp's argument, the last for all that is far
__device__ __forceinline__ int bin_of(const Row& r, float x) {
  return x == r.top ? 0 : (int)fminf((r.top - x) * r.bins, (float)(kBins - 1));
}

// f(logit, index) for the row's elements i0 .. i1 - 1, and for those around them in the same pieces with a logit of
// -inf, which a NaN also becomes: no branch. `lanes` lanes take 16-byte pieces in turn. A row may start at any
// element: the pieces are aligned in memory. (Several pieces in flight a lane, moved up as they are used, took 3 to 10%
// longer: the waves of a unit hide each other's loads.)
template <typename T>
__device__ __forceinline__ u32x4 load_piece(const T* row, int V, int e0) {
  constexpr int E = 16 / sizeof(T);
  if (e0 >= 0 && e0 + E <= V) return *reinterpret_cast<const u32x4*>(row + e0);
  u32x4 raw = {0u, 0u, 0u, 0u};      // the first or last piece of the row
#pragma unroll
  for (int j = 0; j < E; ++j) {
    if (e0 + j < 0 || e0 + j >= V) continue;
    if constexpr (sizeof(T) == 4) raw[j] = __builtin_bit_cast(unsigned int, row[e0 + j]);
    else raw[j / 2] |= (unsigned)__builtin_bit_cast(u16, row[e0 + j]) << (16 * (j & 1));
  }
  return raw;
}
template <typename T, typename F>
__device__ __forceinline__ void use_piece(u32x4 raw, int e0, int i0, int i1, F&& f) {
#pragma unroll
  for (int j = 0; j < (int)(16 / sizeof(T)); ++j) {
    const int i = e0 + j;
    float x;
    if constexpr (sizeof(T) == 4) x = __uint_as_float(raw[j]);
    else x = (j & 1) ? bf16_hi(raw[j / 2]) : bf16_lo(raw[j / 2]);
    f(x > -INFINITY && (unsigned)(i - i0) < (unsigned)(i1 - i0) ? x : -INFINITY, i);
  }
}
template <typename T, typename F>
__device__ __forceinline__ void for_all(const T* row, int V, int i0, int i1, int lane, int lanes, F&& f) {
  constexpr int E = 16 / sizeof(T);
  if (i0 >= i1) return;
  const int off = (int)(((uintptr_t)row & 15u) / sizeof(T));
  const int v1 = (i1 - 1 + off) / E;
  for (int v = (i0 + off) / E + lane; v <= v1; v += lanes)
    use_piece<T>(load_piece(row, V, v * E - off), v * E - off, i0, i1, f);
}
// f(logit, index) for the elements i0 .. i1 - 1 that can be taken: not -inf, no NaN
template <typename T, typename F>
__device__ __forceinline__ void for_range(const T* row, int V, int i0, int i1, int lane, int lanes, F&& f) {
  for_all<T>(row, V, i0, i1, lane, lanes, [&](float x, int i) {
    if (x > -INFINITY) f(x, i);
  });
}

// v plus what another lane of the wave has, by a data-parallel move (0 where there is none)
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 add_moved(u64 v) {
  const unsigned int lo = __builtin_amdgcn_update_dpp(0, (int)(unsigned)v, CTRL, ROWS, 0xf, false);
  const unsigned int hi = __builtin_amdgcn_update_dpp(0, (int)(unsigned)(v >> 32), CTRL, ROWS, 0xf, false);
  return v + (((u64)hi << 32) | lo);
}
// Inclusive prefix sum over a wave: within rows of 16 lanes by shifts of 1, 2, 4 and 8, then a row's last lane to the
// next row, and lane 31 to the upper half.  (Six shuffles through LDS took 600 cycles.)
__device__ __forceinline__ u64 wave_scan(u64 v) {
  v = add_moved<0x111, 0xf>(v);
  v = add_moved<0x112, 0xf>(v);
  v = add_moved<0x114, 0xf>(v);
  v = add_moved<0x118, 0xf>(v);
  v = add_moved<0x142, 0xa>(v);
  return add_moved<0x143, 0xc>(v);
}

// Inclusive prefix sum over the workgroup; `total` is the whole.  s: one value per wave.
template <int NT>
__device__ __forceinline__ u64 block_scan(u64 v, u64* s, u64& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = wave_scan(v);
  __syncthreads();
  if (lane == 63) s[wave] = v;
  __syncthreads();
  u64 before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    const u64 t = s[w];
    if (w < wave) before += t;
    total += t;
  }
  return v + before;
}
template <int NT, typename F>
__device__ __forceinline__ u64 block_reduce(u64 v, u64* s, F&& f) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v = f(v, (u64)__shfl_xor(v, d, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) v = f(v, s[w]);
  return v;
}
template <int NT>
__device__ __forceinline__ u64 block_sum(u64 v, u64* s) {
  u64 total;
  block_scan<NT>(v, s, total);
  return total;
}
template <int NT>
__device__ __forceinline__ u64 block_min(u64 v, u64* s) {
  return block_reduce<NT>(v, s, [](u64 p, u64 q) { return min(p, q); });
}

// Where the filters end among the bins: top-k, if it leaves a token out, or else top-p.
struct Ends {
  u64 n_all, m_all;      // the row's tokens and weight
  bool by_k, both;       // top-k ends there; top-p is still to come
  int last;              // the bin of the last token, kBins where all are kept
  u64 want, base;        // (top-k) that token's place in the bin; the weight before the bin
  u64 in_bin, count;     // tokens of the bin, and up to it
};
// What is gathered: all tokens up to the last bin; where they are too many, the last bin's alone; nothing where these
// are too many too, or where top-p ends somewhere before top-k.
// (Where top-p alone ends, tokens have not been counted: the list may turn out too short.)
enum { kGatherAll, kGatherBin, kGatherNone };
__device__ __forceinline__ int gathered(const Ends& e) {
  return e.count <= kList ? kGatherAll : !e.both && e.in_bin <= kList ? kGatherBin : kGatherNone;
}
// at: eight values in LDS.  COUNTED: the bins' tokens are counted also where there is no top-k.
template <int NT, bool COUNTED>
__device__ __forceinline__ Ends find_ends(const unsigned int* count, const u64* mass, int top_k, float top_p, u64* s,
                                          u64* at) {
  constexpr int B = kBins / NT;
  const int t = B * threadIdx.x;
  unsigned int c[B];
  u64 m[B], cs = 0, ms = 0;
#pragma unroll
  for (int i = 0; i < B; ++i) {
    c[i] = count[t + i];
    m[i] = mass[t + i];
    cs += c[i];
    ms += m[i];
  }
  Ends e;
  const u64 pc = block_scan<NT>(cs, s, e.n_all) - cs, pm = block_scan<NT>(ms, s, e.m_all) - ms;
  const bool by_k = top_k > 0 && (u64)top_k < e.n_all;
  const double target = (double)top_p * (double)e.m_all;
  u64 ec = pc, em = pm;
#pragma unroll
  for (int i = 0; i < B; ++i) {
    const bool here = by_k ? ec < (u64)top_k && (u64)top_k <= ec + c[i]
                           : top_p < 1.0f && (double)em < target && target <= (double)(em + m[i]);
    if (here) {
      at[0] = t + i;
      at[1] = (u64)top_k - ec;
      at[2] = em;
      at[3] = c[i];
      at[4] = ec + c[i];
    }
    ec += c[i];
    em += m[i];
  }
  __syncthreads();
  const bool some = by_k || top_p < 1.0f;
  e.by_k = by_k;
  e.both = by_k && top_p < 1.0f;
  e.last = some ? (int)at[0] : kBins;
  e.want = at[1];
  e.base = some ? at[2] : e.m_all;
  e.in_bin = some ? at[3] : 0;
  e.count = some ? at[4] : e.n_all;
  if (!COUNTED && top_k <= 0) e.count = kList + 1;
  __syncthreads();
  return e;
}

template <int kT>
struct Shared {
  u64 list[kList];        // what has been gathered
  u64 few[kT];            // the last tokens in question
  u64 weight[kT];         // and what they weigh
  u64 mass[kBins];        // the row's bins
  u64 part_mass[kBins];   // parts of one of them
  unsigned int count[kBins];
  unsigned int part_count[kBins];
  u64 wave[kT / 64];
  u64 at[8];
  unsigned int n;
};

// Of N sums in LDS, the one where base + their running sum passes `target` (in s.at: its index, what is before it,
// itself).
template <int N, int kT>
__device__ __forceinline__ void find_passing(Shared<kT>& s, const u64* sums, u64 base, double target) {
  constexpr int B = N >= kT ? N / kT : 1;
  const int t = B * threadIdx.x;
  u64 m[B], ms = 0, all;
#pragma unroll
  for (int i = 0; i < B; ++i) {
    m[i] = t + i < N ? sums[t + i] : 0;
    ms += m[i];
  }
  u64 em = base + block_scan<kT>(ms, s.wave, all) - ms;
#pragma unroll
  for (int i = 0; i < B; ++i) {
    if (!((double)em > target) && (double)(em + m[i]) > target) {
      s.at[0] = t + i;
      s.at[1] = em;
      s.at[2] = m[i];
    }
    em += m[i];
  }
  __syncthreads();
}

// A filter's end in a bin of n tokens.  By count: the first `want` of them are kept.  By mass: those before which
// the mass (`base` before the bin) is below `target`.
struct Cut {
  int bin, n;
  bool by_mass;
  u64 want, base;
  double target;
};
struct Bound {
  u64 c, mass;      // the composite of the last token that is kept, the weight of the bin's up to it
};

// each(f) calls f(logit, composite) for all tokens of the row that may be in the bin; those with c <= most count.
// Where more than `few` (at most kT) are left, the interval of composites in question is cut to one of up to 2048 parts, again
// and again; then a thread for each counts the tokens ahead of its own and their weight.  (Sorting 100 of them took three
// times as long; counting among 500 took 20 us.)
template <int kT, typename Each>
__device__ __forceinline__ Bound cut_bin(Shared<kT>& s, Each&& each, const Row& r, Cut q, u64 most,
                                         int few) {
  u64 lo = 0, hi = most, before = 0;      // composites lo .. hi are in question; the weight of the bin's below lo
  const int t = threadIdx.x;
#pragma unroll 1
  while (q.n > few) {
    u64 least = ~0ull, last = 0;
    each([&](float x, u64 c) {
      if (bin_of(r, x) != q.bin || c < lo || c > hi) return;
      least = min(least, c);
      last = max(last, c);
    });
    lo = block_min<kT>(least, s.wave);
    hi = ~block_min<kT>(~last, s.wave);
    const int bits = 64 - __builtin_clzll((hi - lo) | 1);
    const int shift = bits > 11 ? bits - 11 : 0;
    for (int i = t; i < kBins; i += kT) {
      s.part_count[i] = 0;
      s.part_mass[i] = 0;
    }
    __syncthreads();
    each([&](float x, u64 c) {
      if (bin_of(r, x) != q.bin || c < lo || c > hi) return;
      atomicAdd(&s.part_count[(c - lo) >> shift], 1u);
      atomicAdd(&s.part_mass[(c - lo) >> shift], weight(r, x));
    });
    __syncthreads();
    constexpr int B = kBins / kT;
    u64 cs = 0, ms = 0, all;
#pragma unroll
    for (int k = 0; k < B; ++k) {
      cs += s.part_count[B * t + k];
      ms += s.part_mass[B * t + k];
    }
    u64 ec = block_scan<kT>(cs, s.wave, all) - cs, em = q.base + before + block_scan<kT>(ms, s.wave, all) - ms;
#pragma unroll
    for (int k = 0; k < B; ++k) {
      const u64 c = s.part_count[B * t + k], m = s.part_mass[B * t + k];
      const bool here = q.by_mass ? (double)em < q.target && q.target <= (double)(em + m)
                                  : ec < q.want && q.want <= ec + c;
      if (here) {
        s.at[0] = B * t + k;
        s.at[1] = ec;
        s.at[2] = em - q.base;
        s.at[3] = c;
      }
      ec += c;
      em += m;
    }
    __syncthreads();
    before = s.at[2];
    q.want -= q.by_mass ? 0 : s.at[1];
    q.n = (int)s.at[3];
    lo += s.at[0] << shift;
    hi = min(hi, lo + ((1ull << shift) - 1));
    __syncthreads();
  }
  if (t == 0) s.n = 0;
  __syncthreads();
  each([&](float x, u64 c) {
    if (bin_of(r, x) != q.bin || c < lo || c > hi) return;
    const unsigned int at = atomicAdd(&s.n, 1u);
    if (at < kT) s.few[at] = c;
  });
  __syncthreads();
  const int n = (int)min(s.n, (unsigned)kT);
  const u64 c = t < n ? s.few[t] : 0, m = t < n ? weight(r, logit_of(c)) : 0;
  if (t < n) s.weight[t] = m;
  __syncthreads();
  if (t < n) {
    u64 em = before, rank = 0;
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      const bool ahead = s.few[i] < c;
      rank += ahead ? 1 : 0;
      em += ahead ? s.weight[i] : 0;
    }
    const bool here = q.by_mass ? (double)(q.base + em) < q.target && q.target <= (double)(q.base + em + m)
                                : rank + 1 == q.want;
    if (here) {
      s.at[0] = c;
      s.at[1] = em + m;
    }
  }
  __syncthreads();
  const Bound out = {s.at[0], s.at[1]};
  __syncthreads();
  return out;
}

// ---------------------------------------------------------------- slices of a row

// The first composite of every slice, and the row's bins cleared.
template <typename T>
__global__ __launch_bounds__(kS) void sample_first_kernel(SampleArgs a) {
  __shared__ u64 s_wave[kS / 64];
  const int64_t r0 = blockIdx.y;
  const T* row = static_cast<const T*>(a.logits) + r0 * a.ld;
  RowSpace& sp = a.space[r0];
  const int i0 = blockIdx.x * a.slice, i1 = min(i0 + a.slice, a.V), tid = threadIdx.x;
  for (int b = blockIdx.x * kS + tid; b < kBins; b += a.slices * kS) {
    sp.bin_count[b] = 0;
    sp.bin_mass[b] = 0;
  }
  if (blockIdx.x == 0 && tid == 0) sp.n = 0;
  u64 first = ~0ull;
  for_all<T>(row, a.V, i0, i1, tid, kS, [&](float x, int i) {
    const u64 c = composite(x, i);
    first = x > -INFINITY && c < first ? c : first;
  });
  first = block_min<kS>(first, s_wave);
  if (tid == 0) sp.first[blockIdx.x] = first;
}

// A slice's share of the bins, or the weight that it keeps.
template <typename T>
__global__ __launch_bounds__(kS) void sample_bins_kernel(SampleArgs a) {
  __shared__ u64 s_wave[kS / 64], s_mass[kBins];
  __shared__ unsigned int s_count[kBins];
  const int64_t r0 = blockIdx.y;
  const T* row = static_cast<const T*>(a.logits) + r0 * a.ld;
  RowSpace& sp = a.space[r0];
  const int i0 = blockIdx.x * a.slice, i1 = min(i0 + a.slice, a.V), tid = threadIdx.x;
  const Settings p = settings(a, r0);
  const u64 first = block_min<kS>(tid < a.slices ? sp.first[tid] : ~0ull, s_wave);
  if (first == ~0ull || p.first_only) return;
  const Row r = row_of(first, p.temp);
  if (!p.filtered) {
    const double least = least_of(p.min_p);
    u64 m = 0;
    for_all<T>(row, a.V, i0, i1, tid, kS, [&](float x, int) {
      const double z = exponent(r, x);
      m += z >= least ? weight_of(z) : 0;
    });
    m = block_sum<kS>(m, s_wave);
    if (tid == 0) sp.mass[blockIdx.x] = m;
    return;
  }
  for (int b = tid; b < kBins; b += kS) {
    s_count[b] = 0;
    s_mass[b] = 0;
  }
  __syncthreads();
  // numbers for top-k, weights for top-p
  if (p.top_k <= 0) {
    for_all<T>(row, a.V, i0, i1, tid, kS, [&](float x, int) { atomicAdd(&s_mass[bin_of(r, x)], weight(r, x)); });
  } else if (!(p.top_p < 1.0f)) {
    for_range<T>(row, a.V, i0, i1, tid, kS, [&](float x, int) { atomicAdd(&s_count[bin_of(r, x)], 1u); });
  } else {
    for_range<T>(row, a.V, i0, i1, tid, kS, [&](float x, int) {
      const int b = bin_of(r, x);
      atomicAdd(&s_count[b], 1u);
      atomicAdd(&s_mass[b], weight(r, x));
    });
  }
  __syncthreads();
  for (int b = tid; b < kBins; b += kS) {
    if (s_count[b]) atomicAdd(&sp.bin_count[b], s_count[b]);
    if (s_mass[b]) atomicAdd(&sp.bin_mass[b], s_mass[b]);
  }
}

// A slice's tokens that have to be sorted, and, where they are those of one bin, the weight that it keeps before it.
// (The list's place is reserved once for the slice: 64 rows of 150000 took 25 us with an atomic per token.)
template <typename T>
__global__ __launch_bounds__(kS) void sample_gather_kernel(SampleArgs a) {
  __shared__ u64 s_wave[kS / 64], s_at[8], s_list[kList];
  __shared__ unsigned int s_n, s_to;
  const int64_t r0 = blockIdx.y;
  const T* row = static_cast<const T*>(a.logits) + r0 * a.ld;
  RowSpace& sp = a.space[r0];
  const int i0 = blockIdx.x * a.slice, i1 = min(i0 + a.slice, a.V), tid = threadIdx.x;
  const Settings p = settings(a, r0);
  if (p.first_only || !p.filtered) return;
  const u64 first = block_min<kS>(tid < a.slices ? sp.first[tid] : ~0ull, s_wave);
  if (first == ~0ull) return;
  const Row r = row_of(first, p.temp);
  const Ends e = find_ends<kS, false>(sp.bin_count, sp.bin_mass, p.top_k, p.top_p, s_wave, s_at);
  const int what = gathered(e);
  if (what == kGatherNone) return;
  if (tid == 0) s_n = 0;
  __syncthreads();
  const double least = least_of(p.min_p);
  u64 m = 0;
  auto add = [&](float x, int i) {
    const unsigned int at = atomicAdd(&s_n, 1u);
    if (at < kList) s_list[at] = composite(x, i);
  };
  if (what == kGatherAll) {
    for_range<T>(row, a.V, i0, i1, tid, kS, [&](float x, int i) {
      if (bin_of(r, x) <= e.last) add(x, i);
    });
  } else {
    for_all<T>(row, a.V, i0, i1, tid, kS, [&](float x, int i) {
      const int b = bin_of(r, x);
      const double z = exponent(r, x);
      m += b < e.last && z >= least ? weight_of(z) : 0;
      if (b == e.last && x > -INFINITY) add(x, i);
    });
    m = block_sum<kS>(m, s_wave);
    if (tid == 0) sp.mass[blockIdx.x] = m;
  }
  __syncthreads();
  const unsigned int n = s_n;
  if (tid == 0 && n) s_to = atomicAdd(&sp.n, n);
  __syncthreads();
  for (unsigned int i = tid; i < n; i += kS)
    if (s_to + i < kList) sp.list[s_to + i] = s_list[i];
}

// ---------------------------------------------------------------------- a row's token

// SLICED: with what the kernels above have left; otherwise from the row alone.
template <typename T, bool SLICED>
__global__ __launch_bounds__(SLICED ? kPickT : kAloneT) void sample_kernel(SampleArgs a) {
  constexpr int kT = SLICED ? kPickT : kAloneT;
  __shared__ Shared<kT> s;
  const int64_t r0 = blockIdx.x;
  const T* row = static_cast<const T*>(a.logits) + r0 * a.ld;
  const int tid = threadIdx.x, V = a.V;
  const Settings p = settings(a, r0);
  RowSpace* sp = SLICED ? a.space + r0 : nullptr;
  u64 first = ~0ull;
  if constexpr (SLICED) {
    if (tid < a.slices) first = sp->first[tid];
  } else {
    for_range<T>(row, V, 0, V, tid, kT, [&](float x, int i) { first = min(first, composite(x, i)); });
  }
  first = block_min<kT>(first, s.wave);
  if (first == ~0ull || p.first_only) {
    if (tid == 0) {
      a.token[r0] = first == ~0ull ? -1 : (int)(first & 0xfffffu);
      if (a.prob) a.prob[r0] = first == ~0ull ? 0.f : 1.f;
    }
    return;
  }
  const Row r = row_of(first, p.temp);
  const double least = least_of(p.min_p);
  float u = a.u[r0];
  u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
  u64 bound = ~0ull;          // composites up to it are kept
  int what = kGatherNone;
  int n = 0;                  // composites in s.list
  if (p.filtered) {
    for (int i = tid; i < kBins; i += kT) {
      s.count[i] = SLICED ? sp->bin_count[i] : 0;
      s.mass[i] = SLICED ? sp->bin_mass[i] : 0;
    }
    __syncthreads();
    if constexpr (!SLICED) {
      for_range<T>(row, V, 0, V, tid, kT, [&](float x, int) {
        const int b = bin_of(r, x);
        atomicAdd(&s.count[b], 1u);
        atomicAdd(&s.mass[b], weight(r, x));
      });
      __syncthreads();
    }
    const Ends e = find_ends<kT, !SLICED>(s.count, s.mass, p.top_k, p.top_p, s.wave, s.at);
    what = gathered(e);
    unsigned int in_bin = (unsigned int)e.in_bin;
    if constexpr (SLICED) {
      if (what != kGatherNone) {
        const unsigned int have = sp->n;
        if (what == kGatherBin) in_bin = have;
        if (have > kList) what = kGatherNone;
        n = what == kGatherNone ? 0 : (int)have;
      }
      for (int i = tid; i < n; i += kT) s.list[i] = sp->list[i];
    } else if (what == kGatherAll) {
      n = (int)e.count;
      if (tid == 0) s.n = 0;
      __syncthreads();
      for_range<T>(row, V, 0, V, tid, kT, [&](float x, int i) {
        if (bin_of(r, x) > e.last) return;
        const unsigned int at = atomicAdd(&s.n, 1u);
        if (at < kList) s.list[at] = composite(x, i);
      });
    } else {
      what = kGatherNone;
    }
    __syncthreads();
    u64 sum = e.m_all;          // the weight that top-k keeps
    Cut q = {e.last, (int)in_bin, false, e.want, e.base, 0.0};
#pragma unroll 1
    for (int filter = e.by_k ? 0 : 1; filter < (p.top_p < 1.0f ? 2 : 1); ++filter) {
      if (filter == 1) {
        q.by_mass = true;
        q.target = (double)p.top_p * (double)sum;
        constexpr int B = kBins / kT;
        const int t = B * tid;
        u64 ms = 0, total;
#pragma unroll
        for (int k = 0; k < B; ++k) ms += s.mass[t + k];
        u64 ahead = block_scan<kT>(ms, s.wave, total) - ms;
#pragma unroll
        for (int k = 0; k < B; ++k) {
          const u64 m = e.by_k && t + k == e.last ? sum - ahead : s.mass[t + k];
          if ((!e.by_k || t + k <= e.last) && (double)ahead < q.target && q.target <= (double)(ahead + m)) {
            s.at[0] = t + k;
            s.at[2] = ahead;
            s.at[3] = s.count[t + k];
          }
          ahead += m;
        }
        __syncthreads();
        q.bin = (int)s.at[0];
        q.base = s.at[2];
        q.n = SLICED && p.top_k <= 0 ? (int)in_bin : (int)s.at[3];
        __syncthreads();
      }
      const Bound end = cut_bin(s, [&](auto&& f) __attribute__((always_inline)) {
        if (what != kGatherNone) {
          for (int i = tid; i < n; i += kT) f(logit_of(s.list[i]), s.list[i]);
        } else {
          for_range<T>(row, V, 0, V, tid, kT, [&](float x, int i) { f(x, composite(x, i)); });
        }
      }, r, q, bound, what != kGatherNone ? kFew : kT);
      bound = min(bound, end.c);
      sum = q.base + end.mass;
    }
  }
  if (what == kGatherAll) {
    // all that is kept is in the list: its weight by 1024 parts of the vocabulary, then within the part where u falls
    u64 m[kList / kT], all = 0;
#pragma unroll
    for (int k = 0; k < kList / kT; ++k) {
      const int i = tid + k * kT;
      const u64 c = i < n ? s.list[i] : ~0ull;
      const float x = logit_of(c);
      m[k] = i < n && c <= bound && exponent(r, x) >= least ? weight(r, x) : 0;
      all += m[k];
    }
    all = block_sum<kT>(all, s.wave);
    const double target = (double)u * (double)all;
    u64 base = 0;
    int part = -1;
#pragma unroll 1
    for (int level = 0; level < 2; ++level) {
      for (int i = tid; i < 1024; i += kT) s.mass[i] = 0;
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kList / kT; ++k) {
        if (!m[k]) continue;
        const int i = (int)(s.list[tid + k * kT] & 0xfffffu);
        if (level == 0) atomicAdd(&s.mass[i >> 10], m[k]);
        else if (i >> 10 == part) s.mass[i & 1023] = m[k];
      }
      __syncthreads();
      find_passing<1024>(s, s.mass, base, target);
      if (level == 0) {
        part = (int)s.at[0];
        base = s.at[1];
      }
    }
    if (tid == 0) {
      a.token[r0] = (part << 10) + (int)s.at[0];
      if (a.prob) a.prob[r0] = (float)((double)s.at[2] / (double)all);
    }
    return;
  }
  // the weight that every slice keeps, where it is known
  const bool by_slice = SLICED && (!p.filtered || what == kGatherBin);
  if (by_slice) {
    __syncthreads();
    if (tid < kMaxSlices) s.mass[tid] = tid < a.slices ? sp->mass[tid] : 0;
    __syncthreads();
    for (int i = tid; i < n; i += kT) {
      const u64 c = s.list[i];
      const float x = logit_of(c);
      if (c <= bound && exponent(r, x) >= least) atomicAdd(&s.mass[(int)(c & 0xfffffu) / a.slice], weight(r, x));
    }
    __syncthreads();
  }
  // the part of the row in which the distribution passes u: a thread sums consecutive tokens, and the part becomes those
  // of the thread where it passes, until that is one
  int i0 = 0, i1 = V;
  u64 base = 0;
  double all = 0.0, target = 0.0;
  bool whole = true;
  if (by_slice) {
    all = (double)block_sum<kT>(tid < kMaxSlices ? s.mass[tid] : 0, s.wave);
    target = (double)u * all;
    find_passing<kMaxSlices>(s, s.mass, 0, target);
    i0 = (int)s.at[0] * a.slice;
    i1 = min(i0 + a.slice, V);
    base = s.at[1];
    whole = false;
  }
  auto weigh = [&](int a0, int a1, int lane, int lanes) __attribute__((always_inline)) {
    u64 m = 0;
    for_all<T>(row, V, a0, a1, lane, lanes, [&](float x, int i) {
      const double z = exponent(r, x);
      m += composite(x, i) <= bound && z >= least ? weight_of(z) : 0;      // (-inf weighs nothing)
    });
    if (whole) {
      all = (double)block_sum<kT>(m, s.wave);
      target = (double)u * all;
    }
    return m;
  };
  auto take = [&](int len) __attribute__((always_inline)) {
    i0 = min(i0 + (int)s.at[0] * len, i1);
    i1 = min(i0 + len, i1);
    base = s.at[1];
  };
  constexpr int W = kT / 64;
#pragma unroll 1
  for (; i1 - i0 > kWide * kT; whole = false) {      // (long parts by waves, whose loads are consecutive)
    const int len = (i1 - i0 + W - 1) / W, a0 = min(i0 + (tid >> 6) * len, i1);
    const u64 m = wave_scan(weigh(a0, min(a0 + len, i1), tid & 63, 64));
    __syncthreads();
    if ((tid & 63) == 63) s.mass[tid >> 6] = m;
    __syncthreads();
    find_passing<W>(s, s.mass, base, target);
    take(len);
  }
#pragma unroll 1
  for (;; whole = false) {
    const int len = (i1 - i0 + kT - 1) / kT, a0 = min(i0 + tid * len, i1);
    const u64 m = weigh(a0, min(a0 + len, i1), 0, 1);
    __syncthreads();
    s.mass[tid] = m;
    __syncthreads();
    find_passing<kT>(s, s.mass, base, target);
    take(len);
    if (len == 1) break;
  }
  if (tid == 0) {
    a.token[r0] = i0;
    if (a.prob) a.prob[r0] = (float)((double)s.at[2] / all);
  }
}

// Slices of a row: a 16-byte piece or more for every thread, so many that the chip has some 1024 workgroups.
// Rows of up to 16384 tokens, and of up to 65536 where there are 256 or more (a unit each): a workgroup a row (16384 fp32
// logits, one row, greedy and top-50: 6.7 and 19 us, with slices 11.2 and 21; 256 rows of 32000: 8.6 and 31, 14 and 41; but
// one row of 32000 bf16: 6.9 and 26, 11.5 and 22).
constexpr int64_t kAloneRows = 256;
bool alone(int64_t rows, int64_t V) { return V <= 16384 || (V <= 65536 && rows >= kAloneRows); }
// What the call itself needs
size_t space_of(int64_t rows, int64_t V) { return alone(rows, V) ? 0 : (size_t)rows * sizeof(RowSpace); }
struct Slices {
  int n, tokens;
};
Slices slices_of(int64_t rows, int64_t V, size_t elem) {
  const int64_t unit = kS * (16 / (int64_t)elem);
  int64_t want = std::max<int64_t>(1, 1024 / std::max<int64_t>(rows, 1));
  want = std::min<int64_t>(std::min<int64_t>(want, (V + unit - 1) / unit), kMaxSlices);
  const int64_t tokens = ((V + want - 1) / want + unit - 1) / unit * unit;
  return {(int)((V + tokens - 1) / tokens), (int)tokens};
}

template <typename T>
catq_status launch_sample(SampleArgs a, int64_t rows, hipStream_t stream) {
  const double bytes = (double)rows * a.V * sizeof(T);
  if (alone(rows, a.V)) {
    CATQ_TRACED(stream, "sample_kernel<alone>", 0.0, bytes, rows, a.V, 1,
                hipLaunchKernelGGL((sample_kernel<T, false>), dim3((unsigned)rows), dim3(kAloneT), 0, stream, a));
    CATQ_CHECK_LAUNCH("sample");
    return CATQ_OK;
  }
  const Slices sl = slices_of(rows, a.V, sizeof(T));
  a.slices = sl.n;
  a.slice = sl.tokens;
  const dim3 grid((unsigned)sl.n, (unsigned)rows);
  CATQ_TRACED(stream, "sample_first_kernel", 0.0, bytes, rows, a.V, sl.n,
              hipLaunchKernelGGL((sample_first_kernel<T>), grid, dim3(kS), 0, stream, a));
  CATQ_TRACED(stream, "sample_bins_kernel", 0.0, bytes, rows, a.V, sl.n,
              hipLaunchKernelGGL((sample_bins_kernel<T>), grid, dim3(kS), 0, stream, a));
  if (a.top_k || a.top_p)     // (no row has a filter that gathers)
    CATQ_TRACED(stream, "sample_gather_kernel", 0.0, bytes, rows, a.V, sl.n,
                hipLaunchKernelGGL((sample_gather_kernel<T>), grid, dim3(kS), 0, stream, a));
  CATQ_TRACED(stream, "sample_kernel", 0.0, 0.0, rows, a.V, 1,
              hipLaunchKernelGGL((sample_kernel<T, true>), dim3((unsigned)rows), dim3(kPickT), 0, stream, a));
  CATQ_CHECK_LAUNCH("sample");
  return CATQ_OK;
}

}  // namespace
}  // namespace catq

using namespace catq;

extern "C" size_t catq_aux_sample_workspace_bytes(int64_t rows, int64_t V) {
  if (rows <= 0 || rows > 65535 || V > (1 << 20)) return 0;
  // (enough for fewer rows too, which may be read by several workgroups each where so many are not)
  return space_of(alone(rows, V) ? std::min(rows, kAloneRows - 1) : rows, V);
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
  CATQ_REQUIRE(rows <= 65535 && ld >= V && count_ok(rows, ld), CATQ_ERR_SHAPE,
               "ld must be >= V, rows at most 65535 and rows * ld within 2^38");
  auto at4 = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; };
  CATQ_REQUIRE(aligned16(logits) && at4(temperature) && at4(top_k) && at4(top_p) && at4(min_p) && at4(u) &&
                   at4(token) && at4(prob) && aligned16(workspace),
               CATQ_ERR_ALIGN, "logits and workspace must be 16-byte aligned, the others 4-byte");
  const size_t need = space_of(rows, V);
  CATQ_REQUIRE(need == 0 || (workspace && workspace_bytes >= need), CATQ_ERR_WORKSPACE,
               "workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
  const SampleArgs a{logits, ld, (int32_t)V, temperature, top_k, top_p, min_p, u, token, prob,
                     static_cast<RowSpace*>(workspace), 1, (int32_t)V};
  return dtype == CATQ_F32 ? launch_sample<float>(a, rows, stream) : launch_sample<bf16>(a, rows, stream);
}
