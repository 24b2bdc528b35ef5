// Sampling of tokens from vocabulary logits: temperature, top-k, top-p, min-p, given random numbers.
//
// The tokens of a row are ordered by (logit descending, id ascending); w = exp((z - max z) / T).  top_k keeps the first k of the order,
// top_p of those the shortest prefix with at least top_p of their mass, min_p of those the tokens with w >= min_p: all three keep
// a prefix, so what is kept is a prefix.  The token is the first one, by id, whose cumulative kept mass exceeds u times the kept mass.
//
// Which token that is hangs on borders between masses, and there are as many borders as tokens.  So masses are whole numbers: w in
// units of 2^-42, rounded once, and added in 64 bits.  Sums then depend on no order, atomics included, the borders are where they would be in
// exact arithmetic on those w, and w itself is good to about one unit in its last place (weight()).
#include <algorithm>
#include <cmath>

#include "focus_common.h"
#include "focus_kernels.h"

namespace focus {

constexpr int kMassBits = 42;
static_assert(((uint64_t)kSampleMaxVocab << kMassBits) <= ((uint64_t)1 << 63), "the mass of a row fits");

// ---- logits
// as a float32: NaN counts as -inf, +inf as the largest number, -0 as +0
__device__ __forceinline__ float clean(float z) { return z == z ? fminf(z, 3.402823466e38f) + 0.f : -INFINITY; }
// whole numbers in the order of the numbers
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }
constexpr uint32_t kKeyNone = 0x007fffffu;  // key_of(-inf)

// One 16-byte chunk of a row: E consecutive logits from id E * chunk on; ids past the vocabulary give -inf.
template <class T>
struct Chunk {
  static constexpr int E = 16 / sizeof(T);
  float z[E];
};
template <class T>
__device__ __forceinline__ void load_chunk(Chunk<T>& x, const T* row, int chunk, int vocab) {
  constexpr int E = Chunk<T>::E;
  const int i0 = chunk * E;
  if (i0 + E <= vocab) {
    const uint4 w = *reinterpret_cast<const uint4*>(row + i0);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < E; ++e)
      x.z[e] = clean(sizeof(T) == 4 ? __uint_as_float(u[e & 3]) : ((e & 1) ? bf16_hi(u[(e >> 1) & 3]) : bf16_lo(u[(e >> 1) & 3])));
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float z = -INFINITY;
      if (i0 + e < vocab) z = sizeof(T) == 4 ? *reinterpret_cast<const float*>(row + i0 + e) : bf16_lo(*reinterpret_cast<const uint16_t*>(row + i0 + e));
      x.z[e] = clean(z);
    }
  }
}

// ---- masses
// (1 / T) log2(e) as a sum of two floats
struct Scale {
  float hi, lo;
};
__device__ __forceinline__ Scale scale_of(float temperature) {
  const double c = fmin(1.4426950408889634 / (double)temperature, 3e38);
  Scale s;
  s.hi = (float)c;
  s.lo = (float)(c - (double)s.hi);
  return s;
}
// 2^-((top - z) * s): the difference and the product are taken with what their roundings leave over (of a difference of 20 and more that
// would be ten units of the result's last place), which enters as a factor 1 + r ln 2
__device__ __forceinline__ float weight(float z, float top, const Scale& s) {
  const float d = top - z;
  const float b = top - d;
  const float rest = (top - (d + b)) + (b - z);  // top - z = d + rest
  const float x = d * s.hi;
  const float r = __builtin_fmaf(d, s.hi, -x) + __builtin_fmaf(d, s.lo, rest * s.hi);
  const float w = __builtin_amdgcn_exp2f(-x);
  return x < 60.f ? __builtin_fmaf(w * -0.6931471805599453f, r, w) : 0.f;
}
__device__ __forceinline__ uint64_t mass_of(float w) {  // w <= 1 in units of 2^-42, to nearest
  const float high = truncf(w * 1024.f);                // units of 2^-10
  const float low = rintf(__builtin_fmaf(w, 1024.f, -high) * 4294967296.f);  // the rest, below 2^32 + 1
  return ((uint64_t)(uint32_t)high << 32) + (uint64_t)low;
}
__device__ __forceinline__ uint64_t mass(float z, float top, const Scale& s) { return mass_of(weight(z, top, s)); }

// ---- sums over a workgroup of THREADS; every thread receives the result.  `sh`: THREADS / 64 words.
__device__ __forceinline__ uint64_t shfl_xor64(uint64_t v, int o) {
  const uint32_t lo = (uint32_t)__shfl_xor((int)(uint32_t)v, o, kWave), hi = (uint32_t)__shfl_xor((int)(uint32_t)(v >> 32), o, kWave);
  return ((uint64_t)hi << 32) | lo;
}
template <int THREADS, class Op>
__device__ __forceinline__ uint64_t block_reduce64(uint64_t v, uint64_t* sh, const Op op) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = op(v, shfl_xor64(v, o));
  __syncthreads();  // sh may still be read from a previous call
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  v = sh[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) v = op(v, sh[w]);
  return v;
}
struct Add64 {
  __device__ __forceinline__ uint64_t operator()(uint64_t a, uint64_t b) const { return a + b; }
};
struct Max64 {
  __device__ __forceinline__ uint64_t operator()(uint64_t a, uint64_t b) const { return a > b ? a : b; }
};

struct SampleArgs {
  const void* logits;
  int64_t row_stride;
  const uint8_t* masked;
  const float* uniform;
  const float* temperature;  // [n_rows] or null, like the next three
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int n_rows, vocab;
  int32_t* tokens;
  float* conf;
  float* prob;
};
struct RowParams {
  float temperature, top_p, min_p, u;
  int top_k;
};
__device__ __forceinline__ RowParams row_params(const SampleArgs& a, int row) {
  RowParams p;
  p.temperature = a.temperature ? a.temperature[row] : 1.f;
  p.top_p = a.top_p ? a.top_p[row] : 1.f;
  p.min_p = a.min_p ? a.min_p[row] : 0.f;
  p.top_k = a.top_k ? a.top_k[row] : 0;
  p.u = fmaxf(a.uniform[row], 0.f);  // NaN: 0
  return p;
}
__device__ __forceinline__ void write_row(const SampleArgs& a, int row, int token, float conf, float prob) {
  a.tokens[row] = token;
  if (a.conf) a.conf[row] = conf;
  if (a.prob) a.prob[row] = prob;
}
// the smallest key that min_p keeps: w >= min_p <=> z >= top + T ln(min_p)
__device__ __forceinline__ uint32_t min_p_key(float min_p, float temperature, float top) {
  if (!(min_p > 0.f)) return 0u;
  if (min_p >= 1.f) return key_of(top);
  const double cut = (double)top + (double)temperature * log((double)min_p);
  float z = (float)cut;
  if ((double)z < cut) z = of_key(key_of(z) + 1u);
  return key_of(clean(z));
}

// The whole row by one workgroup that walks it as often as it takes: the order is searched bit by bit.  What is kept is
// {key > cut} and of {key == cut} the ids up to `last_id`.
constexpr int kRowThreads = 1024;
template <class T>
__global__ __launch_bounds__(kRowThreads) void sample_row_kernel(const SampleArgs a) {
  constexpr int E = Chunk<T>::E;
  __shared__ uint64_t sh[kRowThreads / 64], sh2[kRowThreads / 64];
  __shared__ uint64_t wave_mass[kRowThreads / 64];
  __shared__ int found_sh;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (a.masked != nullptr && a.masked[row] == 0) {
    if (tid == 0) write_row(a, row, -1, 0.f, 0.f);
    return;
  }
  const T* z = static_cast<const T*>(a.logits) + (int64_t)row * a.row_stride;
  const int n_chunks = (a.vocab + E - 1) / E;
  const RowParams p = row_params(a, row);
  auto each = [&](auto&& f) {  // f(id, logit) over the row
    for (int ch = tid; ch < n_chunks; ch += kRowThreads) {
      Chunk<T> x;
      load_chunk(x, z, ch, a.vocab);
#pragma unroll
      for (int e = 0; e < E; ++e) f(ch * E + e, x.z[e]);
    }
  };
  // the first of the order
  uint64_t best = 0;
  each([&](int id, float v) {
    const uint64_t k = ((uint64_t)key_of(v) << 32) | (uint32_t)~id;
    best = k > best ? k : best;
  });
  best = block_reduce64<kRowThreads>(best, sh, Max64());
  const uint32_t top_key = (uint32_t)(best >> 32);
  const int first_id = (int)~(uint32_t)best;
  if (top_key <= kKeyNone) {  // no number in the row
    if (tid == 0) write_row(a, row, -1, 0.f, 0.f);
    return;
  }
  const float top = of_key(top_key);
  const Scale s1 = scale_of(1.f);
  const bool greedy = !(p.temperature > 0.f);
  const Scale s = scale_of(greedy ? 1.f : p.temperature);
  uint64_t all1 = 0, all = 0;
  each([&](int, float v) {
    all1 += mass(v, top, s1);
    all += mass(v, top, s);
  });
  all1 = block_reduce64<kRowThreads>(all1, sh, Add64());
  all = block_reduce64<kRowThreads>(all, sh2, Add64());
  const double unit = 1.0 / (double)((uint64_t)1 << kMassBits);
  const double denom = (double)all1 * unit;
  if (greedy) {
    if (tid == 0) write_row(a, row, first_id, (float)(1.0 / denom), 1.f);
    return;
  }
  auto at_least = [&](uint32_t key, uint64_t& count, uint64_t& sum) {  // of the tokens with this key or a larger one
    uint64_t c = 0, m = 0;
    each([&](int, float v) {
      if (key_of(v) >= key && key_of(v) > kKeyNone) {
        ++c;
        m += mass(v, top, s);
      }
    });
    count = block_reduce64<kRowThreads>(c, sh, Add64());
    sum = block_reduce64<kRowThreads>(m, sh2, Add64());
  };
  // kept so far: keys above `cut`, and the first `ties` tokens with it
  uint32_t cut = kKeyNone + 1u;
  uint64_t ties = ~(uint64_t)0, kept = all, count, sum;
  auto search = [&](auto&& enough) {  // the largest key with enough(count, mass of the tokens down to it)
    uint32_t k = 0;
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t t = k | (1u << bit);
      if (t > top_key) continue;
      at_least(t, count, sum);
      if (enough(count, sum)) k = t;
    }
    return k;
  };
  if (p.top_k > 0) {
    const uint64_t k = (uint64_t)p.top_k;
    const uint32_t c = max(search([&](uint64_t n, uint64_t) { return n >= k; }), kKeyNone + 1u);
    at_least(c + 1u, count, sum);
    if (count < k) {  // (else: fewer than k numbers in the row)
      const uint64_t n_above = count, m_above = sum;
      at_least(c, count, sum);
      cut = c;
      ties = min(k, count) - n_above;
      kept = m_above + ties * mass(of_key(c), top, s);
    }
  }
  if (p.top_p < 1.f) {
    const double target = (double)p.top_p * (double)kept;
    const uint32_t c = max(search([&](uint64_t, uint64_t m) { return (double)m >= target; }), kKeyNone + 1u);
    at_least(c + 1u, count, sum);
    const uint64_t w = mass(of_key(c), top, s), above = sum;
    uint64_t n = 1;  // the j-th token with this key is kept where above + (j - 1) w < target
    if (w > 0) {
      n = (uint64_t)fmax(floor((target - (double)above) / (double)w), 0.0);
      while ((double)(above + n * w) < target) ++n;
      while (n > 1 && !((double)(above + (n - 1) * w) < target)) --n;
      n = n < 1 ? 1 : n;
    }
    if (c > cut || (c == cut && n < ties)) {
      cut = c;
      ties = n;
    }
  }
  const uint32_t m_key = min(min_p_key(p.min_p, p.temperature, top), top_key);
  if (m_key > cut) {
    cut = m_key;
    ties = p.min_p > 1.f ? 1 : ~(uint64_t)0;
  } else if (m_key == cut && p.min_p > 1.f) {
    ties = 1;
  }
  int last_id = a.vocab;
  if (ties != ~(uint64_t)0) {  // the largest id up to which at most `ties` tokens have the key
    int id = -1;
    for (int bit = 30; bit >= 0; --bit) {
      const int t = id + (1 << bit);
      if (t >= a.vocab || t < 0) continue;
      uint64_t c = 0;
      each([&](int i, float v) { c += key_of(v) == cut && i <= t; });
      if (block_reduce64<kRowThreads>(c, sh, Add64()) <= ties) id = t;
    }
    last_id = id;
  }
  // masses by id: rounds of the workgroup, then wavefronts, lanes, logits
  auto held = [&](int id, float v) {
    const uint32_t k = key_of(v);
    return k > cut || (k == cut && id <= last_id) ? mass(v, top, s) : 0;
  };
  uint64_t total = 0;
  each([&](int id, float v) { total += held(id, v); });
  total = block_reduce64<kRowThreads>(total, sh, Add64());
  const double want = (double)p.u * (double)total;
  if (tid == 0) found_sh = -1;
  uint64_t base = 0;
  for (int c0 = 0; c0 < n_chunks; c0 += kRowThreads) {
    uint64_t m[E], mine = 0;
    Chunk<T> x;
    const int ch = c0 + tid;
    if (ch < n_chunks) load_chunk(x, z, ch, a.vocab);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      m[e] = ch < n_chunks ? held(ch * E + e, x.z[e]) : 0;
      mine += m[e];
    }
    uint64_t before = mine;  // inclusive over the wavefront, then exclusive over the workgroup
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const uint32_t lo = (uint32_t)__shfl_up((int)(uint32_t)before, o, kWave), hi = (uint32_t)__shfl_up((int)(uint32_t)(before >> 32), o, kWave);
      if (lane >= o) before += ((uint64_t)hi << 32) | lo;
    }
    __syncthreads();
    if (lane == 63) wave_mass[wave] = before;
    __syncthreads();
    uint64_t round = 0;
    before += base - mine;
    for (int w = 0; w < kRowThreads / 64; ++w) {
      if (w < wave) before += wave_mass[w];
      round += wave_mass[w];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {  // (the last token with a mass takes what rounding leaves)
      const uint64_t after = before + m[e];
      if (m[e] > 0 && (double)before <= want && (!((double)after <= want) || after == total)) {
        atomicMax(&found_sh, ch * E + e);
      }
      before = after;
    }
    base += round;
  }
  __syncthreads();
  const int token = found_sh;
  if (tid == 0) {
    const float v = token < 0 ? top : clean(sizeof(T) == 4 ? reinterpret_cast<const float*>(z)[token] : bf16_lo(reinterpret_cast<const uint16_t*>(z)[token]));
    const double w1 = weight(v, top, s1), w = weight(v, top, s);
    write_row(a, row, token < 0 ? first_id : token, (float)(w1 / denom), (float)(w / ((double)total * unit)));
  }
}

size_t sample_tokens_workspace(int, int) { return 256; }

hipError_t launch_sample_tokens(const void* logits, int dtype, int64_t row_stride, const uint8_t* masked, const float* uniform, const float* temperature,
                                const int32_t* top_k, const float* top_p, const float* min_p, int n_rows, int vocab, int32_t* tokens, float* conf,
                                float* prob, void*, hipStream_t st) {
  const SampleArgs a = {logits, row_stride, masked, uniform, temperature, top_k, top_p, min_p, n_rows, vocab, tokens, conf, prob};
  if (dtype == FOCUS_F32)
    hipLaunchKernelGGL(sample_row_kernel<float>, dim3(n_rows), dim3(kRowThreads), 0, st, a);
  else
    hipLaunchKernelGGL(sample_row_kernel<uint16_t>, dim3(n_rows), dim3(kRowThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace focus
