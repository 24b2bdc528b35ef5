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
// 2^-((top - z) * s): the product is taken with what its rounding leaves over (of a difference of 20 and more that would be ten units of
// the result's last place), which enters as a factor 1 + r ln 2; so is the difference, unless the logits are bf16, whose differences
// from `top` are float32 numbers but for logits of less than 2^-16 of it.
template <bool BF16>
__device__ __forceinline__ float weight(float z, float top, const Scale& s) {
  const float d = top - z;
  const float x = d * s.hi;
  float r = d * s.lo;
  if (!BF16) {
    const float b = top - d;
    r = __builtin_fmaf((top - (d + b)) + (b - z), s.hi, r);  // top - z = d + that
  }
  r += __builtin_fmaf(d, s.hi, -x);
  const float w = __builtin_amdgcn_exp2f(-x);
  return x < 60.f ? __builtin_fmaf(w * -0.6931471805599453f, r, w) : 0.f;
}
// w < 2^22 in units of 2^-42, to nearest.  Both halves are whole numbers of 32 bits: what is left of w 2^10 has 24 bits and is below 1.
__device__ __forceinline__ uint64_t mass_of(float w) {
  const float x = w * 1024.f;
  const uint32_t high = (uint32_t)x;
  return ((uint64_t)high << 32) | (uint32_t)rintf((x - (float)high) * 4294967296.f);
}
template <bool BF16>
__device__ __forceinline__ uint64_t mass(float z, float top, const Scale& s) {
  return mass_of(weight<BF16>(z, top, s));
}

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
  if (p.top_k == 1 || p.top_p <= 0.f || p.min_p > 1.f) p.temperature = 0.f;  // only the first stays
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
// {key > cut} and of {key == cut} the ids up to `last_id`.  For the rows that the lists below do not hold (hundreds of microseconds).
constexpr int kRowThreads = 1024;
template <class T>
__device__ void search_row(const SampleArgs& a, int row, uint64_t* sh, uint64_t* sh2, uint64_t* wave_mass, int* found) {
  constexpr int E = Chunk<T>::E;
  constexpr bool BF16 = sizeof(T) == 2;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
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
    all1 += mass<BF16>(v, top, s1);
    all += mass<BF16>(v, top, s);
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
        m += mass<BF16>(v, top, s);
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
      kept = m_above + ties * mass<BF16>(of_key(c), top, s);
    }
  }
  if (p.top_p < 1.f) {
    const double target = (double)p.top_p * (double)kept;
    const uint32_t c = max(search([&](uint64_t, uint64_t m) { return (double)m >= target; }), kKeyNone + 1u);
    at_least(c + 1u, count, sum);
    const uint64_t w = mass<BF16>(of_key(c), top, s), above = sum;
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
    ties = ~(uint64_t)0;
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
    return k > cut || (k == cut && id <= last_id) ? mass<BF16>(v, top, s) : 0;
  };
  uint64_t total = 0;
  each([&](int id, float v) { total += held(id, v); });
  total = block_reduce64<kRowThreads>(total, sh, Add64());
  const double want = (double)p.u * (double)total;
  if (tid == 0) (*found) = -1;
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
        atomicMax(found, ch * E + e);
      }
      before = after;
    }
    base += round;
  }
  __syncthreads();
  const int token = (*found);
  if (tid == 0) {
    const float v = token < 0 ? top : clean(sizeof(T) == 4 ? reinterpret_cast<const float*>(z)[token] : bf16_lo(reinterpret_cast<const uint16_t*>(z)[token]));
    const double w1 = weight<BF16>(v, top, s1), w = weight<BF16>(v, top, s);
    write_row(a, row, token < 0 ? first_id : token, (float)(w1 / denom), (float)(w / ((double)total * unit)));
  }
}

// =====================================================================================================
// The ordinary way: three launches, the first two with a workgroup per slice of a row.
//   sample_scan_kernel   the slice's largest logit and weights, and a histogram of the order: bins of 1/16 in logit / T, counts and
//                        masses.  Bins are counted from zero logit up (floor(z * bins per unit)), so that those of all slices are the
//                        same; a bin kBins and more below the largest logit's has no mass.
//   sample_cut_kernel    from the row's histogram the bins in which top_k and top_p end.  Tokens above them are kept whatever comes:
//                        their masses are summed per segment of 64 chunks.  Tokens in them are listed.
//   sample_pick_kernel   a workgroup per row orders the list, finds the end of what is kept in it, adds the kept ones to their segments, and
//                        walks down: segment, chunk, token.
// The row is read twice, the second time from a cache.  The histogram only says where to look: ends are decided by the weights, and
// everything that workgroups add up in no order is a whole number.  A chunk's weights are added as floats, in order, and the sum is rounded
// to a mass once.  Where the lists do not hold the tokens of a bin, or the bins do not resolve the logits (2^18 and more, at T = 1), the
// last launch searches the row instead.
// =====================================================================================================
constexpr int kBins = 512;
constexpr int kScanThreads = 512;
constexpr int kSlice = 32 * kScanThreads, kSliceSmall = 8 * kScanThreads;  // logits of a workgroup
constexpr int kSliceList = 2048, kRowList = 4096;                          // entries of a slice, of a row
constexpr int kSegChunks = 64;
constexpr int kMaxSlices = kSampleMaxVocab / kSlice;
constexpr float kMostBin = 4194304.f;                       // beyond, floats would not hold bin numbers and their neighbours
constexpr float kBinsPerNat = 16.f, kMostPerUnit = 8192.f;  // bins per unit of logit: kBinsPerNat / T at T > 1 / 512

struct SliceStat {
  float top;   // -inf: no number
  int id;      // the first with it
  double at1;  // sum of the weights at T = 1 and at T, relative to `top`
  double atT;
};
// Where a row is cut.
struct RowCut {
  float top;
  int first_id;
  int way;                         // kNone, kFirst, kDraw, kSearch
  double at1, atT;                 // sum of the weights at T = 1 and at T
  int ends;                        // 0: nothing is cut but by min_p; else the list decides
  float sure;                      // logits from here on are kept
  float least;                     // min_p: none below this one
  uint32_t least_key;
  float p_low, k_high, k_low;      // the list: [p_low, sure) and [k_low, k_high), where top_k ends apart from top_p
  bool apart;
  uint32_t count_sure, count_k;    // tokens above `sure`, above k_high
};
enum { kNone = 0, kFirst = 1, kDraw = 2, kSearch = 3 };
struct SampleWs {
  SliceStat* stat;   // [rows, slices]
  uint64_t* bins;    // [rows, slices, kBins]  tokens in the upper half, their masses above that of the bin's lower end in the lower half
  uint64_t* middle;  // [rows, slices]  mass between the two parts of the list
  uint32_t* listed;  // [rows, slices]
  uint64_t* list;    // [rows, slices, kSliceList]  order_of() each
  RowCut* cut;       // [rows]
  uint64_t* seg;     // [rows, segments]
  int slices, segs;
};
__device__ __forceinline__ uint64_t order_of(uint32_t key, int id) { return ((uint64_t)~key << 32) | (uint32_t)id; }  // ascending: first to last
__device__ __forceinline__ uint32_t key_in(uint64_t order) { return ~(uint32_t)(order >> 32); }
__device__ __forceinline__ float bins_per_unit(float temperature) { return fminf(kBinsPerNat / temperature, kMostPerUnit); }
constexpr double kMassUnit = 1.0 / (double)((uint64_t)1 << kMassBits);
__device__ __forceinline__ bool needs_order(const RowParams& p) { return p.top_k > 0 || p.top_p < 1.f; }
template <class T>
__device__ __forceinline__ float logit_at(const void* row, int id) {
  return clean(sizeof(T) == 4 ? static_cast<const float*>(row)[id] : bf16_lo(static_cast<const uint16_t*>(row)[id]));
}

template <class T, int SLICE>
__global__ __launch_bounds__(kScanThreads) void sample_scan_kernel(const SampleArgs a, const SampleWs ws, int row0) {
  constexpr int E = Chunk<T>::E, N = SLICE / E / kScanThreads, kCopies = 4, kWaves = kScanThreads / 64;
  constexpr bool BF16 = sizeof(T) == 2;
  __shared__ unsigned long long bins_sh[kCopies][kBins];
  __shared__ float top_sh[kWaves];
  __shared__ double at1_sh[kWaves], atT_sh[kWaves];
  __shared__ int id_sh;
  const int slice = blockIdx.x, r = blockIdx.y, row = row0 + r, tid = threadIdx.x;
  if (a.masked != nullptr && a.masked[row] == 0) return;
  const T* z = static_cast<const T*>(a.logits) + (int64_t)row * a.row_stride;
  const int c0 = slice * (SLICE / E) + tid, n_chunks = (a.vocab + E - 1) / E;
  Chunk<T> x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) load_chunk(x[i], z, min(c0 + i * kScanThreads, n_chunks), a.vocab);
  const RowParams p = row_params(a, row);
  const bool drawn = p.temperature > 0.f, order = drawn && needs_order(p);  // uniform over the workgroup
  if (order)
    for (int i = tid; i < kCopies * kBins; i += kScanThreads) (&bins_sh[0][0])[i] = 0;
  if (tid == 0) id_sh = 0x7fffffff;
  float mine = -INFINITY;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) mine = fmaxf(mine, x[i].z[e]);
  float top = mine;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
  if ((tid & 63) == 0) top_sh[tid >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, top_sh[w]);
  SliceStat* stat = ws.stat + (int64_t)r * ws.slices + slice;
  if (top == -INFINITY) {
    if (tid == 0) *stat = SliceStat{top, 0, 0.0, 0.0};
    return;
  }
  if (mine == top) {
    int id = 0x7fffffff;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (x[i].z[e] == top) id = min(id, (c0 + i * kScanThreads) * E + e);
    atomicMin(&id_sh, id);
  }
  float at1 = 0.f, atT = 0.f;
  if (a.conf != nullptr) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) at1 += __builtin_amdgcn_exp2f((x[i].z[e] - top) * 1.4426950408889634f);
  }
  if (order && p.top_p < 1.f) {
    const Scale s = scale_of(p.temperature);
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) atT += weight<BF16>(x[i].z[e], top, s);
  }
  if (order) {
    // exp(f / 16) - 1 = g(f) / 16 for the place f of a token in its bin: 1 + f / 32 + f^2 / 1536 times f, in units of 2^-17
    const float per_unit = bins_per_unit(p.temperature), first = floorf(top * per_unit);
    const int copy = tid & (kCopies - 1);
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float t = x[i].z[e] * per_unit, low = floorf(t), b = first - low;
        if (b < (float)kBins) {
          const float f = t - low;
          const uint32_t g = (uint32_t)(f * __builtin_fmaf(f, __builtin_fmaf(f, 131072.f / 1536.f, 131072.f / 32.f), 131072.f));
          atomicAdd(&bins_sh[copy][(int)b], (1ull << 32) | g);
        }
      }
  }
  double d1 = (double)at1, dT = (double)atT;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    d1 += __shfl_xor(d1, o, kWave);
    dT += __shfl_xor(dT, o, kWave);
  }
  if ((tid & 63) == 0) {
    at1_sh[tid >> 6] = d1;
    atT_sh[tid >> 6] = dT;
  }
  __syncthreads();
  if (tid == 0) {
    d1 = dT = 0.0;
    for (int w = 0; w < kWaves; ++w) {
      d1 += at1_sh[w];
      dT += atT_sh[w];
    }
    *stat = SliceStat{top, id_sh, d1, dT};
  }
  if (order) {
    static_assert(kBins == kScanThreads, "a bin a thread");
    uint64_t v = 0;  // 16384 tokens at most: the lower half holds 16384 * 1.04 * 2^17
#pragma unroll
    for (int i = 0; i < kCopies; ++i) v += bins_sh[i][tid];
    ws.bins[((int64_t)r * ws.slices + slice) * kBins + tid] = v;
  }
}

struct CutShared {
  int shift[4 * kMaxSlices];
  double mass[kBins + 1];  // of the bins in front
  uint32_t count[kBins + 1];
  double wave_mass[kScanThreads / 64];
  uint32_t wave_count[kScanThreads / 64];
  int k_bin, p_lo, p_hi;
};
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}
// the smallest logit of the bins up to `last`: floor(z * per_unit) >= first - last
__device__ __forceinline__ float bin_end(float first, int last, float per_unit) {
  const float n = first - (float)last;
  uint32_t k = key_of(clean(n / per_unit));
  for (int i = 0; i < 4 && floorf(of_key(k) * per_unit) >= n; ++i) --k;
  for (int i = 0; i < 8 && !(floorf(of_key(k) * per_unit) >= n); ++i) ++k;
  return of_key(k);
}
// Every workgroup of the second launch works this out, in the same operations; the third reads it.
__device__ __forceinline__ RowCut cut_row(const SampleWs& ws, int r, const RowParams& p, CutShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const SliceStat* stat = ws.stat + (int64_t)r * ws.slices;
  RowCut c;
  uint64_t best = 0;  // the first of the order, in every wavefront
  for (int i = lane; i < ws.slices; i += kWave) {
    const uint64_t t = ((uint64_t)key_of(stat[i].top) << 32) | (uint32_t)~stat[i].id;
    best = t > best ? t : best;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) best = Max64()(best, shfl_xor64(best, o));
  c.top = of_key((uint32_t)(best >> 32));
  c.first_id = (int)~(uint32_t)best;
  const bool drawn = p.temperature > 0.f;
  const float T = drawn ? p.temperature : 1.f;
  const float per_unit = bins_per_unit(T), first = floorf(c.top * per_unit);
  c.way = !(c.top > -INFINITY) ? kNone : (!drawn ? kFirst : (fabsf(first) <= kMostBin ? kDraw : kSearch));
  c.ends = 0;
  c.apart = false;
  c.least_key = c.way == kDraw ? min_p_key(p.min_p, T, c.top) : 0u;
  c.least = c.least_key > kKeyNone ? of_key(c.least_key) : -INFINITY;
  c.sure = -3.402823466e38f;
  c.p_low = c.k_high = c.k_low = INFINITY;
  c.at1 = c.atT = 0.0;
  c.count_sure = c.count_k = 0;
  if (c.way != kFirst && c.way != kDraw) return c;  // uniform over the workgroup, like the others
  for (int i = lane; i < ws.slices; i += kWave) {
    const SliceStat t = stat[i];
    const double down = (double)t.top - (double)c.top;  // (no number in the slice: -inf)
    const float shift = first - floorf(t.top * per_unit);
    c.at1 += t.at1 * exp(down);
    c.atT += t.atT * exp(down / (double)T);
    if (wave == 0) sh.shift[i] = shift < (float)kBins ? (int)shift : kBins;
  }
  c.at1 = wave_sum(c.at1);
  c.atT = wave_sum(c.atT);
  if (!drawn || !needs_order(p)) return c;
  constexpr int kNoBin = 4 * kBins;
  if (tid == 0) sh.k_bin = sh.p_lo = sh.p_hi = kNoBin;
  __syncthreads();
  uint32_t n = 0;
  uint64_t above = 0;
  for (int i = 0; i < ws.slices; ++i) {
    const int from = tid - sh.shift[i];
    if (from >= 0) {
      const uint64_t v = ws.bins[((int64_t)r * ws.slices + i) * kBins + from];
      n += (uint32_t)(v >> 32);
      above += (uint32_t)v;
    }
  }
  const double m = exp(((double)first - (double)tid - (double)c.top * (double)per_unit) / (double)kBinsPerNat) *
                   ((double)n + (double)above / (131072.0 * (double)kBinsPerNat));
  double im = m;
  uint32_t in = n;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const double om = __shfl_up(im, o, kWave);
    const uint32_t on = __shfl_up(in, o, kWave);
    if (lane >= o) {
      im += om;
      in += on;
    }
  }
  if (lane == 63) {
    sh.wave_mass[wave] = im;
    sh.wave_count[wave] = in;
  }
  __syncthreads();
  for (int w = 0; w < wave; ++w) {
    im += sh.wave_mass[w];
    in += sh.wave_count[w];
  }
  if (tid == 0) {
    sh.mass[0] = 0.0;
    sh.count[0] = 0;
  }
  sh.mass[tid + 1] = im;
  sh.count[tid + 1] = in;
  int k_bin = kNoBin, p_lo = kNoBin, p_hi = kNoBin;
  if (p.top_k > 0) {
    if (in >= (uint32_t)p.top_k && in - n < (uint32_t)p.top_k) sh.k_bin = tid;  // (the counts ascend: one thread at most)
    __syncthreads();
    k_bin = sh.k_bin;
  }
  if (p.top_p < 1.f) {
    __syncthreads();
    const bool cut = k_bin < kBins;
    if (per_unit < kMostPerUnit) {
      // a mass is good to 2^-17 and what the product z * per_unit rounds off; which bin holds the end is left open by more than that
      const double off = 1.0 / 65536.0 + ((double)fabsf(first) + kBins) / 33554432.0;
      const double lo = (double)p.top_p * sh.mass[cut ? k_bin : kBins] * (1.0 - off), hi = (double)p.top_p * sh.mass[cut ? k_bin + 1 : kBins] * (1.0 + off);
      if (im * (1.0 + off) >= lo) atomicMin(&sh.p_lo, tid);
      if (im * (1.0 - off) >= hi) atomicMin(&sh.p_hi, tid);
      __syncthreads();
      p_hi = min(sh.p_hi, cut ? k_bin : kBins - 1);
      p_lo = min(sh.p_lo, p_hi);
    } else {  // T below 1 / 512: bins of more than 1/16, and all the mass in a few of them
      p_lo = 0;
      p_hi = min(cut ? k_bin : kBins - 1, (int)(32.f * kMostPerUnit * T) + 1);
    }
  }
  const int sure_bin = min(k_bin, p_lo);
  if (sure_bin >= kBins) return c;
  const float sure = sure_bin > 0 ? bin_end(first, sure_bin - 1, per_unit) : INFINITY;
  if (c.least >= sure) return c;  // min_p ends above: nothing else matters
  c.ends = 1;
  c.sure = sure;
  c.count_sure = sh.count[sure_bin];
  c.p_low = bin_end(first, p_lo < kBins ? p_hi : k_bin, per_unit);
  c.apart = p_lo < kBins && k_bin < kBins && k_bin > p_hi;
  if (c.apart) {
    c.k_high = bin_end(first, k_bin - 1, per_unit);
    c.k_low = bin_end(first, k_bin, per_unit);
    c.count_k = sh.count[k_bin];
  }
  return c;
}

// sum over the wavefront of numbers below 2^48
__device__ __forceinline__ uint64_t wave_mass_sum(uint64_t m) {
  auto add = [](uint32_t x, uint32_t y) { return x + y; };
  const uint32_t lo = wave_reduce_u32((uint32_t)m & 0xffffffu, add), hi = wave_reduce_u32((uint32_t)(m >> 24), add);
  return ((uint64_t)hi << 24) + lo;
}
__device__ __forceinline__ uint64_t wave_inclusive64(uint64_t v, int lane) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const uint32_t lo = (uint32_t)__shfl_up((int)(uint32_t)v, o, kWave), hi = (uint32_t)__shfl_up((int)(uint32_t)(v >> 32), o, kWave);
    if (lane >= o) v += ((uint64_t)hi << 32) | lo;
  }
  return v;
}

template <class T, int SLICE>
__global__ __launch_bounds__(kScanThreads) void sample_cut_kernel(const SampleArgs a, const SampleWs ws, int row0) {
  constexpr int E = Chunk<T>::E, N = SLICE / E / kScanThreads;
  constexpr bool BF16 = sizeof(T) == 2;
  __shared__ CutShared sh;
  __shared__ uint64_t middle_sh[kScanThreads / 64];
  __shared__ uint32_t listed;
  const int slice = blockIdx.x, r = blockIdx.y, row = row0 + r, tid = threadIdx.x;
  if (a.masked != nullptr && a.masked[row] == 0) return;
  const RowParams p = row_params(a, row);
  if (!(p.temperature > 0.f) && slice > 0) return;
  const T* z = static_cast<const T*>(a.logits) + (int64_t)row * a.row_stride;
  const int c0 = slice * (SLICE / E) + tid, n_chunks = (a.vocab + E - 1) / E;
  Chunk<T> x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) load_chunk(x[i], z, min(c0 + i * kScanThreads, n_chunks), a.vocab);
  if (tid == 0) listed = 0;
  const RowCut c = cut_row(ws, r, p, sh);
  if (slice == 0 && tid == 0) ws.cut[r] = c;
  if (c.way != kDraw) return;  // uniform over the workgroup
  __syncthreads();
  const Scale s = scale_of(p.temperature);
  const float from = fmaxf(c.sure, c.least);
  uint64_t* list = ws.list + ((int64_t)r * ws.slices + slice) * kSliceList;
  float middle = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int chunk = c0 + i * kScanThreads;
    bool any = false;
#pragma unroll
    for (int e = 0; e < E; ++e) any |= x[i].z[e] >= from;
    uint64_t m = 0;
    if (__ballot(any) != 0ull) {
      float w = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) w += x[i].z[e] >= from ? weight<BF16>(x[i].z[e], c.top, s) : 0.f;
      m = wave_mass_sum(mass_of(w));
    }
    const int seg = chunk / kSegChunks;
    if ((tid & 63) == 0 && seg < ws.segs) ws.seg[(int64_t)r * ws.segs + seg] = m;
    if (c.ends) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float v = x[i].z[e];
        if ((v >= c.p_low && v < c.sure) || (v >= c.k_low && v < c.k_high)) {
          const uint32_t at = atomicAdd(&listed, 1u);
          if (at < (uint32_t)kSliceList) list[at] = order_of(key_of(v), chunk * E + e);
        }
        if (c.apart && v < c.p_low && v >= c.k_high) middle += weight<BF16>(v, c.top, s);
      }
    }
  }
  if (c.ends) {  // (a float per thread, which its tokens enter in order; whole numbers from there on)
    uint64_t m = wave_mass_sum(mass_of(middle));
    if ((tid & 63) == 0) middle_sh[tid >> 6] = m;
    __syncthreads();
    if (tid == 0) {
      m = 0;
      for (int w = 0; w < kScanThreads / 64; ++w) m += middle_sh[w];
      ws.middle[(int64_t)r * ws.slices + slice] = m;
      ws.listed[(int64_t)r * ws.slices + slice] = listed;
    }
  }
}

// sorts list[0, pad) in ascending order; pad a power of two up to 2 * kRowThreads * 2.  Pairs up to 64 apart are a wavefront's own.
__device__ __forceinline__ void sort_list(unsigned long long* list, int pad) {
  const int tid = threadIdx.x;
  for (int size = 2; size <= pad; size <<= 1)
    for (int step = size >> 1; step > 0; step >>= 1) {
      if (step > 64) __syncthreads();
      for (int i = tid; i < pad / 2; i += kRowThreads) {
        const int lo = 2 * i - (i & (step - 1)), hi = lo + step;
        const unsigned long long x = list[lo], y = list[hi];
        if ((x > y) == ((lo & size) == 0)) {
          list[lo] = y;
          list[hi] = x;
        }
      }
      if (step > 64)
        __syncthreads();
      else
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  __syncthreads();
}

constexpr int kMaxSegs = kSampleMaxVocab / (kSegChunks * 4);
template <class T>
__global__ __launch_bounds__(kRowThreads) void sample_pick_kernel(const SampleArgs a, const SampleWs ws, int row0) {
  constexpr int E = Chunk<T>::E, kWaves = kRowThreads / 64, RUN = kRowList / kRowThreads;
  constexpr bool BF16 = sizeof(T) == 2;
  __shared__ unsigned long long list[kRowList];
  __shared__ unsigned long long seg[kMaxSegs];
  __shared__ uint64_t sum_a[kWaves], sum_b[kWaves], wave_mass[kWaves];
  __shared__ int found, n_kept;
  __shared__ uint64_t found_base;
  const int r = blockIdx.x, row = row0 + r, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (a.masked != nullptr && a.masked[row] == 0) {
    if (tid == 0) write_row(a, row, -1, 0.f, 0.f);
    return;
  }
  const RowParams p = row_params(a, row);
  const RowCut c = ws.cut[r];
  if (c.way == kNone || c.way == kFirst) {
    if (tid == 0) write_row(a, row, c.way == kNone ? -1 : c.first_id, c.way == kNone ? 0.f : (float)(1.0 / c.at1), c.way == kNone ? 0.f : 1.f);
    return;
  }
  const Scale s = scale_of(p.temperature);
  uint32_t n = 0;
  uint64_t middle = 0;
  bool slow = c.way == kSearch;
  if (!slow) {
    for (int i = tid; i < ws.segs; i += kRowThreads) seg[i] = ws.seg[(int64_t)r * ws.segs + i];
    if (c.ends)
      for (int i = 0; i < ws.slices; ++i) {  // the slices' lists one behind the other
        const uint32_t k = ws.listed[(int64_t)r * ws.slices + i];
        slow = slow || k > (uint32_t)kSliceList || n + k > (uint32_t)kRowList;
        if (slow) break;
        for (uint32_t j = tid; j < k; j += kRowThreads) list[n + j] = ws.list[((int64_t)r * ws.slices + i) * kSliceList + j];
        n += k;
        middle += ws.middle[(int64_t)r * ws.slices + i];
      }
  }
  if (slow) {  // uniform over the workgroup
    search_row<T>(a, row, sum_a, sum_b, wave_mass, &found);
    return;
  }
  uint64_t last = 0;  // the last token kept, if the list decides that
  if (c.ends) {
    int pad = 1;
    while (pad < (int)n) pad <<= 1;
    for (int i = (int)n + tid; i < pad; i += kRowThreads) list[i] = ~0ull;
    if (tid == 0) n_kept = 0;
    __syncthreads();
    sort_list(list, pad);
    // the list's masses, a run of it for each thread, and that of everything above it
    uint64_t m[RUN], mine = 0, sure = 0, first_part = 0, upto = 0;
    const int j0 = tid * RUN;
    const uint32_t p_low = key_of(c.p_low);
    int n_first = (int)n;  // of [p_low, sure); behind them where top_k ends
    if (c.apart) {
      int lo = 0, hi = (int)n;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (key_in(list[mid]) >= p_low)
          lo = mid + 1;
        else
          hi = mid;
      }
      n_first = lo;
    }
    auto in_front = [&](int j) { return (j < n_first ? c.count_sure : c.count_k - (uint32_t)n_first) + (uint32_t)j; };  // tokens above the j-th entry
#pragma unroll
    for (int u = 0; u < RUN; ++u) {
      const int j = j0 + u;
      m[u] = j < (int)n ? mass<BF16>(of_key(key_in(list[j])), c.top, s) : 0;
      mine += m[u];
      if (j < n_first) first_part += m[u];
      if (j < (int)n && (!c.apart || j >= n_first) && in_front(j) < (uint32_t)p.top_k) upto += m[u];
    }
    for (int i = tid; i < ws.segs; i += kRowThreads) sure += seg[i];
    sure = block_reduce64<kRowThreads>(sure, sum_a, Add64());
    double target = INFINITY;
    if (p.top_p < 1.f) {
      double all = c.atT / kMassUnit;
      const bool cut = p.top_k > 0 && (c.apart || c.count_sure + n >= (uint32_t)p.top_k);  // the mass of the first top_k
      if (cut) {
        if (c.apart) upto += first_part;
        all = (double)(sure + middle + block_reduce64<kRowThreads>(upto, sum_b, Add64()));
      }
      target = (double)p.top_p * all;
    }
    uint64_t front = wave_inclusive64(mine, lane);
    if (lane == 63) wave_mass[wave] = front;
    __syncthreads();
    front += sure - mine;
    for (int w = 0; w < wave; ++w) front += wave_mass[w];
    int mine_kept = 0;
#pragma unroll
    for (int u = 0; u < RUN; ++u) {
      const int j = j0 + u;
      if (j < n_first) {
        const bool in_k = p.top_k <= 0 || in_front(j) < (uint32_t)p.top_k, in_p = (double)front < target;
        if (in_front(j) == 0 || (in_k && in_p && key_in(list[j]) >= c.least_key)) mine_kept = j + 1;
      }
      front += m[u];
    }
    if (mine_kept > 0) atomicMax(&n_kept, mine_kept);
    __syncthreads();
    const int kept = n_kept;  // a prefix
    if (kept > 0) last = list[kept - 1];
#pragma unroll
    for (int u = 0; u < RUN; ++u)
      if (j0 + u < kept) atomicAdd(&seg[(int)(uint32_t)list[j0 + u] / (E * kSegChunks)], (unsigned long long)m[u]);
  }
  if (tid == 0) found = -1;
  __syncthreads();
  // the segment that the random number falls into
  const int per = (ws.segs + kRowThreads - 1) / kRowThreads, g0 = tid * per, g1 = min(g0 + per, ws.segs);
  uint64_t mine = 0;
  for (int g = g0; g < g1; ++g) mine += seg[g];
  uint64_t before = wave_inclusive64(mine, lane);
  if (lane == 63) sum_a[wave] = before;
  __syncthreads();
  before -= mine;
  uint64_t total = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += sum_a[w];
    total += sum_a[w];
  }
  const double want = (double)p.u * (double)total;
  // whose end is the first past `want`; the last with a mass takes what rounding leaves
  auto here = [&](uint64_t from, uint64_t to) { return from < to && (double)from <= want && (!((double)to <= want) || to == total); };
  for (int g = g0; g < g1; ++g) {
    const uint64_t after = before + seg[g];
    if (here(before, after)) {
      found = g;
      found_base = before;
    }
    before = after;
  }
  __syncthreads();
  if (wave != 0) return;
  const T* z = static_cast<const T*>(a.logits) + (int64_t)row * a.row_stride;
  const int chunk = found * kSegChunks + lane, n_chunks = (a.vocab + E - 1) / E;
  Chunk<T> x;
  load_chunk(x, z, min(chunk, n_chunks), a.vocab);
  const float from = fmaxf(c.sure, c.least);
  uint64_t end[E], extra = 0;  // masses up to each token of the chunk: the sum of the sure ones, as in the second launch, and the listed ones
  float w = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float v = x.z[e];
    if (v >= from)
      w += weight<BF16>(v, c.top, s);
    else if (c.ends && order_of(key_of(v), chunk * E + e) <= last)
      extra += mass<BF16>(v, c.top, s);
    end[e] = mass_of(w) + extra;
  }
  before = wave_inclusive64(end[E - 1], lane) - end[E - 1] + found_base;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (here(before + (e > 0 ? end[e > 0 ? e - 1 : 0] : 0), before + end[e])) {
      const float v = x.z[e];
      write_row(a, row, chunk * E + e, (float)((double)weight<BF16>(v, c.top, scale_of(1.f)) / c.at1),
                (float)((double)weight<BF16>(v, c.top, s) / ((double)total * kMassUnit)));
    }
  }
}

struct SamplePlan {
  int slice, slices, segs, rows;  // logits of a slice; rows of a pass
  size_t stat, bins, middle, listed, list, cut, seg, total;
};
// Few rows: slices of a quarter, so that more compute units share a row.
static SamplePlan plan_sample(int n_rows, int vocab) {
  SamplePlan p;
  auto align = [](size_t x) { return (x + 255) & ~(size_t)255; };
  p.slice = (int64_t)n_rows * ceil_div(vocab, kSlice) <= 64 && ceil_div(vocab, kSliceSmall) <= 4 * kMaxSlices ? kSliceSmall : kSlice;
  p.slices = ceil_div(vocab, p.slice);
  p.segs = ceil_div(vocab, kSegChunks * 4);  // of float32, which has the shorter chunks
  p.rows = std::max(1, std::min({n_rows, 1024, 4096 / p.slices}));
  const size_t n = (size_t)p.rows * p.slices;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += align(bytes);
    return at;
  };
  p.stat = take(n * sizeof(SliceStat));
  p.bins = take(n * kBins * sizeof(uint64_t));
  p.middle = take(n * sizeof(uint64_t));
  p.listed = take(n * sizeof(uint32_t));
  p.list = take(n * kSliceList * sizeof(uint64_t));
  p.cut = take((size_t)p.rows * sizeof(RowCut));
  p.seg = take((size_t)p.rows * p.segs * sizeof(uint64_t));
  p.total = off;
  return p;
}
size_t sample_tokens_workspace(int n_rows, int vocab) { return plan_sample(n_rows, vocab).total; }

template <class T>
static hipError_t launch_sample_t(const SampleArgs& a, const SamplePlan& p, char* w, hipStream_t st) {
  SampleWs ws;
  ws.stat = reinterpret_cast<SliceStat*>(w + p.stat);
  ws.bins = reinterpret_cast<uint64_t*>(w + p.bins);
  ws.middle = reinterpret_cast<uint64_t*>(w + p.middle);
  ws.listed = reinterpret_cast<uint32_t*>(w + p.listed);
  ws.list = reinterpret_cast<uint64_t*>(w + p.list);
  ws.cut = reinterpret_cast<RowCut*>(w + p.cut);
  ws.seg = reinterpret_cast<uint64_t*>(w + p.seg);
  ws.slices = p.slices;
  ws.segs = ceil_div(a.vocab, kSegChunks * Chunk<T>::E);
  for (int row0 = 0; row0 < a.n_rows; row0 += p.rows) {  // the passes use the workspace one after the other
    const int rows = std::min(p.rows, a.n_rows - row0);
    const dim3 grid(p.slices, rows), block(kScanThreads);
    if (p.slice == kSlice) {
      hipLaunchKernelGGL((sample_scan_kernel<T, kSlice>), grid, block, 0, st, a, ws, row0);
      hipLaunchKernelGGL((sample_cut_kernel<T, kSlice>), grid, block, 0, st, a, ws, row0);
    } else {
      hipLaunchKernelGGL((sample_scan_kernel<T, kSliceSmall>), grid, block, 0, st, a, ws, row0);
      hipLaunchKernelGGL((sample_cut_kernel<T, kSliceSmall>), grid, block, 0, st, a, ws, row0);
    }
    hipLaunchKernelGGL(sample_pick_kernel<T>, dim3(rows), dim3(kRowThreads), 0, st, a, ws, row0);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_sample_tokens(const void* logits, int dtype, int64_t row_stride, const uint8_t* masked, const float* uniform, const float* temperature,
                                const int32_t* top_k, const float* top_p, const float* min_p, int n_rows, int vocab, int32_t* tokens, float* conf,
                                float* prob, void* workspace, hipStream_t st) {
  const SampleArgs a = {logits, row_stride, masked, uniform, temperature, top_k, top_p, min_p, n_rows, vocab, tokens, conf, prob};
  const SamplePlan p = plan_sample(n_rows, vocab);
  return dtype == FOCUS_F32 ? launch_sample_t<float>(a, p, static_cast<char*>(workspace), st) : launch_sample_t<uint16_t>(a, p, static_cast<char*>(workspace), st);
}

}  // namespace focus
