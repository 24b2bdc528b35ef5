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
// as a float32: NaN counts as -inf, +inf as the largest number
__device__ __forceinline__ float clean(float z) { return fminf(fmaxf(z, -INFINITY), 3.402823466e38f); }
// whole numbers in the order of the numbers, -0 as +0
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
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
__device__ __forceinline__ void unpack(Chunk<T>& x, const uint4& w) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int e = 0; e < Chunk<T>::E; ++e)
    x.z[e] = clean(sizeof(T) == 4 ? __uint_as_float(u[e & 3]) : ((e & 1) ? bf16_hi(u[(e >> 1) & 3]) : bf16_lo(u[(e >> 1) & 3])));
}
template <class T>
__device__ __forceinline__ float logit_at(const T* row, int id) {
  return clean(sizeof(T) == 4 ? *reinterpret_cast<const float*>(row + id) : bf16_lo(*reinterpret_cast<const uint16_t*>(row + id)));
}
// The N chunks c0, c0 + step, ... of a thread, packed: all requests first, none of them conditional.  A row's last, shorter chunk is read
// logit by logit, by whoever has it.
template <class T, int N>
struct Chunks {
  uint4 w[N];
  // f(i, chunk) for each of them, in a loop that is not unrolled: it takes the first and turns the others around.  (These launches
  // are a few microseconds long and start with a cold instruction cache: 32 logits unrolled took twice as long as four times eight.)
  // Eight logits a turn, because turning costs two moves per chunk held (511 rows of 32 003 float32 70.0 -> 67.2 us a call; sixteen: 78.7,
  // the code's own length).
  static constexpr int kTurn = N % 2 == 0 && Chunk<T>::E == 4 ? 2 : 1;
  template <class F>
  __device__ __forceinline__ void each(F&& f) {
#pragma unroll 1
    for (int i = 0; i < N; i += kTurn) {
#pragma unroll
      for (int j = 0; j < kTurn; ++j) {
        Chunk<T> x;
        unpack(x, w[j]);
        f(i + j, x);
      }
      turn<kTurn>();
    }
  }
  template <int STEP>
  __device__ __forceinline__ void turn() {
    uint4 first[STEP];
#pragma unroll
    for (int j = 0; j < STEP; ++j) first[j] = w[j];
#pragma unroll
    for (int j = 0; j + STEP < N; ++j) w[j] = w[j + STEP];
#pragma unroll
    for (int j = 0; j < STEP; ++j) w[N - STEP + j] = first[j];
  }
  __device__ __forceinline__ void load(const T* row, int c0, int step, int vocab) {
    constexpr int E = Chunk<T>::E;
    const int whole = vocab / E;
    if (whole > 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = *reinterpret_cast<const uint4*>(row + (int64_t)min(c0 + i * step, whole - 1) * E);
    }
    if (__ballot(c0 + (N - 1) * step >= whole) != 0ull) {
#pragma unroll 1
      for (int i = 0; i < N; ++i) {
        const int ch = c0 + i * step;
        if (ch >= whole) {
          uint32_t u[4];
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const bool in = ch == whole && ch * E + e < vocab;
            if constexpr (sizeof(T) == 4) {
              u[e] = in ? *reinterpret_cast<const uint32_t*>(row + ch * E + e) : 0xff800000u;
            } else {
              const uint32_t b = in ? *reinterpret_cast<const uint16_t*>(row + ch * E + e) : 0xff80u;
              u[e / 2] = (e & 1) ? u[e / 2] | (b << 16) : b;
            }
          }
          w[0] = make_uint4(u[0], u[1], u[2], u[3]);
        }
        turn<1>();
      }
    }
  }
};
template <class T>
__device__ __forceinline__ void load_chunk(Chunk<T>& x, const T* row, int chunk, int vocab) {
  Chunks<T, 1> c;
  c.load(row, chunk, 0, vocab);
  unpack(x, c.w[0]);
}

// ---- masses
// (1 / T) log2(e) as a sum of two floats
struct Scale {
  float hi, lo;
};
__device__ __forceinline__ Scale scale_of(float temperature) {
  constexpr float kHi = 1.44269504f, kLo = (float)(1.4426950408889634 - (double)kHi);
  Scale s;
  s.hi = fminf(kHi / temperature, 3e38f);
  s.lo = (__builtin_fmaf(-s.hi, temperature, kHi) + kLo) / temperature;  // what the division leaves over
  if (!(s.hi > 1e-30f && s.hi < 1e30f)) s.lo = 0.f;
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
  return x < 126.f ? __builtin_fmaf(w * -0.6931471805599453f, r, w) : 0.f;  // (a mass is none from 43 on, a confidence counts as far as floats go)
}
// 0 <= w < 512 in units of 2^-42, to nearest: the doubles of [1024, 2048) are 2^-42 apart
__device__ __forceinline__ uint64_t mass_of(float w) {
  constexpr double kAt = 1536.0;
  static_assert(kMassBits == 42, "the last place of kAt");
  return (uint64_t)(__double_as_longlong((double)w + kAt) - __double_as_longlong(kAt));
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

__device__ __forceinline__ uint64_t wave_inclusive64(uint64_t v, int lane) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const uint32_t lo = (uint32_t)__shfl_up((int)(uint32_t)v, o, kWave), hi = (uint32_t)__shfl_up((int)(uint32_t)(v >> 32), o, kWave);
    if (lane >= o) v += ((uint64_t)hi << 32) | lo;
  }
  return v;
}

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
// the same address for every lane, of memory that nobody writes meanwhile: a scalar load
template <class V>
__device__ __forceinline__ V uniform_load(const V* ptr) {
  typedef const __attribute__((address_space(4))) V* cptr_t;
  return *(cptr_t)(uintptr_t)ptr;
}
__device__ __forceinline__ RowParams row_params(const SampleArgs& a, int row) {
  // all requests at once: what is not given is read from `uniform` and replaced
  const float temperature = uniform_load((a.temperature ? a.temperature : a.uniform) + row), top_p = uniform_load((a.top_p ? a.top_p : a.uniform) + row),
              min_p = uniform_load((a.min_p ? a.min_p : a.uniform) + row), u = uniform_load(a.uniform + row);
  const int top_k = uniform_load((a.top_k ? a.top_k : reinterpret_cast<const int32_t*>(a.uniform)) + row);
  RowParams p;
  p.temperature = a.temperature ? temperature : 1.f;
  p.top_p = a.top_p ? top_p : 1.f;
  p.min_p = a.min_p ? min_p : 0.f;
  p.top_k = a.top_k ? top_k : 0;
  p.u = fmaxf(u, 0.f);  // NaN: 0
  if (p.top_k == 1 || p.top_p <= 0.f || p.min_p > 1.f) p.temperature = 0.f;  // only the first stays
  return p;
}
__device__ __forceinline__ void write_row(const SampleArgs& a, int row, int token, float conf, float prob) {
  a.tokens[row] = token;
  if (a.conf) a.conf[row] = conf;
  if (a.prob) a.prob[row] = prob;
}
// the smallest key that min_p keeps: w >= min_p <=> z >= top + T ln(min_p); `down`: T ln(min_p), of a min_p between 0 and 1
__device__ __forceinline__ uint32_t min_p_key(float min_p, double down, float top) {
  if (!(min_p > 0.f)) return 0u;
  if (min_p >= 1.f) return key_of(top);
  const double cut = (double)top + down;
  float z = (float)cut;
  if ((double)z < cut) z = of_key(key_of(z) + 1u);
  return key_of(clean(z));
}

// The whole row by one workgroup that walks it as often as it takes: the order is searched bit by bit.  What is kept is
// {key > cut} and of {key == cut} the ids up to `last_id`.  For the rows that the lists below do not hold, which are more than
// those of logits all alike.  Normal logits, top_p 0.7 to 0.9: more than 4096 tokens lie within 1/16 of T where the end is at a spread over T of 0.5 and
// less for 126 464 (64 rows: in some of them at 0.75), of 1 for 200 000, 1.5 for 262 144, 2 for a million.  And where top_p is close to
// 1 and ends among the many tokens of small weight, or nearer to the last than the bins' error: 126 464 at a spread of 3, from 0.999 on.
// A pass is bound by what one compute unit computes, so passes are what counts: 126 464 logits, top_p: 517 us a row, as float32 962 (33 where the lists
// hold the end); 64 rows 549 to 558; 32 003 170 and 301; 200 000 840; a million 3.7 ms (65 us).  (One bit of the order a pass, and of the ids, took
// two and a half times as long.)
constexpr int kRowThreads = 512;
template <class T>
__device__ void search_row(const SampleArgs& a, int row, uint64_t* sh, uint64_t* sh2, uint64_t* wave_mass, int* found) {
  constexpr int E = Chunk<T>::E;
  constexpr bool BF16 = sizeof(T) == 2;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const T* z = static_cast<const T*>(a.logits) + (int64_t)row * a.row_stride;
  const int n_chunks = (a.vocab + E - 1) / E;
  const RowParams p = row_params(a, row);
  auto each = [&](auto&& f) {  // f(id, logit) over the row
    constexpr int kAhead = 8;
    for (int c0 = tid; c0 < n_chunks; c0 += kAhead * kRowThreads) {
      Chunks<T, kAhead> chunks;  // (past the row: -inf)
      chunks.load(z, c0, kRowThreads, a.vocab);
      chunks.each([&](int i, const Chunk<T>& x) {
#pragma unroll
        for (int e = 0; e < E; ++e) f((c0 + i * kRowThreads) * E + e, x.z[e]);
      });
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
  // the largest key with enough(count, mass of the tokens down to it), two bits at a time; the lower half of a bf16 number's key follows
  // from its sign (+inf stands for a float32 that is none)
  const bool half = BF16 && top < 3.402823466e38f;
  auto search = [&](auto&& enough) {
    uint32_t k = 0;
    for (int bit = 30; bit >= (half ? 16 : 0); bit -= 2) {
      uint32_t c[3] = {0, 0, 0};
      uint64_t m[3] = {0, 0, 0};
      each([&](int, float v) {
        const uint32_t key = key_of(v);
        if (key > kKeyNone && key >= k + (1u << bit)) {
          const uint64_t w = mass<BF16>(v, top, s);
#pragma unroll
          for (uint32_t j = 0; j < 3; ++j) {
            const bool in = key >= k + ((j + 1u) << bit);
            c[j] += in ? 1 : 0;
            m[j] += in ? w : 0;
          }
        }
      });
      uint32_t step = 0;
#pragma unroll
      for (uint32_t j = 0; j < 3; ++j) {  // (what is enough for one is so for those in front)
        const uint64_t n = block_reduce64<kRowThreads>(c[j], sh, Add64()), w = block_reduce64<kRowThreads>(m[j], sh2, Add64());
        if (enough(n, w)) step = j + 1u;
      }
      k += step << bit;
    }
    return half && !(k & 0x80000000u) ? k | 0xffffu : k;
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
  const uint32_t m_key = min(min_p_key(p.min_p, (double)p.temperature * log((double)p.min_p), top), top_key);
  if (m_key > cut) {
    cut = m_key;
    ties = ~(uint64_t)0;
  }
  // f(id, sum of `of(id, logit)` over the ids in front, up to this one), in rounds of the workgroup
  auto walk = [&](auto&& of, auto&& f) {
    uint64_t base = 0;
    for (int c0 = 0; c0 < n_chunks; c0 += kRowThreads) {
      uint64_t m[E], mine = 0;
      const int ch = c0 + tid;
      Chunk<T> x;
      load_chunk(x, z, ch, a.vocab);  // (past the row: -inf)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        m[e] = of(ch * E + e, x.z[e]);
        mine += m[e];
      }
      uint64_t before = wave_inclusive64(mine, lane);  // then exclusive over the workgroup
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
      for (int e = 0; e < E; ++e) {
        f(ch * E + e, before, before + m[e]);
        before += m[e];
      }
      base += round;
    }
  };
  int last_id = a.vocab;
  if (ties != ~(uint64_t)0) {  // that of the last of them
    if (tid == 0) (*found) = a.vocab;
    walk([&](int, float v) -> uint64_t { return key_of(v) == cut ? 1 : 0; },
         [&](int id, uint64_t before, uint64_t after) {
           if (before < ties && after == ties) (*found) = id;
         });
    __syncthreads();
    last_id = *found;
    __syncthreads();
  }
  auto held = [&](int id, float v) {
    const uint32_t k = key_of(v);
    return k > kKeyNone && (k > cut || (k == cut && id <= last_id)) ? mass<BF16>(v, top, s) : (uint64_t)0;
  };
  uint64_t total = 0;
  each([&](int id, float v) { total += held(id, v); });
  total = block_reduce64<kRowThreads>(total, sh, Add64());
  const double want = (double)p.u * (double)total;
  if (tid == 0) (*found) = -1;
  walk(held, [&](int id, uint64_t before, uint64_t after) {  // (the last token with a mass takes what rounding leaves)
    if (before < after && (double)before <= want && (!((double)after <= want) || after == total)) atomicMax(found, id);
  });
  __syncthreads();
  const int token = (*found);
  if (tid == 0) {
    const float v = token < 0 ? top : logit_at(z, token);
    const double w1 = weight<BF16>(v, top, s1), w = weight<BF16>(v, top, s);
    write_row(a, row, token < 0 ? first_id : token, (float)(w1 / denom), (float)(w / ((double)total * unit)));
  }
}

// =====================================================================================================
// The ordinary way: three launches, the first two with a workgroup per slice of a row.
//   sample_scan_kernel   the slice's largest logit and its weights at T = 1, and a histogram of the order: bins of 1/16 in logit / T, counts and
//                        masses.  Bins are counted from zero logit up (floor(z * bins per unit)), so that those of all slices are the
//                        same; a bin kBins and more below the largest logit's has no mass.
//   sample_cut_kernel    from the row's histogram the bins in which top_k and top_p end.  Tokens above them are kept whatever comes:
//                        their masses are summed per segment of 64 chunks.  Tokens in them are listed.
//   sample_pick_kernel   a workgroup per row orders the list, finds the end of what is kept in it, adds the kept ones to their segments, and
//                        walks down: segment, chunk, token.
// The row is read twice, the second time from a cache.  The histogram only says where to look: ends and borders are decided by the masses,
// token for token, so they are the same whichever way a row takes and however it is cut into slices.  (The confidence's sum alone is of
// floats, 8 or 32 of a thread at a time.  With chunks of weights added as floats rows without a filter took 3 to 4 us less, 64 bf16 rows
// of 126 464 24.3 -> 26.4, 511 of 32 003 38.8 -> 42.7 and as float32 49.5 -> 52.9, filtered ones up to 2 us less or more; a weight
// below 2^-24 of its chunk's sum then got no share.)  Where the lists do not hold the tokens of a bin, or the bins do not resolve
// the logits (2^18 and more, at T = 1), the last launch searches the row instead.
//
// What bounds it.  One row of 126 464: three launches of 3.9, 10.5 and 8.7 us, each a chain of round trips (3.3, 2.4 and 2.1 where the largest
// logit is taken).  64 such rows (bf16, 16 MB, three quarters of them drawn from) 11.2, 16.6 and 9.7 us, 511 rows of 32 003 (float32,
// 65 MB) 20.8, 38.9 and 14.8: the arithmetic on each logit, an exponential, a bin and an atomic in the first launch, a weight with
// its rounding kept and its mass in the second where the bulk of a row carries the mass, at a quarter to a half of the rate at which
// HBM would deliver (511 float32 rows without a filter 55.5 us a call, of which the largest are taken 30.4).  One workgroup that keeps a whole row in registers through all three parts (up to 65 536 bf16 logits) saves two
// launches and the second read, and is slower: it holds 128 registers and 68 KB of LDS and computes the same, with fewer wavefronts to hide
// the parts in which one waits (511 rows 72 -> 81 us).
// =====================================================================================================
constexpr int kBins = 512;
constexpr int kScanThreads = 512;
constexpr int kSlice = 32 * kScanThreads, kSliceSmall = 8 * kScanThreads;  // logits of a workgroup
// Entries of the list of a slice and of a row: what eight tokens a thread hold in the last launch, 32 KB of its LDS; 16 KB of workspace a slice.
constexpr int kSliceList = 2048, kRowList = 4096;
constexpr int kSegChunks = 64;
constexpr int kMaxSlices = kSampleMaxVocab / kSlice;
constexpr float kMostBin = 4194304.f;                       // beyond, floats would not hold bin numbers and their neighbours
constexpr float kBinsPerNat = 16.f, kMostPerUnit = 8192.f;  // bins per unit of logit: kBinsPerNat / T at T > 1 / 512

struct SliceStat {
  float top;   // -inf: no number
  int id;      // the first with it
  double at1;  // sum of the weights at T = 1, relative to `top`
};
// Where a row is cut.
struct RowCut {
  float top;
  int first_id;
  int way;                         // kNone, kFirst, kDraw, kSearch
  int ends;                        // 0: nothing is cut but by min_p; else the list decides
  float per_unit;                  // bins per unit of logit; the next four are logits times that
  float sure;                      // tokens from here on are kept
  float p_low, k_high, k_low;      // the list: [p_low, sure) and [k_low, k_high), where top_k ends apart from top_p
  float rest_low, rest_high;       // tokens whose masses top_p counts beside those of the sure and the listed ones that top_k leaves: [k_high, p_low)
                                   // where that is apart, all but the sure ones where top_k ends nothing, else none
  bool apart;
  uint32_t count_sure, count_k;    // tokens above `sure`, above k_high
  float least;                     // min_p: no logit below this one
  uint32_t least_key;
};
enum { kNone = 0, kFirst = 1, kDraw = 2, kSearch = 3 };
struct SampleWs {
  SliceStat* stat;   // [rows, slices]
  uint64_t* bins;    // [rows, slices, kBins]  tokens in the upper half, their masses above that of the bin's lower end in the lower half
  uint64_t* rest;    // [rows, slices]  mass of [rest_low, rest_high)
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
// sum over the wavefront of numbers below 2^48
__device__ __forceinline__ uint64_t wave_mass_sum(uint64_t m) {
  auto add = [](uint32_t x, uint32_t y) { return x + y; };
  const uint32_t lo = wave_reduce_u32((uint32_t)m & 0xffffffu, add), hi = wave_reduce_u32((uint32_t)(m >> 24), add);
  return ((uint64_t)hi << 24) + lo;
}

template <class T, int SLICE>
__global__ __launch_bounds__(kScanThreads) void sample_scan_kernel(const SampleArgs a, const SampleWs ws, int row0) {
  constexpr int E = Chunk<T>::E, N = SLICE / E / kScanThreads, kCopies = 4, kWaves = kScanThreads / 64;
  __shared__ unsigned long long bins_sh[kCopies][kBins];
  __shared__ float top_sh[kWaves];
  __shared__ unsigned long long at1_sh;
  __shared__ int id_sh;
  const int slice = blockIdx.x, r = blockIdx.y, row = row0 + r, tid = threadIdx.x;
  const RowParams p = row_params(a, row);
  if (a.masked != nullptr && a.masked[row] == 0) return;
  const int c0 = slice * (SLICE / E) + tid;
  Chunks<T, N> chunks;
  chunks.load(static_cast<const T*>(a.logits) + (int64_t)row * a.row_stride, c0, kScanThreads, a.vocab);
  const bool drawn = p.temperature > 0.f, order = drawn && needs_order(p);  // uniform over the workgroup
  if (order) {
#pragma unroll
    for (int i = 0; i < kCopies; ++i) bins_sh[i][tid] = 0;
  }
  if (tid == 0) {
    id_sh = 0x7fffffff;
    at1_sh = 0;
  }
  float mine = -INFINITY;
  chunks.each([&](int, const Chunk<T>& x) {
#pragma unroll
    for (int e = 0; e < E; ++e) mine = fmaxf(mine, x.z[e]);
  });
  auto larger = [](uint32_t x, uint32_t y) { return x > y ? x : y; };
  float top = of_key(wave_reduce_u32(key_of(mine), larger));
  if ((tid & 63) == 0) top_sh[tid >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, top_sh[w]);
  SliceStat* stat = ws.stat + (int64_t)r * ws.slices + slice;
  if (top == -INFINITY) {
    if (tid == 0) *stat = SliceStat{top, 0, 0.0};
    return;
  }
  if (mine == top) {
    int id = 0x7fffffff;
    chunks.each([&](int i, const Chunk<T>& x) {
#pragma unroll
      for (int e = E - 1; e >= 0; --e)
        if (x.z[e] == top) id = min(id, (c0 + i * kScanThreads) * E + e);
    });
    atomicMin(&id_sh, id);
  }
  // exp(f / 16) - 1 = g(f) / 16 for the place f of a token in its bin: 1 + f / 32 + f^2 / 1536 times f, in units of 2^-17
  const float T_ = drawn ? p.temperature : 1.f, per_unit = bins_per_unit(T_), first = floorf(top * per_unit);
  const bool conf = a.conf != nullptr;
  unsigned long long* bins = bins_sh[tid & (kCopies - 1)];
  float at1 = 0.f;
  chunks.each([&](int, const Chunk<T>& x) {
    if (conf) {
#pragma unroll
      for (int e = 0; e < E; ++e) at1 += __builtin_amdgcn_exp2f((x.z[e] - top) * 1.4426950408889634f);
    }
    if (order) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float t = x.z[e] * per_unit, low = floorf(t), b = first - low;
        if (b < (float)kBins) {
          const float f = t - low;
          const uint32_t g = (uint32_t)(f * __builtin_fmaf(f, __builtin_fmaf(f, 131072.f / 1536.f, 131072.f / 32.f), 131072.f));
          atomicAdd(&bins[(int)b], (1ull << 32) | g);
        }
      }
    }
  });
  const uint64_t w1 = wave_mass_sum(mass_of(at1));  // (32 at most each: below 2^48)
  if ((tid & 63) == 0) atomicAdd(&at1_sh, (unsigned long long)w1);
  __syncthreads();
  if (tid == 0) *stat = SliceStat{top, id_sh, (double)at1_sh * kMassUnit};
  if (order) {
    static_assert(kBins == kScanThreads, "a bin a thread");
    uint64_t v = 0;  // 16384 tokens at most: the lower half holds 16384 * 1.04 * 2^17
#pragma unroll
    for (int i = 0; i < kCopies; ++i) v += bins_sh[i][tid];
    ws.bins[((int64_t)r * ws.slices + slice) * kBins + tid] = v;
  }
}

constexpr int kNoBin = 4 * kBins;
constexpr int kEarly = 4;  // slices whose bins are requested beside the statistics, before it is known how far down they begin
struct CutShared {
  RowCut cut;
  int shift[4 * kMaxSlices];
  uint64_t early[kEarly][kBins];
  float mass[kBins + 1];  // of the bins in front
  uint32_t count[kBins + 1];
  float wave_mass[kScanThreads / 64];
  uint32_t wave_count[kScanThreads / 64];
  double down_min_p;
  int k_bin, p_lo, p_hi;
};
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}
// Every workgroup of the second launch works this out, in the same operations; the third reads it.  The slices' statistics are one
// wavefront's work, the logarithm of min_p another's.  Nothing but latency: the bins of the first slices are requested beside the
// statistics, before it is known how far down they begin, and wait in LDS; those of the others AHEAD at a time, from where they belong.  (A
// thread adds up one bin; with atomics into LDS instead a row of 126 464 bf16 logits takes 24.4 us and not 23.4, one of 1 000 000
// 60 and not 54.)
template <int AHEAD>
__device__ __forceinline__ RowCut cut_row(const SampleWs& ws, int r, const RowParams& p, CutShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const SliceStat* stat = ws.stat + (int64_t)r * ws.slices;
  const bool drawn = p.temperature > 0.f, order = drawn && needs_order(p);
  const float T = drawn ? p.temperature : 1.f;
  const float per_unit = bins_per_unit(T);
  const uint64_t* bins = ws.bins + (int64_t)r * ws.slices * kBins;
  uint64_t early[kEarly];
  if (order) {
#pragma unroll
    for (int u = 0; u < kEarly; ++u) early[u] = bins[(int64_t)min(u, ws.slices - 1) * kBins + tid];  // (of a slice without a number: whatever lies there)
  }
  if (wave == 0) {
    RowCut c;
    auto larger = [](uint32_t x, uint32_t y) { return x > y ? x : y; };
    uint32_t key = 0;
    for (int i0 = 0; i0 < ws.slices; i0 += kWave) {
      const int i = i0 + lane;
      key = larger(key, i < ws.slices ? key_of(stat[i].top) : 0u);
    }
    key = wave_reduce_u32(key, larger);
    c.top = of_key(key);
    const float first = floorf(c.top * per_unit);
    c.first_id = 0x7fffffff;
    for (int i0 = 0; i0 < ws.slices; i0 += kWave) {
      const int i = i0 + lane;
      const float t = i < ws.slices ? stat[i].top : -INFINITY;
      const int id = i < ws.slices ? stat[i].id : 0;
      const unsigned long long at = __ballot(t == c.top);  // (slices are in the order of the ids)
      if (at != 0ull && c.first_id == 0x7fffffff) c.first_id = __builtin_amdgcn_readlane(id, __ffsll((long long)at) - 1);
      if (i < ws.slices) {  // (no number in the slice: -inf)
        const float shift = first - floorf(t * per_unit);
        sh.shift[i] = shift < (float)kBins ? (int)shift : kBins;
      }
    }
    c.way = !(c.top > -INFINITY) ? kNone : (!drawn ? kFirst : (fabsf(first) <= kMostBin ? kDraw : kSearch));
    c.ends = 0;
    c.per_unit = per_unit;
    c.sure = -INFINITY;
    c.p_low = c.k_high = c.k_low = c.rest_low = INFINITY;
    c.rest_high = -INFINITY;
    c.apart = false;
    c.count_sure = c.count_k = 0;
    if (lane == 0) {
      sh.cut = c;
      sh.k_bin = sh.p_lo = sh.p_hi = kNoBin;
      sh.mass[0] = 0.f;
      sh.count[0] = 0;
    }
  }
  if (wave == 1 && lane == 0) sh.down_min_p = p.min_p > 0.f && p.min_p < 1.f ? (double)T * log((double)p.min_p) : 0.0;
  if (order) {
#pragma unroll
    for (int u = 0; u < kEarly; ++u) sh.early[u][tid] = early[u];
  }
  __syncthreads();
  RowCut c = sh.cut;
  c.least_key = c.way == kDraw ? min_p_key(p.min_p, sh.down_min_p, c.top) : 0u;
  c.least = c.least_key > kKeyNone ? of_key(c.least_key) : -3.402823466e38f;
  if (c.way != kDraw || !order) return c;  // uniform over the workgroup, like the others
  const float first = floorf(c.top * per_unit);
  uint32_t n = 0;
  uint64_t above = 0;
#pragma unroll
  for (int u = 0; u < kEarly; ++u) {
    const int shift = u < ws.slices ? sh.shift[u] : kBins;
    const uint64_t v = sh.early[u][max(tid - shift, 0)];
    n += tid >= shift ? (uint32_t)(v >> 32) : 0u;
    above += tid >= shift ? (uint32_t)v : 0u;
  }
  for (int i0 = kEarly; i0 < ws.slices; i0 += AHEAD) {
    uint64_t v[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {  // all requests first; a slice whose bins lie lower begins further down (shift), one past the last has none
      const int i = min(i0 + u, ws.slices - 1);
      v[u] = bins[(int64_t)i * kBins + max(tid - sh.shift[i], 0)];
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const bool in = i0 + u < ws.slices && tid >= sh.shift[min(i0 + u, ws.slices - 1)];
      n += in ? (uint32_t)(v[u] >> 32) : 0u;
      above += in ? (uint32_t)v[u] : 0u;
    }
  }
  const float down = (first - (float)tid - c.top * per_unit) * (1.4426950408889634f / kBinsPerNat);
  float im = __builtin_amdgcn_exp2f(down) * ((float)n + (float)above * (1.f / (131072.f * kBinsPerNat)));
  uint32_t in = n;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const float om = __shfl_up(im, o, kWave);
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
  sh.mass[tid + 1] = im;
  sh.count[tid + 1] = in;
  if (p.top_k > 0 && in >= (uint32_t)p.top_k && in - n < (uint32_t)p.top_k) sh.k_bin = tid;  // (the counts ascend: one thread at most)
  __syncthreads();
  const int k_bin = sh.k_bin;
  int p_lo = kNoBin, p_hi = kNoBin;
  if (p.top_p < 1.f) {
    const bool cut = k_bin < kBins;
    if (per_unit < kMostPerUnit) {
      // a mass is good to 2^-17, a sum of them to 2^-20, and to what the product z * per_unit rounds off; which bin holds the end is left
      // open by more than that
      const float off = 1.f / 32768.f + (fabsf(first) + kBins) / 33554432.f;
      const float lo = p.top_p * sh.mass[cut ? k_bin : kBins] * (1.f - off), hi = p.top_p * sh.mass[cut ? k_bin + 1 : kBins] * (1.f + off);
      const unsigned long long at_lo = __ballot(im * (1.f + off) >= lo), at_hi = __ballot(im * (1.f - off) >= hi);  // the masses ascend
      if (lane == 0 && at_lo != 0ull) atomicMin(&sh.p_lo, tid + __ffsll((long long)at_lo) - 1);
      if (lane == 0 && at_hi != 0ull) atomicMin(&sh.p_hi, tid + __ffsll((long long)at_hi) - 1);
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
  const float sure = sure_bin > 0 ? first - (float)(sure_bin - 1) : INFINITY;  // floor(t) >= n <=> t >= n
  if (c.least * per_unit >= sure) return c;                                    // min_p ends above: nothing else matters
  c.ends = 1;
  c.sure = sure;
  c.count_sure = sh.count[sure_bin];
  c.p_low = first - (float)(p_lo < kBins ? p_hi : k_bin);
  c.apart = p_lo < kBins && k_bin < kBins && k_bin > p_hi;
  if (c.apart) {
    c.k_high = first - (float)(k_bin - 1);
    c.k_low = first - (float)k_bin;
    c.count_k = sh.count[k_bin];
    c.rest_low = c.k_high;
    c.rest_high = c.p_low;
  } else if (k_bin >= kBins) {
    c.rest_low = -INFINITY;
    c.rest_high = c.sure;
  }
  return c;
}

template <class T, int SLICE>
__global__ __launch_bounds__(kScanThreads, 6) void sample_cut_kernel(const SampleArgs a, const SampleWs ws, int row0) {
  constexpr int E = Chunk<T>::E, N = SLICE / E / kScanThreads;
  constexpr bool BF16 = sizeof(T) == 2;
  __shared__ CutShared sh;
  __shared__ uint64_t rest_sh[kScanThreads / 64];
  __shared__ uint32_t listed;
  const int slice = blockIdx.x, r = blockIdx.y, row = row0 + r, tid = threadIdx.x;
  const RowParams p = row_params(a, row);
  if (a.masked != nullptr && a.masked[row] == 0) return;
  if (!(p.temperature > 0.f) && slice > 0) return;
  const int c0 = slice * (SLICE / E) + tid;
  Chunks<T, N> chunks;
  chunks.load(static_cast<const T*>(a.logits) + (int64_t)row * a.row_stride, c0, kScanThreads, a.vocab);
  if (tid == 0) listed = 0;
  const RowCut c = cut_row<SLICE == kSlice ? 8 : 16>(ws, r, p, sh);
  if (slice == 0 && tid == 0) ws.cut[r] = c;
  if (c.way != kDraw) return;  // uniform over the workgroup
  __syncthreads();
  const Scale s = scale_of(p.temperature);
  uint64_t* list = ws.list + ((int64_t)r * ws.slices + slice) * kSliceList;
  uint64_t rest = 0;
  chunks.each([&](int i, const Chunk<T>& x) {
    const int chunk = c0 + i * kScanThreads, seg = chunk / kSegChunks;
    uint32_t sure = 0, other = 0, hits = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float t = x.z[e] * c.per_unit;
      sure |= t >= c.sure && x.z[e] >= c.least ? 1u << e : 0u;
      other |= t >= c.rest_low && t < c.rest_high ? 1u << e : 0u;
      hits |= (t >= c.p_low && t < c.sure) || (t >= c.k_low && t < c.k_high) ? 1u << e : 0u;
    }
    uint64_t m = 0;
    if (__ballot((sure | other) != 0u) != 0ull) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (((sure | other) >> e) & 1u) {
          const uint64_t w = mass<BF16>(x.z[e], c.top, s);
          m += (sure >> e) & 1u ? w : 0;
          rest += (sure >> e) & 1u ? 0 : w;
        }
      m = wave_mass_sum(m);
    }
    if ((tid & 63) == 0 && seg < ws.segs) ws.seg[(int64_t)r * ws.segs + seg] = m;
    if (hits != 0u) {
      uint32_t at = atomicAdd(&listed, (uint32_t)__popc(hits));
#pragma unroll
      for (int e = 0; e < E; ++e)
        if ((hits >> e) & 1u) {
          if (at < (uint32_t)kSliceList) list[at] = order_of(key_of(x.z[e]), chunk * E + e);
          ++at;
        }
    }
  });
  if (c.ends) {
    uint64_t m = wave_mass_sum(rest);  // (32 tokens of at most 1 each: below 2^48)
    if ((tid & 63) == 0) rest_sh[tid >> 6] = m;
    __syncthreads();
    if (tid == 0) {
      m = 0;
      for (int w = 0; w < kScanThreads / 64; ++w) m += rest_sh[w];
      ws.rest[(int64_t)r * ws.slices + slice] = m;
      ws.listed[(int64_t)r * ws.slices + slice] = listed;
    }
  }
}

// The end of a prefix of the order.  Every thread holds some tokens: order (order_of) and mass.  Kept are the tokens for which what lies in
// front of them is below a limit: their number, or their mass.  The last one kept is found by narrowing: a histogram of 128 bins over
// what is left of the order, and the last bin that begins below the limit is what is left.  Tokens of one logit part by their ids, the
// lower bits of the order.  A round narrows 64 bits by seven; two to four of them are usual, 3 us each: for lists that are too long
// to rank.  Copies of the bins: tokens of one logit would otherwise queue for one address, 64 of a wavefront at a time.
constexpr int kNarrowBins = 128, kNarrowCopies = 4;
struct NarrowShared {
  unsigned long long mass[kNarrowCopies][kNarrowBins];
  uint32_t count[kNarrowCopies][kNarrowBins];
  uint64_t wave_lo[kRowThreads / 64], wave_hi[kRowThreads / 64];
  int bin;
  uint64_t front_mass;
  uint32_t front_count;
};
struct End {
  uint64_t last;  // 0: nothing is kept
  uint64_t mass;  // of what is kept
};
template <int RUN>
__device__ __forceinline__ End find_end(const uint64_t (&order)[RUN], const uint64_t (&m)[RUN], uint32_t alive, bool by_count, uint32_t count, uint32_t most,
                                        uint64_t base, double limit, NarrowShared& sh) {
  static_assert(kNarrowBins * kNarrowCopies == kRowThreads && kNarrowBins == 2 * kWave, "a cell a thread, two bins a lane");
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, copy = tid & (kNarrowCopies - 1);
  constexpr int kWaves = kRowThreads / 64;
  uint64_t front = 0;
  if (by_count ? count >= most : !((double)base < limit)) return End{0, 0};
  for (;;) {
    uint64_t lo = ~(uint64_t)0, hi = 0;
#pragma unroll
    for (int u = 0; u < RUN; ++u)
      if ((alive >> u) & 1u) {
        lo = order[u] < lo ? order[u] : lo;
        hi = order[u] > hi ? order[u] : hi;
      }
    if (__ballot(alive != 0u) != 0ull) {
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        const uint64_t l = shfl_xor64(lo, o), h = shfl_xor64(hi, o);
        lo = l < lo ? l : lo;
        hi = h > hi ? h : hi;
      }
    }
    (&sh.mass[0][0])[tid] = 0;
    (&sh.count[0][0])[tid] = 0;
    if (lane == 0) {
      sh.wave_lo[wave] = lo;
      sh.wave_hi[wave] = hi;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      lo = sh.wave_lo[w] < lo ? sh.wave_lo[w] : lo;
      hi = sh.wave_hi[w] > hi ? sh.wave_hi[w] : hi;
    }
    if (lo > hi) return End{0, 0};  // (no token at all)
    const int shift = max(0, 64 - __clzll((long long)((hi - lo) | 1ull)) - 7);
#pragma unroll
    for (int u = 0; u < RUN; ++u)
      if ((alive >> u) & 1u) {
        const int b = (int)((order[u] - lo) >> shift);
        atomicAdd(&sh.mass[copy][b], (unsigned long long)m[u]);
        atomicAdd(&sh.count[copy][b], 1u);
      }
    __syncthreads();
    if (wave == 0) {
      uint64_t bm[2] = {0, 0};
      uint32_t bn[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < kNarrowCopies; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          bm[u] += sh.mass[i][2 * lane + u];
          bn[u] += sh.count[i][2 * lane + u];
        }
      uint64_t before = wave_inclusive64(bm[0] + bm[1], lane) - bm[0] - bm[1];
      uint32_t n_before = bn[0] + bn[1];
#pragma unroll
      for (int o = 1; o < kWave; o <<= 1) {
        const uint32_t t = __shfl_up(n_before, o, kWave);
        if (lane >= o) n_before += t;
      }
      n_before -= bn[0] + bn[1];
      auto begins = [&](uint32_t c, uint64_t x) { return by_count ? count + c < most : (double)(base + front + x) < limit; };
      const bool second = bn[1] > 0 && begins(n_before + bn[0], before + bm[0]);
      const unsigned long long some = __ballot(second || (bn[0] > 0 && begins(n_before, before)));
      if (lane == 63 - __clzll((long long)some)) {  // (the first token of all begins below the limit)
        sh.bin = 2 * lane + (second ? 1 : 0);
        sh.front_mass = before + (second ? bm[0] : 0) + (lo == hi ? bm[second ? 1 : 0] : 0);
        sh.front_count = n_before + (second ? bn[0] : 0);
      }
    }
    __syncthreads();
    front += sh.front_mass;
    if (lo == hi) return End{lo, front};  // one token is left: it is the last
    count += sh.front_count;
    const int bin = sh.bin;
#pragma unroll
    for (int u = 0; u < RUN; ++u)
      if (((alive >> u) & 1u) && (int)((order[u] - lo) >> shift) != bin) alive &= ~(1u << u);
  }
}

// Tokens that are ranked each against every other, a thread's one at most; LDS reads under way.  (Lists of 65 to 512 narrowed instead: 511 float32
// rows of 32 003, top_p 0.9 70.0 -> 75.6 us, 0.95 73.5 -> 76.9; 64 bf16 rows of 126 464, top_k 50 to 800 within 0.3 us.)
constexpr int kRankMost = 512, kRankAhead = 8;
// SEGS: the most segments of a row; fewer leave LDS for a second workgroup per compute unit.
constexpr int kFewSegs = 1024, kMaxSegs = kSampleMaxVocab / (kSegChunks * 4);
template <class T, int SEGS>
__global__ __launch_bounds__(kRowThreads) void sample_pick_kernel(const SampleArgs a, const SampleWs ws, int row0) {
  constexpr int E = Chunk<T>::E, kWaves = kRowThreads / 64, RUN = kRowList / kRowThreads;
  constexpr bool BF16 = sizeof(T) == 2;
  __shared__ __attribute__((aligned(16))) unsigned long long list[kRowList];
  __shared__ unsigned long long seg[SEGS];
  __shared__ uint64_t sum_a[kWaves], sum_b[kWaves], wave_mass[kWaves];
  __shared__ int found, n_first, n_kept;
  __shared__ double at1_sh;
  __shared__ uint64_t found_base;
  __shared__ unsigned long long listed_mass;
  __shared__ uint32_t begin_sh[4 * kMaxSlices];
  __shared__ uint64_t sorted[kRankMost];
  __shared__ NarrowShared narrow;
  const int r = blockIdx.x, row = row0 + r, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (a.masked != nullptr && a.masked[row] == 0) {
    if (tid == 0) write_row(a, row, -1, 0.f, 0.f);
    return;
  }
  const RowParams p = row_params(a, row);
  const RowCut c = ws.cut[r];
  if (c.way == kNone) {
    if (tid == 0) write_row(a, row, -1, 0.f, 0.f);
    return;
  }
  if (wave == kWaves - 1) {  // the sum of the weights at T = 1 over the slices, beside what the others do
    double at1 = 0.0;
    for (int i = lane; i < ws.slices; i += kWave) {
      const SliceStat t = ws.stat[(int64_t)r * ws.slices + i];
      if (t.top > -INFINITY) at1 += t.at1 * exp((double)t.top - (double)c.top);
    }
    at1_sh = wave_sum(at1);
  }
  if (c.way == kFirst) {
    __syncthreads();
    if (tid == 0) write_row(a, row, c.first_id, (float)(1.0 / at1_sh), 1.f);
    return;
  }
  const Scale s = scale_of(p.temperature);
  uint32_t n = 0;
  uint64_t rest = 0;
  bool slow = c.way == kSearch;
  if (!slow) {
    for (int i = tid; i < ws.segs; i += kRowThreads) seg[i] = ws.seg[(int64_t)r * ws.segs + i];
    if (c.ends) {  // the slices' lists one behind the other: where each begins, then their entries
      for (int i0 = 0; i0 < ws.slices; i0 += kWave) {  // (every wavefront)
        const int i = min(i0 + lane, ws.slices - 1);
        uint32_t k = ws.listed[(int64_t)r * ws.slices + i];
        uint64_t beside = ws.rest[(int64_t)r * ws.slices + i];
        if (i0 + lane >= ws.slices) {
          k = 0;
          beside = 0;
        }
        slow = slow || __ballot(k > (uint32_t)kSliceList) != 0ull;
        uint32_t upto = k;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
          const uint32_t t = __shfl_up(upto, o, kWave);
          if (lane >= o) upto += t;
        }
        if (wave == 0 && i0 + lane < ws.slices) begin_sh[i0 + lane] = n + upto - k;
        n += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) beside += shfl_xor64(beside, o);
        rest += beside;
      }
      slow = slow || n > (uint32_t)kRowList;
      __syncthreads();
      for (uint32_t j = tid; !slow && j < n; j += kRowThreads) {
        int lo = 0, hi = ws.slices - 1;  // the last slice that begins at or in front of j
        while (lo < hi) {
          const int mid = (lo + hi + 1) >> 1;
          if (begin_sh[mid] <= j)
            lo = mid;
          else
            hi = mid - 1;
        }
        list[j] = ws.list[((int64_t)r * ws.slices + lo) * kSliceList + (j - begin_sh[lo])];
      }
    }
  }
  if (slow) {  // uniform over the workgroup
    search_row<T>(a, row, sum_a, sum_b, wave_mass, &found);
    return;
  }
  uint64_t last = 0;  // the last token kept, if the list decides that
  if (tid == 0) {
    n_first = n_kept = 0;
    listed_mass = 0;
  }
  __syncthreads();
  if (c.ends) {
    uint64_t sure = 0;
    for (int i = tid; i < ws.segs; i += kRowThreads) sure += seg[i];
    sure = block_reduce64<kRowThreads>(sure, sum_a, Add64());
    const uint32_t k = (uint32_t)p.top_k;
    const bool cut = p.top_k > 0 && (c.apart || c.count_sure + n >= k);  // top_k ends in the list
    const uint64_t least = order_of(c.least_key, -1);                    // the last that min_p leaves
    auto in_first = [&](uint64_t order) { return !c.apart || of_key(key_in(order)) * c.per_unit >= c.p_low; };  // of [p_low, sure)
    if (n <= (uint32_t)kRankMost) {  // every token against every other: its place in the order; then one thread per place
      int group = kRowThreads;       // threads per token
      while (group > 64 || (uint32_t)(kRowThreads / group) < n) group >>= 1;
      const int e = tid / group, unit = tid & (group - 1);
      const int end = ((int)n + group * kRankAhead - 1) / (group * kRankAhead) * (group * kRankAhead);  // at most 1024
      for (int j = (int)n + tid; j < end; j += kRowThreads) list[j] = ~0ull;
      __syncthreads();
      const uint64_t mine = list[min(e, kRankMost - 1)];
      uint32_t rank = 0;
      for (int j = unit * kRankAhead; j < end; j += group * kRankAhead) {  // eight neighbours at a time
        ulonglong2 other[kRankAhead / 2];
#pragma unroll
        for (int u = 0; u < kRankAhead / 2; ++u) other[u] = *reinterpret_cast<const ulonglong2*>(list + j + 2 * u);
#pragma unroll
        for (int u = 0; u < kRankAhead / 2; ++u) rank += (other[u].x < mine ? 1u : 0u) + (other[u].y < mine ? 1u : 0u);
      }
      for (int o = 1; o < group; o <<= 1) rank += __shfl_xor(rank, o, kWave);
      if (e < (int)n && unit == 0) sorted[rank] = mine;
      __syncthreads();
      const bool live = tid < (int)n;
      const uint64_t order = live ? sorted[tid] : ~(uint64_t)0;
      const uint64_t m = live ? mass<BF16>(of_key(key_in(order)), c.top, s) : 0;
      const bool first = live && in_first(order);
      const unsigned long long firsts = __ballot(first);
      if (lane == 0 && firsts != 0ull) atomicAdd(&n_first, (int)__popcll(firsts));
      uint64_t front = wave_inclusive64(m, lane);
      if (lane == 63) sum_b[wave] = front;
      __syncthreads();
      front -= m;
      for (int w = 0; w < wave; ++w) front += sum_b[w];
      const uint32_t in_front = tid < n_first ? c.count_sure + (uint32_t)tid : c.count_k + (uint32_t)(tid - n_first);  // tokens above
      if (cut && live && in_front < k && (in_front + 1 == k || tid + 1 == (int)n)) listed_mass = front + m;  // the mass of the first top_k
      __syncthreads();
      const double target = p.top_p < 1.f ? (double)p.top_p * (double)(sure + rest + (cut ? listed_mass : 0)) : INFINITY;
      const bool kept = first && (!cut || in_front < k) && (double)(sure + front) < target && order <= least;
      const unsigned long long some = __ballot(kept);
      if (some != 0ull && lane == 0) atomicAdd(&n_kept, (int)__popcll(some));
      if (kept) atomicAdd(&seg[(int)(uint32_t)order / (E * kSegChunks)], (unsigned long long)m);
      __syncthreads();
      last = n_kept > 0 ? sorted[n_kept - 1] : 0;  // a prefix
    } else {
      uint64_t order[RUN], m[RUN], first_part = 0;
      uint32_t first = 0, second = 0;
#pragma unroll
      for (int u = 0; u < RUN; ++u) {
        const int j = tid + u * kRowThreads;
        order[u] = j < (int)n ? list[j] : 0;
        m[u] = j < (int)n ? mass<BF16>(of_key(key_in(order[u])), c.top, s) : 0;
        if (j < (int)n) {
          if (in_first(order[u])) {
            first |= 1u << u;
            first_part += m[u];
          } else {
            second |= 1u << u;
          }
        }
      }
      End end{0, 0};
      if (cut) end = find_end<RUN>(order, m, c.apart ? second : first, true, c.apart ? c.count_k : c.count_sure, k, 0, 0.0, narrow);
      if (p.top_p < 1.f) {
        uint64_t all = sure + rest + end.mass;  // (nothing is cut: end.mass = 0)
        if (c.apart) all += block_reduce64<kRowThreads>(first_part, sum_b, Add64());
        end = find_end<RUN>(order, m, first, false, 0, 0, sure, (double)p.top_p * (double)all, narrow);
      }
      last = end.last < least ? end.last : least;
#pragma unroll
      for (int u = 0; u < RUN; ++u)
        if (((first >> u) & 1u) && order[u] <= last) atomicAdd(&seg[(int)(uint32_t)order[u] / (E * kSegChunks)], (unsigned long long)m[u]);
    }
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
  uint64_t end[E], upto = 0;  // masses of the kept ones, the sure and the listed, up to each token of the chunk
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float v = x.z[e];
    if ((v * c.per_unit >= c.sure && v >= c.least) || (c.ends && order_of(key_of(v), chunk * E + e) <= last)) upto += mass<BF16>(v, c.top, s);
    end[e] = upto;
  }
  before = wave_inclusive64(end[E - 1], lane) - end[E - 1] + found_base;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (here(before + (e > 0 ? end[e > 0 ? e - 1 : 0] : 0), before + end[e])) {
      const float v = x.z[e];
      write_row(a, row, chunk * E + e, (float)((double)weight<BF16>(v, c.top, scale_of(1.f)) / at1_sh),
                (float)((double)weight<BF16>(v, c.top, s) / ((double)total * kMassUnit)));
    }
  }
}

struct SamplePlan {
  int slice, slices, segs, rows;  // logits of a slice; rows of a pass
  size_t stat, bins, rest, listed, list, cut, seg, total;
};
// Slices of kSlice of a call that takes quarters instead: a quarter of the work a workgroup, and four times the histograms to add up.  Top_k 50, top_p
// 0.95, slices and quarters: 126 464 logits, 1 row (8 slices) 27.1 and 23.3 us, 8 rows 28.4 and 24.9, 12 28.4 and 28.2, 24 29.2 and 33.3, 64 37.3 and 57.2;
// 32 003, 1 row (2 slices) 26.3 and 21.3, 32 rows 28.0 and 23.5, 64 28.7 and 27.1, 128 29.2 and 37.3.
constexpr int kSmallPlans = 64;
constexpr int kMostRows = 1024, kMostRowSlices = 4096;  // rows and slices of a pass
// Where the parts of a workspace lie for so many rows, slices of all rows and segments of all rows.
static void place_parts(SamplePlan& p, size_t rows, size_t n, size_t segs) {
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += (bytes + 255) & ~(size_t)255;
    return at;
  };
  p.stat = take(n * sizeof(SliceStat));
  p.bins = take(n * kBins * sizeof(uint64_t));
  p.rest = take(n * sizeof(uint64_t));
  p.listed = take(n * sizeof(uint32_t));
  p.list = take(n * kSliceList * sizeof(uint64_t));
  p.cut = take(rows * sizeof(RowCut));
  p.seg = take(segs * sizeof(uint64_t));
  p.total = off;
}
// Few rows: slices of a quarter, so that more compute units share a row.
static SamplePlan plan_sample(int n_rows, int vocab) {
  SamplePlan p;
  p.slice = (int64_t)n_rows * ceil_div(vocab, kSlice) <= kSmallPlans && ceil_div(vocab, kSliceSmall) <= 4 * kMaxSlices ? kSliceSmall : kSlice;
  p.slices = ceil_div(vocab, p.slice);
  p.segs = ceil_div(vocab, kSegChunks * 4);  // of float32, which has the shorter chunks
  p.rows = std::max(1, std::min({n_rows, kMostRows, kMostRowSlices / p.slices}));
  place_parts(p, p.rows, (size_t)p.rows * p.slices, (size_t)p.rows * p.segs);
  return p;
}
// What every plan of up to so many rows and so large a vocabulary fits into, part for part, so that a caller's workspace for its largest call
// serves the smaller ones: fewer rows can mean more slices.  A quarter's plan has at most 4 * kSmallPlans slices; a slice has
// kSlice / (4 * kSegChunks) segments.
size_t sample_tokens_workspace(int n_rows, int vocab) {
  const size_t rows = std::min(n_rows, kMostRows);
  const size_t quarters = std::min<size_t>(rows * ceil_div(vocab, kSliceSmall), 4 * kSmallPlans);
  const size_t slices = std::min<size_t>(rows * ceil_div(vocab, kSlice), kMostRowSlices);
  SamplePlan p;
  place_parts(p, rows, std::max(quarters, slices), std::min<size_t>(rows * ceil_div(vocab, kSegChunks * 4), (size_t)kMostRowSlices * (kSlice / (4 * kSegChunks))));
  return p.total;
}

template <class T>
static hipError_t launch_sample_t(const SampleArgs& a, const SamplePlan& p, char* w, hipStream_t st) {
  SampleWs ws;
  ws.stat = reinterpret_cast<SliceStat*>(w + p.stat);
  ws.bins = reinterpret_cast<uint64_t*>(w + p.bins);
  ws.rest = reinterpret_cast<uint64_t*>(w + p.rest);
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
    if (ws.segs <= kFewSegs)
      hipLaunchKernelGGL((sample_pick_kernel<T, kFewSegs>), dim3(rows), dim3(kRowThreads), 0, st, a, ws, row0);
    else
      hipLaunchKernelGGL((sample_pick_kernel<T, kMaxSegs>), dim3(rows), dim3(kRowThreads), 0, st, a, ws, row0);
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
