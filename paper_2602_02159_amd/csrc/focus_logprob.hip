// Log probabilities of given tokens, entropies and the likeliest tokens.
//
// With m the largest logit of a row and y_v = z_v - m, what has to be known is r = sum of exp(y_v) over all tokens but one of the largest, and
// A = sum of exp(y_v) y_v:
//   log sum exp(z) = m + log1p(r)        log p_t = z_t - m - log1p(r)        entropy = log1p(r) - A / (1 + r)
// Leaving the largest out of the sum keeps the digits of rows that are all but certain: 1 + r would round them away.
//
//   logprob_part_kernel  a workgroup has 8192 logits of a row, 32 a thread, in registers: their largest, r and A, and the largest of each four threads
//   logprob_join_kernel  a workgroup a row: the parts together; the likeliest tokens
// The likeliest: 64 numbers of a part, each the largest of 128 logits, are all that the first launch writes.  A number that top_n of all of them reach is
// reached by top_n logits, and what reaches it lies in some 1.2 top_n of those 128s, which the second launch reads once more.  (Each part with a list of its own
// likeliest: 500 rows of 126 464, 20 alternatives 43.4 us instead of 32.3.)
// Every logit is read once.  What bounds it: many rows, HBM and the exponentials: 500 x 126 464 bf16, 126 MB, in 24.6 us = 5.1 TB/s
// and 8.9 us for the rows' ends; 511 x 32 003 fp32 in 13.5 + 6.6.  One row (3.5 + 6 us): the chain of round trips in two launches that depend on each other.
// Not better: parts of 2048 for few rows (one row 14.5 us instead of 14.0 at that time), 16 logits a thread (50 instead of 43), 24 (42.4 instead of 43.3, but
// more parts than one a thread).
#include <type_traits>

#include "focus_common.h"
#include "focus_kernels.h"
#include "focus_topk.h"

namespace focus {

constexpr int kLogitsThread = 32, kLogitsPart = 256 * kLogitsThread;
// candidates and fours that are listed at most (more: list_in_turn); up to 96 candidates are compared each with all (5 x 1000 logits, of which all are: 65 us
// that way, 17 narrowed first)
constexpr int kTopCandidates = 1024, kTopFours = 1024, kTopRanked = 96;

// NaN as -inf, +inf as the largest number
__device__ __forceinline__ float tame(float x) { return fminf(fmaxf(x, -INFINITY), 3.4028234663852886e38f); }
// place in the order of the logits, 0 for those that are no candidate
__device__ __forceinline__ uint32_t top_key(float z) { return z == -INFINITY ? 0u : order_key(z); }

struct LogprobArgs {
  const void* logits;
  const int32_t* targets;
  const uint8_t* masked;
  float* logprob;
  float* entropy;
  int32_t* top_ids;
  float* top_logprobs;
  float4* part;     // [n_rows, n_parts] (m, r, A in units of log 2, -)
  float* part_top;  // [n_rows, n_parts, 64] the largest logit of each four threads, -inf: none
  int64_t row_stride;
  int vocab, n_parts, top_n;
};

// one logit of a row
template <class T>
__device__ __forceinline__ float logit(const T* row, int id) {
  return tame(sizeof(T) == 4 ? *reinterpret_cast<const float*>(row + id) : bf16_lo(*reinterpret_cast<const uint16_t*>(row + id)));
}

// over the wavefront, in a fixed order; every lane receives the result
__device__ __forceinline__ float wave_sum_fast(float x) { return group_sum(row_sum16(x)); }
__device__ __forceinline__ float four_max(float x) {  // of four threads
  x = fmaxf(x, lane_dpp<0xB1>(x));
  return fmaxf(x, lane_dpp<0x4E>(x));
}
__device__ __forceinline__ float wave_max_fours(float x) {
  x = fmaxf(x, lane_dpp<0x141>(x));
  x = fmaxf(x, lane_dpp<0x140>(x));
  return group_max(x);
}
// over the workgroup of four wavefronts; `sh` of four entries
__device__ __forceinline__ float block_max4(float x, float* sh) {
  x = wave_max_fours(four_max(x));
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  return fmaxf(fmaxf(sh[0], sh[1]), fmaxf(sh[2], sh[3]));
}

struct TopShared256 {
  uint32_t best[64];
  unsigned long long list[kTopCandidates];
  unsigned long long shares[64];
  int fours[kTopFours];
  uint32_t count, n_fours;
};
// (key, id) as one number: larger = earlier in the order, the lower id first
__device__ __forceinline__ unsigned long long place_of(uint32_t key, int id) { return ((unsigned long long)key << 32) | (uint32_t)~id; }

// A number that at least top_n entries reach, to sixteen bits: the top_n-th largest of the best of each four threads (1 where fewer have one).  64 of
// them are one a lane, and the search one ballot a bit.
__device__ __forceinline__ uint32_t top_threshold(TopShared256& sm, uint32_t best, int top_n) {
  const int tid = threadIdx.x;
  best = max(best, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)best, 0xB1, 0xF, 0xF, false));  // quad_perm [1,0,3,2]
  best = max(best, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)best, 0x4E, 0xF, 0xF, false));  // quad_perm [2,3,0,1]
  if ((tid & 3) == 0) sm.best[tid >> 2] = best;
  if (tid == 0) sm.count = sm.n_fours = 0u;
  __syncthreads();
  const uint32_t k = sm.best[tid & 63] >> 16;  // every wavefront searches for itself
  uint32_t t = 0u;
#pragma unroll 1
  for (int bit = 15; bit >= 0; --bit) {
    const uint32_t with = t | (1u << bit);
    const int n = __popcll(__ballot(k >= with));
    t = n >= top_n ? with : t;
    if (n == top_n) break;  // exactly these
  }
  return max(t << 16, 1u);
}
__device__ __forceinline__ void list_candidate(TopShared256& sm, uint32_t key, int id) {
  const uint32_t at = atomicAdd(&sm.count, 1u);  // (the list's order does not matter)
  if (at < (uint32_t)kTopCandidates) sm.list[at] = place_of(key, id);
}
// The first top_n of the n listed candidates, found by comparing each with all, four threads a candidate: emit(rank, key, id)
template <class Emit>
__device__ __forceinline__ void rank_candidates(const TopShared256& sm, int n, int top_n, const Emit emit) {
  const int part = threadIdx.x & 3;
  for (int i = threadIdx.x >> 2; i < n; i += 64) {
    const unsigned long long mine = sm.list[i];
    uint32_t rank = 0u;
#pragma unroll 1
    for (int j0 = part; j0 < n; j0 += 32) {
#pragma unroll
      for (int j = 0; j < 32; j += 4) rank += j0 + j < n && sm.list[min(j0 + j, kTopCandidates - 1)] > mine ? 1u : 0u;
    }
    rank += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)rank, 0xB1, 0xF, 0xF, false);
    rank += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)rank, 0x4E, 0xF, 0xF, false);
    if (part == 0 && (int)rank < top_n) emit((int)rank, (uint32_t)(mine >> 32), (int)~(uint32_t)mine);
  }
}
// Drops listed candidates that cannot be among the first top_n of n: those behind the top_n-th of the best of 64 shares of the list, ids counted.  Returns that
// one's place (0: fewer shares have any).  Up to 16 top_n stay, some 1.2 top_n where the list is in no order.
__device__ __forceinline__ unsigned long long narrow_list(TopShared256& sm, int n, int top_n) {
  constexpr int kEach = kTopCandidates / 256;
  const int tid = threadIdx.x;
  unsigned long long mine[kEach], best = 0ull;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    mine[i] = tid + 256 * i < n ? sm.list[tid + 256 * i] : 0ull;
    best = mine[i] > best ? mine[i] : best;
  }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    const unsigned long long other = __shfl_xor(best, o, kWave);
    best = other > best ? other : best;
  }
  if ((tid & 3) == 0) sm.shares[tid >> 2] = best;
  __syncthreads();
  if (tid == 0) sm.count = 0u;
  const unsigned long long share = sm.shares[tid & 63];
  int rank = 0;
#pragma unroll 8
  for (int j = 0; j < 64; ++j) rank += sm.shares[j] > share ? 1 : 0;
  const unsigned long long last = __ballot(rank == top_n - 1 && share != 0ull);
  const unsigned long long bound = last == 0ull ? 0ull : sm.shares[__builtin_ctzll(last)];
  __syncthreads();
#pragma unroll 1
  for (int i = 0; i < kEach; ++i) {
    const unsigned long long x = i == 0 ? mine[0] : (i == 1 ? mine[1] : (i == 2 ? mine[2] : mine[3]));
    if (x != 0ull && x >= bound) sm.list[atomicAdd(&sm.count, 1u)] = x;
  }
  __syncthreads();
  return bound;
}
// More candidates than the list holds (equal logits): the row from its first id on.  Where the list fills up it is narrowed, and from there on only larger logits
// come in than the bound's, as equal ones have higher ids.  key_at(id): 0 for none
template <class Key>
__device__ __forceinline__ void list_in_turn(TopShared256& sm, uint32_t bound, int vocab, int top_n, const Key key_at) {
  constexpr int U = 8;
  const int tid = threadIdx.x;
  __syncthreads();
  if (tid == 0) sm.count = 0u;
  __syncthreads();
#pragma unroll 1
  for (int base = 0; base < vocab; base += U * 256) {
    uint32_t key[U], any = 0u;
#pragma unroll
    for (int u = 0; u < U; ++u) key[u] = base + u * 256 + tid < vocab ? key_at(base + u * 256 + tid) : 0u;
#pragma unroll
    for (int u = 0; u < U; ++u) any |= key[u] >= bound ? 1u : 0u;
    if (__syncthreads_or((int)any) == 0) continue;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (key[u] >= bound) list_candidate(sm, key[u], base + u * 256 + tid);
      __syncthreads();
      const int n = (int)sm.count;
      if (n > kTopCandidates - 256) {  // whole workgroup
        bound = max((uint32_t)(narrow_list(sm, n, top_n) >> 32) + 1u, bound);
      }
      __syncthreads();
    }
  }
}

constexpr float kLog2eF = 1.4426950408889634f, kLn2F = 0.6931471805599453f;
constexpr float kNothing = -200.f;  // 2^-200 is zero: exponents below are taken as this one, so that no 0 times infinity comes up

template <class T>
__global__ __launch_bounds__(256, 6) void logprob_part_kernel(const LogprobArgs p) {
  constexpr int E = 16 / sizeof(T), V = kLogitsThread / E;  // logits a load, loads
  __shared__ float max_sh[4];
  __shared__ float4 sum_sh[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = blockIdx.y, part = blockIdx.x;
  const T* z_row = static_cast<const T*>(p.logits) + (int64_t)row * p.row_stride;
  const int first = part * kLogitsPart + tid * E;
  float z[kLogitsThread];
  {
    uint4 w[V];
    const int whole = p.vocab / E * E - E;  // the last id from which sixteen bytes can be read, if any
    if (whole >= 0) {
#pragma unroll
      for (int k = 0; k < V; ++k) w[k] = *reinterpret_cast<const uint4*>(z_row + min(first + k * 256 * E, whole));
    }
    if (p.masked && p.masked[row] == 0) return;  // whole workgroup
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const uint32_t u[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
      const bool in = first + k * 256 * E <= whole;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float x = sizeof(T) == 4 ? __uint_as_float(u[e & 3]) : ((e & 1) ? bf16_hi(u[(e >> 1) & 3]) : bf16_lo(u[(e >> 1) & 3]));
        z[k * E + e] = in ? x : -INFINITY;  // as it is: see below
      }
    }
    if (part == (int)gridDim.x - 1) {  // a row's last, shorter piece, logit by logit
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int id = first + k * 256 * E;
        if (id > whole && id < p.vocab) {
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (id + e < p.vocab) z[k * E + e] = logit(z_row, id + e);
        }
      }
    }
  }
  // A NaN needs no care: the largest of it and a number is the number, its weight that of kNothing, and no comparison takes it.  (v_med3_f32 with
  // an infinity is a maximum that asks for no other form of its operands.)  +inf is made the largest number where a part has one.
  float mine = -INFINITY;
#pragma unroll
  for (int i = 0; i < kLogitsThread; ++i) mine = __builtin_amdgcn_fmed3f(mine, z[i], INFINITY);
  const float best = four_max(mine);
  if (p.top_n > 0 && (tid & 3) == 0) p.part_top[((int64_t)row * p.n_parts + part) * 64 + (tid >> 2)] = tame(best);
  float m = block_max4(best, max_sh);
  if (m == INFINITY) {  // whole workgroup
#pragma unroll
    for (int i = 0; i < kLogitsThread; ++i) z[i] = tame(z[i]);
    mine = tame(mine);
    m = tame(m);
  }
  const float m_use = m == -INFINITY ? 0.f : m;

  float rest = 0.f, A = 0.f;  // of the logits below m;
  int equal = 0;              // how many equal it
  auto weight = [&](float x, float& y) __attribute__((always_inline)) {
    y = __builtin_amdgcn_fmed3f((x - m_use) * kLog2eF, kNothing, INFINITY);
    return __builtin_amdgcn_exp2f(y);
  };
  if (__ballot(mine == m) != 0ull) {
#pragma unroll
    for (int i = 0; i < kLogitsThread; ++i) {
      float y;
      const float e = weight(z[i], y);
      A = __builtin_fmaf(e, y, A);
      const bool top = z[i] == m;
      rest += top ? 0.f : e;
      equal += top ? 1 : 0;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kLogitsThread; ++i) {
      float y;
      const float e = weight(z[i], y);
      A = __builtin_fmaf(e, y, A);
      rest += e;
    }
  }
  rest = wave_sum_fast(rest);
  A = wave_sum_fast(A);
  const float n_equal = wave_sum_fast((float)equal);
  if (lane == 0) sum_sh[wave] = make_float4(rest, A, n_equal, 0.f);
  __syncthreads();
  if (tid == 0) {
    float r = 0.f, a = 0.f, n = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      r += sum_sh[k].x;
      a += sum_sh[k].y;
      n += sum_sh[k].z;
    }
    p.part[(int64_t)row * p.n_parts + part] = m == -INFINITY ? make_float4(-INFINITY, 0.f, 0.f, 0.f) : make_float4(m, r + (n - 1.f), a, 0.f);
  }
}

template <class T>
__global__ __launch_bounds__(256) void logprob_join_kernel(const LogprobArgs p) {
  constexpr int E = 16 / sizeof(T), V = kLogitsThread / E;
  constexpr int kFours = 4, kLoads = V / 2;  // (a logit of 32 bits has twice the loads)
  __shared__ float max_sh[4];
  __shared__ float2 sum_sh[4];
  __shared__ TopShared256 top_sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = blockIdx.x;
  const bool live = !p.masked || p.masked[row] != 0;
  int target = -1;
  float z_t = -INFINITY;
  if (p.targets && live) {
    target = p.targets[row];
    if (target >= 0 && target < p.vocab) {
      z_t = logit(static_cast<const T*>(p.logits) + (int64_t)row * p.row_stride, target);
    }
  }
  if (!live) {  // whole workgroup
    if (tid == 0) {
      if (p.logprob) p.logprob[row] = 0.f;
      if (p.entropy) p.entropy[row] = 0.f;
    }
    for (int i = tid; i < p.top_n; i += 256) {
      p.top_ids[(int64_t)row * p.top_n + i] = -1;
      p.top_logprobs[(int64_t)row * p.top_n + i] = -INFINITY;
    }
    return;
  }
  float4 s = make_float4(-INFINITY, 0.f, 0.f, 0.f);  // at most 256 parts: one a thread
  if (tid < p.n_parts) s = p.part[(int64_t)row * p.n_parts + tid];
  const float* tops = p.part_top + (int64_t)row * p.n_parts * 64;
  // Thread t has the (t / 4)-th of the parts t % 4, t % 4 + 4, ...: four threads together have one of every part, a part alone is spread over all
  const int n = p.top_n > 0 ? p.n_parts * 64 : 0, mine0 = (tid & 3) * 64 + (tid >> 2);
  float top_of[kFours];  // those of the first 16 parts, here before the statistics are
#pragma unroll
  for (int i = 0; i < kFours; ++i) top_of[i] = mine0 + 256 * i < n ? tops[mine0 + 256 * i] : -INFINITY;
  const float m = block_max4(s.x, max_sh), m_use = m == -INFINITY ? 0.f : m;
  // Of the parts whose largest logit is the row's the first one's is left out of r
  const unsigned long long top = __ballot(s.x == m && m != -INFINITY);
  int before = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) before += w < wave && max_sh[w] == m ? 1 : 0;
  const bool first = before == 0 && top != 0ull && lane == __builtin_ctzll(top | (1ull << 63));
  const float d = fmaxf((s.x - m_use) * kLog2eF, kNothing), f = __builtin_amdgcn_exp2f(d);
  const float whole = s.x == -INFINITY ? 0.f : 1.f + s.y;
  const float r_mine = wave_sum_fast(first ? s.y : f * whole), a_mine = wave_sum_fast(f * (s.z + whole * d));
  if (lane == 0) sum_sh[wave] = make_float2(r_mine, a_mine);
  __syncthreads();
  float r = 0.f, a = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    r += sum_sh[w].x;
    a += sum_sh[w].y;
  }
  const float log_sum = log1pf(r);
  if (tid == 0) {
    if (p.logprob) p.logprob[row] = target < 0 || target >= p.vocab ? 0.f : (m == -INFINITY ? -INFINITY : (z_t - m) - log_sum);
    if (p.entropy) p.entropy[row] = m == -INFINITY ? 0.f : log_sum - kLn2F * a / (1.f + r);
  }
  if (p.top_n == 0) return;
  // The threads that had a candidate, four by four, then their logits once more
  uint32_t best = 0u;
#pragma unroll
  for (int i = 0; i < kFours; ++i) best = max(best, top_key(top_of[i]));
  for (int i = mine0 + 256 * kFours; i < n; i += 256) best = max(best, top_key(tops[i]));
  const uint32_t threshold = top_threshold(top_sh, best, p.top_n);
  if (best >= threshold) {
    auto take = [&](float x, int i) __attribute__((always_inline)) {
      if (top_key(x) < threshold) return;
      const uint32_t at = atomicAdd(&top_sh.n_fours, 1u);
      if (at < (uint32_t)kTopFours) top_sh.fours[at] = i;
    };
#pragma unroll
    for (int i = 0; i < kFours; ++i) take(top_of[i], mine0 + 256 * i);
    for (int i = mine0 + 256 * kFours; i < n; i += 256) take(tops[i], i);
  }
  __syncthreads();
  const T* z_row = static_cast<const T*>(p.logits) + (int64_t)row * p.row_stride;
  const int n_fours = (int)top_sh.n_fours, n_loads = n_fours <= kTopFours ? n_fours * 4 * V : 0;
  const float least = threshold < 0x00800000u ? -3.4028234663852886e38f : order_value(threshold);  // (0x00800000: the lowest number's key)
  auto id_of = [&](int i) __attribute__((always_inline)) {
    const int four = top_sh.fours[i / (4 * V)], k = i % (4 * V) / 4;
    return (four / 64) * kLogitsPart + k * (256 * E) + ((four % 64) * 4 + i % 4) * E;
  };
#pragma unroll 1
  for (int i0 = tid; i0 < n_loads; i0 += 256 * kLoads) {
    uint4 w[kLoads];
    uint32_t some = 0u;  // those that reach the threshold, and all at a row's end
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
      w[l] = make_uint4(0u, 0u, 0u, 0u);
      if (i0 - tid + 256 * l >= n_loads) continue;  // whole workgroup
      const int i = i0 + 256 * l, id = id_of(min(i, n_loads - 1));
      if (id + E <= p.vocab) w[l] = *reinterpret_cast<const uint4*>(z_row + id);
      if (i < n_loads && id + E > p.vocab) some |= ((1u << E) - 1u) << (E * l);
    }
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
      const uint32_t u[4] = {w[l].x, w[l].y, w[l].z, w[l].w};
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float x = sizeof(T) == 4 ? __uint_as_float(u[e & 3]) : ((e & 1) ? bf16_hi(u[(e >> 1) & 3]) : bf16_lo(u[(e >> 1) & 3]));
        some |= x >= least ? 1u << (E * l + e) : 0u;
      }
    }
    while (some != 0u) {  // few, which come from the cache
      const int bit = __builtin_ctz(some), i = i0 + bit / E * 256;
      some &= some - 1u;
      if (i >= n_loads) break;
      const int id = id_of(i) + bit % E;
      const uint32_t key = id < p.vocab ? top_key(logit(z_row, id)) : 0u;
      if (key >= threshold) list_candidate(top_sh, key, id);
    }
  }
  __syncthreads();
  if (n_fours > kTopFours || top_sh.count > (uint32_t)kTopCandidates)  // whole workgroup
    list_in_turn(top_sh, threshold, p.vocab, p.top_n, [&](int id) __attribute__((always_inline)) { return top_key(logit(z_row, id)); });
  __syncthreads();
  auto emit = [&](int rank, uint32_t key, int id) __attribute__((always_inline)) {
    p.top_ids[(int64_t)row * p.top_n + rank] = id;
    p.top_logprobs[(int64_t)row * p.top_n + rank] = id < 0 ? -INFINITY : (order_value(key) - m) - log_sum;
  };
  int listed = (int)top_sh.count;
  if (listed > kTopRanked) {
    narrow_list(top_sh, listed, p.top_n);
    listed = (int)top_sh.count;
  }
  rank_candidates(top_sh, listed, p.top_n, emit);
  for (int i = listed + tid; i < p.top_n; i += 256) emit(i, 0u, -1);
}

static size_t logprob_parts_bytes(int n_rows, int n_parts) { return (size_t)n_rows * n_parts * sizeof(float4); }
size_t token_logprobs_workspace(int n_rows, int vocab, int top_n) {
  const int n_parts = ceil_div(vocab, kLogitsPart);
  return logprob_parts_bytes(n_rows, n_parts) + (top_n > 0 ? (size_t)n_rows * n_parts * 64 * sizeof(float) : 0);
}

template <class T>
static hipError_t launch_logprobs_t(const LogprobArgs& p, int n_rows, hipStream_t st) {
  hipLaunchKernelGGL(logprob_part_kernel<T>, dim3(p.n_parts, n_rows), dim3(256), 0, st, p);
  hipLaunchKernelGGL(logprob_join_kernel<T>, dim3(n_rows), dim3(256), 0, st, p);
  return hipGetLastError();
}
hipError_t launch_token_logprobs(const void* logits, int dtype, int64_t row_stride, const int32_t* targets, const uint8_t* masked, int n_rows, int vocab,
                                 int top_n, float* logprob, float* entropy, int32_t* top_ids, float* top_logprobs, void* workspace, hipStream_t st) {
  LogprobArgs p;
  p.logits = logits;
  p.targets = targets;
  p.masked = masked;
  p.logprob = logprob;
  p.entropy = entropy;
  p.top_ids = top_ids;
  p.top_logprobs = top_logprobs;
  p.row_stride = row_stride;
  p.vocab = vocab;
  p.n_parts = ceil_div(vocab, kLogitsPart);
  p.top_n = top_n;
  p.part = static_cast<float4*>(workspace);
  p.part_top = reinterpret_cast<float*>(static_cast<char*>(workspace) + logprob_parts_bytes(n_rows, p.n_parts));
  return dtype == FOCUS_F32 ? launch_logprobs_t<float>(p, n_rows, st) : launch_logprobs_t<uint16_t>(p, n_rows, st);
}

}  // namespace focus
