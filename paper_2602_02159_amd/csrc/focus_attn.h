// Device code that the attention kernels share: sub-tiles of the key list, the loads of their rows, operand layouts, the softmax
// step, the arguments, the ranking of the blocks in a prologue, the order of the rounds of a key split.
#pragma once

#include <type_traits>

#include "focus_common.h"
#include "focus_kernels.h"
#include "focus_topk.h"

namespace focus {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <int D>
struct Geo {
  static constexpr int kChunks = D / 8;               // 16-byte chunks per row
  static constexpr int kRowsPerLoad = 64 / kChunks;   // rows covered by one wave-wide 16-byte load
  static constexpr int kLoads = kSubTile / kRowsPerLoad;
  static constexpr int kKSteps = D / 32;              // MFMA k-steps of the QK^T product
  static constexpr int kColTiles = D / 16;            // 16-wide d tiles of the PV product
  static constexpr int kRowBytes = D * 2;
  static constexpr int kStageBytes = kSubTile * kRowBytes;  // one staged K (or V) sub-tile
};

// byte offset of 16-byte chunk `chunk` of staged row `row`: position chunk ^ (row mod chunks-per-row)
template <int D>
__device__ __forceinline__ int stage_off(int row, int chunk) {
  return row * Geo<D>::kRowBytes + ((chunk ^ (row & (Geo<D>::kChunks - 1))) << 4);
}

// swizzle of a V stage that is read in transposed 32x32x16 operands (see read_v_operand32)
template <int D>
__device__ __forceinline__ int vstage_swz(int row) {
  return D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2;
}

// cache policy of the K/V row loads: non-temporal (every row is read once per launch)
constexpr int kStreamPolicy = 2;

// s_waitcnt vmcnt(0): every outstanding global load, LDS-direct ones included, has landed
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }
// s_waitcnt vmcnt(N): every global load and store but the N issued last has completed
template <int N>
__device__ __forceinline__ void wait_loads_but() {
  static_assert(N < 64, "six bits");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
  __builtin_amdgcn_sched_barrier(0);
}
// s_waitcnt lgkmcnt(0): every LDS read of this wavefront has returned.  Placed before an LDS-direct load that
// overwrites a stage the wavefront has just read: that write-after-read order is not covered by vmcnt, and the fence
// keeps the compiler from moving the load above the wait.
__device__ __forceinline__ void wait_lds_reads() {
  __builtin_amdgcn_s_waitcnt(0xC07F);
  __builtin_amdgcn_sched_barrier(0);
}

// ---------------------------------------------------------------------------------------- sub-tiles
// Which rows of K/V a sub-tile covers.  Wave-uniform.
struct SubTile {
  int row0;        // first row when contiguous (kind 0), first sink entry when kind 1
  int kind;        // 0: contiguous rows row0 .. ; 1: scattered rows sink_idx[row0 + slot]
  uint32_t vmask;  // bit s set: slot s holds a key that takes part
  int sink_row;    // kind 1, per lane: the row that slot `lane` stages (lanes 0..31; see subtile_row)
};

__device__ __forceinline__ uint32_t low_mask(int n) { return n >= 32 ? 0xffffffffu : (n > 0 ? ((1u << n) - 1u) : 0u); }

// Locate sub-tile `st` of the attention key list: kept blocks first (n_keep * sub_per_block sub-tiles), then
// the response rows, then the sinks.  Block ids outside [0, n_b) are skipped.  The union of Eq. 8 is a set:
// a sink is dropped when it is outside the prompt, inside a kept block or listed earlier in sink_idx (the block
// list itself must not repeat a block).  For sink sub-tiles lane r < 32 owns slot r.  dense_rows > 0 replaces all of
// that by "all of the first dense_rows rows".
//   "inside a kept block": one look-up in `kept_bits` (bit b set <=> block b is kept; LDS, built by the workgroup)
//   when that is given, else the block list is scanned 64 entries per load.
//   "listed earlier": a strictly ascending list (what focus_find_sinks writes) cannot repeat an entry; `ascending`
//   says so (1 / 0, established once by the workgroup), or -1: not known, then a scan of 64 entries per step
//   establishes it here.  Only lists that are not ascending pay for the all-pairs comparison.
// A list of at most one sub-tile (n_sink <= 32) costs no memory access here: lane r < n_sink holds its entry r in `few_sinks`
// (-1 in the other lanes), requested at the start of the kernel.
constexpr int kBitmapBlocks = 8192;  // largest n_b for which workgroups keep a bitmap of the kept blocks
// A wave-uniform 4-byte read of global memory that no kernel writes while this one runs, issued as a scalar load: it
// returns through the scalar cache instead of queueing behind the wavefront's vector loads (which return in order), and
// a hit there is much quicker than a vector load's trip through L2.
__device__ __forceinline__ int32_t uniform_load(const int32_t* ptr) {
  typedef const __attribute__((address_space(4))) int32_t* cptr_t;
  return *(cptr_t)(uintptr_t)ptr;
}
__device__ __forceinline__ int32_t uniform_load(const uint16_t* ptr) { return *ptr; }  // (lists of 16 bits lie in LDS: KeptList)
// Sub-tile `st` of the sink list
template <class Id>
__device__ __forceinline__ SubTile locate_sinks(int st, int lane, int M, int B, const Id* __restrict__ kept_blocks, int n_keep,
                                                const int32_t* __restrict__ sink_idx, int n_sink, const uint32_t* kept_bits, int ascending,
                                                int few_sinks) {
  SubTile t;
  t.kind = 1;
  t.row0 = st * kSubTile;
  const int e = t.row0 + lane;
  const bool few = n_sink <= kSubTile;  // the list is one sub-tile, which the caller holds in registers
  const int mine = few ? few_sinks : ((lane < kSubTile && e < n_sink) ? sink_idx[e] : -1);
  const int n_slots = min(n_sink - t.row0, kSubTile);
  const bool in_prompt = mine >= 0 && mine < M;
  const int my_block = in_prompt ? mine / B : -1;
  uint32_t bad = 0u;
  if (kept_bits != nullptr) {
    const bool kept = my_block >= 0 && ((kept_bits[my_block >> 5] >> (my_block & 31)) & 1u);
    bad = (uint32_t)(__ballot(kept) & 0xffffffffull);
  } else {
    for (int j0 = 0; j0 < n_keep; j0 += kWave) {
      const int v = j0 + lane < n_keep ? kept_blocks[j0 + lane] : -2;
      for (int r = 0; r < n_slots; ++r) {
        const int sb = __builtin_amdgcn_readlane(my_block, r);
        if (__ballot(v == sb) != 0ull) bad |= 1u << r;
      }
    }
  }
  const int e_end = min(t.row0 + kSubTile, n_sink);
  if (few) {
    const int before = __shfl_up(mine, 1, kWave);
    ascending = 1;
    if (__ballot(lane > 0 && lane < n_sink && mine <= before) != 0ull) {
      for (int r = 1; r < n_slots; ++r)
        if (__ballot(mine == __builtin_amdgcn_readlane(mine, r) && lane < r) != 0ull) bad |= 1u << r;
    }
  }
  if (ascending < 0) {  // sink_idx[0 .. e_end) strictly ascending?
    ascending = 1;
    for (int j0 = 0; j0 + 1 < e_end; j0 += kWave) {
      const int idx = j0 + lane;
      const bool pair = idx + 1 < e_end;
      const int a = pair ? sink_idx[idx] : 0, b = pair ? sink_idx[idx + 1] : 1;
      if (__ballot(b <= a) != 0ull) ascending = 0;
    }
  }
  if (ascending == 0) {
    for (int j0 = 0; j0 < e_end; j0 += kWave) {
      const int idx = j0 + lane;
      const int v = idx < e_end ? sink_idx[idx] : -2;
      for (int r = 0; r < n_slots; ++r) {
        const int s = __builtin_amdgcn_readlane(mine, r);
        if (__ballot(v == s && idx < t.row0 + r) != 0ull) bad |= 1u << r;
      }
    }
  }
  t.vmask = (uint32_t)(__ballot(in_prompt) & 0xffffffffull) & ~bad;
  // a slot whose sink was dropped stages the sub-tile's first valid sink instead
  const int fallback = __shfl(mine, t.vmask != 0u ? __builtin_ctz(t.vmask) : 0, kWave);
  t.sink_row = ((t.vmask >> (lane & 31)) & 1u) ? mine : fallback;
  return t;
}

template <class Id>
__device__ __forceinline__ SubTile locate_subtile(int st, int lane, int M, int N, int B, int n_b, int sub_per_block,
                                                  const Id* __restrict__ kept_blocks, int n_keep,
                                                  const int32_t* __restrict__ sink_idx, int n_sink,
                                                  const uint32_t* kept_bits = nullptr, int ascending = -1,
                                                  int dense_rows = 0, bool blocks_in_lds = false, int few_sinks = -1) {
  SubTile t;
  t.kind = 0;
  t.row0 = 0;
  t.vmask = 0u;
  t.sink_row = 0;
  if (dense_rows > 0) {  // every key row takes part (dense layers): sub-tile st is rows [32 st, 32 st + 32)
    t.row0 = st * kSubTile;
    t.vmask = low_mask(min(dense_rows - t.row0, kSubTile));
    return t;
  }
  const int n_blk_sub = n_keep * sub_per_block;
  const int n_resp_sub = (N + kSubTile - 1) / kSubTile;
  if (st < n_blk_sub) {
    const int slot = st / sub_per_block, sub = st % sub_per_block;
    const int b = blocks_in_lds ? kept_blocks[slot] : uniform_load(kept_blocks + slot);
    if (b < 0 || b >= n_b) return t;
    const int first = b * B + sub * kSubTile;
    const int end = min(min((b + 1) * B, M), first + kSubTile);
    t.row0 = first;
    t.vmask = low_mask(end - first);
    return t;
  }
  st -= n_blk_sub;
  if (st < n_resp_sub) {
    const int first = M + st * kSubTile;
    t.row0 = first;
    t.vmask = low_mask(min(M + N - first, kSubTile));
    return t;
  }
  return locate_sinks(st - n_resp_sub, lane, M, B, kept_blocks, n_keep, sink_idx, n_sink, kept_bits, ascending, few_sinks);
}

// Row of K/V that staged slot `slot` of sub-tile t reads.  Every slot reads a row of the key set, also the slots that
// hold no key (they are masked out of the softmax, but their V row still meets a zero probability in the PV product,
// and 0 x inf would poison the output): past the end of a contiguous tile the tile's last valid row, for a dropped
// sink the sub-tile's first valid sink.  `last` = highest valid slot.  Requires t.vmask != 0.
__device__ __forceinline__ int subtile_row(const SubTile& t, int slot, int last) {
  if (t.kind == 0) return t.row0 + min(slot, last);
  return __shfl(t.sink_row, slot, kWave);  // wave-uniform branch; the list was read once, when the sub-tile was located
}

// HBM -> LDS for one 32-row sub-tile of a [rows, D] bf16 matrix.  Lane l of load i supplies the 16 bytes that
// land at stage + 1024 i + 16 l, i.e. position (l mod chunks) of staged row i * rows_per_load + l / chunks; with
// the swizzle that position holds logical chunk (l mod chunks) ^ (row mod chunks).  No load is predicated: a
// slot that holds no key reads another row of the key set instead (subtile_row) and is masked out of the softmax.
// Requires t.vmask != 0.
// The loads [first, first + NL) of a sub-tile, straight into LDS (all of them, or a wavefront's share when several
// wavefronts stage one sub-tile).  A whole contiguous sub-tile — the common case — takes the short way: one scalar base
// address per sub-tile plus per-lane byte offsets that depend on the lane and the load only (the compiler keeps them
// across a key loop), so a request costs no per-lane address arithmetic; ragged and scattered sub-tiles work out a row
// per lane and load.
// VSWZ: the rows are swizzled for the transposed reads of the 32x32 tiles (vstage_swz) instead of for row reads.
template <int D, int NL, bool VSWZ = false, int POLICY = kStreamPolicy>
__device__ __forceinline__ void issue_subtile_part(const uint16_t* __restrict__ base, int64_t sn, const SubTile& t, char* stage,
                                                   int lane, int first) {
  using G = Geo<D>;
  typedef const __attribute__((address_space(1))) void* gptr_t;
  typedef __attribute__((address_space(3))) void* lptr_t;
  const int sub = lane / G::kChunks, pos = lane % G::kChunks;
  if (t.kind == 0 && t.vmask == 0xffffffffu && sn < (int64_t(1) << 26)) {  // wave-uniform; 31 rows of the stride fit 32 bits
    // load i starts rows_per_load * i rows further down (scalar), so the per-lane offset depends on i only through the
    // swizzle: at most four different ones per matrix
    const char* tile = reinterpret_cast<const char*>(base + (int64_t)__builtin_amdgcn_readfirstlane(t.row0) * sn);
    const uint32_t lane_row = (uint32_t)sub * (uint32_t)(sn * 2);  // a sub-tile spans < 4 GB
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int slot = (first + i) * G::kRowsPerLoad + sub;
      const int chunk = pos ^ (VSWZ ? vstage_swz<D>(slot) : (slot & (G::kChunks - 1)));
      const char* rows = tile + (int64_t)((first + i) * G::kRowsPerLoad) * (sn * 2);
      __builtin_amdgcn_global_load_lds((gptr_t)(rows + (lane_row + (uint32_t)(chunk * 16))), (lptr_t)(stage + (first + i) * 1024), 16, 0,
                                       POLICY);
    }
    return;
  }
  const int last = 31 - __builtin_clz(t.vmask);
  int lane_now = lane;  // ragged and scattered sub-tiles are rare: nothing of theirs is kept in registers across a key loop
  asm volatile("" : "+v"(lane_now));
  const int sub_now = lane_now / G::kChunks, pos_now = lane_now % G::kChunks;
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int slot = (first + i) * G::kRowsPerLoad + sub_now;
    const int row = subtile_row(t, slot, last);
    const int chunk = pos_now ^ (VSWZ ? vstage_swz<D>(slot) : (slot & (G::kChunks - 1)));
    const uint16_t* src = base + (int64_t)row * sn + chunk * 8;
    __builtin_amdgcn_global_load_lds((gptr_t)src, (lptr_t)(stage + (first + i) * 1024), 16, 0, POLICY);
  }
}
template <int D, bool VSWZ = false, int POLICY = kStreamPolicy>
__device__ __forceinline__ void issue_subtile(const uint16_t* __restrict__ base, int64_t sn, const SubTile& t, char* stage,
                                              int lane) {
  issue_subtile_part<D, Geo<D>::kLoads, VSWZ, POLICY>(base, sn, t, stage, lane, 0);
}

typedef unsigned uintx4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------------------- queries
// Row of Q for query slot q0 + (lane % 16), or -1.  The index is fetched for every slot below max_active
// without waiting for the device-side count; slots at or past the count are zeroed afterwards (mask_q_tile),
// which keeps the count out of the load chain.
__device__ __forceinline__ int fetch_q_row(const int32_t* __restrict__ active_idx, int q0, int max_active, int n_gen,
                                           int lane) {
  const int a = q0 + (lane & 15);
  int row = -1;
  if (a < max_active) row = active_idx[a];
  return (row >= 0 && row < n_gen) ? row : -1;
}
// Q rows of one 16-query tile in B-operand layout: lane (c, g) holds Q[query c][32*kk + 8g .. +7].
template <int D>
__device__ __forceinline__ void load_q_tile(bf16x8 (&q)[Geo<D>::kKSteps], const uint16_t* __restrict__ Qh, int64_t qsn,
                                            int row, int lane) {
  const int g = lane >> 4;
  const uint16_t* src = Qh + (int64_t)max(row, 0) * qsn + g * 8;
#pragma unroll
  for (int kk = 0; kk < Geo<D>::kKSteps; ++kk) {
    const uint4 v = *reinterpret_cast<const uint4*>(src + kk * 32);
    q[kk] = as_bf16x8(row >= 0 ? v : make_uint4(0u, 0u, 0u, 0u));
  }
}
template <int D>
__device__ __forceinline__ void mask_q_tile(bf16x8 (&q)[Geo<D>::kKSteps], int q0, int n_act, int lane) {
  if (q0 + (lane & 15) >= n_act) {
#pragma unroll
    for (int kk = 0; kk < Geo<D>::kKSteps; ++kk) q[kk] = as_bf16x8(make_uint4(0u, 0u, 0u, 0u));
  }
}

// ---------------------------------------------------------------------------------------- tile math
// S^T tiles of one staged K sub-tile: acc[kt][r] = logit of key 16kt + 4g + r.
template <int D>
__device__ __forceinline__ void qk_subtile(floatx4 (&acc)[2], const char* stageK, const bf16x8 (&q)[Geo<D>::kKSteps], int lane) {
  const int c = lane & 15, g = lane >> 4;
#pragma unroll
  for (int kt = 0; kt < 2; ++kt) {
    acc[kt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < Geo<D>::kKSteps; ++kk) {
      const bf16x8 a = as_bf16x8(*reinterpret_cast<const uint4*>(stageK + stage_off<D>(kt * 16 + c, kk * 4 + g)));
      acc[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, q[kk], acc[kt], 0, 0, 0);
    }
  }
}

// eight fp32 -> eight bf16 (round to nearest even) with v_cvt_pk_bf16_f32
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t cvt_pk_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2){lo, hi}, bf16x2));
}
// sum + lo + hi of a packed pair, in fp32
__device__ __forceinline__ float add_bf16_pair(float sum, uint32_t pair) {
  const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), ones, sum, false);
}
__device__ __forceinline__ bf16x8 pack_bf16x8(const float (&v)[8]) {
  return as_bf16x8(make_uint4(cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]), cvt_pk_bf16(v[4], v[5]), cvt_pk_bf16(v[6], v[7])));
}

// A operand of the PV product for d-column tile `ct`: lane (c, g) needs V[key slot (g, e)][16 ct + c], e = 0..7,
// i.e. eight different rows at one column of the row-major staged tile.  ds_read_b64_tr_b16 does that
// transposition in the LDS unit: within a block of 16 lanes, lane i receives element (i % 4) of the 8-byte
// groups addressed by lanes i/4, i/4 + 4, i/4 + 8, i/4 + 12.  Lane s therefore points at row 4g + s/4 (first
// read) or 16 + 4g + s/4 (second read), columns 16 ct + 4 (s % 4) .. + 3.
typedef short shortx4 __attribute__((ext_vector_type(4)));
template <int D>
__device__ __forceinline__ bf16x8 read_v_operand(const char* stageV, int ct, int lane) {
  const int s = lane & 15, g = lane >> 4;
  const int row = 4 * g + (s >> 2);
  const int col = 16 * ct + 4 * (s & 3);
  const int off0 = stage_off<D>(row, col >> 3) + (col & 7) * 2;
  const int off1 = stage_off<D>(row + 16, col >> 3) + (col & 7) * 2;
  typedef shortx4 __attribute__((address_space(3))) * lds_ptr;
  const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(stageV + off0));
  const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(stageV + off1));
  struct { shortx4 a, b; } both = {lo, hi};
  return __builtin_bit_cast(bf16x8, both);
}

// All K (V) operands of a staged sub-tile into registers, complete on return.  Key loops that request the next K rows while the V
// rows of this sub-tile are still under way need the reads outside the compiler's sight: it would wait for every outstanding
// LDS-direct load in front of them.  The callers wait for the rows (wait_loads_but).  Stages are aligned to 256 bytes, so that the
// swizzle of a chunk is an exclusive or of the address.
__device__ __forceinline__ uint32_t lds_address(const char* p) {
  typedef const __attribute__((address_space(3))) char* lds_ptr;
  return (uint32_t)(uintptr_t)(lds_ptr)p;
}
template <int D>
__device__ __forceinline__ void read_k_operands16(bf16x8 (&k)[2][D / 32], const char* stageK, int lane) {
  const uint32_t a = lds_address(stageK) + stage_off<D>(lane & 15, lane >> 4);  // chunk 4 kk + g, row 16 kt + c
  if constexpr (D == 128) {
    asm volatile(
        "ds_read_b128 %0, %8\n\tds_read_b128 %1, %9\n\tds_read_b128 %2, %10\n\tds_read_b128 %3, %11\n\t"
        "ds_read_b128 %4, %8 offset:4096\n\tds_read_b128 %5, %9 offset:4096\n\tds_read_b128 %6, %10 offset:4096\n\t"
        "ds_read_b128 %7, %11 offset:4096\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(k[0][0]), "=&v"(k[0][1]), "=&v"(k[0][2]), "=&v"(k[0][3]), "=&v"(k[1][0]), "=&v"(k[1][1]), "=&v"(k[1][2]), "=&v"(k[1][3])
        : "v"(a), "v"(a ^ 64u), "v"(a ^ 128u), "v"(a ^ 192u)
        : "memory");
  } else {
    asm volatile(
        "ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %4 offset:2048\n\tds_read_b128 %3, %5 offset:2048\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(k[0][0]), "=&v"(k[0][1]), "=&v"(k[1][0]), "=&v"(k[1][1])
        : "v"(a), "v"(a ^ 64u)
        : "memory");
  }
}
template <int D>
__device__ __forceinline__ void read_v_operands16(bf16x8 (&v)[D / 16], const char* stageV, int lane) {
  const int s = lane & 15, g = lane >> 4, col = 4 * (s & 3);
  const uint32_t a = lds_address(stageV) + stage_off<D>(4 * g + (s >> 2), col >> 3) + (col & 7) * 2;  // column tile ct: chunk 2 ct further
  shortx4 r[D / 16][2];
  if constexpr (D == 128) {
    asm volatile(
        "ds_read_b64_tr_b16 %0, %16\n\tds_read_b64_tr_b16 %1, %16 offset:4096\n\t"
        "ds_read_b64_tr_b16 %2, %17\n\tds_read_b64_tr_b16 %3, %17 offset:4096\n\t"
        "ds_read_b64_tr_b16 %4, %18\n\tds_read_b64_tr_b16 %5, %18 offset:4096\n\t"
        "ds_read_b64_tr_b16 %6, %19\n\tds_read_b64_tr_b16 %7, %19 offset:4096\n\t"
        "ds_read_b64_tr_b16 %8, %20\n\tds_read_b64_tr_b16 %9, %20 offset:4096\n\t"
        "ds_read_b64_tr_b16 %10, %21\n\tds_read_b64_tr_b16 %11, %21 offset:4096\n\t"
        "ds_read_b64_tr_b16 %12, %22\n\tds_read_b64_tr_b16 %13, %22 offset:4096\n\t"
        "ds_read_b64_tr_b16 %14, %23\n\tds_read_b64_tr_b16 %15, %23 offset:4096\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(r[0][0]), "=&v"(r[0][1]), "=&v"(r[1][0]), "=&v"(r[1][1]), "=&v"(r[2][0]), "=&v"(r[2][1]), "=&v"(r[3][0]), "=&v"(r[3][1]),
          "=&v"(r[4][0]), "=&v"(r[4][1]), "=&v"(r[5][0]), "=&v"(r[5][1]), "=&v"(r[6][0]), "=&v"(r[6][1]), "=&v"(r[7][0]), "=&v"(r[7][1])
        : "v"(a), "v"(a ^ 32u), "v"(a ^ 64u), "v"(a ^ 96u), "v"(a ^ 128u), "v"(a ^ 160u), "v"(a ^ 192u), "v"(a ^ 224u)
        : "memory");
  } else {
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:2048\n\t"
        "ds_read_b64_tr_b16 %2, %9\n\tds_read_b64_tr_b16 %3, %9 offset:2048\n\t"
        "ds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:2048\n\t"
        "ds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:2048\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(r[0][0]), "=&v"(r[0][1]), "=&v"(r[1][0]), "=&v"(r[1][1]), "=&v"(r[2][0]), "=&v"(r[2][1]), "=&v"(r[3][0]), "=&v"(r[3][1])
        : "v"(a), "v"(a ^ 32u), "v"(a ^ 64u), "v"(a ^ 96u)
        : "memory");
  }
#pragma unroll
  for (int ct = 0; ct < D / 16; ++ct) {
    struct { shortx4 a, b; } both = {r[ct][0], r[ct][1]};
    v[ct] = __builtin_bit_cast(bf16x8, both);
  }
}

typedef float floatx16 __attribute__((ext_vector_type(16)));
// A operand of O^T += V^T P^T (32x32x16) for d tile `dt` and k-step `ks`: lane (dcol = lane % 32, hh) needs
// V[16 ks + 8 (e / 4) + 4 hh + e % 4][32 dt + dcol], e = 0..7 — two transposed reads of four consecutive rows each.
// A V staged for the 32x32 tiles is only ever read this way — one instruction touches eight rows (four per half of the
// wavefront) and 64 bytes of each — so its rows are swizzled for that: rows that would fall on the same banks
// (consecutive rows at d = 128, every other row at d = 64) get different 64-byte segments.
template <int D>
__device__ __forceinline__ int vstage_off(int row, int chunk) {
  return row * Geo<D>::kRowBytes + ((chunk ^ vstage_swz<D>(row)) << 4);
}
template <int D>
__device__ __forceinline__ bf16x8 read_v_operand32(const char* stageV, int dt, int ks, int lane) {
  const int s = lane & 15, b = lane >> 4;
  const int row = 16 * ks + 4 * (b >> 1) + (s >> 2);
  const int col = 32 * dt + 16 * (b & 1) + 4 * (s & 3);
  const int off0 = vstage_off<D>(row, col >> 3) + (col & 7) * 2;
  const int off1 = vstage_off<D>(row + 8, col >> 3) + (col & 7) * 2;
  typedef shortx4 __attribute__((address_space(3))) * lds_ptr;
  const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(stageV + off0));
  const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(stageV + off1));
  struct { shortx4 a, b; } both = {lo, hi};
  return __builtin_bit_cast(bf16x8, both);
}

// Scaled logits of one 32-key sub-tile (contiguous rows row0 .., row0 a multiple of 32) against up to 16 queries, kept
// for the column-mass kernel in the layout [head][key quad][query][key within the quad] (fp32): a lane holds, per
// 16-key tile, the logits of ONE query for four consecutive keys — one 16-byte store — and the 64 lanes of a store
// instruction cover 1 KB of consecutive bytes (query fastest, then the four quads of the tile).  Quads that start at or
// past key L are not written; the padding keys of the last quad hold finite values nobody reads.  Neither are the slots of queries past
// the capacity n_q of the list, and the column-mass kernel does not fetch them: at eight queries half of the traffic beside K (32 heads, sink
// chain of 8192 keys 28.8 -> 26.7 us, 32 832 73.5 -> 67.1, 131 136 255 -> 232; probe layer of 32 832 128 -> 118; four queries take as
// long as eight, a line of 128 bytes; sixteen as before).  The device-side count would come too late for the second kernel's first loads.
// n_q >= 1, which the launchers check: a whole sub-tile is then kSpillStores store instructions, whatever the list, and the key loops count
// them among the requests under way.
constexpr int kSpillStores = 2;
__device__ __forceinline__ void spill_logits(float* __restrict__ logits, int h, int L, int n_q, int row0, const floatx4 (&acc)[2],
                                             float scale_log2, int lane) {
  const int c = lane & 15, g = lane >> 4;
  const int64_t n_quads = (L + 3) >> 2;
#pragma unroll
  for (int kt = 0; kt < kSpillStores; ++kt) {
    const int key0 = row0 + 16 * kt + 4 * g;
    if (key0 < L && c < n_q) {
      floatx4* dst = reinterpret_cast<floatx4*>(logits + (((int64_t)h * n_quads + (key0 >> 2)) * 16 + c) * 4);
      *dst = acc[kt] * scale_log2;
    }
  }
}

// One step of the base-2 online softmax for the 8 logits a lane holds of one query; returns the rescale factor
// of the running state and leaves exp2(scale * s - m) in ps.  The running maximum m is kept in the scaled domain;
// the scale (> 0) is applied to the raw maximum once and folded into the exponent's multiply-add for the rest.
// A sub-tile whose 32 slots all hold keys (the common case) skips the per-slot masking.
__device__ __forceinline__ float softmax_step(const floatx4 (&acc)[2], uint32_t vmask, int g, float scale_log2, float& m_run,
                                              float& l_run, float (&ps)[8]) {
  float s[8];
  float mx = -INFINITY;
  if (vmask == 0xffffffffu) {  // wave-uniform
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s[e] = acc[e >> 2][e & 3];
      mx = fmaxf(mx, s[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int slot = 16 * (e >> 2) + 4 * g + (e & 3);
      s[e] = ((vmask >> slot) & 1u) ? acc[e >> 2][e & 3] : -INFINITY;
      mx = fmaxf(mx, s[e]);
    }
  }
  mx = group_max(mx) * scale_log2;  // -inf stays -inf
  const float m_new = fmaxf(m_run, mx);
  const float m_use = (m_new == -INFINITY) ? 0.f : m_new;
  const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
  float lsum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    ps[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], scale_log2, -m_use));
    lsum += ps[e];
  }
  lsum = group_sum(lsum);
  l_run = l_run * alpha + lsum;
  m_run = m_new;
  return alpha;
}

// =====================================================================================================
// Sparse attention
// =====================================================================================================
struct AttnArgs {
  const uint16_t* Q;
  const uint16_t* K;
  const uint16_t* V;
  const int32_t* active_idx;
  const int32_t* counts;
  const int32_t* kept_blocks;
  const int32_t* sink_idx;
  uint16_t* out;
  float* lse;
  float* part_o;   // [H, q_pad, n_split, D]
  float* part_ml;  // [H, q_pad, n_split, 2]
  int64_t qsh, qsn, ksh, ksn, vsh, vsn, osh, osn;
  int H, M, N, B, n_b, n_gen, n_keep, n_sink, max_active;
  int sub_per_block, n_sub, n_split, q_pad, q_groups;
  float scale_log2;
  uint32_t head_turn;                // (2^32 - 1) / H      see SplitRounds
  int split_rounds, split_rounds_more;  // every split has so many rounds, the first so many splits one more
  // fused layer path only: partial relevances in, scores / kept blocks out
  // (where the kernel works the relevances out itself rel_part is the representative keys [H, n_b, D] and kept_blocks the focus rows' ids)
  const float* rel_part;  // [ceil(H / 4), n_b], or with rel_per_head [H, n_b]
  bool rel_per_head;
  float* scores_out;      // [n_b] or null
  int32_t* kept_out;      // [n_keep]
  int n_focus_max;
  // dense (probe) layer only
  int dense_rows;     // > 0: attend to all of the first dense_rows = M + N key rows, block and sink lists unused
  float* logits_out;  // [H, ceil(L / 4), 16, 4] scaled base-2 logits of the (at most 16) active queries (spill_logits), or null
  float* lse2_out;    // [H, q_pad] base-2 log-sum-exp per row (+inf for an empty row), or null
};

// of a launch over kept blocks, sinks and response rows; `fused`: the blocks are ranked by the kernel
AttnArgs attention_args(const void* Q, const int32_t* active_idx, const int32_t* counts, int max_active, const void* K, const void* V,
                        const focus_shape& s, const int32_t* kept_blocks, int n_keep, const int32_t* sink_idx, int n_sink, const SplitPlan& p,
                        void* out, float* lse, float* part_o, float* part_ml, const FusedTopC* fused);
// merges the key splits (p.n_split > 1) into out and lse
hipError_t launch_attn_combine(const AttnArgs& a, const SplitPlan& p, int head_dim, hipStream_t st);

// |I_focus| and |I_active| as they lie in memory (or the capacities of the lists): scalar loads that a kernel requests at its start and
// waits for once its first vector loads are out (one that first looked whether its query group is past the count, and read the other
// count when the relevances had come, spent two memory round trips on it: layers of more than 16 queries 0.3 to 0.7 us).
struct Counts {
  int focus, active;
  __device__ __forceinline__ explicit Counts(const AttnArgs& p) : focus(p.n_focus_max), active(p.max_active) {
    if (p.counts) {
      focus = p.counts[0];
      active = p.counts[1];
    }
  }
  __device__ __forceinline__ int n_active(const AttnArgs& p) const { return min(max(active, 0), p.max_active); }
};

// The arguments that the first memory requests of an attention kernel need, once more as leading scalar parameters: those (14
// dwords) are in scalar registers when a wavefront starts (-amdgpu-kernarg-preload-count), while a member of AttnArgs is a load
// of its own in front of everything that depends on it.  H arrives negative where the partial relevances are per head.
#define ATTN_FIRST_PARAMS                                                                                                  \
  const float *rel_part, const int32_t *active_idx, const uint16_t *Q, const int32_t *counts, int n_b, int H, int max_active, \
      int n_gen, int n_split, int n_sub
#define ATTN_FIRST_NAMES rel_part, active_idx, Q, counts, n_b, H, max_active, n_gen, n_split, n_sub
// wide_attn_kernel: n_gen is needed later, the number of query groups at once
#define WIDE_FIRST_PARAMS                                                                                                     \
  const float *rel_part, const int32_t *active_idx, const uint16_t *Q, const int32_t *counts, int n_b, int H, int max_active, \
      int q_groups, int n_split, int n_sub
__device__ __forceinline__ AttnArgs with_first(AttnArgs p, ATTN_FIRST_PARAMS) {
  p.rel_part = rel_part;
  p.active_idx = active_idx;
  p.Q = Q;
  p.counts = counts;
  p.n_b = n_b;
  p.H = abs(H);
  p.rel_per_head = H < 0;
  p.max_active = max_active;
  p.n_gen = n_gen;
  p.n_split = n_split;
  p.n_sub = n_sub;
  return p;
}
#define WIDE_LAUNCH(kernel, grid, block, st, a)                                                                            \
  hipLaunchKernelGGL(kernel, grid, block, 0, st, (a).rel_part, (a).active_idx, (a).Q, (a).counts, (a).n_b, (a).rel_per_head ? -(a).H : (a).H, (a).max_active, \
                     (a).q_groups, (a).n_split, (a).n_sub, a)
#define ATTN_LAUNCH(kernel, grid, block, st, a)                                                                            \
  hipLaunchKernelGGL(kernel, grid, block, 0, st, (a).rel_part, (a).active_idx, (a).Q, (a).counts, (a).n_b, (a).rel_per_head ? -(a).H : (a).H, (a).max_active, \
                     (a).n_gen, (a).n_split, (a).n_sub, a)

// Where a workgroup that ranks the blocks itself keeps the list.  Up to 256 blocks: beside the ranking's scratch memory.  More: in 16 bits
// per block, in the place of the histograms, which everyone has read by then; beside them and in 32 bits a workgroup of
// sparse_attn_kernel<64, .> without a key loop took 43 620 bytes (up to 1024 blocks) and 47 716 (2048), and of the four that the plan
// of the key splits counts on per compute unit (kAttnGroupsSmall) three fitted (32 heads, d = 64, whole layer: 512 blocks, 97 sub-tiles
// 20.4 -> 16.5 us, 127 21.7 -> 18.1; 2048 blocks 27.9 -> 22.6, 29.3 -> 23.6).
template <bool FUSED, int BLOCKS>
struct KeptList {
  static constexpr bool kInScratch = FUSED && BLOCKS > 256;
  using Id = std::conditional_t<kInScratch, uint16_t, int32_t>;
  static constexpr int kEntriesBeside = FUSED && !kInScratch ? BLOCKS : 1;
  static_assert(!kInScratch || BLOCKS * sizeof(Id) <= sizeof(TopkShared::keys), "fits the histograms");
  static __device__ __forceinline__ Id* place(char* scratch, int32_t* beside) {
    if constexpr (kInScratch)
      return reinterpret_cast<Id*>(reinterpret_cast<TopkShared*>(scratch)->keys);
    else
      return beside;
  }
};

// What the attention kernels prepare before their first K/V request.
// R_b = (1 / (|I_focus| H)) sum_h qsum^h . kbar^h_b, then Top-C into kept_sh; the workgroup with `writer` set also writes scores
// and kept blocks out.  First use of `sm`.  Thread t of THREADS ranks the blocks t, t + THREADS, ...; n_b <= kFusedMaxBlocks.
// FirstParts holds the loads of the first NP parts (32 heads in groups of four are 8 parts), which the caller requests before it
// waits for anything.  BLOCKS: the most blocks of the variant, 256, kFusedManyBlocks or kFusedMaxBlocks.  Few blocks to keep of up to 256: the tournament of block_topk_small; else
// block_topk_planes.  Repeating it in every workgroup takes less time than the launch of a kernel that ranks the blocks once
// (sparse layer at 128K, 30 of 1024 blocks, 34.7 -> 29.0 us; half of 512 64-row blocks 63.2 -> 60.1).
template <int NP, int THREADS, int BLOCKS>
struct FirstParts {
  static constexpr int kPlanes = BLOCKS > 256 ? BLOCKS / THREADS : 1;
  float part[kPlanes][NP];
};
template <int NP, int THREADS, int BLOCKS>
__device__ __forceinline__ void first_partials(FirstParts<NP, THREADS, BLOCKS>& f, const AttnArgs& p, bool per_head) {
  const int last = (per_head ? p.H : (p.H + kRelGroup - 1) / kRelGroup) - 1;
#pragma unroll
  for (int l = 0; l < f.kPlanes; ++l) {
    const uint32_t b = min((int)threadIdx.x + l * THREADS, p.n_b - 1);  // n_b <= kFusedMaxBlocks: small offsets
#pragma unroll
    for (int i = 0; i < NP; ++i) f.part[l][i] = p.rel_part[(uint32_t)(min(i, last) * p.n_b) + b];
  }
  __builtin_amdgcn_sched_barrier(0);  // (the scheduler would move the wait for the row ids in front of these loads)
}
// The whole relevance in the attention kernel (relevance_in_attention): a wavefront takes one head and kInnerBlocks consecutive blocks, all
// of its representative keys requested before the focus rows, and the sums of the groups of four heads go to the thread that ranks the
// block, in the order of relevance_partial_kernel.
constexpr int kInnerBlocks = 16, kInnerGroups = 4;  // WAVES <= 16 heads
template <int D, int WAVES, int NP, int BLOCKS>
__device__ __forceinline__ void relevance_parts(FirstParts<NP, 64 * WAVES, BLOCKS>& f, const AttnArgs& p, int entry, int n_focus, float* dots,
                                                int wave, int lane) {
  constexpr int CPR = D / 8, R = kWave / CPR, P = kInnerBlocks / R;
  static_assert(WAVES <= kInnerGroups * kRelGroup && kInnerGroups <= NP && FirstParts<NP, 64 * WAVES, BLOCKS>::kPlanes == 1,
                "a thread ranks one block and holds the sums of all groups");
  const int c = lane % CPR, r = lane / CPR;
  const int per_head = (p.n_b + kInnerBlocks - 1) / kInnerBlocks;
  const int h = wave / per_head, b0 = (wave - h * per_head) * kInnerBlocks;
  if (h < p.H) {
    float4 k0[P], k1[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const float4* kp = reinterpret_cast<const float4*>(p.rel_part + ((int64_t)h * p.n_b + min(b0 + i * R + r, p.n_b - 1)) * D + c * 8);
      k0[i] = kp[0];
      k1[i] = kp[1];
    }
    __builtin_amdgcn_sched_barrier(0);
    float qs[8];
    focus_row_sum<D, true>(qs, p.Q + (int64_t)h * p.qsh, p.qsn, p.kept_blocks, entry, min(max(n_focus, 0), p.n_focus_max), p.n_gen);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const float dot = chunk_dot_reduce<CPR>(qs, k0[i], k1[i]);
      if (c == 0) dots[wave * kInnerBlocks + i * R + r] = dot;
    }
  }
  __syncthreads();
  const int b = min((int)threadIdx.x, p.n_b - 1);
#pragma unroll
  for (int g = 0; g < kInnerGroups; ++g) {
    const int h0 = g * kRelGroup;
    float acc = h0 < p.H ? dots[h0 * per_head * kInnerBlocks + b] : 0.f;
#pragma unroll
    for (int w = 1; w < kRelGroup; ++w) acc = h0 + w < p.H ? acc + dots[(h0 + w) * per_head * kInnerBlocks + b] : acc;
    f.part[0][g] = acc;
  }
}
template <int NP, int THREADS, int BLOCKS>
__device__ __forceinline__ void rank_blocks(const AttnArgs& p, const FirstParts<NP, THREADS, BLOCKS>& f, bool per_head, int n_focus,
                                            typename KeptList<true, BLOCKS>::Id* kept_sh, TopkShared& sm, bool writer) {
  constexpr int kPlanes = FirstParts<NP, THREADS, BLOCKS>::kPlanes;
  const int tid = threadIdx.x;
  // more than eight wavefronts (one_split_waves: at most 256 blocks, at most 16 to keep): the first four rank
  constexpr int kRankWaves = THREADS > 512 ? 4 : THREADS / kWave;
  const bool tournament = BLOCKS <= 256 && (THREADS > 512 || p.n_keep * kRankWaves <= kWave);  // uniform
  if (!tournament) {
    block_topk_clear<THREADS>(sm);
    __syncthreads();
  }
  const int n_f = min(max(n_focus, 0), p.n_focus_max);
  const float scale = n_f > 0 ? 1.f / ((float)n_f * (float)p.H) : 0.f;
  const int n_groups = (p.H + kRelGroup - 1) / kRelGroup;
  float rel[kPlanes];
#pragma unroll
  for (int l = 0; l < kPlanes; ++l) {
    const float(&part)[NP] = f.part[l];
    const int b = tid + l * THREADS;
    float r = 0.f;  // in the order of sum_partials
    if (per_head) {
#pragma unroll
      for (int h = 0; h < NP; h += kRelGroup) {
        float g = part[h];
#pragma unroll
        for (int i = 1; i < kRelGroup; ++i) g = h + i < p.H ? g + part[h + i] : g;
        r = h < p.H ? r + g : r;
      }
      if (p.H > NP && b < p.n_b) r = sum_partials(p.rel_part, p.H, false, p.n_b, b, NP, r);
    } else {
#pragma unroll
      for (int g = 0; g < NP; ++g) r = g < n_groups ? r + part[g] : r;
      if (n_groups > NP && b < p.n_b) r = sum_partials(p.rel_part, n_groups, true, p.n_b, b, NP, r);
    }
    rel[l] = r * scale;
    if (writer && p.scores_out && b < p.n_b) p.scores_out[b] = rel[l];
  }
  if (tournament) {
    auto keyfn = [&](int, uint32_t& key) -> bool {
      key = order_key(rel[0]);
      return true;
    };
    if constexpr (BLOCKS <= 256)
      block_topk_small<256, true, (THREADS > 512 ? kRankWaves : 0)>(keyfn, p.n_b, p.n_keep, kept_sh, nullptr, sm);
  } else if constexpr (THREADS <= 512) {
    uint32_t key1[kPlanes];
#pragma unroll
    for (int l = 0; l < kPlanes; ++l) key1[l] = tid + l * THREADS < p.n_b ? order_key(rel[l]) + 1u : 0u;
    block_topk_planes<kPlanes, THREADS>(key1, p.n_b, p.n_keep, kept_sh, sm);
  }
  if (writer)
    for (int i = tid; i < p.n_keep; i += THREADS) p.kept_out[i] = kept_sh[i];
}

// Workgroups whose key range reaches the sink sub-tiles prepare the union of Eq. 8 once: a bitmap of the kept blocks, and
// whether the sink list is strictly ascending (then it cannot name a position twice).  A list of one sub-tile needs neither: its
// wavefront holds it in registers (few_sinks; three memory round trips behind the Top-C became none, 1 us of the 32K layer).
__device__ __forceinline__ int request_few_sinks(const AttnArgs& p, int lane) {
  return p.n_sink <= kSubTile && lane < p.n_sink && p.dense_rows == 0 ? p.sink_idx[lane] : -1;
}
struct SinkUnion {
  const uint32_t* kept_bits;  // see locate_subtile; null when there is none
  int ascending;
};
template <class Id>
__device__ __forceinline__ SinkUnion prepare_union(const AttnArgs& p, int split, const Id* kept_blocks, uint32_t* bits_sh,
                                                   int* unsorted_sh) {
  SinkUnion u;
  u.kept_bits = nullptr;
  u.ascending = -1;
  const int first_sink_sub = p.n_keep * p.sub_per_block + (p.N + kSubTile - 1) / kSubTile;
  const int n_round = (p.n_sub + kWavesPerGroup - 1) / kWavesPerGroup;                      // rounds of four sub-tiles ...
  const int last = n_round - 1 - (n_round - 1 - split) % p.n_split;                         // ... the last one of this split
  if (p.dense_rows == 0 && p.n_sink > kSubTile && (last + 1) * kWavesPerGroup > first_sink_sub) {  // uniform over the workgroup
    const bool bitmap = p.n_keep > 0 && p.n_b <= kBitmapBlocks;
    const int words = bitmap ? (p.n_b + 31) >> 5 : 0;
    for (int i = threadIdx.x; i < words; i += blockDim.x) bits_sh[i] = 0u;
    if (threadIdx.x == 0) *unsorted_sh = 0;
    __syncthreads();
    if (bitmap) {
      for (int i = threadIdx.x; i < p.n_keep; i += blockDim.x) {
        const int b = kept_blocks[i];
        if (b >= 0 && b < p.n_b) atomicOr(&bits_sh[b >> 5], 1u << (b & 31));
      }
    }
    for (int i = threadIdx.x; i + 1 < p.n_sink; i += blockDim.x)
      if (p.sink_idx[i + 1] <= p.sink_idx[i]) *unsorted_sh = 1;
    __syncthreads();
    if (bitmap) u.kept_bits = bits_sh;
    u.ascending = *unsorted_sh ? 0 : 1;
  }
  return u;
}

// The rounds of four sub-tiles of one key split (see SplitPlan) in the order in which a key loop takes them: head h begins h / H of the
// way down the list and wraps around.  All heads sweep their keys at the same time, and with the same place in the sweep the rows
// being fetched are the head stride apart, which for some lengths keeps meeting the same memory channels (32 heads, 16 queries:
// 33 024 rows 92 us from the top for every head, 87.5 this way; 32 832 rows 86.5 either way; 256 of 512 blocks, 256 response
// rows, 25 queries, whole layer 66 and 60).
struct SplitRounds {
  int first, step, n_rounds, turn, n_sub;
  __device__ __forceinline__ SplitRounds(const AttnArgs& p, int split, int h) {
    first = split * kWavesPerGroup;
    step = p.n_split * kWavesPerGroup;
    n_sub = p.n_sub;
    n_rounds = p.split_rounds + (split < p.split_rounds_more);
    turn = (int)__umulhi((uint32_t)h * p.head_turn, (uint32_t)n_rounds);  // < n_rounds
  }
  // sub-tile of slot `slot` in the i-th round; n_sub or more: none
  __device__ __forceinline__ int sub(int i, int slot) const {
    if (i >= n_rounds) return n_sub;
    const int r = i + turn;
    return first + slot + (r >= n_rounds ? r - n_rounds : r) * step;
  }
};

// The sub-tiles of 64 rounds at a time, lane i those of round i0 + i: a key loop takes them by lane reads, where working one out per round
// put a division and the wait for a block id in front of the products (a call of 32 heads, 8256 keys, 16 queries 27.4 -> 26.9 us, 28
// queries 28.8 -> 28.0; half of 512 blocks, 25 queries 50.5 -> 49.0; 8 heads, 16 448 keys 19.3 -> 18.6).  n: rows, -1: sub-tile row0 of
// the sink list.
struct RoundTable {
  int row0, n;
};
template <class Id>
__device__ __forceinline__ RoundTable tabulate_rounds(const AttnArgs& p, const SplitRounds& rounds, int slot, int i0, int lane, const Id* kept_blocks) {
  RoundTable r{0, 0};
  int sub = rounds.sub(i0 + lane, slot);
  if (sub >= p.n_sub) return r;
  if (p.dense_rows > 0) {
    r.row0 = sub * kSubTile;
    r.n = min(p.dense_rows - r.row0, kSubTile);
    return r;
  }
  const int n_blk_sub = p.n_keep * p.sub_per_block, n_resp_sub = (p.N + kSubTile - 1) / kSubTile;
  if (sub < n_blk_sub) {
    const int i = sub / p.sub_per_block, b = kept_blocks[i];
    if (b >= 0 && b < p.n_b) {
      r.row0 = b * p.B + (sub - i * p.sub_per_block) * kSubTile;
      r.n = max(min(min((b + 1) * p.B, p.M) - r.row0, kSubTile), 0);
    }
    return r;
  }
  sub -= n_blk_sub;
  if (sub < n_resp_sub) {
    r.row0 = p.M + sub * kSubTile;
    r.n = min(p.M + p.N - r.row0, kSubTile);
  } else {
    r.row0 = sub - n_resp_sub;
    r.n = -1;
  }
  return r;
}
// rounds 0, 1, 2, ... of a slot, one call each
template <class Id>
struct RoundList {
  const AttnArgs& p;
  const SplitRounds& rounds;
  const SinkUnion& uni;
  const Id* kept_blocks;
  int slot, lane, few_sinks, next = 0;
  RoundTable table{0, 0};
  __device__ __forceinline__ SubTile take() {
    const int i = next & (kWave - 1);
    if (i == 0) table = tabulate_rounds(p, rounds, slot, next, lane, kept_blocks);
    ++next;
    const int n = __builtin_amdgcn_readlane(table.n, i), row0 = __builtin_amdgcn_readlane(table.row0, i);
    if (n < 0) return locate_sinks(row0, lane, p.M, p.B, kept_blocks, p.n_keep, p.sink_idx, p.n_sink, uni.kept_bits, uni.ascending, few_sinks);
    SubTile t;
    t.kind = 0;
    t.row0 = row0;
    t.vmask = low_mask(n);
    t.sink_row = 0;
    return t;
  }
};

}  // namespace focus
