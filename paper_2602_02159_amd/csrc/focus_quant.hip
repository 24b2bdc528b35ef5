// The quantised KV cache: rows of e4m3 codes with one power of two each.
//
//   quant_update_kernel    Eq. 3: the cache rows of the active positions take new states, quantised on the way
//   quant_refresh_kernel   block entry: all rows, and the block means of what they read back as, in one pass
//   quant_read_kernel      a range of rows back as bf16
//   quant_attn_kernel      Eq. 8 + Eq. 9 over the quantised rows (v_mfma_f32_16x16x32_bf16)
//
// A row x[0 .. d) of one head stands for code_i * 2^E.  E is the smallest integer with max |x_i| <= 448 * 2^E (448 = the largest e4m3
// number), within [-110, 119]; code_i = x_i / 2^E to the nearest e4m3, ties to even.  Dividing by a power of two rounds nothing, a code
// times a power of two is a bf16 number, and powers of two commute with every later rounding: what the library computes over
// the quantised cache is what it computes over the bf16 cache that this one reads back as.  One power of two per row of a
// head is enough because the codes have an exponent of their own: a value keeps its three bits down to 2^-14 of the row's largest.
// The limits of E keep every value that is not a rounding of zero within the normal numbers, here and in the products.
#include <algorithm>

#include "focus_attn.h"
#include "focus_cache.h"
#include "focus_codes.h"
#include "focus_common.h"
#include "focus_kernels.h"

namespace focus {

// The rows of a wavefront's lanes, eight values a lane: N = D / 8 neighbouring lanes hold one row.  Its power of two, as stored.
template <int N>
__device__ __forceinline__ uint32_t row_exponent(const uint4& x) {
  auto largest = [](uint32_t w) {  // of the two magnitudes, those that are finite
    const uint32_t a = w & 0x7fffu, b = (w >> 16) & 0x7fffu;
    return max(a < 0x7f80u ? a : 0u, b < 0x7f80u ? b : 0u);
  };
  uint32_t m = max(max(largest(x.x), largest(x.y)), max(largest(x.z), largest(x.w)));
#pragma unroll
  for (int o = 1; o < N; o <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, kWave));
  // 448 = 1.75 * 2^8: a mantissa past 0x60 / 0x80 takes the next power of two
  return (uint32_t)min(max((int)((m + 0x1fu) >> 7) - 8, kExpMin), kExpMax);
}

// eight values as codes; `inv` = 2^-E
__device__ __forceinline__ uint2 encode8(const uint4& x, float inv) {
  auto scaled = [&](float v) { return scaled_for_code(v, inv); };
  auto four = [&](uint32_t a, uint32_t b) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(bf16_lo(a)), scaled(bf16_hi(a)), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(scaled(bf16_lo(b)), scaled(bf16_hi(b)), w, true);
  };
  return make_uint2(four(x.x, x.y), four(x.z, x.w));
}

// ---------------------------------------------------------------------------------------- writing and reading
// One row's share of a thread: the codes of its eight values, and the exponent from the row's first lane.
template <int D>
__device__ __forceinline__ uint2 store_row(const uint4& x, bool live, uint8_t* codes, uint8_t* exponent, int c) {
  const uint32_t e = row_exponent<D / 8>(x);
  const uint2 w = encode8(x, exp_value(254u - e));
  if (live) {
    *reinterpret_cast<uint2*>(codes) = w;
    if (c == 0) *exponent = (uint8_t)e;
  }
  return w;
}

// Slots a of the list, D / 8 threads each: the rows of K and V, requested together with the position, the count and the entries behind
// it.  A position that is listed again further down is left to that entry: its codes and its exponent come from one state.  One launch and two
// dependent round trips, nothing else counts (8 rows, 4 heads: 2.5 us a call in a graph, 2.8 traced).
template <int D>
__global__ __launch_bounds__(256) void quant_update_kernel(const CacheUpdate u, const QuantCache q) {
  constexpr int kChunks = D / 8, kAhead = 4;
  const int a = blockIdx.x * (256 / kChunks) + (int)threadIdx.x / kChunks, c = (int)threadIdx.x % kChunks, h = blockIdx.y;
  const int slot = min(a, u.max_active - 1);
  const int64_t src = (int64_t)h * u.nsh + (int64_t)slot * u.nsn + c * 8;
  const uint4 k = *reinterpret_cast<const uint4*>(u.Kn + src);
  const uint4 v = *reinterpret_cast<const uint4*>(u.Vn + src);
  const int i = u.active_idx[slot];
  const int n_act = u.counts ? min(max(u.counts[1], 0), u.max_active) : u.max_active;
  const int64_t row = (int64_t)u.row_base + i;
  bool again = false;
  for (int t0 = a + 1 + c; t0 < n_act; t0 += kChunks * kAhead) {
    int later[kAhead];
#pragma unroll
    for (int s = 0; s < kAhead; ++s) later[s] = u.active_idx[min(t0 + s * kChunks, u.max_active - 1)];
#pragma unroll
    for (int s = 0; s < kAhead; ++s) again |= t0 + s * kChunks < n_act && later[s] == i;
  }
  const unsigned long long mine = ((1ull << kChunks) - 1ull) << ((threadIdx.x & 63) / kChunks * kChunks);
  const bool live = a < n_act && i >= 0 && row >= 0 && row < u.n_rows && (__ballot(again) & mine) == 0ull;
  const int64_t at = live ? row : 0;
  const int64_t e = (int64_t)h * q.esh + at * q.esn;
  store_row<D>(k, live, q.K + (int64_t)h * u.ksh + at * u.ksn + c * 8, q.k_exp + e, c);
  store_row<D>(v, live, q.V + (int64_t)h * u.vsh + at * u.vsn + c * 8, q.v_exp + e, c);
}

// The same of a long list, which is compared with itself once for several heads: every entry behind the workgroup's first slot is read by
// one thread and compared with all its slots.  By its bytes 4096 rows of 32 heads would take 20 us and 32 768 rows 158, at the rate of a copy, and not
// 26.5 and 207: the copy waits for the comparison, quadratic in the length of the list (32 768 entries: 5e8 pairs, some 40 us by the
// instructions).  (At d = 64 the slots' 32 positions are more scalars than fit; lanes of vector registers hold what is left over.)
template <int D>
__global__ __launch_bounds__(256) void quant_update_many_kernel(const CacheUpdate u, const QuantCache q, int heads) {
  constexpr int kChunks = D / 8, kSlots = 256 / kChunks, kAhead = 2;
  __shared__ uint32_t again_sh;
  const int a0 = blockIdx.x * kSlots, j = (int)threadIdx.x / kChunks, a = a0 + j, c = (int)threadIdx.x % kChunks;
  const int slot = min(a, u.max_active - 1);
  if (threadIdx.x == 0) again_sh = 0;
  const int n_act = u.counts ? min(max(u.counts[1], 0), u.max_active) : u.max_active;
  if (a0 >= n_act) return;  // whole workgroup
  const int i = u.active_idx[slot];
  int mine[kSlots];
#pragma unroll
  for (int s = 0; s < kSlots; ++s) mine[s] = uniform_load(u.active_idx + min(a0 + s, u.max_active - 1));
  uint32_t again = 0;
  for (int t0 = a0 + 1 + (int)threadIdx.x; t0 < n_act; t0 += 256 * kAhead) {
    int later[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) later[k] = u.active_idx[min(t0 + k * 256, u.max_active - 1)];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int t = t0 + k * 256;
      const int id = t < n_act ? later[k] : -1;  // (no row)
#pragma unroll
      for (int s = 0; s < kSlots; ++s) again |= id == mine[s] && t > a0 + s ? 1u << s : 0u;
    }
  }
  __syncthreads();
  if (again != 0u) atomicOr(&again_sh, again);
  __syncthreads();
  const int64_t row = (int64_t)u.row_base + i;
  const bool live = a < n_act && i >= 0 && row >= 0 && row < u.n_rows && !((again_sh >> j) & 1u);
  const int64_t at = live ? row : 0;
  const int h0 = (int)blockIdx.y * heads, h1 = min(h0 + heads, u.n_heads);
  for (int h = h0; h < h1; ++h) {
    const int64_t src = (int64_t)h * u.nsh + (int64_t)slot * u.nsn + c * 8, e = (int64_t)h * q.esh + at * q.esn;
    const uint4 k = *reinterpret_cast<const uint4*>(u.Kn + src);
    const uint4 v = *reinterpret_cast<const uint4*>(u.Vn + src);
    store_row<D>(k, live, q.K + (int64_t)h * u.ksh + at * u.ksn + c * 8, q.k_exp + e, c);
    store_row<D>(v, live, q.V + (int64_t)h * u.vsh + at * u.vsn + c * 8, q.v_exp + e, c);
  }
}

// One workgroup per (chunk of B rows, head), as in cache_refresh_chunk; the means are those of the values that the rows read back as,
// accumulated in the order of block_means_kernel.  Bound by HBM: 538 MB read, 275 written at 32 heads, 32 832 rows of 128 in 148 to 151 us a
// call = 5.4 TB/s (copying them as bf16: 186 us, 1.08 GB); four rows of K and of V a thread under way, read past the caches because
// nothing reads them again.
template <int D>
__global__ __launch_bounds__(256) void quant_refresh_kernel(const CacheRefresh p, const QuantCache q) {
  constexpr int TPR = D / 8, RPP = 256 / TPR, UNROLL = 4;
  __shared__ __attribute__((aligned(16))) float red[RPP * D];
  const int b = blockIdx.x, h = blockIdx.y;
  const bool prompt = b < p.n_b;
  const int r0 = prompt ? b * p.B : p.M + (b - p.n_b) * p.B;
  const int len = min(p.B, (prompt ? p.M : p.L) - r0);
  const int c = threadIdx.x % TPR, rr = threadIdx.x / TPR;
  const uint16_t* ksrc = p.Kn + (int64_t)h * p.nsh + (int64_t)r0 * p.nsn + c * 8;
  const uint16_t* vsrc = p.Vn + (int64_t)h * p.nsh + (int64_t)r0 * p.nsn + c * 8;
  uint8_t* kdst = q.K + (int64_t)h * p.ksh + (int64_t)r0 * p.ksn + c * 8;
  uint8_t* vdst = q.V + (int64_t)h * p.vsh + (int64_t)r0 * p.vsn + c * 8;
  const int64_t e0 = (int64_t)h * q.esh + (int64_t)r0 * q.esn;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int r = rr; r < len + rr; r += RPP * UNROLL) {  // (uniform: the lanes of a row meet)
    uint4 k[UNROLL], v[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int64_t row = min(r + u * RPP, len - 1);
      k[u] = load_stream16(ksrc + row * p.nsn);
      v[u] = load_stream16(vsrc + row * p.nsn);
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int row = r + u * RPP;
      const bool live = row < len;
      const int64_t at = min(row, len - 1);
      const uint32_t e = row_exponent<TPR>(k[u]);
      const uint2 w = store_row<D>(k[u], live, kdst + at * p.ksn, q.k_exp + e0 + at * q.esn, c);
      if (live) add_bf16x8(acc, decode8(w, exp_value(e)));
      store_row<D>(v[u], live, vdst + at * p.vsn, q.v_exp + e0 + at * q.esn, c);
    }
  }
  if (!p.kbar || !prompt) return;  // uniform over the workgroup
#pragma unroll
  for (int e = 0; e < 8; ++e) red[rr * D + c * 8 + e] = acc[e];
  __syncthreads();
  if (threadIdx.x < D) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < RPP; ++i) s += red[i * D + threadIdx.x];
    p.kbar[((int64_t)h * p.n_b + b) * D + threadIdx.x] = s / (float)len;
  }
}

// Bound by HBM: 271 MB read, 538 written in 115 to 120 us = 6.8 to 7.0 TB/s, part of the codes from the memory-side cache; 131 us a call.
// Stores pass the caches by.
constexpr int kReadRows = 4;  // rows of K and of V per thread
template <int D>
__global__ __launch_bounds__(256) void quant_read_kernel(const QuantRead p, const QuantCache q) {
  constexpr int TPR = D / 8, RPP = 256 / TPR;
  const int h = blockIdx.y, c = threadIdx.x % TPR;
  const int r0 = blockIdx.x * (RPP * kReadRows) + threadIdx.x / TPR;
  uint2 k[kReadRows], v[kReadRows];
  uint32_t ke[kReadRows], ve[kReadRows];
#pragma unroll
  for (int u = 0; u < kReadRows; ++u) {
    const int64_t row = p.row0 + min(r0 + u * RPP, p.n_rows - 1);
    k[u] = *reinterpret_cast<const uint2*>(q.K + (int64_t)h * p.ksh + row * p.ksn + c * 8);
    v[u] = *reinterpret_cast<const uint2*>(q.V + (int64_t)h * p.vsh + row * p.vsn + c * 8);
    ke[u] = q.k_exp[(int64_t)h * q.esh + row * q.esn];
    ve[u] = q.v_exp[(int64_t)h * q.esh + row * q.esn];
  }
#pragma unroll
  for (int u = 0; u < kReadRows; ++u) {
    const int r = r0 + u * RPP;
    if (r >= p.n_rows) return;
    const int64_t to = (int64_t)h * p.osh + (int64_t)r * p.osn + c * 8;
    __builtin_nontemporal_store(__builtin_bit_cast(uintx4_t, decode8(k[u], exp_value(ke[u]))), reinterpret_cast<uintx4_t*>(p.K_out + to));
    __builtin_nontemporal_store(__builtin_bit_cast(uintx4_t, decode8(v[u], exp_value(ve[u]))), reinterpret_cast<uintx4_t*>(p.V_out + to));
  }
}

// Long lists: 32 heads, rows of 128, 4096 rows 75.6 -> 26.5 us, 32 768 2854 -> 207 (as bf16 21 and 182); 1024 rows 13.0 -> 10.9; up to 512 rows
// both are launch and latency, 6 to 8 us.  As many heads a workgroup as leave eight workgroups per compute unit.
constexpr int kUpdateMany = 512, kUpdateGroups = 2048;
template <int D>
static void launch_quant_update_t(const CacheUpdate& u, const QuantCache& q, hipStream_t st) {
  const int groups = ceil_div(u.max_active, 2048 / D);
  if (u.max_active <= kUpdateMany) {
    hipLaunchKernelGGL(quant_update_kernel<D>, dim3(groups, u.n_heads), dim3(256), 0, st, u, q);
    return;
  }
  const int heads = std::max((int)std::min<int64_t>((int64_t)groups * u.n_heads / kUpdateGroups, u.n_heads), 1);
  hipLaunchKernelGGL(quant_update_many_kernel<D>, dim3(groups, ceil_div(u.n_heads, heads)), dim3(256), 0, st, u, q, heads);
}
hipError_t launch_quant_update(const CacheUpdate& u, const QuantCache& q, int head_dim, hipStream_t st) {
  if (head_dim == 128)
    launch_quant_update_t<128>(u, q, st);
  else
    launch_quant_update_t<64>(u, q, st);
  return hipGetLastError();
}
hipError_t launch_quant_refresh(const CacheRefresh& p, const QuantCache& q, int head_dim, hipStream_t st) {
  const dim3 grid(p.n_chunks, p.n_heads);
  if (head_dim == 128)
    hipLaunchKernelGGL(quant_refresh_kernel<128>, grid, dim3(256), 0, st, p, q);
  else
    hipLaunchKernelGGL(quant_refresh_kernel<64>, grid, dim3(256), 0, st, p, q);
  return hipGetLastError();
}
hipError_t launch_quant_read(const QuantRead& p, const QuantCache& q, int n_heads, int head_dim, hipStream_t st) {
  const dim3 grid(ceil_div(p.n_rows, 2048 / head_dim * kReadRows), n_heads);
  if (head_dim == 128)
    hipLaunchKernelGGL(quant_read_kernel<128>, grid, dim3(256), 0, st, p, q);
  else
    hipLaunchKernelGGL(quant_read_kernel<64>, grid, dim3(256), 0, st, p, q);
  return hipGetLastError();
}

// =====================================================================================================
// Attention over the quantised rows.  The decomposition is that of sparse_attn_kernel: a workgroup works on one (head, key split,
// query group), its four wavefronts own a 32-row sub-tile each and keep a running softmax, and the states meet at the end.
// But the rows go from memory straight into the registers in which the products take them:
//   S^T = K Q^T   the contraction runs over d in any order, so lane (c, g) takes bytes 64 j + 16 g .. + 15 of the rows c and 16 + c
//                 (16-byte loads, a row's 64 bytes side by side) and the query operand is loaded in the same order;
//   O^T = V^T P^T the rows of the product are d columns in any order, so column tile ct has the columns c * D / 16 + ct: lane (c, g)
//                 takes D / 16 neighbouring bytes of the eight rows 4 g + i and 16 + 4 g + i whose probabilities it holds, and a
//                 byte permutation brings the codes of two rows next to each other before they are widened in pairs.
// No stage in LDS, no transposing read, no barrier: a sub-tile is 128 bytes a lane in registers.  The codes are widened
// without their power of two; 2^E of a K row multiplies its logits and that of a V row its probabilities, eight of each a lane,
// which takes a sixteenth of the multiplications and is exact.
//
// What bounds it (16 queries, 32 heads, d = 128): over every one of 32 832 rows HBM, 271 MB in 46 us = 5.9 TB/s (the bf16 cache: 81 us);
// half of the blocks, 25 queries, 139 MB in 32 us, of which the key loop runs at 6.7 TB/s and the rest is the start (2.9 us), uneven splits
// and the states' meeting; seven of 256 blocks, 8 MB in 6.7 to 8.3 us, the chain of dependent round trips, as over a bf16 cache.  With
// many query groups (175 queries, 4 heads) widening the codes, which every group of 32 repeats: 19 us against 18.5 over the bf16 cache.
// =====================================================================================================
struct QuantAttnArgs {
  AttnArgs a;  // K and V: strides in bytes
  QuantCache q;
};
template <int D>
struct QuantTile {
  uint4 k[2][D / 64];
  uint32_t v[8][D / 64];
  uint32_t e;  // exponent of row lane % 32, of K in the lower half of the wavefront, of V in the upper
};

// `exps`: the exponents of the head, of K or V by the half of the wavefront.  Requires t.vmask != 0; slots without a key read another
// row of the key set, as in issue_subtile_part.
template <int D, bool STREAM>
__device__ __forceinline__ void load_tile(QuantTile<D>& x, const AttnArgs& p, int64_t esn, const uint8_t* Kh, const uint8_t* Vh, const uint8_t* exps,
                                          const SubTile& t, int lane) {
  const int c = lane & 15, g = lane >> 4;
  if (t.kind == 0 && t.vmask == 0xffffffffu && max(p.ksn, p.vsn) < (int64_t(1) << 26)) {  // wave-uniform; 31 rows of the stride fit 32 bits
    const int64_t row0 = __builtin_amdgcn_readfirstlane(t.row0);
    const uint8_t* kt = Kh + row0 * p.ksn;
    const uint8_t* vt = Vh + row0 * p.vsn;
    const uint32_t ko = (uint32_t)c * (uint32_t)p.ksn + (uint32_t)(g * 16), vo = (uint32_t)(4 * g) * (uint32_t)p.vsn + (uint32_t)(c * (D / 16));
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < D / 64; ++j) x.k[i][j] = load_codes16<STREAM>(kt + 16 * i * p.ksn + 64 * j + ko);
#pragma unroll
    for (int e = 0; e < 8; ++e) load_codes<D, STREAM>(x.v[e], vt + (16 * (e >> 2) + (e & 3)) * p.vsn + vo);
    x.e = exps[(row0 + (lane & 31)) * esn];
    return;
  }
  // lane i < 32 holds the row of slot i (subtile_row)
  const int mine = t.kind == 0 ? t.row0 + min(lane & 31, 31 - __builtin_clz(t.vmask)) : __shfl(t.sink_row, lane & 31, kWave);
  auto row = [&](int slot) __attribute__((always_inline)) { return (int64_t)__shfl(mine, slot, kWave); };
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint8_t* k = Kh + row(16 * i + c) * p.ksn + 16 * g;
#pragma unroll
    for (int j = 0; j < D / 64; ++j) x.k[i][j] = load_codes16<STREAM>(k + 64 * j);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) load_codes<D, STREAM>(x.v[e], Vh + row(16 * (e >> 2) + 4 * g + (e & 3)) * p.vsn + c * (D / 16));
  x.e = exps[(int64_t)mine * esn];
}

// MODE bit 0: Top-C in the prologue; bit 1: key loop; bit 3: rows pass the caches by; bits 4, 5: more than 256, 1024 blocks to rank.  NT: 16-query tiles of a query group.
template <int D, int NT, int MODE>
__global__ __launch_bounds__(256, 2) void quant_attn_kernel(WIDE_FIRST_PARAMS, const QuantAttnArgs args) {
  AttnArgs p = with_first(args.a, rel_part, active_idx, Q, counts, n_b, H, max_active, args.a.n_gen, n_split, n_sub);
  p.q_groups = q_groups;
  constexpr bool FUSED = (MODE & 1) != 0, PIPE = (MODE & 2) != 0, STREAM = (MODE & 8) != 0;
  constexpr int BLOCKS = (MODE & 32) != 0 ? kFusedMaxBlocks : ((MODE & 16) != 0 ? kFusedManyBlocks : 256);
  constexpr int kKS = D / 32, kCT = D / 16;
  __shared__ __attribute__((aligned(16))) char ldsO[kWavesPerGroup * 16 * D * 4];  // the wavefronts' O tiles at the end
  __shared__ float2 ml_sh[kWavesPerGroup][16];
  __shared__ __attribute__((aligned(16))) float exps_sh[kWavesPerGroup][64];
  __shared__ __attribute__((aligned(16))) char topk_raw[FUSED ? sizeof(TopkShared) : 16];
  using Kept = KeptList<FUSED, BLOCKS>;
  __shared__ int32_t kept_beside[Kept::kEntriesBeside];
  __shared__ uint32_t kept_bits_sh[kBitmapBlocks / 32];
  __shared__ int sinks_unsorted_sh;

  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int slot8 = list_index() >> 3;
  int first8 = slot8, qg = 0;
  if (p.q_groups > 1) {
    first8 = slot8 / p.q_groups;
    qg = slot8 - first8 * p.q_groups;
  }
  const int pair = first8 * 8 + (int)(blockIdx.x & 7u);
  if (pair >= p.n_split * p.H) return;  // whole workgroup
  const int h = pair / p.n_split, split = pair - h * p.n_split;
  const Counts counted(p);
  const int q0 = qg * NT * 16;
  const uint16_t* Qh = p.Q + (int64_t)h * p.qsh;
  const uint8_t* Kh = args.q.K + (int64_t)h * p.ksh;
  const uint8_t* Vh = args.q.V + (int64_t)h * p.vsh;
  const uint8_t* exps = (lane < 32 ? args.q.k_exp : args.q.v_exp) + (int64_t)h * args.q.esh;
  const int64_t esn = args.q.esn;

  int qrow[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) qrow[n] = fetch_q_row(p.active_idx, q0 + 16 * n, p.max_active, p.n_gen, lane);
  bf16x8 q[NT][kKS];  // lane (query, g), k-step 2 j + t: Q[query][64 j + 16 g + 8 t .. + 7]
  auto load_q = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const uint16_t* src = Qh + (int64_t)max(qrow[n], 0) * p.qsn + g * 16;
#pragma unroll
      for (int kk = 0; kk < kKS; ++kk) {
        const uint4 v = *reinterpret_cast<const uint4*>(src + 64 * (kk >> 1) + 8 * (kk & 1));
        q[n][kk] = as_bf16x8(qrow[n] >= 0 ? v : make_uint4(0u, 0u, 0u, 0u));
      }
    }
  };
  typename Kept::Id* kept_sh = Kept::place(topk_raw, kept_beside);
  const typename Kept::Id* kept_blocks = kept_sh;
  if constexpr (!FUSED) kept_blocks = p.kept_blocks;
  int few_sinks;
  if (FUSED) {  // the query rows travel while the blocks are ranked
    FirstParts<8, 256, BLOCKS> first;
    first_partials(first, p, false);
    few_sinks = request_few_sinks(p, lane);
    if (qg > 0 && q0 >= counted.n_active(p)) return;  // a query group past the device-side count has nothing to do
    load_q();
    rank_blocks(p, first, false, counted.focus, kept_sh, *reinterpret_cast<TopkShared*>(topk_raw), pair == 0 && qg == 0);
  } else {
    few_sinks = request_few_sinks(p, lane);
    if (qg > 0 && q0 >= counted.n_active(p)) return;
  }
  const SinkUnion uni = prepare_union(p, split, kept_blocks, kept_bits_sh, &sinks_unsorted_sh);

  const SplitRounds rounds(p, split, h);
  RoundList<typename Kept::Id> list{p, rounds, uni, kept_blocks, wave, lane, few_sinks};
  QuantTile<D> x;
  SubTile t;
  t.kind = 0;
  t.row0 = 0;
  t.vmask = 0u;
  t.sink_row = 0;
  if (!PIPE && split * kWavesPerGroup + wave < p.n_sub)
    t = locate_subtile(split * kWavesPerGroup + wave, lane, p.M, p.N, p.B, p.n_b, p.sub_per_block, kept_blocks, p.n_keep, p.sink_idx, p.n_sink,
                       uni.kept_bits, uni.ascending, 0, FUSED, few_sinks);
  if (!PIPE && t.vmask != 0u) load_tile<D, STREAM>(x, p, esn, Kh, Vh, exps, t, lane);
  if (!FUSED) load_q();
  const int n_act = counted.n_active(p);
#pragma unroll
  for (int n = 0; n < NT; ++n)
    if (q0 + 16 * n + c >= n_act) {
#pragma unroll
      for (int kk = 0; kk < kKS; ++kk) q[n][kk] = as_bf16x8(make_uint4(0u, 0u, 0u, 0u));
    }

  float m_run[NT], l_run[NT];
  floatx4 o[NT][kCT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    m_run[n] = -INFINITY;
    l_run[n] = 0.f;
#pragma unroll
    for (int ct = 0; ct < kCT; ++ct) o[n][ct] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  auto consume = [&](const QuantTile<D>& x, uint32_t vmask) __attribute__((always_inline)) {  // one sub-tile into the running softmax
    float* es = exps_sh[wave];
    es[lane] = exp_value(x.e);
    floatx4 acc[NT][2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
      for (int n = 0; n < NT; ++n) acc[n][kt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < D / 64; ++j) {
        const uint4 w = x.k[kt][j];
        const bf16x8 k0 = as_bf16x8(decode8(make_uint2(w.x, w.y), 1.f)), k1 = as_bf16x8(decode8(make_uint2(w.z, w.w), 1.f));
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          acc[n][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, q[n][2 * j], acc[n][kt], 0, 0, 0);
          acc[n][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, q[n][2 * j + 1], acc[n][kt], 0, 0, 0);
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const floatx4 ek[2] = {*reinterpret_cast<const floatx4*>(es + 4 * g), *reinterpret_cast<const floatx4*>(es + 16 + 4 * g)};
    const floatx4 ev[2] = {*reinterpret_cast<const floatx4*>(es + 32 + 4 * g), *reinterpret_cast<const floatx4*>(es + 48 + 4 * g)};
    bf16x8 pb[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      acc[n][0] *= ek[0];
      acc[n][1] *= ek[1];
      float ps[8];
      const float alpha = softmax_step(acc[n], vmask, g, p.scale_log2, m_run[n], l_run[n], ps);
      if (__ballot(alpha != 1.f) != 0ull) {
#pragma unroll
        for (int ct = 0; ct < kCT; ++ct) o[n][ct] *= alpha;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) ps[e] *= ev[e >> 2][e & 3];
      pb[n] = pack_bf16x8(ps);  // the second product's operand: P is bf16 there as in the attention over the bf16 cache
    }
#pragma unroll
    for (int w = 0; w < D / 64; ++w) {
      uint32_t lo[4], hi[4];  // codes of two rows next to each other: columns 0, 1 and 2, 3 of the word
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        lo[m] = __builtin_amdgcn_perm(x.v[2 * m + 1][w], x.v[2 * m][w], 0x05010400u);
        hi[m] = __builtin_amdgcn_perm(x.v[2 * m + 1][w], x.v[2 * m][w], 0x07030602u);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t(&s)[4] = i < 2 ? lo : hi;
        const bf16x8 v = as_bf16x8(make_uint4(decode2(s[0], i & 1, 1.f), decode2(s[1], i & 1, 1.f), decode2(s[2], i & 1, 1.f), decode2(s[3], i & 1, 1.f)));
#pragma unroll
        for (int n = 0; n < NT; ++n) o[n][4 * w + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pb[n], o[n][4 * w + i], 0, 0, 0);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the next sub-tile's exponents follow these reads
  };
  if (!PIPE) {  // one sub-tile per wavefront at most
    if (t.vmask != 0u) consume(x, t.vmask);
  } else {
    // The next sub-tile's rows travel while one is multiplied.  They are requested in any case, past the end those of row 0, so that it is
    // known how many requests lie behind the ones waited for; and in one place each, because these kernels start with a cold
    // instruction cache.
#pragma unroll 1
    for (int i = -1; i < rounds.n_rounds; ++i) {
      const SubTile next = list.take();
      SubTile there = next;
      if (there.vmask == 0u) {
        there.kind = 0;
        there.row0 = 0;
        there.vmask = 1u;
      }
      QuantTile<D> y;
      load_tile<D, STREAM>(y, p, esn, Kh, Vh, exps, there, lane);
      __builtin_amdgcn_sched_barrier(0);
      if (t.vmask != 0u) consume(x, t.vmask);
      x = y;
      t = next;
    }
  }

  // ---- the four wavefronts' states, one query tile at a time.  A lane holds D / 16 neighbouring columns of one query four times over;
  // 16-byte chunks of a row are permuted by its number (see sparse_attn_kernel).
  constexpr int kVec = D / 64, kRowChunks = D / 4;
  auto chunk_at = [&](int w, int row, int ch) __attribute__((always_inline)) {
    return reinterpret_cast<floatx4*>(ldsO + w * (16 * D * 4) + (row * kRowChunks + (ch ^ row)) * 16);
  };
  const int mq = threadIdx.x >> 4, mc = threadIdx.x & 15;  // query this thread merges
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    if (n > 0) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int w = 0; w < kVec; ++w)
        *chunk_at(wave, c, (4 * g + i) * kVec + w) = floatx4{o[n][4 * w][i], o[n][4 * w + 1][i], o[n][4 * w + 2][i], o[n][4 * w + 3][i]};
    if (g == 0) ml_sh[wave][c] = make_float2(m_run[n], l_run[n]);
    __syncthreads();
    float2 ml[kWavesPerGroup];
    float mmax = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWavesPerGroup; ++w) {
      ml[w] = ml_sh[w][mq];
      mmax = fmaxf(mmax, ml[w].x);
    }
    floatx4 acc_o[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) acc_o[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    float lsum = 0.f;
#pragma unroll
    for (int w = 0; w < kWavesPerGroup; ++w) {
      const float f = ml[w].y > 0.f ? __builtin_amdgcn_exp2f(ml[w].x - mmax) : 0.f;
      lsum += f * ml[w].y;
#pragma unroll
      for (int i = 0; i < kVec; ++i) acc_o[i] += f * *chunk_at(w, mq, mc + 16 * i);
    }
    const int a = q0 + 16 * n + mq;  // position in the active list
    if (a < n_act) {
      if (p.n_split == 1) {
        const float inv = lsum > 0.f ? 1.f / lsum : 0.f;
        uint16_t* dst = p.out + (int64_t)h * p.osh + (int64_t)a * p.osn + mc * 4;
#pragma unroll
        for (int i = 0; i < kVec; ++i)
          *reinterpret_cast<uint2*>(dst + 64 * i) =
              make_uint2(cvt_pk_bf16(acc_o[i][0] * inv, acc_o[i][1] * inv), cvt_pk_bf16(acc_o[i][2] * inv, acc_o[i][3] * inv));
        if (p.lse && mc == 0)
          p.lse[(int64_t)h * p.max_active + a] = lsum > 0.f ? (mmax + __builtin_amdgcn_logf(lsum)) * kLn2 : -INFINITY;
      } else {
        const int64_t row = ((int64_t)h * p.q_pad + a) * p.n_split + split;
#pragma unroll
        for (int i = 0; i < kVec; ++i) *reinterpret_cast<floatx4*>(p.part_o + row * D + mc * 4 + 64 * i) = acc_o[i];
        if (mc == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * row) = make_float2(lsum > 0.f ? mmax : -INFINITY, lsum);
      }
    }
  }
}

#define QUANT_LAUNCH(kernel, x)                                                                                                  \
  hipLaunchKernelGGL(kernel, grid_list(query_group_list(p, (x).a.H)), dim3(256), 0, st, (x).a.rel_part, (x).a.active_idx, (x).a.Q, \
                     (x).a.counts, (x).a.n_b, (x).a.H, (x).a.max_active, (x).a.q_groups, (x).a.n_split, (x).a.n_sub, x)

template <int D, int NT, int STREAM>
static void launch_quant_loop(const QuantAttnArgs& x, const SplitPlan& p, bool fused, hipStream_t st) {
  if (!fused)
    QUANT_LAUNCH((quant_attn_kernel<D, NT, STREAM | 2>), x);
  else if (x.a.n_b > kFusedManyBlocks)
    QUANT_LAUNCH((quant_attn_kernel<D, NT, STREAM | 35>), x);
  else if (x.a.n_b > 256)
    QUANT_LAUNCH((quant_attn_kernel<D, NT, STREAM | 19>), x);
  else
    QUANT_LAUNCH((quant_attn_kernel<D, NT, STREAM | 3>), x);
}
template <int D, int NT>
static void launch_quant_nt(const QuantAttnArgs& x, const SplitPlan& p, bool fused, hipStream_t st) {
  if (p.stream)
    launch_quant_loop<D, NT, 8>(x, p, fused, st);
  else if (p.pipelined)
    launch_quant_loop<D, NT, 0>(x, p, fused, st);
  else if (!fused)
    QUANT_LAUNCH((quant_attn_kernel<D, NT, 0>), x);
  else if (x.a.n_b > kFusedManyBlocks)
    QUANT_LAUNCH((quant_attn_kernel<D, NT, 33>), x);
  else if (x.a.n_b > 256)
    QUANT_LAUNCH((quant_attn_kernel<D, NT, 17>), x);
  else
    QUANT_LAUNCH((quant_attn_kernel<D, NT, 1>), x);
}
template <int D>
static hipError_t launch_quant_t(const QuantAttnArgs& x, const SplitPlan& p, bool fused, hipStream_t st) {
  if (!p.pipelined && p.n_split * kWavesPerGroup < p.n_sub) return hipErrorInvalidValue;  // one sub-tile per wavefront
  if (query_group_list(p, x.a.H) > kMaxList) return hipErrorInvalidValue;
  if (p.q_tiles_per_group == 1)
    launch_quant_nt<D, 1>(x, p, fused, st);
  else
    launch_quant_nt<D, 2>(x, p, fused, st);
  return hipGetLastError();
}

hipError_t launch_quant_attn(const void* Q, const int32_t* active_idx, const int32_t* counts, int max_active, const QuantCache& q, const focus_shape& s,
                             const int32_t* kept_blocks, int n_keep, const int32_t* sink_idx, int n_sink, const SplitPlan& p, void* out, float* lse,
                             float* part_o, float* part_ml, const FusedTopC* fused, hipStream_t st) {
  QuantAttnArgs x;
  x.q = q;
  x.a = attention_args(Q, active_idx, counts, max_active, nullptr, nullptr, s, kept_blocks, n_keep, sink_idx, n_sink, p, out, lse, part_o, part_ml, fused);
  const hipError_t e = s.head_dim == 128 ? launch_quant_t<128>(x, p, fused != nullptr, st) : launch_quant_t<64>(x, p, fused != nullptr, st);
  return e != hipSuccess || p.n_split == 1 ? e : launch_attn_combine(x.a, p, s.head_dim, st);
}

}  // namespace focus
