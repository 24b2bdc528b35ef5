// Rows turned by their positions, and new rows into the pages of a cache.
//
//   turn_rows_kernel<D, false, false>   focus_rotary: out = X turned
//   turn_rows_kernel<D, QUANT, true>    focus_paged_append: K turned and V as it is into their pages, Q turned beside them
//
// A pair (a, b) at position p becomes (a c - b s, b c + a s) with c, s = scale * cos, sin of p * freq[j].  Nothing but the rows has to be moved
// (four bytes a value); the angles, in 64 bits, are worked out once for all heads of a row.
#include <algorithm>

#include "focus_codes.h"
#include "focus_rows.h"

namespace focus {

// A workgroup has R = 512 / D rows, whose R * D / 2 angles are one a thread; cos and sin meet the heads in LDS.  The items of a workgroup are its
// rows times its slots (heads of Q, of K, of V); D / 16 neighbouring threads have one item, sixteen values each: where pairs are halves
// apart eight of each half (so that a pair is in one thread), else sixteen neighbours.  Values that are not turned are divided the same way.
// Items under way per thread, read past the caches, where nothing else reads them.  Bound by HBM: 32 768 rows of 32 heads of 128, 537 MB, in 92.3 us =
// 5.8 TB/s (a copy of a gigabyte: 5.2); prompts of 8 000 rows into eight-bit pages, 185 MB, in 41.6.  One, two, three, four, six items 99.9, 96.2, 99.2, 99.6, 95.7
// and 45.8, 44.3, 46.5, 45.5, 51.4 us through the caches; past them two 92.3 and 41.6.  A few rows are one launch and two round trips: 2.9 us.
constexpr int kTurnItems = 2;

template <int D, bool QUANT, bool PAGES>
__global__ __launch_bounds__(256) void turn_rows_kernel(const TurnRows p) {
  constexpr int kThreads = D / 16, kRows = 512 / D, kItems = 256 / kThreads, kPairs = D / 2;
  __shared__ __attribute__((aligned(16))) float2 turn_sh[kRows][kPairs];
  __shared__ int2 place_sh[kRows];  // page and place in it, page < 0: nowhere
  __shared__ int live_sh[kRows], again_sh[kRows];
  const int tid = threadIdx.x, c = tid % kThreads, r = PAGES ? (int)blockIdx.y : 0;
  RequestRows q;
  if constexpr (PAGES) {
    q = request_rows(p.b, r);
  } else {
    q.first = 0;
    q.n = q.count = p.b.n_rows;
  }
  const int i0 = (int)blockIdx.x * kRows, rows = min(q.n - i0, kRows);
  if (rows <= 0) return;  // whole workgroup
  const int lg = rows > 4 ? 3 : (rows > 2 ? 2 : (rows > 1 ? 1 : 0));
  const int slots = p.n_q_heads + (PAGES ? 2 * p.n_heads : 0), share = (slots + (int)gridDim.z - 1) / (int)gridDim.z;
  const int slot0 = (int)blockIdx.z * share, n_items = max(min(share, slots - slot0), 0) << lg;

  const int half = p.rot_dim / 2;
  const bool turned = c < p.rot_dim / 16, apart = turned && !p.interleaved;
  const int turn_a = apart ? 8 * c : 16 * c, turn_b = apart ? half + 8 * c : 16 * c + 8;  // of Q and K
  struct Item {
    int slot, row;
    bool valid;
  };
  auto item_of = [&](int it) __attribute__((always_inline)) {
    Item x;
    x.row = it & ((1 << lg) - 1);
    x.slot = slot0 + (it >> lg);
    x.valid = it < n_items && x.row < rows;
    if (!x.valid) x.row = 0, x.slot = slot0;
    return x;
  };
  uint4 a[kTurnItems], b[kTurnItems];
  auto load = [&](int it0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kTurnItems; ++u) {
      const Item x = item_of(it0 + u * kItems);
      if (!x.valid) continue;
      const int64_t row = q.first + i0 + x.row;
      const bool is_v = PAGES && x.slot >= p.n_q_heads + p.n_heads;
      const uint16_t* src;
      if (!PAGES || x.slot < p.n_q_heads)
        src = p.Q + row * p.qsn + (int64_t)x.slot * p.qsh;
      else
        src = (is_v ? p.Vn : p.Kn) + row * p.nsn + (int64_t)(x.slot - p.n_q_heads - (is_v ? p.n_heads : 0)) * p.nsh;
      a[u] = load_stream16(src + (is_v ? 16 * c : turn_a));
      b[u] = load_stream16(src + (is_v ? 16 * c + 8 : turn_b));
    }
  };
  load(tid / kThreads);

  {
    const int k = tid / kPairs, j = tid % kPairs, i = i0 + min(k, rows - 1);
    const int len = PAGES ? max(uniform_load(p.b.seq_len + r), 0) : 0;
    const double freq = j < half ? p.freq[j] : 0.0;
    const int pos = p.b.positions ? p.b.positions[q.first + i] : (PAGES ? len - q.count + i : i);
    if (j < half) {
      double cosine, sine;
      cos_sin((double)((int64_t)p.pos_base + pos) * freq, cosine, sine);
      turn_sh[k][j] = make_float2((float)(p.scale * cosine), (float)(p.scale * sine));
    }
    if (j == 0) {
      live_sh[k] = !p.b.positions && !PAGES ? 1 : pos >= 0;
      if constexpr (PAGES) {
        int2 at = make_int2(-1, 0);
        if (pos >= 0) {
          const int entry = pos / p.page;
          if (entry < p.b.table_width) {
            const int id = p.b.page_table[(int64_t)r * p.b.table_stride + entry];
            if (id >= 0 && id < p.n_pages) at = make_int2(id, pos - entry * p.page);
          }
        }
        place_sh[k] = at;
        again_sh[k] = 0;
      }
    }
  }
  __syncthreads();
  if constexpr (PAGES) {
    if (p.b.positions) {  // a position that a later row of the request has as well is left to that row
      int mine[kRows];
#pragma unroll
      for (int k = 0; k < kRows; ++k) mine[k] = p.b.positions[q.first + i0 + min(k, rows - 1)];
      for (int j = i0 + 1 + tid; j < q.n; j += 256) {
        const int other = p.b.positions[q.first + j];
#pragma unroll
        for (int k = 0; k < kRows; ++k)
          if (other == mine[k] && j > i0 + k) again_sh[k] = 1;
      }
      __syncthreads();
    }
  }

  for (int it0 = tid / kThreads; it0 < n_items; it0 += kItems * kTurnItems) {
    if (it0 != tid / kThreads) load(it0);
#pragma unroll
    for (int u = 0; u < kTurnItems; ++u) {
      const Item x = item_of(it0 + u * kItems);
      if (!x.valid || !live_sh[x.row]) continue;
      const bool is_q = !PAGES || x.slot < p.n_q_heads, is_v = !is_q && x.slot >= p.n_q_heads + p.n_heads;
      const int at_a = is_v ? 16 * c : turn_a, at_b = is_v ? 16 * c + 8 : turn_b;
      const bool turn = turned && !is_v;
      float va[8] = {bf16_lo(a[u].x), bf16_hi(a[u].x), bf16_lo(a[u].y), bf16_hi(a[u].y), bf16_lo(a[u].z), bf16_hi(a[u].z), bf16_lo(a[u].w), bf16_hi(a[u].w)};
      float vb[8] = {bf16_lo(b[u].x), bf16_hi(b[u].x), bf16_lo(b[u].y), bf16_hi(b[u].y), bf16_lo(b[u].z), bf16_hi(b[u].z), bf16_lo(b[u].w), bf16_hi(b[u].w)};
      if (turn) {
#pragma clang fp contract(off)  // (products and sums rounded one by one: the same bits wherever they are worked out)
        const float4* cs = reinterpret_cast<const float4*>(&turn_sh[x.row][8 * c]);
        float cosine[8], sine[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 w = cs[i];
          cosine[2 * i] = w.x;
          sine[2 * i] = w.y;
          cosine[2 * i + 1] = w.z;
          sine[2 * i + 1] = w.w;
        }
        if (p.interleaved) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float a0 = va[2 * i], a1 = va[2 * i + 1], b0 = vb[2 * i], b1 = vb[2 * i + 1];
            va[2 * i] = a0 * cosine[i] - a1 * sine[i];
            va[2 * i + 1] = a1 * cosine[i] + a0 * sine[i];
            vb[2 * i] = b0 * cosine[4 + i] - b1 * sine[4 + i];
            vb[2 * i + 1] = b1 * cosine[4 + i] + b0 * sine[4 + i];
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float x0 = va[i], x1 = vb[i];
            va[i] = x0 * cosine[i] - x1 * sine[i];
            vb[i] = x1 * cosine[i] + x0 * sine[i];
          }
        }
      }
      uint16_t* dst = nullptr;
      if (is_q) {
        dst = p.Qo + (int64_t)(q.first + i0 + x.row) * p.qosn + (int64_t)x.slot * p.qosh;
      } else if constexpr (PAGES) {
        const int2 at = place_sh[x.row];
        const bool there = at.x >= 0 && !again_sh[x.row];
        const int h = x.slot - p.n_q_heads - (is_v ? p.n_heads : 0);
        const int64_t off = is_v ? (int64_t)at.x * p.vsp + (int64_t)h * p.vsh + (int64_t)at.y * p.vsn
                                 : (int64_t)at.x * p.ksp + (int64_t)h * p.ksh + (int64_t)at.y * p.ksn;
        if constexpr (QUANT) {
          uint32_t m = 0u;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint32_t x0 = __float_as_uint(va[i]) & 0x7fffffffu, x1 = __float_as_uint(vb[i]) & 0x7fffffffu;
            m = max(m, max(x0 < 0x7f800000u ? x0 : 0u, x1 < 0x7f800000u ? x1 : 0u));
          }
#pragma unroll
          for (int o = 1; o < kThreads; o <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, kWave));
          // 448 = 1.75 * 2^8: a mantissa past 0x600000 takes the next power of two
          const uint32_t e = (uint32_t)min(max((int)((m + 0x1fffffu) >> 23) - 8, kExpMin), kExpMax);
          const float inv = exp_value(254u - e);
          auto four = [&](const float* v) __attribute__((always_inline)) {
            const int w = __builtin_amdgcn_cvt_pk_fp8_f32(scaled_for_code(v[0], inv), scaled_for_code(v[1], inv), 0, false);
            return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(scaled_for_code(v[2], inv), scaled_for_code(v[3], inv), w, true);
          };
          if (there) {
            uint8_t* to = static_cast<uint8_t*>(is_v ? p.V : p.K) + off;
            *reinterpret_cast<uint2*>(to + at_a) = make_uint2(four(va), four(va + 4));
            *reinterpret_cast<uint2*>(to + at_b) = make_uint2(four(vb), four(vb + 4));
            if (c == 0) (is_v ? p.v_exp : p.k_exp)[(int64_t)at.x * p.esp + (int64_t)h * p.esh + (int64_t)at.y * p.esn] = (uint8_t)e;
          }
          continue;
        }
        if (!there) continue;
        dst = static_cast<uint16_t*>(is_v ? p.V : p.K) + off;
      }
      uint4 oa = a[u], ob = b[u];
      if (turn) {
        oa = __builtin_bit_cast(uint4, pack_bf16x8(va));
        ob = __builtin_bit_cast(uint4, pack_bf16x8(vb));
      }
      *reinterpret_cast<uint4*>(dst + at_a) = oa;
      *reinterpret_cast<uint4*>(dst + at_b) = ob;
    }
  }
}

// Heads of a row are divided among workgroups until there are enough of them to fill the chip, as long as each has an item a thread.
constexpr int kTurnGroups = 512;
template <int D>
static hipError_t launch_turn_rows_t(const TurnRows& p, bool pages, bool quant, hipStream_t st) {
  constexpr int kRows = 512 / D, kItems = 4096 / D;
  const int most = pages ? p.b.max_rows : p.b.n_rows, chunks = ceil_div(most, kRows), requests = pages ? p.b.n_req : 1;
  const int slots = p.n_q_heads + (pages ? 2 * p.n_heads : 0);
  const int64_t groups = (int64_t)chunks * requests;
  const int64_t wanted = std::min<int64_t>(ceil_div64(kTurnGroups, groups), ceil_div64((int64_t)std::min(most, kRows) * slots, kItems));
  const dim3 grid(chunks, requests, (uint32_t)std::max<int64_t>(wanted, 1));
  if (!pages)
    hipLaunchKernelGGL((turn_rows_kernel<D, false, false>), grid, dim3(256), 0, st, p);
  else if (quant)
    hipLaunchKernelGGL((turn_rows_kernel<D, true, true>), grid, dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL((turn_rows_kernel<D, false, true>), grid, dim3(256), 0, st, p);
  return hipGetLastError();
}
hipError_t launch_turn_rows(const TurnRows& p, int head_dim, bool pages, bool quant, hipStream_t st) {
  return head_dim == 128 ? launch_turn_rows_t<128>(p, pages, quant, st) : launch_turn_rows_t<64>(p, pages, quant, st);
}

}  // namespace focus
