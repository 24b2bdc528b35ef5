// Attention of the requests' few new rows over their pages.
//
// The keys of a request are cut into tiles of 32, and a unit is what shares them: the rows of a request times the query heads of one K/V head, sixteen
// (or 32) of those at a time.  All tiles of all units, in the order request, head, group of rows, tile, are divided evenly among the wavefronts
// of one launch, by the lengths that they find in memory: a batch of one long and many short requests keeps the whole chip busy, and a captured graph
// does so for lengths that nobody knew when it was captured.  A wavefront keeps the running softmax of the unit that it is in; a unit that
// lies within one wavefront is written out by it, the pieces of the others go to the workspace, and a second launch joins them.
//
// The products are those of the attention over the quantised cache: rows go from memory straight into the registers in which
// v_mfma_f32_16x16x32_bf16 takes them.
//   S^T = K Q^T   lane (c, g) has 16 bytes at a time of the rows c and 16 + c, 64 bytes of a row side by side
//   O^T = V^T P^T column tile ct has the columns c * D / 16 + ct: lane (c, g) has D / 16 neighbouring values of the eight rows 4 g + i and
//                 16 + 4 g + i whose probabilities it holds, and byte permutations put those of two rows next to each other
// P is split into two bf16 numbers, p = hi + lo to 2^-17, and multiplied twice: rounded to one it would cost the result as much
// again as its own rounding, and the matrix unit has nothing else to do (a tile is 16 KB from memory and 24 products).
#include <algorithm>

#include "focus_codes.h"
#include "focus_rows.h"

namespace focus {

constexpr int kTile = 32;

// What a wavefront knows of a request; the same in all lanes
struct Request {
  int first, n, count;  // RequestRows
  int len, tiles;       // keys; tiles of a unit, one at least (of no key: it writes the empty rows)
  int groups;           // units of a K/V head
};
template <int NT>
__device__ __forceinline__ Request make_request(const PagedAttn& p, const RequestRows& q, int len) {
  Request x;
  x.first = q.first;
  x.n = q.n;
  x.count = q.count;
  x.len = (int)min((int64_t)max(len, 0), (int64_t)p.b.table_width * p.page);
  x.tiles = max((x.len + kTile - 1) / kTile, 1);
  x.groups = (x.n * p.group + 16 * NT - 1) / (16 * NT);
  return x;
}
template <int NT>
__device__ __forceinline__ Request load_request(const PagedAttn& p, int r) {
  return make_request<NT>(p, request_rows(p.b, r), uniform_load(p.b.seq_len + r));
}
// tiles of one K/V head of request r (r per lane)
template <int NT>
__device__ __forceinline__ uint32_t head_tiles(const PagedAttn& p, int r) {
  if (r >= p.b.n_req) return 0u;
  const int len = p.b.seq_len[r];
  RequestRows q;
  if (p.b.row_start == nullptr)
    q = clip_rows(p.b, r, r + 1);
  else
    q = clip_rows(p.b, p.b.row_start[r], p.b.row_start[r + 1]);
  const Request x = make_request<NT>(p, q, len);
  return (uint32_t)(x.groups * x.tiles);
}

__device__ __forceinline__ uint32_t wave_total(uint32_t x) {
  return wave_reduce_u32(x, [](uint32_t a, uint32_t b) { return a + b; });
}

// The requests' tiles as one wavefront adds them up, 64 requests a turn; those of the first kKept turns stay in registers.
template <int NT>
struct Prefix {
  static constexpr int kKept = 4;
  uint32_t x[kKept];
  uint32_t total;
  __device__ __forceinline__ Prefix(const PagedAttn& p, int lane) {
    uint32_t sum = 0u;
#pragma unroll
    for (int u = 0; u < kKept; ++u) {
      x[u] = 0u;
      if (u * kWave < p.b.n_req) x[u] = head_tiles<NT>(p, u * kWave + lane);
      sum += x[u];
    }
    for (int r0 = kKept * kWave; r0 < p.b.n_req; r0 += kWave) sum += head_tiles<NT>(p, r0 + lane);
    total = wave_total(sum);
  }
  // the tiles of a head before those of request r
  __device__ __forceinline__ uint32_t before(const PagedAttn& p, int r, int lane) const {
    uint32_t sum = 0u;
#pragma unroll
    for (int u = 0; u < kKept; ++u) sum += u * kWave + lane < r ? x[u] : 0u;
    for (int r0 = kKept * kWave; r0 < r; r0 += kWave) sum += r0 + lane < r ? head_tiles<NT>(p, r0 + lane) : 0u;
    return wave_total(sum);
  }
  // the request in which tile t < total of a head lies
  __device__ __forceinline__ int find(const PagedAttn& p, uint32_t t, uint32_t& before, int lane) const {
    uint32_t mine = 0u, done = 0u;
    int r0 = 0;
#pragma unroll 1
    for (; r0 < p.b.n_req; r0 += kWave) {
      mine = r0 < kKept * kWave ? x[0] : 0u;
#pragma unroll
      for (int u = 1; u < kKept; ++u) mine = r0 == u * kWave ? x[u] : mine;
      if (r0 >= kKept * kWave) mine = head_tiles<NT>(p, r0 + lane);
      const uint32_t sum = wave_total(mine);
      if (t < done + sum) break;
      done += sum;
    }
    uint32_t incl = mine;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const uint32_t y = __shfl_up(incl, o, kWave);
      if (lane >= o) incl += y;
    }
    const int at = __builtin_ctzll(__ballot(done + incl > t) | (1ull << 63));
    before = done + (uint32_t)__builtin_amdgcn_readlane((int)(incl - mine), at);
    return r0 + at;
  }
};

// The tiles of all requests, R of them, among W wavefronts: floor(i R / W) is the first one of wavefront i.
struct Shares {
  int64_t base;  // R = base * W + rest
  uint32_t rest, workers;
  __device__ __forceinline__ Shares(int64_t R, int W) {
    base = R / W;
    rest = (uint32_t)(R - base * W);
    workers = (uint32_t)W;
  }
  __device__ __forceinline__ int64_t begin(int i) const { return base * i + rest * (uint32_t)i / workers; }  // W <= 2^16
  // the last wavefront that begins with tile s or before it
  __device__ __forceinline__ int of(int64_t s) const {
    const double per = (double)base + (double)rest / (double)workers;
    int i = min(max((int)((double)s / per), 0), (int)workers - 1);
    while (i > 0 && begin(i) > s) --i;
    while (i + 1 < (int)workers && begin(i + 1) <= s) ++i;
    return i;
  }
};

// A tile's place
struct Tile {
  Request q;
  int r, h, qg, t;
  bool first, last;  // of the piece of its unit that the wavefront has
};

template <int D, bool QUANT>
struct TileRows {
  static constexpr int kK = QUANT ? D / 64 : D / 32, kV = QUANT ? D / 64 : D / 32;  // 16-byte pieces of a K row, dwords of a V row's piece
  uint4 k[2][kK];
  uint32_t v[8][kV];
  uint32_t e;     // QUANT: exponent of row lane % 32, of K in the lower half of the wavefront, of V in the upper
  uint32_t mask;  // bit s: slot s holds a key
};

template <int N>
__device__ __forceinline__ void load_piece(uint32_t (&v)[N], const uint8_t* p) {
  if constexpr (N == 4) {
    const uintx4 w = *reinterpret_cast<const uintx4*>(p);
    v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
  } else if constexpr (N == 2) {
    const uintx2 w = *reinterpret_cast<const uintx2*>(p);
    v[0] = w.x; v[1] = w.y;
  } else {
    v[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

// page of slot lane % 32 of a tile (any entry for slots past the keys)
__device__ __forceinline__ int load_entry(const PagedAttn& p, const Tile& t, int lane) {
  const int row = min(t.t * kTile + (lane & 31), max(t.q.len - 1, 0));
  return p.b.page_table[(int64_t)t.r * p.b.table_stride + row / p.page];
}

// Rows of a tile; `entry` from load_entry.  Slots without a key read another row of the tile, all of them row 0 of page 0 where it has none
// (what is read there is not used, but zero times an infinity would be).
template <int D, bool QUANT>
__device__ __forceinline__ void load_tile_rows(TileRows<D, QUANT>& x, const PagedAttn& p, const Tile& t, int entry, int lane) {
  constexpr int kPiece = D / 16 * (QUANT ? 1 : 2);  // bytes of a V row that a lane takes
  const int c = lane & 15, g = lane >> 4, row0 = t.t * kTile;
  const int mine = min(row0 + (lane & 31), max(t.q.len - 1, 0));
  const bool there = row0 + (lane & 31) < t.q.len && entry >= 0 && entry < p.n_pages;
  x.mask = (uint32_t)__ballot(there);  // (the upper half of the wavefront repeats the lower one)
  const uint8_t* Kh = p.K + (int64_t)t.h * p.ksh;
  const uint8_t* Vh = p.V + (int64_t)t.h * p.vsh;
  if (x.mask == 0xffffffffu && (p.page & 15) == 0) {  // sixteen rows lie in one page
    const int page0 = __builtin_amdgcn_readlane(entry, 0), page1 = __builtin_amdgcn_readlane(entry, 16);
    const int at0 = row0 % p.page, at1 = (row0 + 16) % p.page;
    const uint8_t* kp[2] = {Kh + (int64_t)page0 * p.ksp + (int64_t)at0 * p.ksn, Kh + (int64_t)page1 * p.ksp + (int64_t)at1 * p.ksn};
    const uint8_t* vp[2] = {Vh + (int64_t)page0 * p.vsp + (int64_t)at0 * p.vsn, Vh + (int64_t)page1 * p.vsp + (int64_t)at1 * p.vsn};
    const uint32_t ko = (uint32_t)c * (uint32_t)p.ksn + (uint32_t)(g * 16), vo = (uint32_t)(4 * g) * (uint32_t)p.vsn + (uint32_t)(c * kPiece);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < x.kK; ++j) x.k[i][j] = *reinterpret_cast<const uint4*>(kp[i] + 64 * j + ko);
#pragma unroll
    for (int e = 0; e < 8; ++e) load_piece(x.v[e], vp[e >> 2] + (e & 3) * p.vsn + vo);
    if constexpr (QUANT) {
      const int page = (lane & 16) ? page1 : page0, at = ((lane & 16) ? at1 : at0) + (lane & 15);
      x.e = (lane < 32 ? p.k_exp : p.v_exp)[(int64_t)page * p.esp + (int64_t)t.h * p.esh + (int64_t)at * p.esn];
    }
    return;
  }
  int page = 0, at = 0;
  if (x.mask != 0u) {
    const int from = there ? lane : __builtin_ctz(x.mask);
    page = __shfl(entry, from, kWave);
    const int row = __shfl(mine, from, kWave);
    at = row - row / p.page * p.page;
  }
  const int64_t k_off = (int64_t)page * p.ksp + (int64_t)at * p.ksn, v_off = (int64_t)page * p.vsp + (int64_t)at * p.vsn;
  auto of_slot = [&](int64_t off, int slot) __attribute__((always_inline)) {
    const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)off, slot, kWave), hi = (uint32_t)__shfl((int)(uint32_t)((uint64_t)off >> 32), slot, kWave);
    return (int64_t)(((uint64_t)hi << 32) | lo);
  };
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint8_t* k = Kh + of_slot(k_off, 16 * i + c) + 16 * g;
#pragma unroll
    for (int j = 0; j < x.kK; ++j) x.k[i][j] = *reinterpret_cast<const uint4*>(k + 64 * j);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) load_piece(x.v[e], Vh + of_slot(v_off, 16 * (e >> 2) + 4 * g + (e & 3)) + c * kPiece);
  if constexpr (QUANT) x.e = (lane < 32 ? p.k_exp : p.v_exp)[(int64_t)page * p.esp + (int64_t)t.h * p.esh + (int64_t)at * p.esn];
}

// Query rows of tile n of a unit: lane (c, g) has row 16 n + c in the order of the K rows' pieces, zeros past the unit's rows
template <int D, bool QUANT>
__device__ __forceinline__ void load_queries(bf16x8 (&q)[D / 32], const PagedAttn& p, const Tile& t, int at, int lane) {
  const int g = lane >> 4, i = at / p.group;
  const bool there = i < t.q.n;
  const int64_t row = t.q.first + (there ? i : 0);
  const uint16_t* src = p.Q + row * p.qsn + (int64_t)(t.h * p.group + (there ? at - i * p.group : 0)) * p.qsh + (QUANT ? 16 * g : 8 * g);
#pragma unroll
  for (int kk = 0; kk < D / 32; ++kk) {
    const uint4 v = *reinterpret_cast<const uint4*>(src + (QUANT ? 64 * (kk >> 1) + 8 * (kk & 1) : 32 * kk));
    q[kk] = as_bf16x8(there ? v : make_uint4(0u, 0u, 0u, 0u));
  }
}

// workgroups per compute unit, by the registers
static constexpr int groups_per_cu(int head_dim, int q_tiles) { return head_dim == 64 && q_tiles == 1 ? 3 : 2; }
template <int D, bool QUANT, int NT>
__global__ __launch_bounds__(256, groups_per_cu(D, NT)) void paged_attn_kernel(const PagedAttn p) {
  constexpr int kKS = D / 32, kCT = D / 16, kV = TileRows<D, QUANT>::kV, kVec = D / 64;
  __shared__ __attribute__((aligned(16))) float exps_sh[QUANT ? 4 : 1][64];
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int worker = (int)blockIdx.x * 4 + wave;

  const Prefix<NT> prefix(p, lane);
  const Shares shares((int64_t)prefix.total * p.H, p.workers);
  const int64_t begin = shares.begin(worker);
  const int n_tiles = (int)(shares.begin(worker + 1) - begin);
  if (n_tiles <= 0) return;

  Tile here;
  {
    uint32_t before;
    here.r = prefix.find(p, (uint32_t)((uint64_t)begin / (uint32_t)p.H), before, lane);
    here.q = load_request<NT>(p, here.r);
    const uint32_t local = (uint32_t)(begin - (int64_t)before * p.H), unit = local / (uint32_t)here.q.tiles;
    here.t = (int)(local - unit * (uint32_t)here.q.tiles);
    here.h = (int)(unit / (uint32_t)here.q.groups);
    here.qg = (int)unit - here.h * here.q.groups;
    here.first = true;
    here.last = here.t == here.q.tiles - 1 || n_tiles == 1;
  }
  // the tile behind `t`, the i-th of the wavefront
  auto advance = [&](Tile t, int i) __attribute__((always_inline)) {
    ++t.t;
    t.first = t.t >= t.q.tiles;
    if (t.first) {
      t.t = 0;
      ++t.qg;
      if (t.qg >= t.q.groups) {
        t.qg = 0;
        ++t.h;
        if (t.h >= p.H) {
          t.h = 0;
          do {  // requests without a row have no tile
            ++t.r;
            t.q = load_request<NT>(p, t.r);
          } while (t.q.n == 0);
        }
      }
    }
    t.last = t.t == t.q.tiles - 1 || i == n_tiles - 1;
    return t;
  };

  bf16x8 q[NT][kKS];
  int limit[NT];  // keys that the lane's row may attend to
  float m_run[NT], l_run[NT];
  floatx4 o[NT][kCT];

  auto begin_unit = [&](const Tile& t) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int at = (t.qg * NT + n) * 16 + c;
      load_queries<D, QUANT>(q[n], p, t, at, lane);
      limit[n] = t.q.len;
      if (p.causal) {
        const int i = min(at / p.group, max(t.q.n - 1, 0));
        const int position = p.b.positions ? p.b.positions[t.q.first + i] : max(p.b.seq_len[t.r], 0) - t.q.count + i;
        limit[n] = min(position, t.q.len - 1) + 1;
      }
      m_run[n] = -INFINITY;
      l_run[n] = 0.f;
#pragma unroll
      for (int ct = 0; ct < kCT; ++ct) o[n][ct] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
  };

  // operands of the second product for the columns 2 w and 2 w + 1 (codes: 4 w + i) of a lane's piece
  auto v_operand = [&](const uint32_t (&v)[8][kV], int w, int i) __attribute__((always_inline)) {
    uint32_t s[4];
    if constexpr (QUANT) {
#pragma unroll
      for (int m = 0; m < 4; ++m) s[m] = decode2(__builtin_amdgcn_perm(v[2 * m + 1][w], v[2 * m][w], i < 2 ? 0x05010400u : 0x07030602u), i & 1, 1.f);
    } else {
#pragma unroll
      for (int m = 0; m < 4; ++m) s[m] = __builtin_amdgcn_perm(v[2 * m + 1][w], v[2 * m][w], i == 0 ? 0x05040100u : 0x07060302u);
    }
    return make_uint4(s[0], s[1], s[2], s[3]);
  };
  constexpr int kPer = QUANT ? 4 : 2;  // columns a dword

  auto consume = [&](const TileRows<D, QUANT>& x, const Tile& t) __attribute__((always_inline)) {
    floatx4 acc[NT][2];
    floatx4 ek[2], ev[2];
    if constexpr (QUANT) exps_sh[wave][lane] = exp_value(x.e);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
      for (int n = 0; n < NT; ++n) acc[n][kt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < TileRows<D, QUANT>::kK; ++j) {
        const uint4 w = x.k[kt][j];
        if constexpr (QUANT) {
          const bf16x8 k0 = as_bf16x8(decode8(make_uint2(w.x, w.y), 1.f)), k1 = as_bf16x8(decode8(make_uint2(w.z, w.w), 1.f));
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            acc[n][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, q[n][2 * j], acc[n][kt], 0, 0, 0);
            acc[n][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, q[n][2 * j + 1], acc[n][kt], 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int n = 0; n < NT; ++n) acc[n][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(w), q[n][j], acc[n][kt], 0, 0, 0);
        }
      }
    }
    if constexpr (QUANT) {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      const float* es = exps_sh[wave];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        ek[i] = *reinterpret_cast<const floatx4*>(es + 16 * i + 4 * g);
        ev[i] = *reinterpret_cast<const floatx4*>(es + 32 + 16 * i + 4 * g);
      }
    }
    bf16x8 hi[NT], lo[NT];
    uint32_t seen[NT];
    bool apart = false;  // rows of the unit that see different keys
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if constexpr (QUANT) {
        acc[n][0] *= ek[0];
        acc[n][1] *= ek[1];
      }
      seen[n] = x.mask;
      if (p.causal) {
        seen[n] &= low_mask(limit[n] - t.t * kTile);
        apart |= seen[n] != x.mask;
      }
      float ps[8];
      const float alpha = softmax_step(acc[n], seen[n], g, p.scale_log2, m_run[n], l_run[n], ps);
      if (__ballot(alpha != 1.f) != 0ull) {
#pragma unroll
        for (int ct = 0; ct < kCT; ++ct) o[n][ct] *= alpha;
      }
      float rest[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (QUANT) ps[e] *= ev[e >> 2][e & 3];
      }
      hi[n] = pack_bf16x8(ps);
      const uint4 w = __builtin_bit_cast(uint4, hi[n]);
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) rest[e] = ps[e] - ((e & 1) ? bf16_hi(u[e >> 1]) : bf16_lo(u[e >> 1]));
      lo[n] = pack_bf16x8(rest);
    }
    // A key that some rows of the unit may not see has probability zero there, and zero times an infinity or a NaN of its V would still reach
    // them.  Where that can be, the products are those of the finite values, and what infinities and NaN do to the rows that see them is added.
    bool beyond = false;
    if (p.causal && __ballot(apart) != 0ull) {
      bool any = false;
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int w = 0; w < kV; ++w) {
          const uint32_t y = x.v[e][w];
          if constexpr (QUANT)
            any |= ((~y & 0x7fu) == 0u) | ((~y & 0x7f00u) == 0u) | ((~y & 0x7f0000u) == 0u) | ((~y & 0x7f000000u) == 0u);
          else
            any |= ((~y & 0x7f80u) == 0u) | ((~y & 0x7f800000u) == 0u);
        }
      beyond = __ballot(any) != 0ull;
    }
    if (!beyond) {
#pragma unroll
      for (int w = 0; w < kV; ++w)
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const bf16x8 v = as_bf16x8(v_operand(x.v, w, i));
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            o[n][kPer * w + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, hi[n], o[n][kPer * w + i], 0, 0, 0);
            o[n][kPer * w + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, lo[n], o[n][kPer * w + i], 0, 0, 0);
          }
        }
    } else {
      bf16x8 sees[NT];  // one where the row may attend to the key
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        uint32_t u[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const uint32_t two = seen[n] >> (16 * (m >> 1) + 4 * g + 2 * (m & 1));
          u[m] = ((two & 1u) ? 0x3f80u : 0u) | ((two & 2u) ? 0x3f800000u : 0u);
        }
        sees[n] = as_bf16x8(make_uint4(u[0], u[1], u[2], u[3]));
      }
#pragma unroll
      for (int w = 0; w < kV; ++w)
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const uint4 v = v_operand(x.v, w, i);
          const uint32_t u[4] = {v.x, v.y, v.z, v.w};
          uint32_t finite[4], above[4], below[4];  // the value or 0; one where it is +inf or NaN; one where it is -inf or NaN
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            finite[m] = above[m] = below[m] = 0u;
#pragma unroll
            for (int half = 0; half < 32; half += 16) {
              const uint32_t y = (u[m] >> half) & 0xffffu, size = y & 0x7fffu;
              finite[m] |= size < 0x7f80u ? y << half : 0u;
              above[m] |= size > 0x7f80u || y == 0x7f80u ? 0x3f80u << half : 0u;
              below[m] |= size > 0x7f80u || y == 0xff80u ? 0x3f80u << half : 0u;
            }
          }
          const bf16x8 f = as_bf16x8(make_uint4(finite[0], finite[1], finite[2], finite[3]));
          const bf16x8 up = as_bf16x8(make_uint4(above[0], above[1], above[2], above[3]));
          const bf16x8 down = as_bf16x8(make_uint4(below[0], below[1], below[2], below[3]));
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            floatx4& y = o[n][kPer * w + i];
            y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, hi[n], y, 0, 0, 0);
            y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, lo[n], y, 0, 0, 0);
            const floatx4 none = {0.f, 0.f, 0.f, 0.f};
            const floatx4 more = __builtin_amdgcn_mfma_f32_16x16x32_bf16(up, sees[n], none, 0, 0, 0);
            const floatx4 less = __builtin_amdgcn_mfma_f32_16x16x32_bf16(down, sees[n], none, 0, 0, 0);
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] += (more[k] > 0.f ? INFINITY : 0.f) + (less[k] > 0.f ? -INFINITY : 0.f);
          }
        }
    }
    if constexpr (QUANT) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the next tile's exponents follow these reads
  };

  // `t`: the last tile of the piece, which began with tile `start` of the unit.  Lane (c, g) has the columns (4 g + i) * D / 16 + ct of row c.
  auto end_piece = [&](const Tile& t, int start) __attribute__((always_inline)) {
    const bool whole = start == 0 && t.t == t.q.tiles - 1;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int at = (t.qg * NT + n) * 16 + c, i = at / p.group, head = t.h * p.group + at - i * p.group;
      if (i >= t.q.n) continue;
      if (whole) {
        const float inv = l_run[n] == 0.f ? 0.f : 1.f / l_run[n];
        uint16_t* dst = p.out + (int64_t)(t.q.first + i) * p.osn + (int64_t)head * p.osh;
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          uint32_t w[kCT / 2];
#pragma unroll
          for (int ct = 0; ct < kCT; ct += 2) w[ct / 2] = cvt_pk_bf16(o[n][ct][m] * inv, o[n][ct + 1][m] * inv);
          if constexpr (D == 128)
            *reinterpret_cast<uint4*>(dst + (4 * g + m) * kCT) = make_uint4(w[0], w[1], w[2], w[3]);
          else
            *reinterpret_cast<uint2*>(dst + (4 * g + m) * kCT) = make_uint2(w[0], w[1]);
        }
        if (p.lse && g == 0)
          p.lse[(int64_t)(t.q.first + i) * (p.H * p.group) + head] = l_run[n] == 0.f ? -INFINITY : (m_run[n] + __builtin_amdgcn_logf(l_run[n])) * kLn2;
      } else {
        const int64_t row = (int64_t)(2 * worker + (start == 0)) * p.unit_rows + 16 * n + c;
        float* dst = p.part_o + row * D;
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
          for (int v = 0; v < kVec; ++v)
            *reinterpret_cast<floatx4*>(dst + (4 * g + m) * kCT + 4 * v) = floatx4{o[n][4 * v][m], o[n][4 * v + 1][m], o[n][4 * v + 2][m], o[n][4 * v + 3][m]};
        if (g == 0) p.part_ml[row] = make_float2(m_run[n], l_run[n]);
      }
    }
  };

  int start = 0, entry = load_entry(p, here, lane);
#pragma unroll 1
  for (int i = 0; i < n_tiles; ++i) {
    if (here.first) {
      start = here.t;
      begin_unit(here);
    }
    TileRows<D, QUANT> x;
    load_tile_rows<D, QUANT>(x, p, here, entry, lane);
    Tile next = here;
    if (i + 1 < n_tiles) {
      next = advance(here, i + 1);
      entry = load_entry(p, next, lane);  // travels with the rows
    }
    __builtin_amdgcn_sched_barrier(0);
    if (x.mask != 0u) consume(x, here);
    if (here.last) end_piece(here, start);
    here = next;
  }
}

// Joins the pieces of the units that several wavefronts worked on: NW wavefronts for one row of one query head.  The wavefront that had tile s of all
// tiles follows from s alone, and with it where the pieces lie.
template <int D, int NT, int NW>
__global__ __launch_bounds__(256) void paged_join_kernel(const PagedAttn p) {
  constexpr int kVec = D / 64, kAhead = 8;
  __shared__ float2 ml_sh[NW];
  __shared__ float o_sh[NW][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int Hq = p.H * p.group;
  const int64_t at = NW == 1 ? (int64_t)list_index() * 4 + wave : (int64_t)list_index();
  const int64_t row_at = at / Hq;
  const int head = (int)(at - row_at * Hq);
  const int r = (int)(row_at / p.b.max_rows), i = (int)(row_at - (int64_t)r * p.b.max_rows);
  if (r >= p.b.n_req) return;  // (the same in the whole workgroup where it has a barrier)
  const Prefix<NT> prefix(p, lane);
  const Request q = load_request<NT>(p, r);
  if (i >= q.n) return;
  const int h = head / p.group, unit_row = i * p.group + head - h * p.group, qg = unit_row / (16 * NT), in_unit = unit_row - qg * 16 * NT;
  const Shares shares((int64_t)prefix.total * p.H, p.workers);
  const int64_t s = (int64_t)prefix.before(p, r, lane) * p.H + ((int64_t)h * q.groups + qg) * q.tiles;
  const int w0 = shares.of(s), w1 = shares.of(s + q.tiles - 1);
  if (w0 == w1) return;
  const int n = w1 - w0 + 1;  // (some of them may have no tile)
  float m_run = -INFINITY, l_run = 0.f, o[kVec];
#pragma unroll
  for (int v = 0; v < kVec; ++v) o[v] = 0.f;
  for (int j0 = NW == 1 ? 0 : wave * kWave; j0 < n; j0 += NW * kWave) {
    const int j = j0 + lane, w = w0 + j;
    float2 ml = make_float2(-INFINITY, 0.f);
    const int64_t row = (int64_t)(2 * w + (j == 0)) * p.unit_rows + in_unit;
    if (j < n && shares.begin(w) < shares.begin(w + 1)) ml = p.part_ml[row];
    float top = ml.x;
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor(top, k, kWave));
    const float m_new = fmaxf(m_run, top), m_use = m_new == -INFINITY ? 0.f : m_new;
    const float f = ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - m_use), old = __builtin_amdgcn_exp2f(m_run - m_use);
    l_run = l_run * old + wave_sum(f * ml.y);
#pragma unroll
    for (int v = 0; v < kVec; ++v) o[v] *= old;
    m_run = m_new;
    const unsigned long long some = __ballot(ml.y != 0.f);
    const int n_here = min(n - j0, kWave);
    for (int k0 = 0; k0 < n_here; k0 += kAhead) {
      float y[kAhead][kVec];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
#pragma unroll
        for (int v = 0; v < kVec; ++v) y[k][v] = 0.f;
        if (k0 + k < n_here && ((some >> (k0 + k)) & 1ull)) {
          const float* src = p.part_o + ((int64_t)(2 * (w0 + j0 + k0 + k) + (j0 + k0 + k == 0)) * p.unit_rows + in_unit) * D + lane * kVec;
          if constexpr (kVec == 2) {
            const float2 t = *reinterpret_cast<const float2*>(src);
            y[k][0] = t.x;
            y[k][1] = t.y;
          } else {
            y[k][0] = *src;
          }
        }
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const float w = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), (k0 + k) & 63));
        if (k0 + k < n_here && ((some >> (k0 + k)) & 1ull)) {
#pragma unroll
          for (int v = 0; v < kVec; ++v) o[v] += w * y[k][v];
        }
      }
    }
  }
  if constexpr (NW > 1) {
    if (lane == 0) ml_sh[wave] = make_float2(m_run, l_run);
#pragma unroll
    for (int v = 0; v < kVec; ++v) o_sh[wave][lane * kVec + v] = o[v];
    __syncthreads();
    if (wave != 0) return;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, ml_sh[w].x);
    const float m_use = top == -INFINITY ? 0.f : top;
    m_run = top;
    l_run = 0.f;
#pragma unroll
    for (int v = 0; v < kVec; ++v) o[v] = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float2 ml = ml_sh[w];
      const float f = ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - m_use);
      l_run += f * ml.y;
#pragma unroll
      for (int v = 0; v < kVec; ++v) o[v] += f * o_sh[w][lane * kVec + v];
    }
  }
  const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
  uint16_t* dst = p.out + (int64_t)(q.first + i) * p.osn + (int64_t)head * p.osh + lane * kVec;
  if constexpr (kVec == 2)
    *reinterpret_cast<uint32_t*>(dst) = cvt_pk_bf16(o[0] * inv, o[1] * inv);
  else
    *dst = (uint16_t)cvt_pk_bf16(o[0] * inv, 0.f);
  if (p.lse && lane == 0) p.lse[(int64_t)(q.first + i) * Hq + head] = l_run == 0.f ? -INFINITY : (m_run + __builtin_amdgcn_logf(l_run)) * kLn2;
}

// Wavefronts: as many as are resident at once, and no more than the batch may have tiles.
constexpr int kPagedGroups = 256;  // compute units
PagedPlan plan_paged_attn(int n_heads, int group, int head_dim, const PagedBatch& b, int page) {
  PagedPlan p;
  const int64_t rows = (int64_t)b.max_rows * group;
  p.q_tiles = rows <= 16 ? 1 : 2;
  p.unit_rows = (int)std::min<int64_t>(rows, 16 * p.q_tiles);
  const int64_t tiles = ceil_div64((int64_t)b.table_width * page, kTile), units = ceil_div64(rows, 16 * p.q_tiles) * n_heads;
  const int64_t most = tiles * units >= (int64_t(1) << 31) ? int64_t(1) << 31 : tiles * units * b.n_req;
  p.workers = (int)std::min<int64_t>((int64_t)kPagedGroups * kWavesPerGroup * groups_per_cu(head_dim, p.q_tiles), ceil_div64(most, kWavesPerGroup) * kWavesPerGroup);
  const size_t slots = (size_t)2 * p.workers;
  p.part_ml = (slots * p.unit_rows * head_dim * sizeof(float) + 255) & ~(size_t)255;
  p.total = p.part_ml + slots * p.unit_rows * sizeof(float2);
  return p;
}

// Few rows: four wavefronts for each, so that all its pieces are requested at once.
constexpr int kJoinGroups = 1024;
template <int D, int NT>
static hipError_t launch_paged_t(const PagedAttn& a, const PagedPlan& p, hipStream_t st) {
  const int groups = p.workers / kWavesPerGroup;
  if (a.k_exp != nullptr)
    hipLaunchKernelGGL((paged_attn_kernel<D, true, NT>), dim3(groups), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((paged_attn_kernel<D, false, NT>), dim3(groups), dim3(256), 0, st, a);
  if ((int64_t)a.b.table_width * a.page <= kTile) return hipGetLastError();  // no unit has two tiles
  const int64_t rows = (int64_t)a.b.n_req * a.b.max_rows * a.H * a.group;
  if (rows <= kJoinGroups)
    hipLaunchKernelGGL((paged_join_kernel<D, NT, 4>), grid_list(rows), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((paged_join_kernel<D, NT, 1>), grid_list(ceil_div64(rows, 4)), dim3(256), 0, st, a);
  return hipGetLastError();
}
hipError_t launch_paged_attn(const PagedAttn& a, const PagedPlan& p, int head_dim, hipStream_t st) {
  if (head_dim == 128) return p.q_tiles == 1 ? launch_paged_t<128, 1>(a, p, st) : launch_paged_t<128, 2>(a, p, st);
  return p.q_tiles == 1 ? launch_paged_t<64, 1>(a, p, st) : launch_paged_t<64, 2>(a, p, st);
}

}  // namespace focus
