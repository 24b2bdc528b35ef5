// Attention of the requests' few new rows over their pages.
//
// The keys of a request are cut into tiles of 32, and a unit is what shares them: the rows of a request times the query heads of one K/V head, sixteen
// (or 32) of those at a time.  All tiles of all units, in the order request, heads, group of rows, tile, are divided evenly among the wavefronts
// of one launch, by the lengths that they find in memory: a batch of one long and many short requests keeps the whole chip busy, and a captured graph
// does so for lengths that nobody knew when it was captured.  A wavefront keeps the running softmax of the unit that it is in; a unit that
// lies within one wavefront is written out by it, the pieces of the others go to the workspace, and a second launch joins them.  The wavefronts of
// a workgroup take neighbouring heads of the same tiles: where the heads of a row lie side by side their rows are then fetched at about the same time.
//
// Products, from tiles of 32 rows that lie in LDS (Ring):
//   S^T = K Q^T   v_mfma_f32_16x16x32_bf16, lane (c, g) with 16 bytes at a time of the rows c and 16 + c
//   O^T = V^T P^T bf16: column tile ct has the columns 16 ct + c, by transposed reads; codes: c * D / 16 + ct, D / 16 neighbouring codes of each of the
//                 rows 4 g + i and 16 + 4 g + i, of which byte permutations put those of two rows next to each other
// P is split into two bf16 numbers, p = hi + lo to 2^-17, and multiplied twice: rounded to one it would cost the result as much
// again as its own rounding.  Of few query rows a tile is 16 KB from memory and 24 products, and the matrix unit has nothing else to do; of many, where the
// products count, it is a third of them.
//
// What bounds it is HBM, every row read once: one request of 32 832 rows, 32 heads, 538 MB, in 84 us = 6.4 TB/s and 4.7 for the join; 64 of up to
// 16 384 rows with 7 query heads on each of 4, 869 MB, in 136 and 6; eight-bit rows, 227 MB for 37 requests with 16 rows a unit, in 58 and 6: some 8 us are the
// start, 8 the pieces of 16 rows each (16 KB a wavefront), and half as many bytes a tile leave the instructions half the time.  A thousand
// rows of four heads: 5.9 + 3.9 us, dependent round trips (lengths, table, rows, products; pieces).  Many query rows of a K/V head are far from their bounds: each
// 32 of them read all rows of the request again, those that causal limits hide from all 32 among them (64 rows of 4 query heads on each of 8, 32 requests of
// 2048: 268 MB and 69 GFLOP, either 55 us, in 312 to 334, causal or not).
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
  x.tiles = max((int)(((uint32_t)x.len + kTile - 1) / kTile), 1);  // (len up to 2^31 - 1)
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
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)wave_reduce_u32(x, [](uint32_t a, uint32_t b) { return a + b; }));
}
// a number that is the same in all lanes, in a scalar register: what follows from it is worked out once a wavefront
__device__ __forceinline__ int same(int x) { return __builtin_amdgcn_readfirstlane(x); }

// sum of x over the lanes up to this one
__device__ __forceinline__ uint32_t wave_scan(uint32_t x, int lane) {
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, true);  // row_shr 1, 2, 4, 8: within sixteen lanes
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, true);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, true);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, true);
  const uint32_t a = (uint32_t)__builtin_amdgcn_readlane((int)x, 15), b = (uint32_t)__builtin_amdgcn_readlane((int)x, 31), c = (uint32_t)__builtin_amdgcn_readlane((int)x, 47);
  return x + (lane >= 16 ? a : 0u) + (lane >= 32 ? b : 0u) + (lane >= 48 ? c : 0u);
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
    const uint32_t incl = wave_scan(mine, lane);
    const int at = __builtin_ctzll(__ballot(done + incl > t) | (1ull << 63));
    before = done + (uint32_t)__builtin_amdgcn_readlane((int)(incl - mine), at);
    return r0 + at;
  }
};

// The tiles of all requests, R < 2^31 of them, among W bundles of wavefronts: floor(i R / W) is the first one of the i-th.  In 64-bit floating point, where
// products are exact and quotients are moved off the whole numbers by half of the least distance from them (a division of integers is as
// long as a round trip to L2).
struct Shares {
  double R, workers, per_worker;
  __device__ __forceinline__ Shares(uint32_t tiles, int W, double reciprocal) : R((double)tiles), workers((double)W), per_worker(reciprocal) {}
  __device__ __forceinline__ int begin(int i) const { return (int)((R * (double)i + 0.5) * per_worker); }
  // the last one that begins with tile s or before it: floor(((s + 1) W - 1) / R)
  __device__ __forceinline__ int of(int s) const { return (int)(((double)(s + 1) * workers - 0.5) / R); }
};

// A group of rows of a request and a bundle of K/V heads, one a wavefront
struct Unit {
  Request q;
  int r, b, qg;
};

// The rows of a tile lie in LDS between memory and the products: every wavefront has a ring of its own, 16 KB of rows (one tile of 128 bf16
// columns, two of codes), whose loads go to LDS directly and are waited for by their number; K's place is asked for again while V is worked on.  Two workgroups
// a compute unit hide each other's joints.  32 heads, 32 832 keys: 83 us; the same bytes under way in registers 91.5, and spills with 32 query rows.  Rings of
// 32 KB and one workgroup: eight-bit rows 94 to 101 us instead of 64 to 73.
template <int D, bool QUANT>
struct Ring {
  static constexpr int kRow = QUANT ? D : 2 * D, kRows = kTile * kRow;  // bytes of a row, of a tile's K (or V)
  static constexpr int kChunks = kRow / 16, kPerLoad = 64 / kChunks, kLoads = kTile / kPerLoad;
  static constexpr int kDepth = 8192 / kRows;  // tiles
  static constexpr int kExps = QUANT ? 256 : 0;  // an exponent a row, in 32 bits: of K, of V
  static constexpr int kStage = 2 * kRows + kExps, kTileLoads = 2 * kLoads + (QUANT ? 1 : 0);
  static constexpr int kBytes = kDepth * kStage;
  // chunk `x` of a row lies at place x ^ turn(row): reads of one chunk of several rows meet different banks
  static __device__ __forceinline__ int turn(int row) { return kRow == 64 ? (row >> 1) & 3 : row & (kChunks - 1); }
};
typedef const __attribute__((address_space(1))) void* gptr_t;
typedef __attribute__((address_space(3))) void* lptr_t;

// Pages as a wavefront holds them: lane l has entry `first` + l of request r's table.
struct Window {
  int r, first, entry;
};
// Where the rows of a tile lie.  Slots without a key take another row of the tile, all of them row 0 of page 0 where it has none (what
// is read there is not used, but zero times an infinity would be).
struct TilePlace {
  uint32_t mask;  // bit s: slot s holds a key
  bool plain;     // every slot does, and sixteen rows lie in one page: page0, at0 and page1, at1; else page and at of slot lane % 32
  int page0, at0, page1, at1, page, at;
};
__device__ __forceinline__ TilePlace locate(const PagedAttn& p, const Unit& u, int t, Window& win, int lane) {
  TilePlace x;
  x.page = x.at = x.page0 = x.page1 = x.at0 = x.at1 = 0;
  x.mask = 0u;
  x.plain = false;
  const int row0 = t * kTile, n = min(u.q.len - row0, kTile);
  if (n <= 0) return x;
  auto entry_of = [&](int row) __attribute__((always_inline)) { return p.page_shift >= 0 ? row >> p.page_shift : row / p.page; };
  const int e0 = entry_of(row0), e_last = entry_of(row0 + n - 1);
  if (u.r != win.r || e0 < win.first || e_last >= win.first + kWave) {
    win.r = u.r;
    win.first = e0;
    win.entry = p.b.page_table[(int64_t)u.r * p.b.table_stride + min(e0 + lane, p.b.table_width - 1)];
  }
  if (n == kTile && (p.page & 15) == 0) {
    const int e1 = entry_of(row0 + 16);
    x.page0 = __builtin_amdgcn_readlane(win.entry, e0 - win.first);
    x.page1 = __builtin_amdgcn_readlane(win.entry, e1 - win.first);
    x.at0 = row0 - e0 * p.page;
    x.at1 = row0 + 16 - e1 * p.page;
    if ((uint32_t)x.page0 < (uint32_t)p.n_pages && (uint32_t)x.page1 < (uint32_t)p.n_pages) {
      x.plain = true;
      x.mask = 0xffffffffu;
      return x;
    }
  }
  const int row = row0 + min(lane & 31, n - 1), e = entry_of(row);
  const int entry = __shfl(win.entry, e - win.first, kWave), at = row - e * p.page;
  const bool there = (lane & 31) < n && entry >= 0 && entry < p.n_pages;
  x.mask = (uint32_t)__ballot(there);  // (the upper half of the wavefront repeats the lower one)
  if (x.mask != 0u) {
    const int from = there ? lane : __builtin_ctz(x.mask);
    x.page = __shfl(entry, from, kWave);
    x.at = __shfl(at, from, kWave);
  }
  return x;
}
__device__ __forceinline__ int64_t offset_of_slot(int64_t off, int slot) {
  const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)off, slot, kWave), hi = (uint32_t)__shfl((int)(uint32_t)((uint64_t)off >> 32), slot, kWave);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}
// The rows of a tile to `stage`.  Lane l of load i supplies the 16 bytes that land at stage + 1024 i + 16 l: place l mod kChunks of row
// i * kPerLoad + l / kChunks.
template <int D, bool QUANT, int POLICY>
__device__ __forceinline__ void request_rows_as(const uint8_t* base, int64_t stride_p, int64_t stride_n, TilePlace x, char* stage, int lane) {
  using G = Ring<D, QUANT>;
  const int sub = lane / G::kChunks, pos = lane % G::kChunks;
  if (x.plain) {
    const uint8_t* rows[2] = {base + (int64_t)x.page0 * stride_p + (int64_t)x.at0 * stride_n, base + (int64_t)x.page1 * stride_p + (int64_t)x.at1 * stride_n};
    const uint32_t lane_row = (uint32_t)sub * (uint32_t)stride_n;  // (16 rows of the stride fit 32 bits)
#pragma unroll
    for (int i = 0; i < G::kLoads; ++i) {
      const int slot = i * G::kPerLoad + sub, first = i * G::kPerLoad;
      const uint8_t* src = rows[first >> 4] + (int64_t)(first & 15) * stride_n + (lane_row + (uint32_t)((pos ^ G::turn(slot)) << 4));
      __builtin_amdgcn_global_load_lds((gptr_t)src, (lptr_t)(stage + i * 1024), 16, 0, POLICY);
    }
    return;
  }
  const int64_t mine = (int64_t)x.page * stride_p + (int64_t)x.at * stride_n;
#pragma unroll
  for (int i = 0; i < G::kLoads; ++i) {
    const int slot = i * G::kPerLoad + sub;
    const uint8_t* src = base + offset_of_slot(mine, slot) + ((pos ^ G::turn(slot)) << 4);
    __builtin_amdgcn_global_load_lds((gptr_t)src, (lptr_t)(stage + i * 1024), 16, 0, POLICY);
  }
}
// Past the caches, unless several groups of query rows read the same bf16 rows: 25 rows of 7 query heads on each of 4, 16 requests of 4096 120 us past them, 98 through
// them (causal 122 and 100), 64 of 4 on each of 8, 32 requests of 2048 358 and 334; one group (64 requests, 7 on each of 4) 139 and 159, eight-bit rows (37 requests) 64
// and 69; eight-bit rows of several groups (the 25 rows of 7, causal) 112 and 107
template <int D, bool QUANT, int NT>
__device__ __forceinline__ void request_rows(const PagedAttn& p, const uint8_t* base, int64_t stride_p, int64_t stride_n, TilePlace x, char* stage, int lane) {
  if (!QUANT && NT > 1 && p.most_groups > 1)
    request_rows_as<D, QUANT, 0>(base, stride_p, stride_n, x, stage, lane);
  else
    request_rows_as<D, QUANT, kStreamPolicy>(base, stride_p, stride_n, x, stage, lane);
}
// exponents of slot lane % 32, of K in the lower half of the wavefront, of V in the upper
__device__ __forceinline__ void request_exponents(const PagedAttn& p, TilePlace x, int h, char* stage, int lane) {
  const int page = x.plain ? ((lane & 16) ? x.page1 : x.page0) : x.page, at = x.plain ? ((lane & 16) ? x.at1 : x.at0) + (lane & 15) : x.at;
  const uint8_t* src = (lane < 32 ? p.k_exp : p.v_exp) + (int64_t)page * p.esp + (int64_t)h * p.esh + (int64_t)at * p.esn;
  __builtin_amdgcn_global_load_lds((gptr_t)src, (lptr_t)stage, 1, 0, 0);
}

// Operands from a stage, outside the compiler's sight and complete on return (read_k_operands16): it would wait for every load to LDS.
// K codes: lane (c, g) has the chunks 4 j + g of the rows c and 16 + c
template <int D>
__device__ __forceinline__ void read_k_codes(uint4 (&k)[2][D / 64], const char* stage, int lane) {
  using G = Ring<D, true>;
  const int c = lane & 15, g = lane >> 4;
  const uint32_t a = lds_address(stage) + c * G::kRow + ((g ^ G::turn(c)) << 4);
  uintx4 x[2][D / 64];
  if constexpr (D == 128)
    asm volatile(
        "ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %4 offset:2048\n\tds_read_b128 %3, %5 offset:2048\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1])
        : "v"(a), "v"(a ^ 64u)
        : "memory");
  else
    asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %2 offset:1024\n\ts_waitcnt lgkmcnt(0)" : "=&v"(x[0][0]), "=&v"(x[1][0]) : "v"(a) : "memory");
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < D / 64; ++j) k[i][j] = __builtin_bit_cast(uint4, x[i][j]);
}
// V codes: lane (c, g) has D / 16 neighbouring codes, the c-th of a row, of the rows 4 g + e and 16 + 4 g + e
template <int D>
__device__ __forceinline__ void read_v_codes(uint32_t (&v)[8][D / 64], const char* stage, int lane) {
  using G = Ring<D, true>;
  const int c = lane & 15, g = lane >> 4;
  if constexpr (D == 128) {  // turn(4 g + e) = 4 (g mod 2) ^ e
    const uint32_t a = lds_address(stage) + 4 * g * G::kRow + (((c >> 1) ^ (4 * (g & 1))) << 4) + (c & 1) * 8;
    uintx2 x[8];
    asm volatile(
        "ds_read_b64 %0, %8\n\tds_read_b64 %1, %9 offset:128\n\tds_read_b64 %2, %10 offset:256\n\tds_read_b64 %3, %11 offset:384\n\t"
        "ds_read_b64 %4, %8 offset:2048\n\tds_read_b64 %5, %9 offset:2176\n\tds_read_b64 %6, %10 offset:2304\n\tds_read_b64 %7, %11 offset:2432\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
        : "v"(a), "v"(a ^ 16u), "v"(a ^ 32u), "v"(a ^ 48u)
        : "memory");
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e][0] = x[e].x;
      v[e][1] = x[e].y;
    }
  } else {  // turn(4 g + e) = 2 (g mod 2) ^ e / 2
    const uint32_t a = lds_address(stage) + 4 * g * G::kRow + (((c >> 2) ^ (2 * (g & 1))) << 4) + (c & 3) * 4;
    asm volatile(
        "ds_read_b32 %0, %8\n\tds_read_b32 %1, %8 offset:64\n\tds_read_b32 %2, %9 offset:128\n\tds_read_b32 %3, %9 offset:192\n\t"
        "ds_read_b32 %4, %8 offset:1024\n\tds_read_b32 %5, %8 offset:1088\n\tds_read_b32 %6, %9 offset:1152\n\tds_read_b32 %7, %9 offset:1216\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(v[0][0]), "=&v"(v[1][0]), "=&v"(v[2][0]), "=&v"(v[3][0]), "=&v"(v[4][0]), "=&v"(v[5][0]), "=&v"(v[6][0]), "=&v"(v[7][0])
        : "v"(a), "v"(a ^ 16u)
        : "memory");
  }
}
// 2^E of the rows 4 g + i and 16 + 4 g + i, of K and of V.  A byte of 255, which rows that nobody has written may hold, is an infinity: logits of such rows
// are masked afterwards, but a probability of zero times it would be NaN.
__device__ __forceinline__ void read_exponents(floatx4 (&ek)[2], floatx4 (&ev)[2], const char* stage, int lane) {
  const uint32_t a = lds_address(stage) + 16 * (lane >> 4);
  uintx4 x[4];
  asm volatile(
      "ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:64\n\tds_read_b128 %2, %4 offset:128\n\tds_read_b128 %3, %4 offset:192\n\ts_waitcnt lgkmcnt(0)"
      : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3])
      : "v"(a)
      : "memory");
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      ek[i][e] = exp_value(x[i][e]);
      ev[i][e] = exp_value(min(x[2 + i][e], 254u));
    }
}

// Of a pair of bf16 numbers: the finite ones, zero for the others (which = 0), or one where +inf (which = 2) or -inf (1) or a NaN is, zero elsewhere
__device__ __forceinline__ uint32_t sorted_out(uint32_t w, int which) {
  auto one = [&](uint32_t z) __attribute__((always_inline)) {
    const uint32_t size = z & 0x7fffu;
    if (which == 0) return size < 0x7f80u ? z : 0u;
    return size > 0x7f80u || z == (which == 2 ? 0x7f80u : 0xff80u) ? 0x3f80u : 0u;
  };
  return one(w & 0xffffu) | one(w >> 16) << 16;
}

// Query rows of tile n of a unit: lane (c, g) has row 16 n + c in the order of the K rows' pieces, zeros past the unit's rows
template <int D, bool QUANT>
__device__ __forceinline__ void load_queries(bf16x8 (&q)[D / 32], const PagedAttn& p, const Unit& t, int h, int at, int lane) {
  const int g = lane >> 4, i = at / p.group;
  const bool there = i < t.q.n;
  const int64_t row = t.q.first + (there ? i : 0);
  const uint16_t* src = p.Q + row * p.qsn + (int64_t)(h * p.group + (there ? at - i * p.group : 0)) * p.qsh + (QUANT ? 16 * g : 8 * g);
#pragma unroll
  for (int kk = 0; kk < D / 32; ++kk) {
    const uint4 v = *reinterpret_cast<const uint4*>(src + (QUANT ? 64 * (kk >> 1) + 8 * (kk & 1) : 32 * kk));
    q[kk] = as_bf16x8(there ? v : make_uint4(0u, 0u, 0u, 0u));
  }
}

// What a wavefront has of N operands of sixteen query rows: lane (c, g) of row c
template <int D, int N>
struct QueryRows {
  static constexpr int kN = N;
  bf16x8 q[N][D / 32];
  int limit[N];  // keys that the lane's row may attend to
  float m[N], l[N];
  floatx4 o[N][D / 16];  // of query row 16 n + c four columns of column tile ct, see end_piece
};

template <int D, bool QUANT, bool CAUSAL, int NT>
__global__ __launch_bounds__(256, 2) void paged_attn_kernel(const PagedAttn p) {
  using G = Ring<D, QUANT>;
  constexpr int kKS = D / 32, kCT = D / 16, kDepth = G::kDepth;
  __shared__ __attribute__((aligned(256))) char ring_sh[kWavesPerGroup * G::kBytes];
  int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int in_bundle = wave & ((1 << p.log_bundle) - 1), bundles = p.H >> p.log_bundle;
  const int wave_id = (int)blockIdx.x * kWavesPerGroup + wave, worker = wave_id >> p.log_bundle;
  char* ring = ring_sh + wave * G::kBytes;

  const Prefix<NT> prefix(p, lane);
  const Shares shares(prefix.total * (uint32_t)bundles, p.workers, p.per_worker);
  const int begin = same(shares.begin(worker)), n_tiles = same(shares.begin(worker + 1)) - begin;
  if (n_tiles <= 0) {  // (its pieces count for nothing where the units of its neighbours are joined)
    for (int i = lane; i < p.unit_rows; i += kWave) p.part_ml[(int64_t)2 * wave_id * p.unit_rows + i] = make_float2(-INFINITY, 0.f);
    return;
  }

  Unit u;  // of the tile that is worked on,
  int t;
  {
    uint32_t before;
    u.r = prefix.find(p, (uint32_t)same((int)(((double)begin + 0.5) * p.per_bundle)), before, lane);  // begin / bundles
    u.q = load_request<NT>(p, u.r);
    const uint32_t local = (uint32_t)begin - before * (uint32_t)bundles, unit = local / (uint32_t)u.q.tiles;
    t = (int)(local - unit * (uint32_t)u.q.tiles);
    u.b = (int)(unit / (uint32_t)u.q.groups);
    u.qg = (int)unit - u.b * u.q.groups;
  }
  Unit ahead = u;  // and of the one to be requested next
  int t_ahead = t, asked = 0;
  auto next_unit = [&](Unit& x) __attribute__((always_inline)) {
    if (++x.qg < x.q.groups) return;
    x.qg = 0;
    if (++x.b < bundles) return;
    x.b = 0;
    do {  // requests without a row have no tile
      ++x.r;
      x.q = load_request<NT>(p, x.r);
    } while (x.q.n == 0);
  };
  Window window{-1, 0, 0};
  TilePlace place;
  int masks = 0;  // lane l: the mask of the tile in stage l
  auto stage_of = [&](int i) __attribute__((always_inline)) { return ring + (i & (kDepth - 1)) * G::kStage; };
  auto head_of = [&](const Unit& x) __attribute__((always_inline)) { return (x.b << p.log_bundle) + in_bundle; };
  auto request_k = [&]() __attribute__((always_inline)) {
    place = locate(p, ahead, t_ahead, window, lane);
    char* stage = stage_of(asked);
    if constexpr (QUANT) request_exponents(p, place, head_of(ahead), stage + 2 * G::kRows, lane);
    request_rows<D, QUANT, NT>(p, p.K + (int64_t)head_of(ahead) * p.ksh, p.ksp, p.ksn, place, stage, lane);
    masks = lane == (asked & (kDepth - 1)) ? (int)place.mask : masks;
  };
  auto request_v = [&]() __attribute__((always_inline)) {
    request_rows<D, QUANT, NT>(p, p.V + (int64_t)head_of(ahead) * p.vsh, p.vsp, p.vsn, place, stage_of(asked) + G::kRows, lane);
    ++asked;
    if (++t_ahead >= ahead.q.tiles && asked < n_tiles) {
      t_ahead = 0;
      next_unit(ahead);
    }
  };
  // w: the rows of operand n0 on
  auto begin_unit = [&](auto& w, int n0) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < w.kN; ++n) {
      const int at = (u.qg * NT + n0 + n) * 16 + c;
      load_queries<D, QUANT>(w.q[n], p, u, head_of(u), at, lane);
      w.limit[n] = u.q.len;
      if constexpr (CAUSAL) {
        const int i = min(at / p.group, max(u.q.n - 1, 0));
        const int position = p.b.positions ? p.b.positions[u.q.first + i] : max(p.b.seq_len[u.r], 0) - u.q.count + i;
        w.limit[n] = min(position, u.q.len - 1) + 1;
      }
      w.m[n] = -INFINITY;
      w.l[n] = 0.f;
#pragma unroll
      for (int ct = 0; ct < kCT; ++ct) w.o[n][ct] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
  };

  // S of a tile: lane (c, g) has the logits of row c and the keys 4 g + i, 16 + 4 g + i
  auto multiply_k = [&](auto& acc, const auto& w, const char* stage) __attribute__((always_inline)) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int n = 0; n < w.kN; ++n) acc[n][kt] = floatx4{0.f, 0.f, 0.f, 0.f};
    if constexpr (QUANT) {
      uint4 k[2][D / 64];
      read_k_codes<D>(k, stage, lane);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
          const uint4 x = k[kt][j];
          const bf16x8 k0 = as_bf16x8(decode8(make_uint2(x.x, x.y), 1.f)), k1 = as_bf16x8(decode8(make_uint2(x.z, x.w), 1.f));
#pragma unroll
          for (int n = 0; n < w.kN; ++n) {
            acc[n][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, w.q[n][2 * j], acc[n][kt], 0, 0, 0);
            acc[n][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, w.q[n][2 * j + 1], acc[n][kt], 0, 0, 0);
          }
        }
    } else {
      bf16x8 k[2][kKS];
      read_k_operands16<D>(k, stage, lane);
#pragma unroll
      for (int j = 0; j < kKS; ++j)
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int n = 0; n < w.kN; ++n) acc[n][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[kt][j], w.q[n][j], acc[n][kt], 0, 0, 0);
    }
  };

  // The running softmax.  P as two bf16 numbers, see above
  auto softmax = [&](auto& acc, auto& w, int tile, uint32_t mask, const floatx4 (&ek)[2], const floatx4 (&ev)[2], auto& hi, auto& lo,
                     auto& seen) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < w.kN; ++n) {
      if constexpr (QUANT) {
        acc[n][0] *= ek[0];
        acc[n][1] *= ek[1];
      }
      seen[n] = mask;
      if constexpr (CAUSAL) seen[n] &= low_mask(w.limit[n] - tile * kTile);
      float ps[8];
      const float alpha = softmax_step(acc[n], seen[n], g, p.scale_log2, w.m[n], w.l[n], ps);
      if (__ballot(alpha != 1.f) != 0ull) {
#pragma unroll
        for (int ct = 0; ct < kCT; ++ct) w.o[n][ct] *= alpha;
      }
      if constexpr (QUANT) {
#pragma unroll
        for (int e = 0; e < 8; ++e) ps[e] *= ev[e >> 2][e & 3];
      }
      hi[n] = pack_bf16x8(ps);
      const uint4 x = __builtin_bit_cast(uint4, hi[n]);
      const uint32_t h[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) ps[e] -= (e & 1) ? bf16_hi(h[e >> 1]) : bf16_lo(h[e >> 1]);
      lo[n] = pack_bf16x8(ps);
    }
  };

  auto read_v = [&](bf16x8 (&v)[kCT], const char* stage) __attribute__((always_inline)) {
    if constexpr (QUANT) {
      uint32_t codes[8][D / 64];
      read_v_codes<D>(codes, stage, lane);
#pragma unroll
      for (int ct = 0; ct < kCT; ++ct) {  // the codes of two rows next to each other, widened in pairs
        uint32_t s[4];
#pragma unroll
        for (int m = 0; m < 4; ++m)
          s[m] = decode2(__builtin_amdgcn_perm(codes[2 * m + 1][ct >> 2], codes[2 * m][ct >> 2], (ct & 2) == 0 ? 0x05010400u : 0x07030602u), ct & 1, 1.f);
        v[ct] = as_bf16x8(make_uint4(s[0], s[1], s[2], s[3]));
      }
    } else {
      read_v_operands16<D>(v, stage, lane);
    }
  };
  auto multiply_v = [&](auto& w, const bf16x8 (&v)[kCT], const auto& hi, const auto& lo) __attribute__((always_inline)) {
#pragma unroll
    for (int ct = 0; ct < kCT; ++ct)
#pragma unroll
      for (int n = 0; n < w.kN; ++n) {
        w.o[n][ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[ct], hi[n], w.o[n][ct], 0, 0, 0);
        w.o[n][ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[ct], lo[n], w.o[n][ct], 0, 0, 0);
      }
  };

  // Infinities and NaN in V.  Products with them are not what the definition says: lo may be zero or negative, and the probability of a key that a row does not
  // see, or of one far below the largest, is zero.  Any of them in a tile leaves no finite sum in its column, for all rows, until the piece ends; there one look
  // finds it (0.1 us of 9.6 for a thousand rows, 0.3 of 138 for 64 requests; a look at every tile would be 64 instructions and more each).  The wavefront then works on
  // that piece once more, and on what else it has, tile by tile: with zeros in the place of such values, after it has found out for each sum whether one of
  // them leads up or down among the keys that its row sees, as products of ones for those keys with ones for those values.
  auto not_finite = [&](const auto& w) __attribute__((always_inline)) {
    float x[2] = {0.f, 0.f};
#pragma unroll
    for (int n = 0; n < w.kN; ++n)
#pragma unroll
      for (int ct = 0; ct < kCT; ++ct)
#pragma unroll
        for (int i = 0; i < 4; i += 2)  // (v_maximum3_f32: a NaN stays)
          x[i / 2] = __builtin_elementwise_maximum(__builtin_elementwise_maximum(fabsf(w.o[n][ct][i]), fabsf(w.o[n][ct][i + 1])), x[i / 2]);
    return __ballot(!(x[0] < INFINITY && x[1] < INFINITY)) != 0ull;
  };
  auto same_lane = [&]() __attribute__((always_inline)) {  // what follows from the lane's number is worked out anew, and takes no registers of the loop before
    asm volatile("" : "+v"(lane));
    c = lane & 15;
    g = lane >> 4;
  };
  // The tiles start .. end - 1 for the rows of operand n
  auto repeat = [&](QueryRows<D, 1>& w, int n, int start, int end) __attribute__((always_inline)) {
    uint32_t up = 0u, down = 0u;  // bit 4 ct + i
#pragma unroll 1
    for (int which = 2; which >= 0; --which) {  // whether one leads up, down; the sums
      begin_unit(w, n);
      Window win{-1, 0, 0};
#pragma unroll 1
      for (int tile = start; tile < end; ++tile) {
        const TilePlace here = locate(p, u, tile, win, lane);
        if (here.mask == 0u) continue;
        if constexpr (QUANT) request_exponents(p, here, head_of(u), ring + 2 * G::kRows, lane);
        request_rows_as<D, QUANT, 0>(p.K + (int64_t)head_of(u) * p.ksh, p.ksp, p.ksn, here, ring, lane);
        request_rows_as<D, QUANT, 0>(p.V + (int64_t)head_of(u) * p.vsh, p.vsp, p.vsn, here, ring + G::kRows, lane);
        wait_loads();
        same_lane();
        bf16x8 hi[1], lo[1], v[kCT];
        uint32_t seen[1];
        if (which == 0) {
          floatx4 acc[1][2], ek[2], ev[2];
          multiply_k(acc, w, ring);
          if constexpr (QUANT) read_exponents(ek, ev, ring + 2 * G::kRows, lane);
          softmax(acc, w, tile, here.mask, ek, ev, hi, lo, seen);
        } else {  // ones for the keys that the row sees
          seen[0] = here.mask;
          if constexpr (CAUSAL) seen[0] &= low_mask(w.limit[0] - tile * kTile);
          uint32_t y[4];
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            const uint32_t two = seen[0] >> (16 * (m >> 1) + 4 * g + 2 * (m & 1));
            y[m] = (two & 1u) * 0x3f80u | ((two >> 1) & 1u) * 0x3f800000u;
          }
          hi[0] = as_bf16x8(make_uint4(y[0], y[1], y[2], y[3]));
          lo[0] = as_bf16x8(make_uint4(0u, 0u, 0u, 0u));
        }
        read_v(v, ring + G::kRows);
#pragma unroll
        for (int ct = 0; ct < kCT; ++ct) {
          const uint4 x = __builtin_bit_cast(uint4, v[ct]);
          v[ct] = as_bf16x8(make_uint4(sorted_out(x.x, which), sorted_out(x.y, which), sorted_out(x.z, which), sorted_out(x.w, which)));
          __builtin_amdgcn_sched_barrier(0);  // (one at a time: registers)
        }
        multiply_v(w, v, hi, lo);
      }
      if (which == 0) break;
#pragma unroll
      for (int ct = 0; ct < kCT; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t bit = w.o[0][ct][i] > 0.f ? 1u << (4 * ct + i) : 0u;
          up |= which == 2 ? bit : 0u;
          down |= which == 2 ? 0u : bit;
        }
    }
#pragma unroll
    for (int ct = 0; ct < kCT; ++ct)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t bit = 1u << (4 * ct + i);
        w.o[0][ct][i] += ((up & bit) ? INFINITY : 0.f) + ((down & bit) ? -INFINITY : 0.f);
      }
  };

  // Writes out what the wavefront has of unit u.  Lane (c, g) has of row c the columns 16 ct + 4 g + i of bf16 rows, (4 g + i) * D / 16 + ct of codes.
  auto end_piece = [&](const auto& w, int n0, int start, int end) __attribute__((always_inline)) {
    const bool whole = start == 0 && end == u.q.tiles;
#pragma unroll
    for (int n = 0; n < w.kN; ++n) {
      const int at = (u.qg * NT + n0 + n) * 16 + c, i = at / p.group, head = head_of(u) * p.group + at - i * p.group;
      if (i >= u.q.n) continue;
      const float inv = !whole ? 1.f : (w.l[n] == 0.f ? 0.f : 1.f / w.l[n]);
      uint16_t* out = p.out + (int64_t)(u.q.first + i) * p.osn + (int64_t)head * p.osh;
      const int64_t row = (int64_t)(2 * wave_id + (start == 0)) * p.unit_rows + 16 * (n0 + n) + c;
      float* part = p.part_o + row * D;
      auto put = [&](int column, const floatx4& x) __attribute__((always_inline)) {  // four columns
        if (whole)
          *reinterpret_cast<uint2*>(out + column) = make_uint2(cvt_pk_bf16(x[0] * inv, x[1] * inv), cvt_pk_bf16(x[2] * inv, x[3] * inv));
        else
          *reinterpret_cast<floatx4*>(part + column) = x;
      };
      if constexpr (QUANT) {
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
          for (int ct = 0; ct < kCT; ct += 4) put((4 * g + m) * kCT + ct, floatx4{w.o[n][ct][m], w.o[n][ct + 1][m], w.o[n][ct + 2][m], w.o[n][ct + 3][m]});
      } else {
#pragma unroll
        for (int ct = 0; ct < kCT; ++ct) put(16 * ct + 4 * g, w.o[n][ct]);
      }
      if (g == 0) {
        if (!whole)
          p.part_ml[row] = make_float2(w.m[n], w.l[n]);
        else if (p.lse)
          p.lse[(int64_t)(u.q.first + i) * (p.H * p.group) + head] = w.l[n] == 0.f ? -INFINITY : (w.m[n] + __builtin_amdgcn_logf(w.l[n])) * kLn2;
      }
    }
  };

  // of whom the pieces of a unit are whose last tile is the one `last` of the wavefront
  auto say_whose = [&](int start, int last) __attribute__((always_inline)) {
    if (t < u.q.tiles || lane != 0) return;
    int2 whose = make_int2(0, 0);
    if (start > 0) {
      whose.x = shares.of(begin + last - (u.q.tiles - 1));
      whose.y = worker - whose.x + 1;
    }
    p.whose[((int64_t)u.r * p.H + head_of(u)) * p.most_groups + u.qg] = whose;
  };

  // A stage's K is requested again as soon as it is in registers, its V likewise.  Loads return in order: a wait leaves those under way that were
  // requested behind what is waited for.  Where no more are requested it leaves none.  (The first requests in turns of the loop that do nothing else are half the code,
  // but with the second way out of it the compiler saw no loop there: 0.4 us of 9.6 for a thousand rows, 1 of 138 for 64 requests.)
  int start = t, i = 0;
  QueryRows<D, NT> w;
#pragma unroll 1
  while (asked < min(n_tiles, kDepth)) {
    request_k();
    request_v();
  }
#pragma unroll 1
  for (; i < n_tiles; ++i) {
    const bool more = asked < n_tiles;
    char* stage = stage_of(i);
    const uint32_t mask = (uint32_t)__builtin_amdgcn_readlane(masks, i & (kDepth - 1));
    floatx4 acc[NT][2], ek[2], ev[2];
    if (t == start) begin_unit(w, 0);
    if (i + kDepth <= n_tiles)
      wait_loads_but<G::kLoads + (kDepth - 1) * G::kTileLoads>();
    else
      wait_loads();
    if (mask != 0u) {
      multiply_k(acc, w, stage);
      if constexpr (QUANT) read_exponents(ek, ev, stage + 2 * G::kRows, lane);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (more) request_k();
    __builtin_amdgcn_sched_barrier(0);
    bf16x8 hi[NT], lo[NT];
    uint32_t seen[NT];
    if (mask != 0u) softmax(acc, w, t, mask, ek, ev, hi, lo, seen);
    if (more)
      wait_loads_but<(kDepth - 1) * G::kTileLoads + G::kTileLoads - G::kLoads>();
    else
      wait_loads();
    if (mask != 0u) {
      bf16x8 v[kCT];
      read_v(v, stage + G::kRows);
      multiply_v(w, v, hi, lo);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (more) request_v();
    ++t;
    if (t >= u.q.tiles || i == n_tiles - 1) {
      if (__builtin_expect(not_finite(w), 0)) break;
      say_whose(start, i);
      end_piece(w, 0, start, t);
      start = t = 0;
      if (i < n_tiles - 1) next_unit(u);
    }
  }
  if (i == n_tiles) return;

  wait_loads();  // those of tiles behind, which are requested again
  same_lane();
#pragma unroll 1
  for (;;) {
#pragma unroll 1
    for (int n = 0; n < NT; ++n) {
      QueryRows<D, 1> one;
      repeat(one, n, start, t);
      end_piece(one, n, start, t);
    }
    say_whose(start, i);
    if (i == n_tiles - 1) return;
    next_unit(u);
    start = 0;
    t = min(u.q.tiles, n_tiles - 1 - i);
    i += t;
  }
}

// Joins the pieces of the units that several wavefronts worked on: NW wavefronts for one row of one query head.  The pieces' largest logits are a lane each
// and their sums of weights one reduction, so that 20 pieces are one round trip: 4 to 7 us.  Whose pieces they are the wavefront with
// the last one has left (`whose`: the first of them, how many follow on one another; none: the unit is written).
template <int D, int NT, int NW>
__global__ __launch_bounds__(256) void paged_join_kernel(const PagedAttn p) {
  constexpr int kVec = D / 64, kAhead = 20;
  __shared__ float2 ml_sh[NW];
  __shared__ float o_sh[NW][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int Hq = p.H * p.group;
  const uint32_t at = NW == 1 ? (uint32_t)list_index() * 4u + (uint32_t)wave : (uint32_t)list_index();  // < kPagedMaxJoins and a slice
  const int row_at = (int)(at / (uint32_t)Hq), head = (int)(at - (uint32_t)row_at * (uint32_t)Hq);
  const int r = (int)((uint32_t)row_at / (uint32_t)p.b.max_rows), i = row_at - r * p.b.max_rows;
  if (r >= p.b.n_req) return;  // (the same in the whole workgroup where it has a barrier)
  const int h = (int)((uint32_t)head / (uint32_t)p.group), unit_row = i * p.group + head - h * p.group, qg = unit_row / (16 * NT), in_unit = unit_row - qg * 16 * NT;
  const int32_t* whose = reinterpret_cast<const int32_t*>(p.whose + ((int64_t)r * p.H + h) * p.most_groups + qg);
  const int w0 = uniform_load(whose), n = uniform_load(whose + 1);
  const RequestRows q = request_rows(p.b, r);
  if (i >= q.n) return;  // (nor has anybody written `whose`)
  if (n == 0) return;
  const int in_bundle = h & ((1 << p.log_bundle) - 1);
  // Wavefront w takes the pieces w, w + NW, ..., kAhead of them at a time: their statistics, lane by lane, and their rows, all requested at once.
  float m_run = -INFINITY, l_run = 0.f, o[kVec];
#pragma unroll
  for (int v = 0; v < kVec; ++v) o[v] = 0.f;
  const int mine = NW == 1 ? n : (n - wave + NW - 1) / NW, first = NW == 1 ? 0 : wave;
  auto slot_row = [&](int j) __attribute__((always_inline)) { return (int64_t)(2 * (((w0 + j) << p.log_bundle) + in_bundle) + (j == 0)) * p.unit_rows + in_unit; };
#pragma unroll 1
  for (int k0 = 0; k0 < mine; k0 += kAhead) {
    const int j = first + (k0 + min(lane, kAhead - 1)) * NW;
    const int j_there = min(j, n - 1);
    float2 ml = p.part_ml[slot_row(j_there)];
    float y[kAhead][kVec];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
#pragma unroll
      for (int v = 0; v < kVec; ++v) y[k][v] = 0.f;
      if (k0 + k >= mine) continue;  // (the same in all lanes)
      const float* src = p.part_o + slot_row(first + (k0 + k) * NW) * D + lane * kVec;
      if constexpr (kVec == 2) {
        const float2 x = *reinterpret_cast<const float2*>(src);
        y[k][0] = x.x;
        y[k][1] = x.y;
      } else {
        y[k][0] = *src;
      }
    }
    if (j >= n || lane >= kAhead) ml = make_float2(-INFINITY, 0.f);
    float top = ml.x;
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor(top, k, kWave));
    const float m_new = fmaxf(m_run, top), m_use = m_new == -INFINITY ? 0.f : m_new;
    const float f = ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - m_use), old = __builtin_amdgcn_exp2f(m_run - m_use);
    l_run = l_run * old + wave_sum(f * ml.y);
    m_run = m_new;
    const unsigned long long some = __ballot(ml.y != 0.f);
#pragma unroll
    for (int v = 0; v < kVec; ++v) o[v] *= old;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const float w = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), k));
      const bool take = ((some >> k) & 1ull) != 0ull;
#pragma unroll
      for (int v = 0; v < kVec; ++v) o[v] = take ? __builtin_fmaf(w, y[k][v], o[v]) : o[v];
    }
  }
  // An infinity or a NaN of a piece stays one, also where the piece's weight is zero in 32 bits.  One look at the end: they are rare
  auto stays = [](float x) __attribute__((always_inline)) { return !(fabsf(x) < INFINITY); };
  auto spoilt = [&]() __attribute__((always_inline)) {
    bool some = false;
#pragma unroll
    for (int v = 0; v < kVec; ++v) some |= stays(o[v]);
    return __ballot(some) != 0ull;
  };
  if (__builtin_expect(spoilt(), 0)) {
#pragma unroll
    for (int v = 0; v < kVec; ++v) o[v] = 0.f;
#pragma unroll 1
    for (int j = first; j < n; j += NW) {
      const float2 ml = p.part_ml[slot_row(j)];
      if (ml.y == 0.f) continue;
      const float f = __builtin_amdgcn_exp2f(ml.x - m_run), *src = p.part_o + slot_row(j) * D + lane * kVec;
#pragma unroll
      for (int v = 0; v < kVec; ++v) o[v] += stays(src[v]) ? src[v] : f * src[v];
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
    if (__builtin_expect(spoilt(), 0)) {
#pragma unroll
      for (int v = 0; v < kVec; ++v) o[v] = 0.f;
#pragma unroll 1
      for (int w = 0; w < NW; ++w) {
        const float2 ml = ml_sh[w];
        const float f = ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - m_use);
#pragma unroll
        for (int v = 0; v < kVec; ++v) {
          const float x = o_sh[w][lane * kVec + v];
          o[v] += stays(x) ? x : f * x;
        }
      }
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

// Two workgroups a compute unit, as their rings allow, and no more than the batch may have tiles.  Up to 16 query rows of a K/V head are one operand (NT = 1),
// more are taken 32 at a time, which halves the passes over the rows: 25 rows of 7 query heads on each of 4, 16 requests of 4096 98 us and not 229, 64 of 4
// on each of 8, 32 requests of 2048 334 and not 626.  Bundles of four heads where they divide: 64 requests 139 us, without bundles 149, eight-bit rows 64 and 70,
// the 25 rows of 7 98 and 146; but the 64 rows of 4 334 and 200, and 256 requests of 128 rows, 32 heads side by side 93 to 118, by where the pages lie, and 92.
constexpr int kPagedGroups = 512;
PagedPlan plan_paged_attn(int n_heads, int group, int head_dim, const PagedBatch& b, int page) {
  PagedPlan p;
  const int64_t rows = (int64_t)b.max_rows * group;
  p.q_tiles = rows <= 16 ? 1 : 2;
  p.unit_rows = (int)std::min<int64_t>(rows, 16 * p.q_tiles);
  const int64_t tiles = ceil_div64((int64_t)b.table_width * page, kTile), units = ceil_div64(rows, 16 * p.q_tiles) * n_heads;
  p.log_bundle = (n_heads & 3) == 0 ? 2 : ((n_heads & 1) == 0 ? 1 : 0);
  const int per_group = kWavesPerGroup >> p.log_bundle;  // wavefronts that take different tiles
  const int64_t bundled = (tiles * units >= (int64_t(1) << 31) ? int64_t(1) << 31 : tiles * units * b.n_req) >> p.log_bundle;
  p.groups = (int)std::min<int64_t>(kPagedGroups, ceil_div64(bundled, per_group));
  p.workers = p.groups * per_group;
  const size_t slots = (size_t)2 * p.groups * kWavesPerGroup;
  p.part_ml = (slots * p.unit_rows * head_dim * sizeof(float) + 255) & ~(size_t)255;
  p.whose = (p.part_ml + slots * p.unit_rows * sizeof(float2) + 255) & ~(size_t)255;
  p.most_groups = (int)ceil_div64(rows, 16 * p.q_tiles);
  p.total = p.whose + (size_t)b.n_req * n_heads * p.most_groups * sizeof(int2);
  return p;
}

// Few rows: four wavefronts for each, so that all its pieces (512 of a single unit) are requested within a few round trips; many: one each, which fill the chip.
constexpr int kJoinGroups = 1024;
template <int D, int NT>
static hipError_t launch_paged_t(const PagedAttn& a, const PagedPlan& p, hipStream_t st) {
  const bool causal = a.causal && (a.b.row_start != nullptr || a.b.positions != nullptr);  // (the last row sees every key)
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(p.groups), dim3(256), 0, st, a); };
  if (a.k_exp != nullptr)
    causal ? launch(paged_attn_kernel<D, true, true, NT>) : launch(paged_attn_kernel<D, true, false, NT>);
  else
    causal ? launch(paged_attn_kernel<D, false, true, NT>) : launch(paged_attn_kernel<D, false, false, NT>);
  if ((int64_t)a.b.table_width * a.page <= kTile) return hipGetLastError();  // no unit has two tiles
  const int64_t rows = (int64_t)a.b.n_req * a.b.max_rows * a.H * a.group;
  if (rows <= kJoinGroups)
    hipLaunchKernelGGL((paged_join_kernel<D, NT, 4>), grid_list(rows), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((paged_join_kernel<D, NT, 1>), grid_list(ceil_div64(rows, 4)), dim3(256), 0, st, a);
  return hipGetLastError();
}
template <int D>
static hipError_t launch_paged_d(const PagedAttn& a, const PagedPlan& p, hipStream_t st) {
  return p.q_tiles == 1 ? launch_paged_t<D, 1>(a, p, st) : launch_paged_t<D, 2>(a, p, st);
}
hipError_t launch_paged_attn(const PagedAttn& a, const PagedPlan& p, int head_dim, hipStream_t st) {
  return head_dim == 128 ? launch_paged_d<128>(a, p, st) : launch_paged_d<64>(a, p, st);
}

}  // namespace focus
