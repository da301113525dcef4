// Keys and values of decoding: rows written into a paged cache with the rotation applied on the way, and the attention
// of every sequence's new rows over its cached keys.
//
// A page holds page_len keys of every KV head, [Hkv][page_len][dh]; `pages` [n_seqs][max_pages] names the page of keys
// j page_len .. of a sequence (an entry outside [0, n_pages) is no page: nothing is written there, and its keys do not exist).
// Sequence s has lens[s] keys in front of this call's rows row_start[s] .. row_start[s + 1]; row i of them is key lens[s] + i.
#pragma once

#include <type_traits>

#include "common.h"

namespace armt {

struct KvView {
  const int32_t *pages, *lens, *row_start;
  int n_seqs, n_pages, max_pages, page_shift, n_rows;
  int64_t page_stride;      // elements from page to page
};

// ------------------------------------------------------------------------------------------------ append
// q | k | v rows of the fused projection: q' = R(p) q -> q_out, k' = R(p) k and v -> the pages.  R(p) turns the pair
// (j, j + dh/2) by p theta^(-2j/dh).  The angle is taken in turns and in double, and only its fraction is rounded to fp32: a position
// of 10^9 loses nothing.  A block takes `per` rows: first where each of them goes and the cosines and sines of all of them, into LDS, then VEC pairs
// at a time without another barrier; a thread's first loads are on their way before the first barrier.  Bytes bound it (each
// element read and written once), for few rows the two loads that lead to a row's page.  Many rows are written past the L2, which a row's heads, a
// page apart, would leave in pieces: 16000 rows of (32 + 2 x 8) x 64 bf16 60 -> 38 us (5.1 TB/s).
// grid: ceil(n_rows / per), block: 256.
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Pack { T v[VEC]; };

constexpr int KV_ROWS = 2;               // most rows of a block
constexpr int64_t KV_STREAM_BYTES = 16 << 20;      // what is written bypasses the L2 from here on (half of the L2s of the eight XCDs)

// STREAM: a store that does not stay in the L2.
template <bool STREAM, typename V>
__device__ __forceinline__ void store_pack(void* at, const V& v) {
  typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
  if constexpr (STREAM && sizeof(V) == 16) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), (u32x4*)at);
  else *(V*)at = v;
}

template <typename T, int VEC, bool STREAM>
__global__ __launch_bounds__(256) void kv_append_kernel(const T* __restrict__ qkv, int64_t ld, KvView c, const int32_t* __restrict__ positions,
                                                        T* __restrict__ q_out, T* __restrict__ kc, T* __restrict__ vc,
                                                        int H, int Hkv, int dh, int per, unsigned per_hv, unsigned per_dv, double log2_theta) {
  typedef Pack<T, VEC> V;
  __shared__ float cs[KV_ROWS][128];     // cos dh/2 | sin dh/2
  __shared__ int64_t at[KV_ROWS];        // element of the key in head 0 of its page; -1: no page; -2: nobody's row
  __shared__ int64_t slot[KV_ROWS];
  __shared__ int near;
  const int half = dh >> 1, hv = half / VEC, rot_items = (H + Hkv) * hv, dv = dh / VEC, row_items = rot_items + Hkv * dv;
  const int tid = threadIdx.x, P = 1 << c.page_shift;
  const int64_t row0 = (int64_t)blockIdx.x * per;
  const int rows = (int)min((int64_t)per, c.n_rows - row0);
  // A thread's items are 256 apart: x of row r, either a pair of VEC columns (j, j + half) of rotated head h or VEC columns of a value head
  struct Item { V a, b; int r, x, h, j; };
  auto load = [&](Item& it) __attribute__((always_inline)) {
    while (it.x >= row_items) { it.x -= row_items; ++it.r; }
    if (it.r >= rows) return;
    if (it.x < rot_items) { it.h = hv == 1 ? it.x : (int)__umulhi(it.x, per_hv); it.j = (it.x - it.h * hv) * VEC; }
    else { const int y = it.x - rot_items; it.h = __umulhi(y, per_dv); it.j = (y - it.h * dv) * VEC; it.h += H + Hkv; }
    const T* src = qkv + (row0 + it.r) * ld + it.h * dh + it.j;
    it.a = *(const V*)src;
    if (it.h < H + Hkv) it.b = *(const V*)(src + half);
  };
  Item next[2];
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    next[n].r = 0;
    next[n].x = n * 256 + tid;
    load(next[n]);
  }
  static_assert(KV_ROWS * 64 <= 256, "an angle per thread");
  const int ar = tid / half, aj = tid - ar * half, pos = positions && ar < rows ? positions[row0 + ar] : 0;
  if (tid < KV_ROWS) { at[tid] = -2; slot[tid] = 0; }
  if (tid == 0) near = 0;
  __syncthreads();
  // whose rows these are: the sequences from the last one that starts at or before row0 to the first that starts behind them
  int from = 0;
  for (int n = c.n_seqs; n > 256;) {     // of many sequences, 256 at equal distances at a time
    const int step = (n + 255) / 256, s = from + tid * step;
    if (tid * step < n && c.row_start[s] <= row0) atomicMax(&near, s);
    __syncthreads();
    n = min(step, n - (max(near, from) - from));
    from = max(near, from);
    __syncthreads();
  }
  for (int s = from + tid; s < c.n_seqs; s += 256) {
    const int64_t lo = c.row_start[s], hi = c.row_start[s + 1], len = c.lens[s];
    if (lo >= row0 + rows) break;
    for (int64_t r = max(lo, row0); r < min(hi, row0 + rows); ++r) {
      const int64_t k = len + (r - lo), j = k >> c.page_shift;
      const int page = k >= 0 && j < c.max_pages ? c.pages[(int64_t)s * c.max_pages + j] : -1;
      slot[r - row0] = k;
      at[r - row0] = page >= 0 && page < c.n_pages ? (int64_t)page * c.page_stride + (k & (P - 1)) * dh : -1;
    }
  }
  if (!positions) __syncthreads();
  if (ar < rows) {
    const double turn = (positions ? (double)pos : (double)slot[ar]) * (exp2(-(double)aj / (double)half * log2_theta) * 0.15915494309189533577);
    const float f = 2.f * (float)(turn - rint(turn));
    cs[ar][aj] = cospif(f);
    cs[ar][half + aj] = sinpif(f);
  }
  __syncthreads();
  while (next[0].r < rows) {
    const Item it = next[0];
    const int r = it.r, h = it.h, j = it.j;
    const int64_t to = at[r];
    next[0] = next[1];
    next[1].r = next[0].r;
    next[1].x = next[0].x + 256;
    load(next[1]);
    if (to == -2) continue;              // behind the last sequence: left as it is
    if (h < H + Hkv) {
      V x, y;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float co = cs[r][j + e], si = cs[r][half + j + e], u = to_f32(it.a.v[e]), w = to_f32(it.b.v[e]);
        x.v[e] = from_f32<T>(u * co - w * si);
        y.v[e] = from_f32<T>(w * co + u * si);
      }
      T* dst = h < H ? q_out + (row0 + r) * (int64_t)(H * dh) + h * dh : kc + to + (int64_t)(h - H) * P * dh;
      if (h < H || to >= 0) {
        store_pack<STREAM>(dst + j, x);
        store_pack<STREAM>(dst + half + j, y);
      }
    } else if (to >= 0) {
      store_pack<STREAM>(vc + to + (int64_t)(h - H - Hkv) * P * dh + j, it.a);
    }
  }
}

inline hipError_t launch_kv_append(bool bf, const void* qkv, int64_t ld, const KvView& c, const int32_t* positions, void* q_out,
                                   void* k, void* v, int H, int Hkv, int dh, double theta, hipStream_t st) {
  const int per = c.n_rows > 2048 ? KV_ROWS : 1;        // one row per block as long as the chip holds all blocks at once
  const unsigned grid = (unsigned)(((int64_t)c.n_rows + per - 1) / per);
  const double l2 = log2(theta);
  auto over = [](int d) { return (unsigned)(0xffffffffu / (unsigned)d + 1); };        // x / d = the high word of x over(d) while x d < 2^32 (d > 1)
  const bool stream = (int64_t)c.n_rows * (H + 2 * Hkv) * dh * (bf ? 2 : 4) >= KV_STREAM_BYTES;
#define ARMT_KV(T, VEC, STREAM)                                                                                                    \
  kv_append_kernel<T, VEC, STREAM><<<grid, 256, 0, st>>>((const T*)qkv, ld, c, positions, (T*)q_out, (T*)k, (T*)v, H, Hkv, dh, per, \
                                                         over(dh / 2 / VEC), over(dh / VEC), l2)
  if (bf && stream) ARMT_KV(bf16, 8, true);
  else if (bf) ARMT_KV(bf16, 8, false);
  else if (dh % 8) ARMT_KV(float, 2, false);
  else if (stream) ARMT_KV(float, 4, true);
  else ARMT_KV(float, 4, false);
#undef ARMT_KV
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------ attention
// out = softmax over the visible keys of (q . k / sqrt(dh)), times v, for the rows of every sequence and every head.
// Row i of a sequence sees its context (keys < lens[s]) and, of the call's own keys, those of its mask bits (a tree of drafted
// tokens) or those up to itself (no mask).  The rows of a KV head's query heads stand side by side: qi = i GROUP + g.
//
// A workgroup takes one slot (a run of keys of one sequence), one KV head and one block of 16 QT query rows; its four waves
// take 32-key tiles in turn, every wave with a ring of tiles in LDS of its own that direct copies fill, so there is no barrier
// among them until their results are joined.  Per tile a wave forms S^T = K Q^T (keys along the rows: a lane holds eight scores of ONE
// query row, so the softmax needs no exchange until a reference has to move), P^T stays in the registers in which the second
// product wants it, and V, which that product wants with the keys side by side, is read from its rows by transposing LDS reads.
// Bytes bound it for up to about 64 query rows: 48 tokens over up to 9000 keys of 32 / 8 heads of 64 take 105 us (5.2 TB/s), 3 over 131072 143 us (5.6).  With more, it is the chain of a tile (its reads from LDS,
// the two products, the softmax between them), which the two or three workgroups of a compute unit hide in part: 16 trees of 64 rows
// over 4000 keys 72 us (470 TFLOP/s), chains of 300 rows, head size 128, 104 us (580).
// Only row blocks that exist are units: a batch's sequences have one row or hundreds (us, units of the longest sequence's blocks for all / these: 16 trees
// of up to 64 rows 57 / 39, of up to 48 with 24 / 8 heads of 128 79 / 67 (59 by now), 8 chains of up to 300 158 / 145).
constexpr int KA_WAVES = 4;
constexpr int KA_STEP = 128;              // keys are cut into slots at multiples of this
constexpr int KA_CUS = 256;               // compute units
constexpr int KA_PLANNED = 1024;          // sequences up to which long ones are cut: every workgroup looks at all lengths
constexpr int KA_FEW = 512, KA_FEW_ROWS = 64;      // keys and query rows of a sequence up to which the probabilities are not rounded
constexpr float KA_LAZY_SUM = 4096.f;     // unnormalised probabilities of a lane's keys of a tile may add up to this before the reference moves

// A workgroup's unit: keys [first, last) of a sequence, the slot-th of `count` runs, and block rb of its query rows, of brows each.  The
// sequence's units start at unit0: slot by slot, in each of them its row blocks.
struct KvSeq { int s, len, row0, rows, all, total, first, last, count, slot, blocks, brows, rb, unit0; };

// Sum over the lanes up to this one.
__device__ __forceinline__ int wave_scan(int v) {
#define ARMT_DPP(ctrl, rows) v += __builtin_amdgcn_update_dpp(0, v, ctrl, rows, 0xf, false)
  ARMT_DPP(0x111, 0xf);      // row_shr:1, 2, 4, 8 inside rows of 16 lanes
  ARMT_DPP(0x112, 0xf);
  ARMT_DPP(0x114, 0xf);
  ARMT_DPP(0x118, 0xf);
  ARMT_DPP(0x142, 0xa);      // row_bcast:15, 31
  ARMT_DPP(0x143, 0xc);
#undef ARMT_DPP
  return v;
}

// Unit w.  A sequence of n steps (of `step` keys) has ceil(n / per) slots of equal length, at least one, and each of them one unit per block of at most
// `most` query rows; `per` is the least number for which all units fit in the row blocks of all sequences + spare.  All lanes of a wave work it out
// together, 64 sequences at a time.  Without spare ones a sequence has `blocks` units, alive or not.
__device__ __forceinline__ bool kv_find_unit(const KvView& c, int max_rows, int group, int w, int spare, int blocks, int most, int step, KvSeq& q) {
  const int lane = threadIdx.x & 63;
  int len, row0, rows, all, total, steps, live;
  auto load = [&](int s) __attribute__((always_inline)) {
    const int64_t cap = (int64_t)c.max_pages << c.page_shift;
    len = c.lens[s];
    const int a = c.row_start[s], b = c.row_start[s + 1];
    len = min(max(len, 0), 1 << 30);
    row0 = min(max(a, 0), c.n_rows);
    all = min(max(b, row0), c.n_rows) - row0;
    rows = min(all, max_rows);
    total = (int)min((int64_t)len + rows, cap);
    steps = rows > 0 ? (total + step - 1) / step : 0;
    live = max(1, (int)((unsigned)(rows * group + most - 1) / (unsigned)most));
  };
  int s, unit0, count = 1;
  if (spare == 0) {                        // one slot per sequence
    s = w / blocks;
    if (s >= c.n_seqs) return false;
    load(s);
    unit0 = s * blocks;
  } else {
    int64_t sum = 0;
    int least = 0;                         // units of uncut sequences
    for (int b = 0; b < c.n_seqs; b += 64) {
      load(min(b + lane, c.n_seqs - 1));
      const bool in = b + lane < c.n_seqs;
      const int64_t n = in ? min((int64_t)steps * live, (int64_t)1 << 36) : 0;       // (a wave's sum may pass 32 bits)
      sum += ((int64_t)__builtin_amdgcn_readlane(wave_scan((int)(n >> 20)), 63) << 20) + __builtin_amdgcn_readlane(wave_scan((int)(n & 0xfffff)), 63);
      least += __builtin_amdgcn_readlane(wave_scan(in ? live : 0), 63);
    }
    unsigned per = sum > 0x7fff0000 - spare ? 0x7fffffffu : max(1u, ((unsigned)sum + spare - 1) / (unsigned)spare);
    auto units_of = [&]() __attribute__((always_inline)) { return steps > 0 ? ((int)((unsigned)(steps - 1) / per) + 1) * live : 1; };
    // few long sequences: no more units than `spare`, which fill the chip once (3 x 131072 keys in 264 workgroups of which 8 wait for a second
    // round: 194 us, in 256: 151; 2 chains of 300 rows over 6000 keys, 32 / 8 heads of 128: 128 and 104).  More of them would be as long as the cut that fits allows: 48 tokens
    // over up to 9000 keys 106 -> 110.  (The loop ends: per grows, and uncut sequences fit.)
    if (c.n_seqs <= 64 && least <= spare / 2)
      for (int over; (over = __builtin_amdgcn_readlane(wave_scan(lane < c.n_seqs ? units_of() : 0), 63) - spare) > 0;)
        per += max(1u, (unsigned)((uint64_t)per * over / (2u * spare)));
    int before = 0;
    s = -1;
    for (int b = 0; b < c.n_seqs; b += 64) {
      if (c.n_seqs > 64) load(min(b + lane, c.n_seqs - 1));
      const int n = b + lane < c.n_seqs ? units_of() : 0;
      const int upto = wave_scan(n), start = before + upto - n;
      const unsigned long long hit = __ballot(w >= start && w < start + n);
      if (hit) {
        const int l = __ffsll(hit) - 1;
        s = b + l;
        unit0 = __builtin_amdgcn_readlane(start, l);
        live = __builtin_amdgcn_readlane(live, l);
        count = (int)((unsigned)__builtin_amdgcn_readlane(n, l) / (unsigned)live);
        len = __builtin_amdgcn_readlane(len, l);
        row0 = __builtin_amdgcn_readlane(row0, l);
        rows = __builtin_amdgcn_readlane(rows, l);
        all = __builtin_amdgcn_readlane(all, l);
        total = __builtin_amdgcn_readlane(total, l);
        steps = __builtin_amdgcn_readlane(steps, l);
        break;
      }
      before += __builtin_amdgcn_readlane(upto, 63);
    }
    if (s < 0) return false;
  }
  q.s = __builtin_amdgcn_readfirstlane(s);
  q.unit0 = __builtin_amdgcn_readfirstlane(unit0);
  q.count = __builtin_amdgcn_readfirstlane(count);
  q.len = __builtin_amdgcn_readfirstlane(len);
  q.row0 = __builtin_amdgcn_readfirstlane(row0);
  q.rows = __builtin_amdgcn_readfirstlane(rows);
  q.all = __builtin_amdgcn_readfirstlane(all);
  q.total = __builtin_amdgcn_readfirstlane(total);
  q.blocks = __builtin_amdgcn_readfirstlane(live);
  q.brows = ((int)((unsigned)(q.rows * group + q.blocks - 1) / (unsigned)q.blocks) + 15) & ~15;       // evenly over the blocks, at most `most`
  const unsigned i = w - q.unit0;
  q.slot = q.count > 1 ? (int)(i / (unsigned)q.blocks) : 0;
  q.rb = (int)i - q.slot * q.blocks;
  // the first (steps % count) slots take one step more
  q.first = 0;
  q.last = q.total;
  if (q.count > 1) {
    const unsigned n = __builtin_amdgcn_readfirstlane(steps), k = q.slot, base = n / (unsigned)q.count, more = n - base * q.count;
    q.first = __builtin_amdgcn_readfirstlane((int)(k * base + min(k, more)) * step);
    q.last = __builtin_amdgcn_readfirstlane(min(q.first + (int)(base + (k < more)) * step, q.total));
  }
  return true;
}

// Geometry of a tile in LDS.  bf16: 32 keys, rows of DH x 2 bytes; fp32: 16 keys, rows of DH x 4 bytes (DH: dh rounded up to 32, 64 or
// 128).  16-byte chunks of a row are exchanged (XOR) so that the reads of both products meet no bank twice: K is read
// 16 rows at one chunk, V 8 rows at a pair of chunks (bf16) or whole rows (fp32).
template <typename T, int DH>
struct KvTile {
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int KEYS = BF ? 32 : 16;
  static constexpr int ROWB = DH * (int)sizeof(T);
  static constexpr int BYTES = KEYS * ROWB;           // K or V
  static constexpr int COPIES = BYTES / 1024;         // wave-wide copies of K or V
  static constexpr int RPC = 1024 / ROWB;             // rows per copy
  static constexpr int CHUNKS = ROWB / 16;
  __device__ static __forceinline__ int swz_k(int row) { return ROWB == 128 ? (row >> 1) & 7 : row & 15; }
  __device__ static __forceinline__ int swz_v(int row) { return !BF ? 0 : ROWB == 128 ? ((row >> 1) & 3) << 1 : (row & 7) << 1; }
};

// A sequence's page table, read by scalar loads: the compiler's wait for a vector load would also wait for every copy in flight.
typedef const __attribute__((address_space(4))) int32_t* kv_table_t;

// Where a tile's 16-key halves are: byte offsets from head kvh of page 0, and whether each of them lies on a page (bit h).
template <typename T, int DH>
struct KvHalves {
  static constexpr int N = KvTile<T, DH>::KEYS / 16;
  int64_t off[N];
  int have;
};

// The table's entries for a tile's halves, as they are: nothing waits for them before they are used, a tile later.  Pages of 32 keys and more hold
// both halves.
template <typename T, int DH>
struct KvEntries { int page[KvHalves<T, DH>::N], key0; };

template <typename T, int DH>
__device__ __forceinline__ KvEntries<T, DH> kv_entries(const KvView& c, kv_table_t table, int key0) {
  KvEntries<T, DH> e;
  e.key0 = key0;
  e.page[0] = table[min(key0 >> c.page_shift, c.max_pages - 1)];
  if constexpr (KvHalves<T, DH>::N > 1) {
    e.page[1] = 0;
    if (c.page_shift == 4) e.page[1] = table[min((key0 >> 4) + 1, c.max_pages - 1)];
  }
  return e;
}

// (Halves behind the last key may lie on any page: their keys are not looked at.  A half without a page is read from page 0.)
template <typename T, int DH>
__device__ __forceinline__ KvHalves<T, DH> kv_halves(const KvView& c, const KvEntries<T, DH>& e, int dh) {
  KvHalves<T, DH> r;
  const uint64_t stride = (uint64_t)c.page_stride * sizeof(T);
  const unsigned row = (unsigned)dh * sizeof(T);
  const unsigned p0 = __builtin_amdgcn_readfirstlane(e.page[0]);
  const int ok0 = p0 < (unsigned)c.n_pages ? 1 : 0;
  r.off[0] = (int64_t)((ok0 ? p0 : 0u) * stride + ((unsigned)e.key0 & ((1u << c.page_shift) - 1)) * row);
  r.have = ok0;
  if constexpr (KvHalves<T, DH>::N > 1) {
    if (c.page_shift == 4) {
      const unsigned p1 = __builtin_amdgcn_readfirstlane(e.page[1]);
      const int ok1 = p1 < (unsigned)c.n_pages ? 1 : 0;
      r.off[1] = (int64_t)((ok1 ? p1 : 0u) * stride);
      r.have |= ok1 * 2;
    } else {
      r.off[1] = r.off[0] + 16 * row;
      r.have *= 3;
    }
  }
  return r;
}

// Keys of a tile (bit x: key0 + x) below a limit.
__device__ __forceinline__ unsigned keys_below(int limit, int key0) {
  const int n = limit - key0;
  return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1;
}

// What a query row sees: without a tree the keys below `limit`, with one those in front (uniform: len) and the drafts of its bits.
struct KvMask { unsigned long long bits; int limit; };

__device__ __forceinline__ unsigned keys_seen(const KvMask& m, bool tree, int len, int key0) {
  if (!tree) return keys_below(m.limit, key0);
  const int d = len - key0;          // drafts start at bit d
  return keys_below(len, key0) | (d >= 32 ? 0u : d >= 0 ? (unsigned)(m.bits << d) : d > -64 ? (unsigned)(m.bits >> -d) : 0u);
}

template <int N> __device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory"); }

// Max over the four lanes of a query row (lanes 16 apart).
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, kWave));
  return fmaxf(v, __shfl_xor(v, 32, kWave));
}

// q, out: [n_rows][H dh]; tree: [n_rows] or null; part: [units][Hkv][prows][DH] and pml: the same rows x {reference in log2,
// sum} for sequences of more than one slot, whose rows' {first unit, slots, row in the sequence, row blocks and their length} go to row_unit [n_rows].
// SHARED: every wave has 16 QT query rows of its own and all of them read the same tiles, else all have the same rows and tiles of their own.
// grid: units Hkv.  The heads of a unit run side by side: they share its pages (the other way round, 48 sequences took 115 us instead of 107).
// Workgroup b belongs to XCD b % 8: with eight KV heads the row blocks that read the same keys stay on one XCD, one behind the other.
template <typename T, int DH, int QT, bool SHARED, int S>
__global__ __launch_bounds__(KA_WAVES * 64) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 4 && DH == 128 && QT == 2 ? 1 : SHARED && DH == 128 && QT == 1 ? 3 : 2))) void kv_attention_kernel(const T* __restrict__ q, const T* __restrict__ kc, const T* __restrict__ vc,
                                                               const unsigned long long* __restrict__ tree, KvView c,
                                                               T* __restrict__ out, float* __restrict__ part, float* __restrict__ pml,
                                                               int4* __restrict__ row_unit, int H, int Hkv, int group, int dh, int max_rows,
                                                               int spare, int blocks, int prows, float scale_log2e) {
  typedef KvTile<T, DH> L;
  constexpr int NW = KA_WAVES;
  constexpr bool BF = L::BF;
  constexpr int KEYS = L::KEYS, ROWS = 16 * QT, NT = DH < 64 ? 4 : DH / 16, KS = BF ? DH / 32 : DH / 16, NS = KEYS / 16;
  constexpr int TILE_WAVES = SHARED ? 1 : NW;
  constexpr int STAGE = 2 * L::BYTES, NCOPY = 2 * L::COPIES / (SHARED ? NW : 1);       // copies of a wave per tile
  static_assert(NCOPY * (SHARED ? NW : 1) == 2 * L::COPIES, "every wave issues the same number of copies");
  extern __shared__ __align__(16) unsigned char smem[];      // rings of S stages; then (not SHARED) [waves][ROWS][DH] fp32 and [waves][ROWS][2]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int w = blockIdx.x / (unsigned)Hkv, kvh = blockIdx.x - w * Hkv;
  KvSeq sq;
  if (!kv_find_unit(c, max_rows, group, w, spare, blocks, ROWS * (SHARED ? NW : 1), KA_STEP, sq)) return;
  if (spare && kvh == 0 && w == sq.unit0)
    for (int i = threadIdx.x; i < sq.all; i += NW * 64)
      row_unit[sq.row0 + i] = make_int4(w, i < sq.rows ? sq.count : 0, i, sq.blocks << 8 | sq.brows);
  const int q0 = sq.rb * sq.brows, nq = min(sq.rows * group, q0 + sq.brows);       // query rows of the workgroup: [q0, nq)
  if (q0 >= nq) return;
  // 16-row tile t of a wave: waves that share the keys take the block's tiles in turn, so that a short block is spread over them
  auto qtile = [&](int t) __attribute__((always_inline)) { return q0 + (SHARED ? t * NW + wave : t) * 16; };

  const int col = lane & 15, kg = lane >> 4;
  // ---- query rows: B operand, lane = row col, 16 bytes at chunk 4 ks + kg
  typedef typename std::conditional<BF, bf16x8, f32x4>::type frag_t;
  frag_t qf[QT][KS];
  KvMask mask[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int qi = qtile(t) + col, i = qi / group, g = qi - i * group;
    const bool live = qi < nq;
    const int64_t row = sq.row0 + (live ? i : 0);
    const T* p = q + row * (int64_t)(H * dh) + (kvh * group + g) * dh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int d = (ks * 4 + kg) * (16 / (int)sizeof(T));
#pragma unroll
      for (int e = 0; e < 16 / (int)sizeof(T); ++e) qf[t][ks][e] = (T)0.f;
      if (live && d < dh) qf[t][ks] = *(const frag_t*)(p + d);
    }
    mask[t].bits = live && tree ? tree[row] : ~0ull;         // rows of padding see everything: they must not look empty
    mask[t].limit = live ? sq.len + i + 1 : 0x7fffffff;
  }
  // keys past the last row of the block are of no use without a tree
  int last = sq.last;
  if (!tree) last = __builtin_amdgcn_readfirstlane(min(last, sq.len + (nq - 1) / group + 1));
  const kv_table_t table = (kv_table_t)(uintptr_t)(c.pages + (int64_t)sq.s * c.max_pages);

  // ---- copies: lane -> 16 bytes of row lane / CHUNKS of a copy's RPC rows.  Copy x of a tile: K, then V, 16-key halves in order;
  // a wave that shares its tiles issues NCOPY of them.
  constexpr int PER = L::COPIES / KvHalves<T, DH>::N;       // copies of K, and of V, per 16-key half
  constexpr int NV = SHARED ? NCOPY : 2 * PER;              // a lane's offsets from the half's base; the swizzles repeat every 16 rows
  const int crow = lane / L::CHUNKS, cchunk = lane % L::CHUNKS;
  const char* khead = (const char*)(kc + ((int64_t)kvh << c.page_shift) * dh);       // of this KV head in page 0
  const char* vhead = (const char*)(vc + ((int64_t)kvh << c.page_shift) * dh);
  const unsigned char* ring = smem + (SHARED ? 0 : wave * (S * STAGE));
  const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) const void*)ring;
  unsigned voff[NV];
#pragma unroll
  for (int x = 0; x < NV; ++x) {
    const int y = SHARED ? wave * NCOPY + x : (x / PER) * L::COPIES + x % PER;
    const int row = (y % PER) * L::RPC + crow;
    int chunk = cchunk ^ (y < L::COPIES ? L::swz_k(row) : L::swz_v(row));
    if (!BF && chunk * 16 >= dh * 4) chunk = 0;             // padding of a short row: anything inside it
    voff[x] = (unsigned)(row * dh * (int)sizeof(T) + chunk * 16);
  }
  auto issue = [&](const KvHalves<T, DH>& hv, int stage) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < NCOPY; ++x) {
      const int y = SHARED ? wave * NCOPY + x : x, z = y % L::COPIES;
      const bool is_v = y >= L::COPIES;
      const int64_t off = KvHalves<T, DH>::N == 1 || z / PER == 0 ? hv.off[0] : hv.off[KvHalves<T, DH>::N - 1];
      lds_copy16((is_v ? vhead : khead) + off, voff[SHARED ? x : (y / L::COPIES) * PER + z % PER], lds0 + stage * STAGE + y * 1024);
    }
  };

  f32x4 o[QT][NT];
  float m2[QT], lsum[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m2[t] = -INFINITY;
    lsum[t] = 0.f;
#pragma unroll
    for (int n = 0; n < NT; ++n) o[t][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const int key_first = sq.first + (SHARED ? 0 : wave * KEYS), stride = TILE_WAVES * KEYS;
  const int n = last > key_first ? (last - key_first + stride - 1) / stride : 0;
  int have[S];
#pragma unroll
  for (int x = 0; x < S - 1; ++x)
    if (x < n) {
      const KvHalves<T, DH> hv = kv_halves<T, DH>(c, kv_entries<T, DH>(c, table, key_first + x * stride), dh);
      have[x] = hv.have;
      issue(hv, x);
    }

  bool any_odd = false;       // values that are not finite were left out
  const int whole_until = min(sq.len, last);
  const bool exact_p = sq.total <= KA_FEW || sq.rows * group <= KA_FEW_ROWS;
  auto tile = [&](int it, int stage, int pages_ok) __attribute__((always_inline)) {
    unsigned char* Kt = (unsigned char*)ring + stage * STAGE;
    unsigned char* Vt = Kt + L::BYTES;
    const int key0 = key_first + it * stride;
    const bool edge = key0 + KEYS > whole_until || pages_ok != (1 << KvHalves<T, DH>::N) - 1;       // (uniform) some key is not everybody's
    const unsigned exist = keys_below(sq.total, key0) & ((pages_ok & 1 ? 0xffffu : 0u) | (pages_ok & 2 ? 0xffff0000u : 0u));
    if (edge) {
      // Values of keys that do not exist become zero, since 0 x NaN is not.  So do, of the call's own keys, which some rows see and others do
      // not, single values that are not finite: they are added to the rows that see them behind the loop.  (Waves that share
      // the tile look first, all of them, then clear.)
      const unsigned partly = exist & ~keys_below(sq.len, key0);
      unsigned odd = 0;                  // bit x: not finite in copy x's 16 bytes
#pragma unroll
      for (int x = 0; x < L::COPIES; ++x) {
        const uint4 v = *(const uint4*)(Vt + x * 1024 + lane * 16);
        const unsigned u[4] = {v.x, v.y, v.z, v.w};
        bool no = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) no |= (BF && (u[e] & 0x7f80u) == 0x7f80u) | ((u[e] & 0x7f800000u) == 0x7f800000u);
        odd |= no & ((partly >> (x * L::RPC + crow)) & 1) ? 1u << x : 0u;
      }
      any_odd |= __ballot(odd != 0) != 0;
      if constexpr (SHARED) __syncthreads();
#pragma unroll
      for (int x = 0; x < L::COPIES; ++x) {
        const bool none = !((exist >> (x * L::RPC + crow)) & 1);
        if (none || ((odd >> x) & 1)) {
          const uint4 v = *(const uint4*)(Vt + x * 1024 + lane * 16);
          unsigned u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (none || (u[e] & 0x7f800000u) == 0x7f800000u) u[e] &= BF ? 0xffffu : 0u;
            if (BF && (none || (u[e] & 0x7f80u) == 0x7f80u)) u[e] &= 0xffff0000u;
          }
          *(uint4*)(Vt + x * 1024 + lane * 16) = make_uint4(u[0], u[1], u[2], u[3]);
        }
      }
      if constexpr (SHARED) __syncthreads();
      else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    if (SHARED && qtile(0) >= nq) return;       // a wave without rows only copies
    // ---- fragments: K rows (A operand, lane = key row col), V transposed (A operand, lane = dimension)
    frag_t kf[NS][KS], vf[BF ? NT : 4 * ((NT + 3) / 4)];
#pragma unroll
    for (int a = 0; a < NS; ++a)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int row = a * 16 + col;
        kf[a][ks] = *(const frag_t*)(Kt + row * L::ROWB + (((ks * 4 + kg) ^ L::swz_k(row)) << 4));
        if constexpr (!BF) {
          if ((ks * 4 + kg) * 4 >= dh) kf[a][ks] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
      }
    if constexpr (BF) {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
#pragma unroll
      for (int d = 0; d < NT; ++d) {
        s16x4 part4[2];
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          const int row = a * 16 + kg * 4 + (col >> 2), chunk = 2 * d + ((col & 3) >> 1);
          part4[a] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) s16x4*)(Vt + row * L::ROWB + ((chunk ^ L::swz_v(row)) << 4) + (col & 1) * 8));
        }
        vf[d] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(part4[0], part4[1], 0, 1, 2, 3, 4, 5, 6, 7));
      }
    } else {
#pragma unroll
      for (int b = 0; b < (NT + 3) / 4; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int chunk = b * 16 + (DH < 64 ? min(col, L::CHUNKS - 1) : col);
          vf[b * 4 + r] = *(const f32x4*)(Vt + (kg * 4 + r) * L::ROWB + chunk * 16);
        }
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      if (SHARED && t > 0 && qtile(t) >= nq) break;
      f32x4 sc[NS];
#pragma unroll
      for (int a = 0; a < NS; ++a) {
        sc[a] = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (BF) {
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) sc[a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[a][ks], qf[t][ks], sc[a], 0, 0, 0);
        } else {                         // (two short sums round less than a long one)
          f32x4 odd = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ks = 0; ks < KS; ks += 2)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              sc[a] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[a][ks][e], qf[t][ks][e], sc[a], 0, 0, 0);
              odd = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[a][ks + 1][e], qf[t][ks + 1][e], odd, 0, 0, 0);
            }
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[a][r] += odd[r];
        }
      }
      if (edge) {
        const unsigned mine = (keys_seen(mask[t], tree != nullptr, sq.len, key0) & exist) >> (kg * 4);
#pragma unroll
        for (int a = 0; a < NS; ++a)
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[a][r] = (mine >> (a * 16 + r)) & 1 ? sc[a][r] : -INFINITY;
      }
      // online softmax against a reference m2 (in log2 units) that moves only when a lane's probabilities of a tile add up to more than
      // KA_LAZY_SUM or to nothing sensible (the first tile: exp2(s + inf))
      float pr[NS][4], hs;
      auto form = [&](float ref) __attribute__((always_inline)) {
        hs = 0.f;
#pragma unroll
        for (int a = 0; a < NS; ++a)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            pr[a][r] = __builtin_amdgcn_exp2f(fmaf(sc[a][r], scale_log2e, -ref));
            hs += pr[a][r];
          }
      };
      form(m2[t]);
      if (__builtin_amdgcn_ballot_w64(!(hs <= KA_LAZY_SUM)) != 0) {
        float mx = sc[0][0];
#pragma unroll
        for (int a = 0; a < NS; ++a)
#pragma unroll
          for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sc[a][r]);
        const float m_new = fmaxf(m2[t], row_max(mx) * scale_log2e), ref = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m2[t] - ref);      // 0 for a row that has seen nothing yet
        m2[t] = m_new;
        lsum[t] *= alpha;
#pragma unroll
        for (int d = 0; d < NT; ++d)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[t][d][r] *= alpha;
        form(ref);
      }
      lsum[t] += hs;
      if constexpr (BF) {
        // P in bf16, as the operand of the matrix product: half a step of 2^-8 each.  Where the keys' bytes are what takes time (up to 64 query rows:
        // 48 tokens 106 us with and without, 16 trees of 8 drafts with 32 / 8 heads of 128 61 and 61, of 16 with heads of 64 42 and 43) and where keys are few, so that single
        // roundings show, what they leave follows as a second operand.  (In a chain of 300 rows that would cost 14 %.)
        bf16x8 pf;
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
          for (int r = 0; r < 4; ++r) pf[a * 4 + r] = (bf16)pr[a][r];
#pragma unroll
        for (int d = 0; d < NT; ++d) o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[d], pf, o[t][d], 0, 0, 0);
        if ((QT == 1 && !SHARED) || exact_p) {
#pragma unroll
          for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int r = 0; r < 4; ++r) pf[a * 4 + r] = (bf16)(pr[a][r] - (float)pf[a * 4 + r]);
#pragma unroll
          for (int d = 0; d < NT; ++d) o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[d], pf, o[t][d], 0, 0, 0);
        }
      } else {
        // a tile's 16 keys first, then the tiles: one sum over all keys would round as often as there are keys
#pragma unroll
        for (int d = 0; d < NT; ++d) {
          f32x4 of = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int r = 0; r < 4; ++r) of = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[(d / 4) * 4 + r][d % 4], pr[0][r], of, 0, 0, 0);
#pragma unroll
          for (int r = 0; r < 4; ++r) o[t][d][r] += of[r];
        }
      }
    }
  };

  // query rows and masks are here: a wait of the compiler's for them inside the loop would also wait for the copies in flight
#pragma unroll
  for (int t = 0; t < QT; ++t) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
      u32x4 r = __builtin_bit_cast(u32x4, qf[t][ks]);
      asm volatile("" : "+v"(r));
      qf[t][ks] = __builtin_bit_cast(frag_t, r);
    }
    asm volatile("" : "+v"(mask[t].bits), "+v"(mask[t].limit));
  }
  // ---- the tiles: S - 1 of them in flight while one is worked on (S - 2 at the barrier of waves that share them, which also says
  // that the oldest stage has been read)
  int stage = 0;
  KvEntries<T, DH> nx = kv_entries<T, DH>(c, table, key_first + min(S - 1, n) * stride);
  for (int it = 0; it < n; ++it) {
    auto next = [&]() __attribute__((always_inline)) {
      int into = stage + S - 1;
      into = into >= S ? into - S : into;
      const KvHalves<T, DH> hv = kv_halves<T, DH>(c, nx, dh);
      have[S - 1] = hv.have;
      issue(hv, into);
      nx = kv_entries<T, DH>(c, table, key_first + (it + S) * stride);
    };
    if constexpr (SHARED) {
      if (it + S - 2 < n) wait_copies<(S - 2) * NCOPY>();
      else wait_copies<0>();
      __syncthreads();
      if (it + S - 1 < n) next();
    } else if (it + S - 1 < n) {
      next();
      wait_copies<(S - 1) * NCOPY>();
    } else {
      wait_copies<0>();
    }
    tile(it, stage, have[0]);
#pragma unroll
    for (int x = 0; x + 1 < S; ++x) have[x] = have[x + 1];
    stage = stage + 1 == S ? 0 : stage + 1;
  }

  if (any_odd)
    for (int x = 0; x < n * KEYS; ++x) {
      const int key = key_first + x / KEYS * stride + x % KEYS;
      if (key < sq.len || key >= sq.total) continue;
      const int page = table[min(key >> c.page_shift, c.max_pages - 1)];
      if (page < 0 || page >= c.n_pages) continue;
      const T* v = vc + (int64_t)page * c.page_stride + (int64_t)((kvh << c.page_shift) + (key & ((1 << c.page_shift) - 1))) * dh;
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const bool sees = keys_seen(mask[t], tree != nullptr, sq.len, key) & 1;
#pragma unroll
        for (int d = 0; d < NT; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int dim = BF ? d * 16 + kg * 4 + e : (d / 4) * 64 + kg * 16 + e * 4 + d % 4;
            const float f = to_f32(v[min(dim, dh - 1)]);
            o[t][d][e] += sees && (__float_as_uint(f) & 0x7f800000u) == 0x7f800000u ? f : 0.f;
          }
      }
    }
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    lsum[t] += __shfl_xor(lsum[t], 16, kWave);
    lsum[t] += __shfl_xor(lsum[t], 32, kWave);
  }
  const bool whole = sq.count == 1;
  // four dimensions of a row: to out, or as they are to the slot's place
  auto store = [&](int qi, int d, const f32x4& acc, float ref, float sum) __attribute__((always_inline)) {
    if (whole) {
      const float inv = ref == -INFINITY ? 0.f : 1.f / sum;       // a row that sees nothing is zero
      const int i = qi / group, g = qi - i * group;
      Pack<T, 4> v4;
#pragma unroll
      for (int e = 0; e < 4; ++e) v4.v[e] = from_f32<T>(ref == -INFINITY ? 0.f : acc[e] * inv);
      *(Pack<T, 4>*)(out + (int64_t)(sq.row0 + i) * (H * dh) + (kvh * group + g) * dh + d) = v4;
    } else {
      const int64_t at = ((int64_t)w * Hkv + kvh) * prows + qi - q0;
      *(f32x4*)(part + at * DH + d) = acc;
      if (d == 0) { pml[at * 2] = ref; pml[at * 2 + 1] = sum; }
    }
  };
  auto dims = [&](int t, int x) __attribute__((always_inline)) {       // the x-th four consecutive dimensions of a lane
    if constexpr (BF) return o[t][x];
    else return f32x4{o[t][x / 4 * 4][x % 4], o[t][x / 4 * 4 + 1][x % 4], o[t][x / 4 * 4 + 2][x % 4], o[t][x / 4 * 4 + 3][x % 4]};
  };
  auto dim_of = [&](int x) __attribute__((always_inline)) { return BF ? x * 16 + kg * 4 : x / 4 * 64 + kg * 16 + x % 4 * 4; };
  if constexpr (SHARED) {
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int qi = qtile(t) + col;
      if (qi < nq)
#pragma unroll
        for (int x = 0; x < NT; ++x) store(qi, dim_of(x), dims(t, x), m2[t], lsum[t]);
    }
  } else {
    // ---- join the waves: rows of O (fp32) and {reference, sum} in LDS
    __syncthreads();
    float* Os = (float*)smem;
    float* ML = Os + NW * ROWS * DH;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float* r = Os + (size_t)(wave * ROWS + t * 16 + col) * DH;
#pragma unroll
      for (int x = 0; x < NT; ++x)
        if (dim_of(x) < DH) *(f32x4*)(r + dim_of(x)) = dims(t, x);
      if (kg == 0) { ML[(wave * ROWS + t * 16 + col) * 2] = m2[t]; ML[(wave * ROWS + t * 16 + col) * 2 + 1] = lsum[t]; }
    }
    __syncthreads();
    for (int x = threadIdx.x; x < ROWS * (DH / 4); x += NW * 64) {
      const int r = x / (DH / 4), d = (x - r * (DH / 4)) * 4, qi = q0 + r;
      if (qi >= nq || d >= dh) continue;
      float ref = -INFINITY;
#pragma unroll
      for (int v = 0; v < NW; ++v) ref = fmaxf(ref, ML[(v * ROWS + r) * 2]);
      float sum = 0.f;
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int v = 0; v < NW; ++v) {
        const float mv = ML[(v * ROWS + r) * 2], f = __builtin_amdgcn_exp2f(mv - ref);
        if (mv == -INFINITY) continue;       // a wave without a visible key
        const f32x4 ov = *(const f32x4*)(Os + (size_t)(v * ROWS + r) * DH + d);
        sum = fmaf(f, ML[(v * ROWS + r) * 2 + 1], sum);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = fmaf(f, ov[e], acc[e]);
      }
      store(qi, d, acc, ref, sum);
    }
  }
}

// Rows of sequences that were cut into several slots: the slots' results joined, one wave per row and head.  DH / 4 lanes hold a slot's
// row, so 64 / (DH / 4) slots are read at a time.  grid: ceil(n_rows H / 4), block: 256.
template <typename T, int DH>
__global__ __launch_bounds__(256) void kv_join_kernel(KvView c, T* __restrict__ out, const float* __restrict__ part, const float* __restrict__ pml,
                                                      const int4* __restrict__ row_unit, int H, int Hkv, int dh, int max_rows, int units, int prows) {
  constexpr int LANES = DH / 4, TOGETHER = 64 / LANES;
  const int lane = threadIdx.x & 63, sub = lane / LANES, d = lane % LANES * 4, group = H / Hkv;
  const int64_t x = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), row = x / H;
  const int h = (int)(x - row * H), kvh = h / group;
  if (row >= c.n_rows) return;
  const int4 ru = row_unit[row];
  // rows outside [row_start[0], row_start[n_seqs]) are nobody's, and nobody has written their entry; no entry leads outside the units
  if (row < c.row_start[0] || row >= c.row_start[c.n_seqs]) return;
  const int unit0 = ru.x, count = ru.y, i = ru.z, blocks = ru.w >> 8, brows = ru.w & 255;
  if (count <= 1 || unit0 < 0 || blocks < 1 || (int64_t)unit0 + (int64_t)count * blocks > units || i < 0 || i >= max_rows || brows < 16 || brows > prows) return;
  const int qi = i * group + (h - kvh * group), rb = (int)((unsigned)qi / (unsigned)brows);
  if (rb >= blocks) return;
  const int64_t at0 = ((int64_t)(unit0 + rb) * Hkv + kvh) * prows + qi - rb * brows, step = (int64_t)blocks * Hkv * prows;
  float ref = -INFINITY;
  for (int n = lane; n < count; n += 64) ref = fmaxf(ref, pml[(at0 + n * step) * 2]);
  float sum = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  ref = wave_max(ref);
#pragma unroll 4
  for (int n = sub; n < count; n += TOGETHER) {
    const int64_t at = at0 + n * step;
    const float m = pml[at * 2], l = pml[at * 2 + 1];
    const f32x4 v = d < dh ? *(const f32x4*)(part + at * DH + d) : f32x4{0.f, 0.f, 0.f, 0.f};
    const float f = __builtin_amdgcn_exp2f(m - ref);
    const bool some = m != -INFINITY;       // (a slot whose keys the row does not see)
    sum = some ? fmaf(f, l, sum) : sum;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = some ? fmaf(f, v[e], acc[e]) : acc[e];
  }
#pragma unroll
  for (int o = LANES; o < 64; o <<= 1) {
    sum += __shfl_xor(sum, o, kWave);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], o, kWave);
  }
  if (sub || d >= dh) return;
  Pack<T, 4> v4;
#pragma unroll
  for (int e = 0; e < 4; ++e) v4.v[e] = from_f32<T>(ref == -INFINITY ? 0.f : acc[e] / sum);
  *(Pack<T, 4>*)(out + row * (int64_t)(H * dh) + h * dh + d) = v4;
}

// Shape of a launch, from what the host knows (the lengths are on the device).
struct KvPlan {
  int DH, QT, blocks, prows, units, spare;
  bool shared;
  size_t part, pml, row_unit, total;         // workspace
};

inline KvPlan kv_plan(bool bf, int n_seqs, int n_rows, int max_rows, int64_t max_keys, int H, int Hkv, int dh, int target = 0) {
  KvPlan p;
  p.DH = dh <= 32 ? 32 : dh <= 64 ? 64 : 128;
  const int64_t nq = (int64_t)max_rows * (H / Hkv);
  p.QT = nq <= 16 ? 1 : nq <= 32 || p.DH == 128 || !bf ? 2 : 4;
  p.shared = bf && nq > 16 * p.QT;
  // 128 dimensions: two row tiles take a wave 254 registers, one 146, so that three workgroups share a compute unit.  For few row blocks that is worth more than
  // reading their keys less often (us, two / one: 16 trees of up to 48 rows, 24 / 8 heads, 67 / 59, 32 / 8 heads: 16 of up to 32 87 / 82, 40 of up to 24 92 / 88, 16 of 20 69 / 70, 32 chains of 32
  // 110 / 118; more rows, 8 chains of 64 105 / 110, 2 of 300 105 / 118)
  if (p.shared) p.QT = p.DH == 128 && nq <= 192 ? 1 : 2;
  const int most = 16 * p.QT * (p.shared ? KA_WAVES : 1);       // rows of a block
  p.blocks = (int)((nq + most - 1) / most);
  p.prows = (int)(nq < most ? (nq + 15) / 16 * 16 : most);
  // row blocks of all sequences: those that hold n_rows, and a partial one each
  const int64_t every = (int64_t)n_seqs * p.blocks, held = n_seqs + (int64_t)n_rows * (H / Hkv) / most, least = every < held ? every : held;
  const int64_t steps = (max_keys + KA_STEP - 1) / KA_STEP;
  // workgroups wanted: what the chip holds at once
  const int resident = p.shared ? (p.DH == 64 || p.QT == 1 ? 3 : 2) : p.DH == 32 ? 4 : p.DH == 64 ? 2 : 1;       // (registers; 1 KB x DH of rings in 160 KB of LDS)
  int64_t spare = (target ? target : KA_CUS * resident) / Hkv;
  if (spare > least * (steps - 1)) spare = least * (steps - 1);         // cuts that keys could be made at
  // Short caches of one row tile are not cut: a second launch costs more than the walk through ten steps, sixteen where the workgroups are
  // many (us, cut and joined / whole: 1 x 1040 keys 6.4 + 3.8 / 9.9, 1 x 2000 7.2 + 3.8 / 13.4, 8 x 2000 11.5 + 4.0 / 14.2, 32 x 2000 27.1 + 4.8 / 27.6)
  if (!p.shared && p.QT == 1 && (steps <= 10 || (steps <= 16 && (int64_t)n_seqs * Hkv * p.blocks >= 64))) spare = 0;
  // Nor are those of very many sequences: a workgroup would spend its time on the lengths (us, n sequences of 300 keys and one of 60000, cut / whole:
  // 520 125 / 299, 1024 270 / 322, 4096 2549 / 501; 1024 with eight of 20000 304 / 258)
  if (n_seqs > KA_PLANNED) spare = 0;
  p.spare = (int)(spare < 0 ? 0 : spare);
  p.units = (int)(p.spare ? least + p.spare : every < 0x7fffffff ? every : 0x7fffffff);
  auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  const size_t all = p.spare ? (size_t)p.units * Hkv * p.prows : 0;
  p.part = 0;
  p.pml = up(all * p.DH * 4);
  p.row_unit = p.pml + up(all * 8);
  p.total = p.row_unit + (p.spare ? up((size_t)n_rows * 16) : 0);
  return p;
}

inline int64_t kv_grid(const KvPlan& p, int Hkv) {
  return (int64_t)p.units * Hkv;
}

template <typename T, int DH, int QT, bool SHARED, int S>
hipError_t launch_kv_attention_as(const KvPlan& p, const void* q, const void* k, const void* v, const unsigned long long* tree, const KvView& c,
                                  void* out, char* ws, int H, int Hkv, int dh, int max_rows, hipStream_t st) {
  typedef KvTile<T, DH> L;
  constexpr int ring = (SHARED ? 1 : KA_WAVES) * S * 2 * L::BYTES, join = SHARED ? 0 : KA_WAVES * 16 * QT * (DH + 2) * 4, lds = ring > join ? ring : join;
  static std::atomic<uint64_t> raised{0};
  if (lds > 65536) {
    const hipError_t e = raise_lds_limit((const void*)kv_attention_kernel<T, DH, QT, SHARED, S>, lds, raised);
    if (e != hipSuccess) return e;
  }
  const unsigned grid = (unsigned)kv_grid(p, Hkv);
  float *part = (float*)(ws + p.part), *pml = (float*)(ws + p.pml);
  int4* row_unit = (int4*)(ws + p.row_unit);
  kv_attention_kernel<T, DH, QT, SHARED, S><<<grid, KA_WAVES * 64, lds, st>>>(
      (const T*)q, (const T*)k, (const T*)v, tree, c, (T*)out, part, pml, row_unit, H, Hkv, H / Hkv, dh, max_rows, p.spare, p.blocks, p.prows,
      1.4426950408889634f / sqrtf((float)dh));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.spare) return e;
  kv_join_kernel<T, DH><<<(unsigned)(((int64_t)c.n_rows * H + 3) / 4), 256, 0, st>>>(c, (T*)out, part, pml, row_unit, H, Hkv, dh, max_rows, p.units, p.prows);
  return hipGetLastError();
}

inline hipError_t launch_kv_attention(bool bf, const KvPlan& p, const void* q, const void* k, const void* v, const unsigned long long* tree,
                                      const KvView& c, void* out, char* ws, int H, int Hkv, int dh, int max_rows, hipStream_t st) {
#define ARMT_KA(T, D, Q, SH, S) return launch_kv_attention_as<T, D, Q, SH, S>(p, q, k, v, tree, c, out, ws, H, Hkv, dh, max_rows, st)
  if (bf && p.shared) {
    if (p.DH == 64) ARMT_KA(bf16, 64, 2, true, 4);
    if (p.QT == 1) ARMT_KA(bf16, 128, 1, true, 3);
    ARMT_KA(bf16, 128, 2, true, 4);
  }
  if (bf) {
    if (p.DH == 64) {
      if (p.QT == 1) ARMT_KA(bf16, 64, 1, false, 2);
      if (p.QT == 2) ARMT_KA(bf16, 64, 2, false, 2);
      ARMT_KA(bf16, 64, 4, false, 2);
    }
    if (p.QT == 1) ARMT_KA(bf16, 128, 1, false, 2);
    ARMT_KA(bf16, 128, 2, false, 2);
  }
  if (p.DH == 32) {
    if (p.QT == 1) ARMT_KA(float, 32, 1, false, 2);
    ARMT_KA(float, 32, 2, false, 2);
  }
  if (p.DH == 64) {
    if (p.QT == 1) ARMT_KA(float, 64, 1, false, 2);
    ARMT_KA(float, 64, 2, false, 2);
  }
  if (p.QT == 1) ARMT_KA(float, 128, 1, false, 2);
  ARMT_KA(float, 128, 2, false, 2);
#undef ARMT_KA
}

}  // namespace armt
