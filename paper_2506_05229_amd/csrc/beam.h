// Beam search: the best continuations of every sequence over its beams and the vocabulary, and the gathering of the beams' states.
#pragma once

#include "common.h"

namespace armt {

// ------------------------------------------------------------------------------------------------ selection
// score(b, v) = scores[b] + x[b][v] - log sum_v' exp(x[b][v']); the n_out best of a sequence's beams x vocab, ties to the lowest b vocab + v.
// First launch: a wave holds its part of one row of logits in registers, all loads in flight at once, takes their maximum and sum, and keeps those that
// reach the n_out-th largest of its lanes' maxima: a bound of the n_out-th best that lets little more than n_out through.  The workgroup's survivors
// are ranked by counting, and its n_out best written in order.  Second launch: one workgroup per sequence, the same over the parts' lists.
// Reading the logits once bounds the large cases; the small ones are two launches' latency.
//
// Inside a row the order of the scores is that of the logits, so the lists hold 64-bit keys: the logit in an order-preserving form above the complement
// of its index.  Scores of different rows are compared in 64 bits; the sums are of fp32 exponentials (random errors of 2^-24 each), added in fp32 per lane and in 64
// bits across lanes.
constexpr int BS_MAX = 64;             // n_out: a list lies over the lanes of one wave
constexpr int BS_BEAMS = 64;           // beams of a sequence
constexpr int BS_WAVES = 4;
constexpr int BS_CAP = 256;            // survivors a wave may have; with more (ties, mostly) it sorts by insertion
constexpr int BS_PICK = 8;             // waves of the second launch
constexpr int kMaxBlocks = 0xffffff;   // of 256 threads: a launch has fewer than 2^32

struct BeamPart { double sum; float top; int pad; };      // of one workgroup's part of a row: sum of exp(x - top)

constexpr float BS_MOST = 3.402823466e+38f;

// A logit as it is taken: no NaN (the lowest), no +inf (the largest finite number).
__device__ __forceinline__ float beam_logit(float x) { return x > -INFINITY ? fminf(x, BS_MOST) : -INFINITY; }
__device__ __forceinline__ unsigned beam_order(float x) {
  const unsigned u = __float_as_uint(x + 0.f);       // one zero
  return u ^ ((u & 0x80000000u) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float beam_value(unsigned o) { return __uint_as_float(o ^ ((o & 0x80000000u) ? 0x80000000u : 0xffffffffu)); }

typedef unsigned long long u64;
__device__ __forceinline__ u64 beam_key(float x, int at) { return ((u64)beam_order(x) << 32) | (unsigned)~at; }     // never 0

__device__ __forceinline__ unsigned shift_lanes_up(unsigned v) {       // lane i gets lane i - 1's
  return (unsigned)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x138, 0xf, 0xf, false);
}
__device__ __forceinline__ unsigned read_lane(unsigned v, int l) { return (unsigned)__builtin_amdgcn_readlane((int)v, l); }
__device__ __forceinline__ u64 read_lane(u64 v, int l) { return ((u64)read_lane((unsigned)(v >> 32), l) << 32) | read_lane((unsigned)v, l); }

// A list of 64-bit keys sorted downwards over the lanes.
struct KeyList {
  u64 key;                             // 0: nothing
  __device__ __forceinline__ void insert(u64 k) {                        // k: the same in all lanes
    const u64 up = ((u64)shift_lanes_up((unsigned)(key >> 32)) << 32) | shift_lanes_up((unsigned)key);
    const int pos = __popcll(__ballot(key >= k));
    const int lane = threadIdx.x & 63;
    key = lane < pos ? key : lane == pos ? k : up;
  }
};

// The n-th largest of the lanes' values, or a little less: its leading BITS bits.
template <int BITS>
__device__ __forceinline__ unsigned nth_of_lanes(unsigned v, int n) {
  unsigned low = 0;
#pragma unroll
  for (int b = 31; b >= 32 - BITS; --b) {
    const unsigned mid = low | (1u << b);
    low = __popcll(__ballot(v >= mid)) >= n ? mid : low;
  }
  return low;
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

// grid: rows x parts, block: 256; a part is 4 x 64 E logits.  list: [sequences][n_out][beams][parts], info: [rows][parts].
template <int E>
__global__ __launch_bounds__(BS_WAVES * 64) __attribute__((amdgpu_waves_per_eu(E == 64 ? 5 : 1))) void beam_scan_kernel(const float* __restrict__ logits, int64_t ld, int beams, int vocab, int n_out, int parts,
                                                                   u64* __restrict__ list, BeamPart* __restrict__ info) {
  struct alignas(4) Four { float v[4]; };
  __shared__ __align__(16) u64 keys[BS_WAVES][BS_CAP + 4];
  __shared__ int counts[BS_WAVES];
  __shared__ float tops[BS_WAVES], edges[BS_WAVES];
  __shared__ double sums[BS_WAVES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.x / parts, part = blockIdx.x - row * parts;
  const float* x = logits + (int64_t)row * ld;
  const int at = (int)min((int64_t)(part * BS_WAVES + wave) * (64 * E), (int64_t)vocab);
  constexpr float LOG2E = 1.4426950408889634f;
  // value e of a lane: index at + 256 (e / 4) + 4 lane + e % 4
  float v[E];
#pragma unroll
  for (int g = 0; g < E / 4; ++g) {
    if (at + (int64_t)g * 256 + 256 <= vocab) {
      const Four f = *(const Four*)(x + at + g * 256 + lane * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[g * 4 + e] = f.v[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int64_t i = at + (int64_t)g * 256 + lane * 4 + e;
        v[g * 4 + e] = i < vocab ? x[i] : -INFINITY;
      }
    }
  }
  float mx = -INFINITY;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    v[e] = beam_logit(v[e]);
    mx = fmaxf(mx, v[e]);
  }
  // sum of exp(v - top) as exp2(v log2(e) - t2) with one rounding inside; what t2 is off by comes out of the sum again
  const float top = fmaxf(wave_max(mx), -BS_MOST), t2 = top * LOG2E;
  float sum = 0.f;
  double off = 0.0;
  if (fabsf(top) < 1e38f) {
#pragma unroll
    for (int e = 0; e < E; ++e) sum += __builtin_amdgcn_exp2f(fmaf(v[e], LOG2E, -t2));
    off = -(double)fmaf(top, LOG2E, -t2);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) sum += __builtin_amdgcn_exp2f((v[e] - top) * LOG2E);
  }
  const double wsum = wave_sum((double)sum) * exp2(off);
  // a value that n_out lanes' maxima reach is not above the n_out-th best, of the row neither: the highest of the waves' serves all
  const unsigned low = nth_of_lanes<20>(beam_order(mx), n_out);
  if (lane == 0) edges[wave] = low > beam_order(-INFINITY) ? beam_value(low) : -INFINITY;
  __syncthreads();
  float edge = edges[0];
#pragma unroll
  for (int w = 1; w < BS_WAVES; ++w) edge = fmaxf(edge, edges[w]);
  int have = 0;
  auto index = [&](int e) __attribute__((always_inline)) { return at + (e / 4) * 256 + lane * 4 + e % 4; };
  auto collect = [&](int e, u64 in) __attribute__((always_inline)) {
    const int place = have + __popcll(in & ((1ull << lane) - 1));
    if (((in >> lane) & 1) && place < BS_CAP) keys[wave][place] = beam_key(v[e], index(e));
    have += __popcll(in);
  };
  if (edge > -INFINITY) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const u64 in = __ballot(v[e] >= edge);
      if (in) collect(e, in);
    }
  } else {                               // (few logits, or hardly any above -inf)
#pragma unroll
    for (int e = 0; e < E; ++e) collect(e, __ballot(index(e) < vocab));
  }
  if (have > BS_CAP) {
    KeyList best{0};
    u64 last = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const u64 key = index(e) < vocab ? beam_key(v[e], index(e)) : 0;
      for (u64 in = __ballot(key > last); in; in &= __ballot(key > last)) {
        best.insert(read_lane(key, __ffsll(in) - 1));
        in &= in - 1;
        last = read_lane(best.key, n_out - 1);
      }
    }
    if (lane < n_out) keys[wave][lane] = best.key;       // (all of them: more than BS_CAP were there)
    have = n_out;
  }
  if (lane < 4) keys[wave][have + lane] = 0;             // read four at a time
  if (lane == 0) { counts[wave] = have; tops[wave] = top; sums[wave] = wsum; }
  __syncthreads();
  // ---- the workgroup's list: a key's place is the number of larger ones
  const int seq = row / beams, lists = beams * parts;
  u64* dst = list + (int64_t)seq * n_out * lists + (row - seq * beams) * parts + part;
  int all = 0;
#pragma unroll
  for (int w = 0; w < BS_WAVES; ++w) all += counts[w];
  for (int i = lane; i < have; i += 64) {
    const u64 mine = keys[wave][i];
    int rank = 0;
#pragma unroll
    for (int w = 0; w < BS_WAVES; ++w) {
      const int n = counts[w];
#pragma unroll 2
      for (int j = 0; j < n; j += 4) {
        const ulonglong2 p = *(const ulonglong2*)&keys[w][j], q = *(const ulonglong2*)&keys[w][j + 2];
        rank += (p.x > mine) + (p.y > mine) + (q.x > mine) + (q.y > mine);
      }
    }
    if (rank < n_out) dst[(int64_t)rank * lists] = mine;
  }
  for (int i = all + (int)threadIdx.x; i < n_out; i += BS_WAVES * 64) dst[(int64_t)i * lists] = 0;
  if (threadIdx.x == 0) {
    float t = tops[0];
    for (int i = 1; i < BS_WAVES; ++i) t = fmaxf(t, tops[i]);
    double total = 0.0;
    for (int i = 0; i < BS_WAVES; ++i) total += sums[i] * exp((double)tops[i] - (double)t);
    info[blockIdx.x] = BeamPart{total, t, 0};
  }
}

// A list of {score, flat index} sorted by falling score, then rising index.
__device__ __forceinline__ u64 score_order(double v) {
  const u64 u = (u64)__double_as_longlong(v);
  return u ^ ((u >> 63) ? ~0ull : 1ull << 63);
}
__device__ __forceinline__ double score_value(u64 o) { return __longlong_as_double((long long)(o ^ ((o >> 63) ? 1ull << 63 : ~0ull))); }

struct ScoreList {
  u64 score;                           // 0: nothing
  unsigned at;
  __device__ __forceinline__ static bool before(u64 s, unsigned a, u64 t, unsigned b) { return s > t || (s == t && a < b); }
  __device__ __forceinline__ void insert(u64 s, unsigned a) {
    const u64 us = ((u64)shift_lanes_up((unsigned)(score >> 32)) << 32) | shift_lanes_up((unsigned)score);
    const unsigned ua = shift_lanes_up(at);
    const int pos = __popcll(__ballot(before(score, at, s, a)));
    const int lane = threadIdx.x & 63;
    if (lane == pos) { score = s; at = a; }
    else if (lane > pos) { score = us; at = ua; }
  }
};

// out_scores may be scores: a workgroup has read its sequence's before it writes them.  grid: sequences, block: 512.
__global__ __launch_bounds__(BS_PICK * 64) void beam_pick_kernel(const u64* __restrict__ list, const BeamPart* __restrict__ info, const float* scores,
                                                                  int beams, int vocab, int n_out, int parts, float* out_scores,
                                                                  int32_t* __restrict__ out_parents, int32_t* __restrict__ out_tokens) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int CAP = BS_CAP + 4;
  u64* sc = (u64*)smem;                                     // [waves][CAP]
  unsigned* ix = (unsigned*)(sc + BS_PICK * CAP);           // the same
  int* counts = (int*)(ix + BS_PICK * CAP);                 // [waves], padded to 16
  double* shift = (double*)(counts + 16);                   // [beams] log of the sum
  double* top = shift + beams;                              // [beams] +inf: no continuation of the beam has a score
  double* before = top + beams;                             // [beams]
  const int fin = (BS_PICK * CAP * 12 + 64 + beams * 24 + 15) & ~15;        // the last list: as sc and ix
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), seq = blockIdx.x, lists = beams * parts;
  const int64_t row0 = (int64_t)seq * beams;
  const u64* pl = list + (int64_t)seq * n_out * lists;
  const int n = n_out * lists;                              // (host: below 2^31)
  constexpr int EARLY = 8, STEP = BS_PICK * 64;
  u64 early[EARLY];                                         // the first candidates' keys are on their way while the sums are made
#pragma unroll
  for (int k = 0; k < EARLY; ++k) early[k] = k * STEP + (int)threadIdx.x < n ? pl[k * STEP + threadIdx.x] : 0;
  for (int b = wave; b < beams; b += BS_PICK) {
    const BeamPart* pi = info + (row0 + b) * parts;
    const float score = scores[row0 + b];
    float t = -3.402823466e+38f;
    for (int i = lane; i < parts; i += 64) t = fmaxf(t, pi[i].top);
    t = wave_max(t);
    double sum = 0.0;
    for (int i = lane; i < parts; i += 64) sum += pi[i].sum * exp((double)pi[i].top - (double)t);
    sum = wave_sum(sum);
    const bool dead = !(score > -INFINITY && score < INFINITY) || !(sum > 0.0);
    if (lane == 0) { shift[b] = log(sum); top[b] = dead ? INFINITY : (double)t; before[b] = score; }
  }
  __syncthreads();
  // candidate i: entry i / lists of list i % lists, so that neighbouring lanes have the same entry of different lists and their maxima are alike.
  // Score and flat index; 0: none.  A beam without a score offers its first tokens, at -inf.
  const float per_list = 1.f / (float)lists, per_part = 1.f / (float)parts;
  auto quotient = [](int x, int d, float inv) __attribute__((always_inline)) {      // off by little: put right
    int q = (int)((float)x * inv);
    while (x < q * d) --q;
    while (x - q * d >= d) ++q;
    return q;
  };
  auto candidate = [&](int i, u64 key, u64& s, unsigned& at) __attribute__((always_inline)) {
    const int j = quotient(i, lists, per_list), l = i - j * lists, b = quotient(l, parts, per_part);
    const bool dead = top[b] == INFINITY;
    const unsigned token = dead ? (unsigned)j : ~(unsigned)key;
    const double value = dead ? -INFINITY : before[b] + (((double)beam_value((unsigned)(key >> 32)) - top[b]) - shift[b]);
    s = i < n && (dead ? l == b * parts && j < vocab : key != 0) ? score_order(value) : 0;
    at = (unsigned)b * (unsigned)vocab + token;
  };
  unsigned mx = 0, at_early[EARLY];
#pragma unroll
  for (int k = 0; k < EARLY; ++k) {
    candidate(min(k * STEP + (int)threadIdx.x, n), early[k], early[k], at_early[k]);
    mx = max(mx, (unsigned)(early[k] >> 32));
  }
  for (int i = EARLY * STEP + (int)threadIdx.x; i < n; i += STEP) {
    u64 s;
    unsigned at;
    candidate(i, pl[i], s, at);
    mx = max(mx, (unsigned)(s >> 32));
  }
  const unsigned low = nth_of_lanes<32>(mx, n_out);
  if (lane == 0) counts[wave] = (int)low;
  __syncthreads();
  unsigned edge = 1;                                        // (a score's upper word is never 0)
  for (int w = 0; w < BS_PICK; ++w) edge = max(edge, (unsigned)counts[w]);
  __syncthreads();
  int have = 0;
  auto collect = [&](u64 s, unsigned at) __attribute__((always_inline)) {
    const u64 in = __ballot((unsigned)(s >> 32) >= edge);
    const int place = have + __popcll(in & ((1ull << lane) - 1));
    if (((in >> lane) & 1) && place < BS_CAP) {
      sc[wave * CAP + place] = s;
      ix[wave * CAP + place] = at;
    }
    have += __popcll(in);
  };
#pragma unroll
  for (int k = 0; k < EARLY; ++k) collect(early[k], at_early[k]);
  for (int i0 = EARLY * STEP + wave * 64; i0 < n; i0 += STEP) {
    u64 s = 0;
    unsigned at = 0;
    if (i0 + lane < n) candidate(i0 + lane, pl[i0 + lane], s, at);
    collect(s, at);
  }
  const bool many = have > BS_CAP;
  if (many) {
    ScoreList best{0, 0xffffffffu};
    for (int i0 = wave * 64; i0 < n; i0 += BS_PICK * 64) {
      u64 s = 0;
      unsigned at = 0xffffffffu;
      if (i0 + lane < n) candidate(i0 + lane, pl[i0 + lane], s, at);
      auto better = [&]() __attribute__((always_inline)) {
        return __ballot(s != 0 && ScoreList::before(s, at, read_lane(best.score, n_out - 1), read_lane(best.at, n_out - 1)));
      };
      for (u64 in = better(); in; in &= better()) {
        const int l = __ffsll(in) - 1;
        best.insert(read_lane(s, l), read_lane(at, l));
        in &= in - 1;
      }
    }
    if (lane < n_out) { sc[wave * CAP + lane] = best.score; ix[wave * CAP + lane] = best.at; }
    have = n_out;
  }
  if (lane == 0) counts[wave] = have;
  if (threadIdx.x == 0) counts[BS_PICK] = 0;
  __syncthreads();
  int all = 0;
  for (int w = 0; w < BS_PICK; ++w) all += counts[w];
  if (all > 2 * 64) {                                       // few lanes had most of them: the same once more, among these
    unsigned m = 0;
    for (int i = lane; i < have; i += 64) m = max(m, (unsigned)(sc[wave * CAP + i] >> 32));
    const unsigned l2 = nth_of_lanes<32>(m, n_out);
    __syncthreads();
    if (lane == 0) counts[wave] = (int)l2;
    __syncthreads();
    for (int w = 0; w < BS_PICK; ++w) edge = max(edge, (unsigned)counts[w]);
  }
  // side by side, in any order: a score's place is the number of better ones
  u64* fs = (u64*)(smem + fin);
  unsigned* fi = (unsigned*)(fs + BS_PICK * CAP);
  for (int i0 = 0; i0 < have; i0 += 64) {
    const int i = i0 + lane;
    const u64 s = i < have ? sc[wave * CAP + i] : 0;
    const u64 in = __ballot(s != 0 && (unsigned)(s >> 32) >= edge);
    int base = 0;
    if (lane == 0 && in) base = atomicAdd(&counts[BS_PICK], __popcll(in));
    base = __builtin_amdgcn_readfirstlane(base);
    if ((in >> lane) & 1) {
      const int place = base + __popcll(in & ((1ull << lane) - 1));
      fs[place] = s;
      fi[place] = ix[wave * CAP + i];
    }
  }
  __syncthreads();
  const int m = counts[BS_PICK];
  if (threadIdx.x < 4) fs[m + threadIdx.x] = 0;             // read four at a time; 0 is behind every score
  __syncthreads();
  for (int i = threadIdx.x; i < m; i += STEP) {
    const u64 s = fs[i];
    const unsigned at = fi[i];
    int rank = 0;
#pragma unroll 2
    for (int j = 0; j < m; j += 4) {
      const ulonglong2 p = *(const ulonglong2*)&fs[j], q = *(const ulonglong2*)&fs[j + 2];
      const uint4 x = *(const uint4*)&fi[j];
      rank += ScoreList::before(p.x, x.x, s, at) + ScoreList::before(p.y, x.y, s, at) + ScoreList::before(q.x, x.z, s, at) +
              ScoreList::before(q.y, x.w, s, at);
    }
    if (rank < n_out) {
      const int64_t o = (int64_t)seq * n_out + rank;
      const unsigned beam = at / (unsigned)vocab;
      out_scores[o] = (float)score_value(s);
      out_parents[o] = (int32_t)beam;
      out_tokens[o] = (int32_t)(at - beam * (unsigned)vocab);
    }
  }
}

// Logits per lane of the first launch: as many as leave a wave for most compute units, as fewer and longer lists serve the second launch (4 rows of 128256:
// 8, 16, 32 logits 14.0, 12.4, 12.0 us; 192 rows of 100003: 16, 32, 64 logits 38.7, 32.4, 32.6).
inline int beam_width(int64_t rows, int vocab) {
  for (int e = 64; e > 8; e /= 2)
    if (rows * ((vocab + 64 * e - 1) / (64 * e)) >= 200) return e;
  return 8;
}
inline int beam_parts(int64_t rows, int vocab) {
  const int part = BS_WAVES * 64 * beam_width(rows, vocab);
  return (int)(((int64_t)vocab + part - 1) / part);
}

inline size_t beam_workspace(int64_t rows, int vocab, int n_out) {
  const size_t all = (size_t)rows * beam_parts(rows, vocab);
  return (all * n_out * sizeof(u64) + 255) / 256 * 256 + all * sizeof(BeamPart);
}

inline hipError_t launch_beam_select(const float* logits, int64_t ld, const float* scores, int n_seqs, int beams, int vocab, int n_out, float* out_scores,
                                     int32_t* out_parents, int32_t* out_tokens, char* ws, hipStream_t st) {
  const int64_t rows = (int64_t)n_seqs * beams;
  const int parts = beam_parts(rows, vocab), width = beam_width(rows, vocab);
  u64* list = (u64*)ws;
  BeamPart* info = (BeamPart*)(ws + ((size_t)rows * parts * n_out * sizeof(u64) + 255) / 256 * 256);
#define ARMT_BS(E) beam_scan_kernel<E><<<(unsigned)(rows * parts), BS_WAVES * 64, 0, st>>>(logits, ld, beams, vocab, n_out, parts, list, info)
  if (width == 64) ARMT_BS(64);
  else if (width == 32) ARMT_BS(32);
  else if (width == 16) ARMT_BS(16);
  else ARMT_BS(8);
#undef ARMT_BS
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int lists = BS_PICK * (BS_CAP + 4) * 12, lds = lists + ((64 + beams * 24 + 15) & ~15) + lists;      // under 64 KB for BS_BEAMS beams
  beam_pick_kernel<<<n_seqs, BS_PICK * 64, lds, st>>>(list, info, scores, beams, vocab, n_out, parts, out_scores, out_parents, out_tokens);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------ states
// dst[s][b] = src[s][parents[s][b]] for every state (a row of bytes per beam).  A thread holds one column (UNIT bytes) of all of a sequence's
// beams in registers between its loads and its stores, so that dst may be src, and rows that stay where they are then cost
// nothing.  A parent of several beams is read for each, but by the same threads at once: HBM sees it once.  Bytes bound it; stores past the L2 leave it to the parents that are read again
// (13 beams of 7 MB: 34.6 -> 24.6 us, 8 beams of 50 MB 120 -> 112).
constexpr int BR_STATES = 8;

struct BeamState { const char* src; char* dst; int64_t row_bytes, src_stride, dst_stride; int first_block, cols; };
struct BeamStates { BeamState s[BR_STATES]; int n; };

typedef unsigned br16 __attribute__((ext_vector_type(4), aligned(4)));       // 16 and 8 bytes at any multiple of four
typedef unsigned br8 __attribute__((ext_vector_type(2), aligned(4)));

// Rows that a beam continues, by beam; a beam that stays where it is takes the row of one that does not, which is read anyway.
template <int KMAX, typename U>
__device__ __forceinline__ void reorder_column(const char* src, char* dst, int64_t src_stride, int64_t dst_stride, const int32_t* __restrict__ par, int beams,
                                               bool in_place, int moved) {
  U v[KMAX];
#pragma unroll
  for (int k = 0; k < KMAX; ++k) {
    const int j = min(k, beams - 1), p = min(max(par[j], 0), beams - 1);
    v[k] = *(const U*)(src + (in_place && p == j ? moved : p) * src_stride);
  }
#pragma unroll
  for (int k = 0; k < KMAX; ++k) {
    const int p = k < beams ? min(max(par[k], 0), beams - 1) : k;
    if (k < beams && !(in_place && p == k)) __builtin_nontemporal_store(v[k], (U*)(dst + k * dst_stride));
  }
}

// grid: all states' blocks (a sequence's columns side by side), block: 256.
template <int KMAX, typename U>
__global__ __launch_bounds__(256) void beam_reorder_kernel(BeamStates st, const int32_t* __restrict__ parents, int beams) {
  int i = 0;
  while (i + 1 < st.n && (int)blockIdx.x >= st.s[i + 1].first_block) ++i;
  const BeamState& t = st.s[i];
  const int b = blockIdx.x - t.first_block, seq = b / t.cols;
  const int64_t col = ((int64_t)(b - seq * t.cols) * 256 + threadIdx.x) * (int64_t)sizeof(U);
  const int32_t* par = parents + (int64_t)seq * beams;
  const bool in_place = t.src == t.dst;
  int moved = -1;
  for (int k = 0; k < beams; ++k) {
    const int p = min(max(par[k], 0), beams - 1);
    if (!in_place || p != k) moved = p;
  }
  if (moved < 0) return;
  const char* src = t.src + (int64_t)seq * beams * t.src_stride + col;
  char* dst = t.dst + (int64_t)seq * beams * t.dst_stride + col;
  if (col + (int64_t)sizeof(U) <= t.row_bytes) reorder_column<KMAX, U>(src, dst, t.src_stride, t.dst_stride, par, beams, in_place, moved);
  else if constexpr (sizeof(U) > 4) {                // the last, shorter piece of a row
    for (int64_t x = 0; x < t.row_bytes - col; x += 4)
      reorder_column<KMAX, unsigned>(src + x, dst + x, t.src_stride, t.dst_stride, par, beams, in_place, moved);
  }
}

template <typename U>
hipError_t launch_beam_reorder_as(const BeamStates& st, int64_t grid, const int32_t* parents, int beams, hipStream_t stream) {
  if (beams <= 4) beam_reorder_kernel<4, U><<<(unsigned)grid, 256, 0, stream>>>(st, parents, beams);
  else if (beams <= 8) beam_reorder_kernel<8, U><<<(unsigned)grid, 256, 0, stream>>>(st, parents, beams);
  else if (beams <= 16) beam_reorder_kernel<16, U><<<(unsigned)grid, 256, 0, stream>>>(st, parents, beams);
  else if (beams <= 32) beam_reorder_kernel<32, U><<<(unsigned)grid, 256, 0, stream>>>(st, parents, beams);
  else if constexpr (sizeof(U) <= 8) beam_reorder_kernel<64, U><<<(unsigned)grid, 256, 0, stream>>>(st, parents, beams);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

// A thread's column is 16 bytes (8 for more than 32 beams: 64 of 16 would fill the registers) where all addresses and sizes are multiples of four,
// else 2 or 1.
inline int beam_reorder_unit(const BeamStates& st, int beams) {
  uint64_t all = 0;
  for (int i = 0; i < st.n; ++i)
    all |= (uint64_t)(uintptr_t)st.s[i].src | (uint64_t)(uintptr_t)st.s[i].dst | (uint64_t)st.s[i].row_bytes | (uint64_t)st.s[i].src_stride |
           (uint64_t)st.s[i].dst_stride;
  return all & 1 ? 1 : all & 2 ? 2 : beams > 32 ? 8 : 16;
}

// Fills in first_block and cols; the blocks of the launch.
inline int64_t beam_reorder_blocks(BeamStates& st, int n_seqs, int unit) {
  int64_t grid = 0;
  for (int i = 0; i < st.n; ++i) {
    const int64_t cols = (st.s[i].row_bytes + 256 * unit - 1) / (256 * unit);
    if (cols > kMaxBlocks / n_seqs || grid + cols * n_seqs > kMaxBlocks) return -1;
    st.s[i].first_block = (int)grid;
    st.s[i].cols = (int)cols;
    grid += cols * n_seqs;
  }
  return grid;
}

inline hipError_t launch_beam_reorder(const BeamStates& st, int64_t grid, int unit, const int32_t* parents, int beams, hipStream_t stream) {
  if (unit == 16) return launch_beam_reorder_as<br16>(st, grid, parents, beams, stream);
  if (unit == 8) return launch_beam_reorder_as<br8>(st, grid, parents, beams, stream);
  if (unit == 2) return launch_beam_reorder_as<unsigned short>(st, grid, parents, beams, stream);
  return launch_beam_reorder_as<unsigned char>(st, grid, parents, beams, stream);
}

}  // namespace armt
