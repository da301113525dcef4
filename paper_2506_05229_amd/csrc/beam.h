// Beam search: the best continuations of every sequence over its beams and the vocabulary, and the gathering of the beams' states.
#pragma once

#include "common.h"

namespace armt {

// ------------------------------------------------------------------------------------------------ selection
// score(b, v) = scores[b] + x[b][v] - log sum_v' exp(x[b][v']); the n_out best of a sequence's beams x vocab, ties to the lowest b vocab + v.
// First launch: every workgroup reads its part of one row of logits once, its four waves a quarter each; lanes keep a running maximum and sum,
// and the wave the n_out best of what it has seen, sorted over its lanes (lane i: the i-th), so that a new value costs one comparison unless it
// belongs among them.  Second launch: one workgroup per sequence joins the parts.  Reading the logits once bounds the large cases;
// the small ones are two launches' latency.
//
// Inside a row the order of the scores is that of the logits, so the lists hold 64-bit keys: the logit in an order-preserving form above the complement
// of its index.  Scores of different rows are compared in 64 bits; the sums are of fp32 exponentials (random errors of 2^-24 each), added in fp32 per lane and in 64
// bits across lanes.
constexpr int BS_MAX = 64;             // n_out: a list lies over the lanes of one wave
constexpr int BS_WAVES = 4;
constexpr int BS_E = 8;                // logits per lane and step

struct BeamPart { double sum; float top; int pad; };      // of one workgroup's part of a row: sum of exp(x - top)

// A logit as it is taken: no NaN (the lowest), no +inf (the largest finite number), no -0.
__device__ __forceinline__ float beam_logit(float x) { return x != x ? -INFINITY : fminf(x, 3.402823466e+38f) + 0.f; }
__device__ __forceinline__ unsigned beam_order(float x) {
  const unsigned u = __float_as_uint(x);
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

// grid: rows x parts, block: 256.  list: [rows][parts][n_out], info: [rows][parts].
__global__ __launch_bounds__(BS_WAVES * 64) void beam_scan_kernel(const float* __restrict__ logits, int64_t ld, int vocab, int n_out, int parts,
                                                                   int per_wave, u64* __restrict__ list, BeamPart* __restrict__ info) {
  struct alignas(4) Four { float v[4]; };
  __shared__ u64 keys[BS_WAVES * BS_MAX];
  __shared__ float tops[BS_WAVES];
  __shared__ double sums[BS_WAVES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.x / parts, part = blockIdx.x - row * parts;
  const float* x = logits + (int64_t)row * ld;
  const int64_t lo = min((int64_t)(part * BS_WAVES + wave) * per_wave, (int64_t)vocab), hi = min(lo + per_wave, (int64_t)vocab);
  constexpr float LOG2E = 1.4426950408889634f;
  float top = -3.402823466e+38f, sum = 0.f, edge = -INFINITY;      // edge, edge_key: what a value has to reach to be among the best
  u64 edge_key = 0;
  KeyList best{0};
  for (int64_t at = lo; at < hi; at += 64 * BS_E) {
    float v[BS_E];
    if (at + 64 * BS_E <= hi) {
#pragma unroll
      for (int g = 0; g < BS_E / 4; ++g) {
        const Four f = *(const Four*)(x + at + g * 256 + lane * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[g * 4 + e] = f.v[e];
      }
    } else {
#pragma unroll
      for (int g = 0; g < BS_E / 4; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t i = at + g * 256 + lane * 4 + e;
          v[g * 4 + e] = i < hi ? x[i] : -INFINITY;
        }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < BS_E; ++e) {
      v[e] = beam_logit(v[e]);
      mx = fmaxf(mx, v[e]);
    }
    const float t = fmaxf(top, mx);
    sum *= __builtin_amdgcn_exp2f((top - t) * LOG2E);
#pragma unroll
    for (int e = 0; e < BS_E; ++e) sum += __builtin_amdgcn_exp2f((v[e] - t) * LOG2E);
    top = t;
    const u64 near = __ballot(mx >= edge);
    if (__popcll(near) >= n_out) {       // many at once, as in the first step: a value that n_out lanes' maxima reach bounds the n_out-th best from below
      const unsigned o = beam_order(mx);
      unsigned low = 0;
      for (int b = 31; b >= 12; --b) {
        const unsigned mid = low | (1u << b);
        if (__popcll(__ballot(o >= mid)) >= n_out) low = mid;
      }
      if (low > beam_order(-INFINITY)) edge = fmaxf(edge, beam_value(low));
    }
    if (near) {
#pragma unroll
      for (int e = 0; e < BS_E; ++e) {
        const int64_t i = at + (e / 4) * 256 + lane * 4 + e % 4;
        const u64 key = i < hi ? beam_key(v[e], (int)i) : 0;
        u64 in = __ballot(v[e] >= edge && key > edge_key);
        while (in) {
          const u64 k = read_lane(key, __ffsll(in) - 1);
          best.insert(k);
          in &= in - 1;
          const u64 last = read_lane(best.key, n_out - 1);
          if (last) {
            edge_key = last;
            edge = beam_value((unsigned)(last >> 32));
            in &= __ballot(key > last);
          }
        }
      }
    }
  }
  // ---- the wave's sum against its maximum, the workgroup's list: a key's rank is the number of larger ones
  const float wtop = wave_max(top);
  double s = (double)sum * exp((double)top - (double)wtop);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, kWave);
  if (lane == 0) { tops[wave] = wtop; sums[wave] = s; }
  if (lane < n_out) keys[wave * n_out + lane] = best.key;
  __syncthreads();
  const int n = BS_WAVES * n_out;
  u64* dst = list + (int64_t)blockIdx.x * n_out;
  if (threadIdx.x < n) {
    const u64 mine = keys[threadIdx.x];
    int rank = 0;
    for (int i = 0; i < n; ++i) rank += keys[i] > mine || (keys[i] == mine && i < (int)threadIdx.x);      // equal keys: nothing (0)
    if (rank < n_out) dst[rank] = mine;
  }
  if (threadIdx.x == 0) {
    float t = tops[0];
    for (int i = 1; i < BS_WAVES; ++i) t = fmaxf(t, tops[i]);
    double all = 0.0;
    for (int i = 0; i < BS_WAVES; ++i) all += sums[i] * exp((double)tops[i] - (double)t);
    info[blockIdx.x] = BeamPart{all, t, 0};
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

// grid: sequences, block: 256.  Wave w joins rows w, w + 4, ... of its sequence; the rows' lists then meet in wave 0.
__global__ __launch_bounds__(BS_WAVES * 64) void beam_pick_kernel(const u64* __restrict__ list, const BeamPart* __restrict__ info, const float* __restrict__ scores,
                                                                   int beams, int vocab, int n_out, int parts, float* __restrict__ out_scores,
                                                                   int32_t* __restrict__ out_parents, int32_t* __restrict__ out_tokens) {
  __shared__ u64 sc[BS_WAVES * BS_MAX];
  __shared__ unsigned ix[BS_WAVES * BS_MAX];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), seq = blockIdx.x;
  ScoreList mine{0, 0xffffffffu};
  for (int b = wave; b < beams; b += BS_WAVES) {
    const int64_t row = (int64_t)seq * beams + b;
    const BeamPart* pi = info + row * parts;
    const u64* pl = list + row * parts * n_out;
    float top = -3.402823466e+38f;
    for (int i = lane; i < parts; i += 64) top = fmaxf(top, pi[i].top);
    top = wave_max(top);
    double sum = 0.0;
    for (int i = lane; i < parts; i += 64) sum += pi[i].sum * exp((double)pi[i].top - (double)top);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, kWave);
    const float before = scores[row];
    const bool dead = !(before > -INFINITY && before < INFINITY) || !(sum > 0.0);       // no continuation of it has a score: its candidates are -inf, by index
    const double shift = log(sum);
    // the row's own best, by key
    KeyList best{0};
    if (!dead) {
      u64 edge = 0;
      for (int i0 = 0; i0 < parts * n_out; i0 += 64) {
        const u64 k = i0 + lane < parts * n_out ? pl[i0 + lane] : 0;
        u64 in = __ballot(k > edge);
        while (in) {
          best.insert(read_lane(k, __ffsll(in) - 1));
          edge = read_lane(best.key, n_out - 1);
          in &= in - 1;
          in &= __ballot(k > edge);
        }
      }
    }
    const bool have = dead ? lane < min(n_out, vocab) : lane < n_out && best.key != 0;
    const unsigned token = dead ? (unsigned)lane : ~(unsigned)best.key;
    const double value = dead ? -INFINITY : (double)before + (((double)beam_value((unsigned)(best.key >> 32)) - (double)top) - shift);
    const u64 s = have ? score_order(value) : 0;
    const unsigned at = (unsigned)b * (unsigned)vocab + token;
    // they come in falling order: stop at the first that is not among the wave's best
    for (int l = 0; l < n_out; ++l) {
      const u64 cs = read_lane(s, l);
      const unsigned ca = read_lane(at, l);
      if (cs == 0 || !ScoreList::before(cs, ca, read_lane(mine.score, n_out - 1), read_lane(mine.at, n_out - 1))) break;
      mine.insert(cs, ca);
    }
  }
  if (lane < n_out) { sc[wave * n_out + lane] = mine.score; ix[wave * n_out + lane] = mine.at; }
  __syncthreads();
  const int n = BS_WAVES * n_out;
  if (threadIdx.x >= n) return;
  const u64 s = sc[threadIdx.x];
  const unsigned a = ix[threadIdx.x];
  int rank = 0;
  for (int i = 0; i < n; ++i) rank += ScoreList::before(sc[i], ix[i], s, a) || (sc[i] == s && ix[i] == a && i < (int)threadIdx.x);
  if (rank < n_out && s != 0) {
    const int64_t o = (int64_t)seq * n_out + rank;
    out_scores[o] = (float)score_value(s);
    out_parents[o] = (int32_t)(a / (unsigned)vocab);
    out_tokens[o] = (int32_t)(a % (unsigned)vocab);
  }
}

// Workgroups of a row: enough to fill the chip with few rows, at least one step of every wave each.
inline int beam_parts(int64_t rows, int vocab) {
  const int64_t step = BS_WAVES * 64 * BS_E, most = (vocab + step - 1) / step, want = (1024 + rows - 1) / rows;
  return (int)(want < most ? want : most);
}

inline size_t beam_workspace(int64_t rows, int vocab, int n_out) {
  const size_t lists = (size_t)rows * beam_parts(rows, vocab) * n_out * sizeof(u64);
  return (lists + 255) / 256 * 256 + (size_t)rows * beam_parts(rows, vocab) * sizeof(BeamPart);
}

inline hipError_t launch_beam_select(const float* logits, int64_t ld, const float* scores, int n_seqs, int beams, int vocab, int n_out, float* out_scores,
                                     int32_t* out_parents, int32_t* out_tokens, char* ws, hipStream_t st) {
  const int64_t rows = (int64_t)n_seqs * beams;
  const int parts = beam_parts(rows, vocab);
  const int64_t cut = (int64_t)parts * BS_WAVES;
  const int per_wave = (int)((((int64_t)vocab + cut - 1) / cut + 3) / 4 * 4);
  u64* list = (u64*)ws;
  BeamPart* info = (BeamPart*)(ws + ((size_t)rows * parts * n_out * sizeof(u64) + 255) / 256 * 256);
  beam_scan_kernel<<<(unsigned)(rows * parts), BS_WAVES * 64, 0, st>>>(logits, ld, vocab, n_out, parts, per_wave, list, info);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  beam_pick_kernel<<<n_seqs, BS_WAVES * 64, 0, st>>>(list, info, scores, beams, vocab, n_out, parts, out_scores, out_parents, out_tokens);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------ states
// dst[s][b] = src[s][parents[s][b]] for every state (a row of bytes per beam).  A thread holds one column (UNIT bytes) of all of a sequence's
// beams in registers between its loads and its stores, so that dst may be src, and rows that stay where they are then cost
// nothing.  A parent of several beams is read for each, but by the same threads at once: HBM sees it once.  Bytes bound it.
constexpr int BR_STATES = 8;

struct BeamState { const char* src; char* dst; int64_t row_bytes, src_stride, dst_stride; int first_block, cols; };
struct BeamStates { BeamState s[BR_STATES]; int n; };

typedef unsigned br16 __attribute__((ext_vector_type(4), aligned(4)));       // 16 and 8 bytes at any multiple of four
typedef unsigned br8 __attribute__((ext_vector_type(2), aligned(4)));

template <int KMAX, typename U>
__device__ __forceinline__ void reorder_column(const char* src, char* dst, int64_t src_stride, int64_t dst_stride, const int32_t* __restrict__ par, int beams,
                                               bool in_place) {
  U v[KMAX];
#pragma unroll
  for (int k = 0; k < KMAX; ++k)
    if (k < beams) {
      const int p = min(max(par[k], 0), beams - 1);
      if (!(in_place && p == k)) v[k] = *(const U*)(src + p * src_stride);
    }
#pragma unroll
  for (int k = 0; k < KMAX; ++k)
    if (k < beams) {
      const int p = min(max(par[k], 0), beams - 1);
      if (!(in_place && p == k)) *(U*)(dst + k * dst_stride) = v[k];
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
  const char* src = t.src + (int64_t)seq * beams * t.src_stride + col;
  char* dst = t.dst + (int64_t)seq * beams * t.dst_stride + col;
  if (col + (int64_t)sizeof(U) <= t.row_bytes) reorder_column<KMAX, U>(src, dst, t.src_stride, t.dst_stride, par, beams, in_place);
  else if constexpr (sizeof(U) > 4) {                // the last, shorter piece of a row
    for (int64_t x = 0; x < t.row_bytes - col; x += 4)
      reorder_column<KMAX, unsigned>(src + x, dst + x, t.src_stride, t.dst_stride, par, beams, in_place);
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
    if (cols > 0x7fffffff / n_seqs || grid + cols * n_seqs > 0x7fffffff) return -1;
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
