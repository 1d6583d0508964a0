// A decoding step of several continuations, apart from its attention: the new tokens' queries and keys are normalised per
// head, rotated and put into the cache; the best continuations are chosen over beams and vocabulary; the beams' tails follow
// the chosen ones.
#include "common.h"
#include "kernels.h"
#include <algorithm>

namespace cb {

namespace {

// ---------------------------------------------------------------------------
// Per-head RMSNorm, rotation and cache append.  Bound by memory: every value is read once and written once.  One workgroup per
// row, so that the position, and with it the (cos, sin) values a lane needs, are the same for all of the heads it walks
// through.  A lane holds the 16-byte vectors at channel p N and dh/2 + p N of a head: both rotary orders then find their
// pairs within the lane, the adjacent one inside each vector, the half-split one across the two.
// 4099 rows of 64 + 2 x 8 heads of 128 with norms 33.7 us = 5.0 TB/s, the rate of a copy; 8 rows 3.2 us, an empty launch being 2.6; 4099 rows of 4 + 2 x 2
// float heads of 64 5.6 us.
// ---------------------------------------------------------------------------
template <typename T, int DH, bool HALF>
__global__ __launch_bounds__(256) void qkv_norm_rope_kernel(QkvRows a) {
  using V = Vec16<T>;
  constexpr int N = V::N, LPH = DH / (2 * N), HPP = 256 / LPH;       // lanes per head, heads per pass
  const int r = blockIdx.x, p = threadIdx.x % LPH, h0 = threadIdx.x / LPH;
  const int pos = a.row_pos[r];
  if (pos < 0 || pos >= a.max_tokens) return;
  const int64_t slot = a.cache_row[r];
  const bool store = slot >= 0 && slot < a.n_cache_rows;
  const float2 *tab = a.rope_tab + (size_t)pos * (DH / 2);
  float2 cs[N];
#pragma unroll
  for (int j = 0; j < N; ++j) cs[j] = tab[HALF ? p * N + j : (j < N / 2 ? 0 : DH / 4 - N / 2) + p * (N / 2) + j];
  const int n_heads = a.hq + (store ? 2 * a.hkv : 0);
  for (int hd = h0; hd < n_heads; hd += HPP) {
    const int kind = hd < a.hq ? 0 : hd < a.hq + a.hkv ? 1 : 2, i = kind == 0 ? hd : kind == 1 ? hd - a.hq : hd - a.hq - a.hkv;
    const T *src = kind == 0 ? (const T *)a.q + r * a.q_stride : kind == 1 ? (const T *)a.k + r * a.k_stride : (const T *)a.v + r * a.v_stride;
    T *dst = kind == 0 ? (T *)a.q_out + (size_t)r * a.hq * DH : (T *)(kind == 1 ? a.k_cache : a.v_cache) + (size_t)slot * a.hkv * DH;
    const V *s = reinterpret_cast<const V *>(src + i * DH) + p;
    V *d = reinterpret_cast<V *>(dst + i * DH) + p;
    V lo = s[0], hi = s[LPH];
    if (kind == 2) {
      d[0] = lo;
      d[LPH] = hi;
      continue;
    }
    float x[N], y[N];
#pragma unroll
    for (int j = 0; j < N; ++j) { x[j] = lo.get(j); y[j] = hi.get(j); }
    const T *gain = (const T *)(kind == 0 ? a.q_norm : a.k_norm);
    if (gain) {
      float ss = 0.f;
#pragma unroll
      for (int j = 0; j < N; ++j) ss += x[j] * x[j] + y[j] * y[j];
#pragma unroll
      for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor(ss, o, 64);
      const float inv = rsqrtf(ss / (float)DH + a.eps);
      const V gl = reinterpret_cast<const V *>(gain)[p], gh = reinterpret_cast<const V *>(gain)[p + LPH];
#pragma unroll
      for (int j = 0; j < N; ++j) { x[j] *= inv * gl.get(j); y[j] *= inv * gh.get(j); }
    }
    V ol, oh;                              // rounded once, after the rotation
    if (HALF) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        ol.set(j, x[j] * cs[j].x - y[j] * cs[j].y);
        oh.set(j, x[j] * cs[j].y + y[j] * cs[j].x);
      }
    } else {
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        ol.set(2 * j, x[2 * j] * cs[j].x - x[2 * j + 1] * cs[j].y);
        ol.set(2 * j + 1, x[2 * j] * cs[j].y + x[2 * j + 1] * cs[j].x);
        oh.set(2 * j, y[2 * j] * cs[N / 2 + j].x - y[2 * j + 1] * cs[N / 2 + j].y);
        oh.set(2 * j + 1, y[2 * j] * cs[N / 2 + j].y + y[2 * j + 1] * cs[N / 2 + j].x);
      }
    }
    d[0] = ol;
    d[LPH] = oh;
  }
}

// ---------------------------------------------------------------------------
// Beam selection.  score(beam, token) = scores[beam] + logit - log sum exp(logits of the beam); the order is by score, then lower beam,
// then larger logit, then lower token.  Within a beam the order is that of the logits, so that a first launch can keep
// the best of every stretch of a row without knowing its sum; it reads every logit once.  Scores are compared in double: as
// floats, different logits of a beam would tie.
// The sums of exponentials are float within a round of a lane and over the lanes of a wavefront, double over a lane's rounds and stretches, relative to
// references that move only when a logit exceeds them by 1.  Their relative error, in units of u = 2^-24: 31 additions, 6 levels of lanes twice, 2 for the
// exponential and for either join's factor, 4 roundings, and for every unit of distance between a logit and the references that it is taken relative to
// on its way 3 for the exponent (subtraction, product, constant) or 5 (a move is 1 at least: its factor's 2 as well).  Weighted by their
// probabilities the distances to the maximum average to at most ln vocab, the references' lag adds 2: (63 + 5 ln vocab) u, the same for a
// whole beam.
// ---------------------------------------------------------------------------
constexpr int BS_PER = 32;                 // logits per lane and round
constexpr int BS_CAP = 256;                // candidates a wavefront holds

// larger logit, then lower token <=> larger key; 0 is below every key (logits are neither NaN nor -infinity)
__device__ __forceinline__ unsigned ord32(float v) {
  const unsigned u = __float_as_uint(v + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unord32(unsigned o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
__device__ __forceinline__ unsigned long long logit_key(float v, int token) {
  return v == -INFINITY ? 0ull : ((unsigned long long)ord32(v) << 32) | (0xFFFFFFFFu - (unsigned)token);
}
__device__ __forceinline__ unsigned long long lane_value(unsigned long long v, int lane) {
  const unsigned lo = __builtin_amdgcn_readlane((unsigned)v, lane), hi = __builtin_amdgcn_readlane((unsigned)(v >> 32), lane);
  return ((unsigned long long)hi << 32) | lo;
}

struct BeamScratch {
  float2 *ms;                              // [rows][pieces] reference of a stretch (infinite as its maximum is) and sum of exponentials relative to it
  unsigned long long *keys;                // [rows][pieces][n_keep] its best logits, descending, 0 behind the last
  FastDiv by_lists, by_beams;              // lists of a group, beams of a group
  int pieces, rounds;                      // stretches of a row, each rounds * 64 * BS_PER logits
};

// LDS written by some lanes of the wavefront is read by others
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// One wavefront: a stretch of a row, 64 x BS_PER logits at a time (the next ones on their way meanwhile would take the registers of the wavefronts
// that hide the loads).  Bound by HBM where there are many rows, so the instructions per logit count: the running reference and sum of exponentials, kept per lane and joined at the end
// (a subtraction, a product, an exponential, an addition), and one comparison with the threshold.  The threshold comes from the first
// round: n_keep lanes have maxima at or above the n_keep-th largest of the lanes' maxima, so nothing below it is wanted.  What passes it goes to a list that is ranked at the end, or when it is half full, which
// tightens the threshold; where it overflows (many equal logits), the n_keep-th of those at hand does, and the round is gone through again.
// 256 rows of 64000 floats 17.2 us = 3.8 TB/s, 4 rows of 32000 6.2 us.
template <typename TL>
__global__ __launch_bounds__(64) void beam_stretch_kernel(BeamSelect a, BeamScratch w) {
  using V = Vec16<TL>;
  constexpr int N = V::N, NV = BS_PER / N;
  constexpr float kLog2e = 1.4426950408889634f;
  __shared__ unsigned long long s_list[BS_CAP];
  __shared__ __attribute__((aligned(16))) float s_x[64 * BS_PER];
  const int row = blockIdx.y, piece = blockIdx.x, lane = threadIdx.x, K = a.n_keep;
  if (a.finished && a.finished[row] != 0) return;
  const TL *src = (const TL *)a.logits + (size_t)row * a.row_stride;
  // Which lane adds up which tokens depends on the tokens alone, so that equal rows have equal sums wherever they start: 16-byte loads at any
  // alignment of the type (the hardware takes them), a row's last round element by element.
  const int t0 = piece * w.rounds * (64 * BS_PER) + lane * N;
  const int n_rounds = min(w.rounds, (a.vocab + 64 * BS_PER - 1) / (64 * BS_PER) - piece * w.rounds);
  V raw[NV];
  auto load = [&](int round) {
    const char *base = (const char *)src + (size_t)(piece * w.rounds + round) * (64 * BS_PER) * sizeof(TL);
    const int left = a.vocab - (piece * w.rounds + round) * (64 * BS_PER);
    if (left >= 64 * BS_PER) {             // the same for all lanes: no branch between the loads
#pragma unroll
      for (int i = 0; i < NV; ++i) __builtin_memcpy(&raw[i], base + (unsigned)((i * 64 + lane) * sizeof(V)), sizeof(V));
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const int t = (i * 64 + lane) * N + j;
          const float v = to_f32(*(const TL *)(base + (unsigned)(min(t, left - 1) * (int)sizeof(TL))));
          raw[i].set(j, t < left ? v : -INFINITY);
        }
    }
  };
  float ref = -INFINITY, tv = -INFINITY;
  double ls = 0.0;                         // of exp(logit - ref)
  unsigned long long thr = 0;
  int n = 0;
#pragma unroll 1
  for (int round = 0; round < n_rounds; ++round) {
    load(round);
    float x[BS_PER];
#pragma unroll
    for (int i = 0; i < BS_PER; ++i) x[i] = fmaxf(raw[i / N].get(i % N), -INFINITY);      // NaN counts as -infinity
    const int tr = t0 + round * 64 * BS_PER;
    auto token = [&](int i) { return tr + i / N * 64 * N + i % N; };
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < BS_PER; ++i) m = fmaxf(m, x[i]);
    if (__any(m > ref + 1.f)) {
      const float nr = m > ref + 1.f ? m : ref;
      ls = nr == ref ? ls : nr == INFINITY ? 0.0 : ls * (double)__builtin_amdgcn_exp2f((ref - nr) * kLog2e);
      ref = nr;
    }
    float part = 0.f;
    if (__any(ref == INFINITY)) {          // infinite logits share the probability: the sum is their number
#pragma unroll
      for (int i = 0; i < BS_PER; ++i)
        part += ref == INFINITY ? (x[i] == INFINITY ? 1.f : 0.f) : ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((x[i] - ref) * kLog2e);
    } else {
      const float base = ref == -INFINITY ? 0.f : ref;
#pragma unroll
      for (int i = 0; i < BS_PER; ++i) part += __builtin_amdgcn_exp2f((x[i] - base) * kLog2e);
    }
    ls += (double)part;
    if (round == 0) {
      int at_least = 0;                    // lanes whose maximum is no smaller
#pragma unroll 16
      for (int l = 0; l < 64; ++l) at_least += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(m), l)) >= m;
      tv = wave_max(at_least >= K ? m : -INFINITY);
    }
    const int kept = n;
    const bool last = round + 1 == n_rounds;
    bool over = __any(m >= tv) || last;
    // The logits at or above the threshold, one per lane at a time: which of its registers a lane takes differs, so they are read back
    // from LDS.  (Register by register, each behind a branch, this took 23000 clocks instead of 2000, mostly to fetch the code.)
    if (over) {
#pragma unroll
      for (int i = 0; i < BS_PER; i += 4) *reinterpret_cast<f32x4 *>(&s_x[i * 64 + lane * 4]) = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
    }
    while (over) {
      n = kept;
      unsigned todo = 0;
#pragma unroll
      for (int i = 0; i < BS_PER; ++i) todo |= x[i] >= tv ? 1u << i : 0u;
      while (__any(todo != 0)) {
        const int i = todo ? __ffs((int)todo) - 1 : 0;
        const unsigned long long key = logit_key(s_x[(i & ~3) * 64 + lane * 4 + (i & 3)], token(i));
        const bool in = todo != 0 && key != 0 && key >= thr;
        const unsigned long long who = __ballot(in);
        const int at = n + __popcll(who & ((1ull << lane) - 1));
        if (in && at < BS_CAP) s_list[at] = key;
        n += __popcll(who);
        todo &= todo - 1;
      }
      over = n > BS_CAP;
      if (!over && !last && n <= BS_CAP / 2) break;
      // rank what is at hand, four entries per lane
      wave_sync();
      const int have = min(n, BS_CAP);
      unsigned long long mine[BS_CAP / 64];
      int above[BS_CAP / 64];
#pragma unroll
      for (int j = 0; j < BS_CAP / 64; ++j) {
        mine[j] = j * 64 + lane < have ? s_list[j * 64 + lane] : 0;
        above[j] = mine[j] ? 0 : BS_CAP;
      }
      if (have <= 64) {
#pragma unroll 8
        for (int c = 0; c < have; ++c) above[0] += s_list[c] > mine[0];
      } else {
#pragma unroll 4
        for (int c = 0; c < have; ++c) {
          const unsigned long long k = s_list[c];
#pragma unroll
          for (int j = 0; j < BS_CAP / 64; ++j) above[j] += k > mine[j];
        }
      }
      wave_sync();
      if (!over) n = min(have, K);
#pragma unroll
      for (int j = 0; j < BS_CAP / 64; ++j) {
        if (!over && above[j] < K) s_list[above[j]] = mine[j];
        const unsigned long long kth = __ballot(above[j] == K - 1);
        if (kth) thr = lane_value(mine[j], __ffsll((long long)kth) - 1);
      }
      if (thr) tv = unord32((unsigned)(thr >> 32));
      wave_sync();
    }
  }
  const float wm = wave_max(ref);
  // a lane whose reference is not the infinite one of the row adds nothing to it
  float sum = wm == INFINITY ? (ref == INFINITY ? (float)ls : 0.f) : wm == -INFINITY ? 0.f : (float)ls * __builtin_amdgcn_exp2f((ref - wm) * kLog2e);
  sum = wave_sum(sum);
  const size_t at = (size_t)row * w.pieces + piece;
  if (lane == 0) w.ms[at] = make_float2(wm, sum);
  if (lane < K) w.keys[at * K + lane] = lane < n ? s_list[lane] : 0;
}

// One workgroup per group: the rows' sums, then the best of all stretches' lists.  Its time is latency, so there are few dependent steps: a
// thread reads its share of the lists' entries while the sums are computed, 64 groups of threads take the maxima of theirs, the
// n_keep-th largest of these is at or below n_keep entries and so a bound, and what reaches it (as a rule one to four times n_keep) is ranked by
// counting, several threads to an entry.  Entries are numbered by depth in their list, then stretch, then beam, so that each
// group of threads sees every beam.
// 6.2 us for 4 beams of 16 stretches and n_keep = 8, 7.9 for 8 beams of 16 and 16.
struct Cand { unsigned long long score, key; int beam; };      // score: order-preserving image of the double
__device__ __forceinline__ unsigned long long ord64(double v) {
  const unsigned long long u = (unsigned long long)__double_as_longlong(v + 0.0);
  return u >> 63 ? ~u : u | 0x8000000000000000ull;
}
__device__ __forceinline__ double unord64(unsigned long long o) {
  return __longlong_as_double((long long)(o >> 63 ? o & 0x7FFFFFFFFFFFFFFFull : ~o));
}
__device__ __forceinline__ bool before(const Cand &a, const Cand &b) {      // a goes first
  const bool tie = a.beam < b.beam || (a.beam == b.beam && a.key > b.key);
  return a.score > b.score || (a.score == b.score && tie);
}
__device__ __forceinline__ unsigned long long max64(unsigned long long a, unsigned long long b) { return a > b ? a : b; }

constexpr int BF_WAVES = 8, BF_THREADS = 64 * BF_WAVES;
constexpr int BF_PER = 8;                  // entries per thread and batch
constexpr int BF_CAP = 1024;               // candidates held, those kept from batches before among them
__global__ __launch_bounds__(BF_THREADS) void beam_final_kernel(BeamSelect a, BeamScratch w) {
  __shared__ double s_lse[kReorderBeams], s_score[kReorderBeams];
  __shared__ int s_state[kReorderBeams];   // 1: the row has infinite logits, 2: the beam has ended
  __shared__ unsigned long long s_so[BF_CAP], s_key[BF_CAP], s_max[64], s_keep_so[kBeamKeep], s_keep_key[kBeamKeep];
  __shared__ int s_beam[BF_CAP], s_keep_beam[kBeamKeep], s_n;
  const int grp = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int K = a.n_keep, B = a.n_beams;
  const unsigned lists = B * w.pieces;
  const long entries = (long)lists * K;
  unsigned long long key[BF_PER];
  int beam[BF_PER];
  auto fetch = [&](long e0) {
#pragma unroll
    for (int j = 0; j < BF_PER; ++j) {
      const long e = e0 + j * BF_THREADS + tid;
      key[j] = 0;
      beam[j] = 0;
      if (e0 + j * BF_THREADS < entries) {               // the same for all threads
        const unsigned ec = (unsigned)(e < entries ? e : entries - 1), depth = w.by_lists.div(ec), l = ec - depth * lists, p = w.by_beams.div(l);
        beam[j] = e < entries ? (int)(l - p * B) : -1;
        key[j] = w.keys[(((size_t)grp * B + (l - p * B)) * w.pieces + p) * K + depth];
        if (p == 0 && depth == 0) beam[j] |= 0x10000;    // the entry that stands for a beam that has ended
      }
    }
  };
  fetch(0);
  for (int b = wave; b < B; b += BF_WAVES) {
    const int row = grp * B + b;
    const float2 *ms = w.ms + (size_t)row * w.pieces;
    float2 v = lane < w.pieces ? ms[lane] : make_float2(-INFINITY, 0.f);
    const bool done = a.finished && a.finished[row] != 0;
    const float score = a.scores[row];
    float m = v.x;
    double s = 0.0;
    for (int p = 64 + lane; p < w.pieces; p += 64) m = fmaxf(m, ms[p].x);
    m = wave_max(m);
    const float base = fabsf(m) < INFINITY ? m : 0.f;
    for (int p = lane;; v = ms[p]) {
      if (v.x > -INFINITY) s += m == INFINITY ? (v.x == INFINITY ? (double)v.y : 0.0) : (double)v.y * (double)expf(v.x - base);
      if ((p += 64) >= w.pieces) break;
    }
    const float total = wave_sum((float)s);
    if (lane == 0) {
      s_lse[b] = (double)base + log((double)total);
      s_state[b] = done ? 2 : m == INFINITY;
      s_score[b] = fabsf(score) < INFINITY ? (double)score : -(double)INFINITY;      // not finite: a beam that is not there
    }
  }
  if (tid == 0) s_n = 0;
  __syncthreads();
  unsigned long long kth = 0;              // score of the n_keep-th best of the batches so far
  int kept = 0;
  for (long e0 = 0; e0 < entries; e0 += BF_THREADS * BF_PER) {
    if (e0 > 0) fetch(e0);
    unsigned long long so[BF_PER], best = 0;
#pragma unroll
    for (int j = 0; j < BF_PER; ++j) {
      so[j] = 0;                           // no continuation
      if (e0 + j * BF_THREADS < entries) {
        const bool first = beam[j] >= 0 && (beam[j] & 0x10000);
        const bool real = beam[j] >= 0;
        beam[j] &= 0xFFFF;
        const int b = real ? beam[j] : 0, state = s_state[b];
        const float x = unord32((unsigned)(key[j] >> 32));
        double score = s_score[b] + ((state == 1 ? 0.0 : (double)x) - s_lse[b]);
        bool in = real && key[j] != 0 && (state == 0 || (state == 1 && x == INFINITY));
        if (state == 2) {
          in = real && first;
          score = s_score[b];
          key[j] = logit_key(0.f, a.end_token);
        }
        if (in && score > -INFINITY) so[j] = ord64(score);
        best = max64(best, so[j]);
      }
    }
#pragma unroll
    for (int o = 1; o < BF_THREADS / 64; o <<= 1) best = max64(best, (unsigned long long)__shfl_xor((long long)best, o, 64));
    if (tid % (BF_THREADS / 64) == 0) s_max[tid / (BF_THREADS / 64)] = best;
    __syncthreads();
    {
      const unsigned long long mine = s_max[lane];
      int at_least = 0;
#pragma unroll 8
      for (int i = 0; i < 64; ++i) at_least += s_max[i] >= mine;
      unsigned long long c = at_least >= K ? mine : 0;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) c = max64(c, (unsigned long long)__shfl_xor((long long)c, o, 64));
      kth = max64(kth, c);
    }
    Cand bound = {kth, 0, 0x7FFFFFFF};     // entries with its score are at or before it
    for (;;) {
#pragma unroll
      for (int j = 0; j < BF_PER; ++j) {
        if (e0 + j * BF_THREADS < entries) {
          const bool in = so[j] != 0 && !before(bound, {so[j], key[j], beam[j]});
          const unsigned long long who = __ballot(in);
          if (who) {
            int at = 0;                    // where an entry lies does not matter: they are ranked below
            if (lane == 0) at = atomicAdd(&s_n, __popcll(who));
            at = __builtin_amdgcn_readfirstlane(at) + __popcll(who & ((1ull << lane) - 1));
            if (in && at < BF_CAP) {
              s_so[at] = so[j];
              s_key[at] = key[j];
              s_beam[at] = beam[j];
            }
          }
        }
      }
      __syncthreads();
      const int n = s_n, have = min(n, BF_CAP);
      const bool over = n > BF_CAP, last = e0 + BF_THREADS * BF_PER >= entries;
      // G threads count what goes before an entry
      int G = 1;
      while (G < 64 && 2 * G * have <= BF_THREADS) G *= 2;
      for (int i0 = 0; i0 < have; i0 += BF_THREADS / G) {
        const int i = i0 + tid / G;
        const int ic = min(i, have - 1);
        const Cand c = {s_so[ic], s_key[ic], s_beam[ic]};
        int above = 0;
#pragma unroll 2
        for (int o = tid % G; o < have; o += G) above += before({s_so[o], s_key[o], s_beam[o]}, c);
        for (int o = 1; o < G; o <<= 1) above += __shfl_xor(above, o, 64);
        if (i < have && above < K && tid % G == 0) {
          if (last && !over) {
            const size_t o = (size_t)grp * K + above;
            a.scores_out[o] = (float)unord64(c.score);
            a.beam_out[o] = c.beam;
            a.token_out[o] = (int32_t)(0xFFFFFFFFu - (unsigned)c.key);
          } else {
            s_keep_so[above] = c.score;
            s_keep_key[above] = c.key;
            s_keep_beam[above] = c.beam;
          }
        }
      }
      if (!over && last) {
        for (int i = have + tid; i < K; i += BF_THREADS) {
          const size_t o = (size_t)grp * K + i;
          a.scores_out[o] = -INFINITY;
          a.beam_out[o] = -1;
          a.token_out[o] = -1;
        }
        return;
      }
      __syncthreads();
      if (over) {                          // more than there is room for (many equal scores): the K-th of those at hand bounds more tightly
        bound = {s_keep_so[K - 1], s_keep_key[K - 1], s_keep_beam[K - 1]};
      } else {
        kept = min(have, K);
        for (int i = tid; i < kept; i += BF_THREADS) {
          s_so[i] = s_keep_so[i];
          s_key[i] = s_keep_key[i];
          s_beam[i] = s_keep_beam[i];
        }
        if (kept == K) kth = max64(kth, s_keep_so[K - 1]);
      }
      if (tid == 0) s_n = kept;
      __syncthreads();
      if (!over) break;
    }
  }
}

BeamScratch beam_scratch(int rows, int vocab, int n_keep, void *base, size_t *bytes) {
  // A round of 2048 logits per wavefront, as long as that makes no more wavefronts than the chip holds four to a SIMD: every
  // stretch costs a threshold, a ranking and a list.
  BeamScratch w;
  const int rounds = (vocab + 64 * BS_PER - 1) / (64 * BS_PER), most = std::max(1, 4096 / rows);
  w.rounds = (rounds + most - 1) / most;
  w.pieces = (rounds + w.rounds - 1) / w.rounds;
  const size_t lists = (size_t)rows * w.pieces, ms = align_up(lists * sizeof(float2), 256);
  w.ms = (float2 *)base;
  w.keys = (unsigned long long *)((char *)base + ms);
  *bytes = ms + align_up(lists * n_keep * 8, 256);
  return w;
}

// ---------------------------------------------------------------------------
// Reordering in place.  Every 16-byte piece of a row is moved between the beams of its group by one lane, which reads what all of them will
// receive before it writes any of it: no second buffer, no order between workgroups.  A beam that stays where it is moves nothing.
// 640 slabs of 80 rows of 2 KB 261 us = 5.0 TB/s, the rate of a copy; 32 slabs a layer as 16 beams 299, as 32 beams 356 (a lane holds a piece of
// every beam, so fewer wavefronts fit).
// ---------------------------------------------------------------------------
constexpr int kReorderLayers = 128;
struct ReorderArgs {
  void *layer[2 * kReorderLayers];
};

template <int NB>
__global__ __launch_bounds__(256) void beam_reorder_kernel(ReorderArgs a, int n_beams, int tail_stride, int row_chunks,
                                                           const int32_t *__restrict__ parent, const int32_t *__restrict__ seq_len) {
  const int grp = blockIdx.y;
  int from[NB], rows[NB], most = 0;
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    from[b] = b < n_beams ? parent[grp * n_beams + b] : b;
    const bool moves = from[b] >= 0 && from[b] < n_beams && from[b] != b;
    from[b] = moves ? from[b] : 0;
    rows[b] = !moves ? 0 : seq_len ? min(max(seq_len[grp * n_beams + from[b]], 0), tail_stride) : tail_stride;
    most = max(most, rows[b]);
  }
  const size_t slab = (size_t)tail_stride * row_chunks;
  f32x4 *base = (f32x4 *)a.layer[blockIdx.z] + (size_t)grp * n_beams * slab;
  const long total = (long)most * row_chunks;
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long)gridDim.x * 256) {
    const int t = (int)(i / row_chunks);
    f32x4 v[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
      if (t < rows[b]) v[b] = base[from[b] * slab + i];
#pragma unroll
    for (int b = 0; b < NB; ++b)
      if (t < rows[b]) base[b * slab + i] = v[b];
  }
}

}  // namespace

hipError_t launch_qkv_norm_rope(const QkvRows &a, hipStream_t s) {
#define CB_ROPE(T, DH)                                                                                               \
  do {                                                                                                               \
    if (a.rope_half) hipLaunchKernelGGL((qkv_norm_rope_kernel<T, DH, true>), dim3(a.n_rows), dim3(256), 0, s, a);    \
    else hipLaunchKernelGGL((qkv_norm_rope_kernel<T, DH, false>), dim3(a.n_rows), dim3(256), 0, s, a);               \
  } while (0)
  if (a.dtype == 0) {
    if (a.dh == 64) CB_ROPE(float, 64);
    else CB_ROPE(float, 128);
  } else {
    if (a.dh == 64) CB_ROPE(bf16, 64);
    else CB_ROPE(bf16, 128);
  }
#undef CB_ROPE
  return hipGetLastError();
}

size_t beam_select_bytes(int n_groups, int n_beams, int vocab, int n_keep) {
  size_t bytes;
  beam_scratch(n_groups * n_beams, vocab, n_keep, nullptr, &bytes);
  return bytes;
}

hipError_t launch_beam_select(const BeamSelect &a, void *scratch, hipStream_t s) {
  size_t bytes;
  BeamScratch w = beam_scratch(a.n_groups * a.n_beams, a.vocab, a.n_keep, scratch, &bytes);
  w.by_lists = FastDiv(a.n_beams * w.pieces);
  w.by_beams = FastDiv(a.n_beams);
  const dim3 grid(w.pieces, a.n_groups * a.n_beams);
  if (a.logits_dtype == 0) hipLaunchKernelGGL(beam_stretch_kernel<float>, grid, dim3(64), 0, s, a, w);
  else hipLaunchKernelGGL(beam_stretch_kernel<bf16>, grid, dim3(64), 0, s, a, w);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(beam_final_kernel, dim3(a.n_groups), dim3(BF_THREADS), 0, s, a, w);
  return hipGetLastError();
}

hipError_t launch_beam_reorder(void *const *k_layers, void *const *v_layers, int n_layers, int n_groups, int n_beams, int tail_stride,
                               int row_bytes, const int32_t *parent, const int32_t *seq_len, hipStream_t s) {
  const int chunks = row_bytes / 16;
  for (int l0 = 0; l0 < n_layers; l0 += kReorderLayers) {
    const int nl = std::min(kReorderLayers, n_layers - l0);
    ReorderArgs a;
    for (int i = 0; i < 2 * kReorderLayers; ++i) a.layer[i] = (i & 1 ? v_layers : k_layers)[l0 + std::min(i / 2, nl - 1)];
    // Whole slabs would need `need` workgroups each, tails fill them in part: small arrays take as many workgroups as the chip holds at a time (64
    // slabs of 24 of 128 rows 8.4 us, with 4096 workgroups 10.4), large ones enough to keep it busy to the end (640 of 80 of 96 rows
    // 261 us with 16384, 279 with 4096).  2048 against 16384, by whole slabs' workgroups: 4096 8.4 / 10.6 us, 7680 (24 of 128 rows) 9.6 / 17 and
    // 15.8 / 30, 8192 (64 of 128) 41 / 44; 15360 (40 of 96) 73 / 81, 16384 (64 of 128) 93 / 81, (8 of 512) 8 / 20, (400 of 512) 68 / 62, 30720 (40 of
    // 96) 133 / 122: beyond 8192 it depends on how full the tails are.
    const long need = ((long)tail_stride * chunks + 255) / 256, others = (long)n_groups * nl * 2;
    const long most = need * others <= 8192 ? 2048 : 16384;
    const dim3 grid((unsigned)std::max<long>(1, std::min<long>(need, most / others)), n_groups, 2 * nl);
#define CB_REORDER(NB) hipLaunchKernelGGL(beam_reorder_kernel<NB>, grid, dim3(256), 0, s, a, n_beams, tail_stride, chunks, parent, seq_len)
    if (n_beams <= 4) CB_REORDER(4);
    else if (n_beams <= 8) CB_REORDER(8);
    else if (n_beams <= 16) CB_REORDER(16);
    else if (n_beams <= 32) CB_REORDER(32);
    else CB_REORDER(64);
#undef CB_REORDER
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace cb
