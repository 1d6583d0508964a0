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
// the best of every stretch of a row without knowing its sum; it reads every logit once.  Scores are compared in double:
// two beams' scores are seldom closer than 1e-7 of each other, the float resolution, but they are not never.
// ---------------------------------------------------------------------------
constexpr int BS_PER = 32;                 // logits per lane
constexpr int BS_PIECE = 64 * BS_PER;      // logits per wavefront

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
  float2 *ms;                              // [rows][pieces] maximum and sum of exponentials of a stretch
  unsigned long long *keys;                // [rows][pieces][n_keep] its best logits, descending, 0 behind the last
  int pieces;
};

// One wavefront: a stretch of BS_PIECE logits.  What can be among its n_keep best lies in the n_keep lanes with the largest
// maxima, at or above the n_keep-th largest of them: that threshold leaves little more than n_keep logits to be ranked.
template <typename TL>
__global__ __launch_bounds__(64) void beam_stretch_kernel(BeamSelect a, BeamScratch w) {
  using V = Vec16<TL>;
  constexpr int N = V::N, NV = BS_PER / N;
  __shared__ unsigned long long s_list[BS_PIECE];
  const int row = blockIdx.y, piece = blockIdx.x, lane = threadIdx.x;
  if (a.finished && a.finished[row] != 0) return;
  const TL *src = (const TL *)a.logits + (size_t)row * a.row_stride;
  const int t0 = piece * BS_PIECE;
  const int K = a.n_keep;
  float x[BS_PER];
  int tok[NV];
  // 16-byte loads where the row's address allows them, single elements otherwise
  const bool wide = (reinterpret_cast<uintptr_t>(src) & 15) == 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int t = t0 + (i * 64 + lane) * N;
    tok[i] = t;
    if (wide && t + N <= a.vocab) {
      const V v = *reinterpret_cast<const V *>(src + t);
#pragma unroll
      for (int j = 0; j < N; ++j) x[i * N + j] = v.get(j);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) x[i * N + j] = t + j < a.vocab ? to_f32(src[t + j]) : -INFINITY;
    }
  }
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < BS_PER; ++i) {
    x[i] = x[i] == x[i] ? x[i] : -INFINITY;              // a NaN logit counts as -infinity
    m = fmaxf(m, x[i]);
  }
  unsigned long long best = 0;                           // the lane's best key: its first logit that equals the maximum
#pragma unroll
  for (int i = BS_PER - 1; i >= 0; --i)
    if (x[i] == m) best = logit_key(m, tok[i / N] + i % N);
  const float wm = wave_max(m);
  // sum of the exponentials; with an infinite maximum the infinite logits share the probability
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < BS_PER; ++i) sum += wm == INFINITY ? (x[i] == INFINITY ? 1.f : 0.f) : wm == -INFINITY ? 0.f : expf(x[i] - wm);
  sum = wave_sum(sum);
  const size_t at = (size_t)row * w.pieces + piece;
  if (lane == 0) w.ms[at] = make_float2(wm, sum);
  // threshold: the K-th largest of the lanes' best keys (0 where fewer lanes have any)
  int rank = 0;
#pragma unroll 8
  for (int l = 0; l < 64; ++l) rank += lane_value(best, l) > best;
  unsigned long long thr = 0;
  const unsigned long long kth = __ballot(rank == K - 1 && best != 0);
  if (kth) thr = lane_value(best, __ffsll((long long)kth) - 1);
  const float tv = thr ? unord32((unsigned)(thr >> 32)) : -INFINITY;
  int n = 0;
#pragma unroll
  for (int i = 0; i < BS_PER; ++i) {
    const unsigned long long key = logit_key(x[i], tok[i / N] + i % N);
    const bool in = x[i] >= tv && key >= thr && key != 0;
    const unsigned long long who = __ballot(in);
    if (who) {
      if (in) s_list[n + __popcll(who & ((1ull << lane) - 1))] = key;
      n += __popcll(who);
    }
  }
  __syncthreads();
  unsigned long long *out = w.keys + at * K;
  for (int c0 = 0; c0 < n; c0 += 64) {
    const unsigned long long mine = c0 + lane < n ? s_list[c0 + lane] : 0ull;
    int above = 0;
    for (int c = 0; c < n; ++c) above += s_list[c] > mine;
    if (mine && above < K) out[above] = mine;
  }
  for (int c = n + lane; c < K; c += 64) out[c] = 0;
}

// LDS written by some lanes of the wavefront is read by others
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// One workgroup per group: the rows' sums, then the best of all stretches' lists.  Its time is latency (a few dependent reads of
// some KB), so little of the lists is looked at.  The D-th entries of the lists bound the result: where R of them, R D >= n_keep, are
// at or before an entry, n_keep entries are; the R-th of the D-th entries, taken per wavefront, is such a bound, and only entries
// at or before the tightest one are collected and ranked, as a rule one to three times n_keep.
struct Cand { double score; unsigned long long key; int beam; };
__device__ __forceinline__ bool before(const Cand &a, const Cand &b) {      // a goes first
  if (a.score != b.score) return a.score > b.score;
  return a.beam != b.beam ? a.beam < b.beam : a.key > b.key;
}

constexpr int BF_WAVES = 8;
constexpr int BF_CAP = 1024;               // candidates collected at a time
constexpr int BF_AHEAD = 4;                // entries of a list that are read before they are asked for
__global__ __launch_bounds__(64 * BF_WAVES) void beam_final_kernel(BeamSelect a, BeamScratch w) {
  __shared__ double s_lse[kReorderBeams], s_score[kReorderBeams];
  __shared__ int s_inf[kReorderBeams];     // the row's maximum is infinite
  __shared__ Cand s_cand[BF_CAP], s_bound[BF_WAVES];
  __shared__ int s_n;
  constexpr int NT = 64 * BF_WAVES;
  const int grp = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int K = a.n_keep, B = a.n_beams, lists = B * w.pieces;
  auto ended = [&](int b) { return a.finished && a.finished[grp * B + b] != 0; };
  // the first entries of the thread's first list are on their way while the sums are computed
  unsigned long long ahead[BF_AHEAD] = {};
  const int b0 = min(tid / w.pieces, B - 1);
  const bool done0 = ended(b0);
  const unsigned long long *list0 = w.keys + ((size_t)grp * lists + min(tid, lists - 1)) * K;
  if (tid < lists && !done0) {
#pragma unroll
    for (int i = 0; i < BF_AHEAD; ++i) ahead[i] = list0[min(i, K - 1)];
  }
  for (int b = wave; b < B; b += BF_WAVES) {
    const float2 *ms = w.ms + ((size_t)grp * B + b) * w.pieces;
    const bool done = ended(b);
    float m = -INFINITY;
    double s = 0.0;
    if (!done) {
      for (int p = lane; p < w.pieces; p += 64) m = fmaxf(m, ms[p].x);
      m = wave_max(m);
      for (int p = lane; p < w.pieces; p += 64) {
        const float2 v = ms[p];
        if (v.x > -INFINITY) s += m == INFINITY ? (v.x == INFINITY ? (double)v.y : 0.0) : (double)(v.y * expf(v.x - m));
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    }
    if (lane == 0) {
      s_lse[b] = (m == INFINITY ? 0.0 : (double)m) + log(s);
      s_inf[b] = m == INFINITY;
      s_score[b] = (double)a.scores[grp * B + b];
    }
  }
  if (tid == 0) s_n = 0;
  __syncthreads();
  // entry i of list l; a score of -infinity where there is none (scores that are NaN are no continuations either)
  auto entry = [&](int l, int i) {
    Cand c = {-INFINITY, 0, l / w.pieces};
    const double s = s_score[c.beam];
    if (l == tid ? done0 : ended(c.beam)) {
      if (i == 0 && l - c.beam * w.pieces == 0) {
        c.key = logit_key(0.f, a.end_token);
        c.score = s;
      }
    } else {
      if (l == tid && i < BF_AHEAD) {
#pragma unroll
        for (int j = 0; j < BF_AHEAD; ++j)
          if (j == i) c.key = ahead[j];
      } else {
        c.key = w.keys[((size_t)grp * lists + l) * K + i];
      }
      const float x = unord32((unsigned)(c.key >> 32));
      if (c.key) c.score = s_inf[c.beam] ? (x == INFINITY ? s - s_lse[c.beam] : -INFINITY) : s + ((double)x - s_lse[c.beam]);
    }
    if (!(c.score > -INFINITY)) c = {-INFINITY, 0, c.beam};
    return c;
  };
  const Cand none = {-INFINITY, 0, 0x7FFFFFFF};
  Cand bound = none;
  {
    const int in_wave = min(64, lists - wave * 64), D = in_wave > 0 ? min(K, max(1, 4 * K / in_wave)) : 1, R = (K + D - 1) / D;
    Cand c = wave * 64 + lane < lists ? entry(wave * 64 + lane, D - 1) : none;
    int rank = 0;
    bool equal = false;
    if (in_wave > 0) {
#pragma unroll 8
      for (int l = 0; l < 64; ++l) {
        const double o = __longlong_as_double((long long)lane_value((unsigned long long)__double_as_longlong(c.score), l));
        rank += o > c.score;
        equal |= o == c.score && l != lane;
      }
      if (__any(equal && c.score > -INFINITY)) {
        rank = 0;
        for (int l = 0; l < 64; ++l) {
          const Cand o = {__longlong_as_double((long long)lane_value((unsigned long long)__double_as_longlong(c.score), l)),
                          lane_value(c.key, l), (int)__builtin_amdgcn_readlane((unsigned)c.beam, l)};
          rank += before(o, c);
        }
      }
    }
    if (lane == 0) s_bound[wave] = none;
    wave_sync();
    if (rank == R - 1 && c.score > -INFINITY) s_bound[wave] = c;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < BF_WAVES; ++i)
      if (before(s_bound[i], bound)) bound = s_bound[i];
  }
  int n;
  for (;;) {
    for (int l = tid; l < lists; l += NT)
      for (int i = 0; i < K; ++i) {
        const Cand c = entry(l, i);
        if (!(c.score > -INFINITY) || before(bound, c)) break;
        const int at = atomicAdd(&s_n, 1);                // where an entry lies does not matter: they are ranked below
        if (at < BF_CAP) s_cand[at] = c;
      }
    __syncthreads();
    n = s_n;
    const int have = min(n, BF_CAP);
    for (int i = tid; i < have; i += NT) {
      const Cand c = s_cand[i];
      int above = 0;
      for (int j = 0; j < have; ++j) above += before(s_cand[j], c);
      if (n <= BF_CAP) {
        if (above < K) {
          const size_t o = (size_t)grp * K + above;
          a.scores_out[o] = (float)c.score;
          a.beam_out[o] = c.beam;
          a.token_out[o] = (int32_t)(0xFFFFFFFFu - (unsigned)c.key);
        }
      } else if (above == K - 1) {
        s_bound[0] = c;                    // more than there is room for: the K-th of those at hand is a tighter bound (K < BF_CAP)
      }
    }
    if (n <= BF_CAP) break;
    __syncthreads();
    bound = s_bound[0];
    if (tid == 0) s_n = 0;
    __syncthreads();
  }
  for (int i = n + tid; i < K; i += NT) {
    const size_t o = (size_t)grp * K + i;
    a.scores_out[o] = -INFINITY;
    a.beam_out[o] = -1;
    a.token_out[o] = -1;
  }
}

BeamScratch beam_scratch(int rows, int vocab, int n_keep, void *base, size_t *bytes) {
  BeamScratch w;
  w.pieces = (vocab + BS_PIECE - 1) / BS_PIECE;
  const size_t lists = (size_t)rows * w.pieces, ms = align_up(lists * sizeof(float2), 256);
  w.ms = (float2 *)base;
  w.keys = (unsigned long long *)((char *)base + ms);
  *bytes = ms + align_up(lists * n_keep * 8, 256);
  return w;
}

// ---------------------------------------------------------------------------
// Reordering in place.  Every 16-byte piece of a row is moved between the beams of its group by one lane, which reads what all of them will
// receive before it writes any of it: no second buffer, no order between workgroups.  A beam that stays where it is moves nothing.
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
  const BeamScratch w = beam_scratch(a.n_groups * a.n_beams, a.vocab, a.n_keep, scratch, &bytes);
  const dim3 grid(w.pieces, a.n_groups * a.n_beams);
  if (a.logits_dtype == 0) hipLaunchKernelGGL(beam_stretch_kernel<float>, grid, dim3(64), 0, s, a, w);
  else hipLaunchKernelGGL(beam_stretch_kernel<bf16>, grid, dim3(64), 0, s, a, w);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(beam_final_kernel, dim3(a.n_groups), dim3(64 * BF_WAVES), 0, s, a, w);
  return hipGetLastError();
}

hipError_t launch_beam_reorder(void *const *k_layers, void *const *v_layers, int n_layers, int n_groups, int n_beams, int tail_stride,
                               int row_bytes, const int32_t *parent, const int32_t *seq_len, hipStream_t s) {
  const int chunks = row_bytes / 16;
  for (int l0 = 0; l0 < n_layers; l0 += kReorderLayers) {
    const int nl = std::min(kReorderLayers, n_layers - l0);
    ReorderArgs a;
    for (int i = 0; i < 2 * kReorderLayers; ++i) a.layer[i] = (i & 1 ? v_layers : k_layers)[l0 + std::min(i / 2, nl - 1)];
    // as many workgroups as the slab has work for; a few thousand in all are enough, the rest is walked
    const long need = ((long)tail_stride * chunks + 255) / 256, others = (long)n_groups * nl * 2;
    const dim3 grid((unsigned)std::max<long>(1, std::min<long>(need, 16384 / others)), n_groups, 2 * nl);
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
