// Attention of several continuations of one fused context (beams, samples, questions about the same documents): every
// new token of a continuation sees the whole context, which is stored once, and its continuation's own tail.
//     o = softmax([q Kc^T, q Kt^T] / sqrt(dh)) [Vc; Vt]
// The two parts are computed apart and joined through the softmax statistics: with m the maximum and l the sum of the
// exponentials of a part, o = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s.  The context's part takes the queries of ALL
// continuations together, so its keys and values are read once for all of them; a tail meets its own queries only.
//
// A single new token per continuation leaves few queries (continuations x query heads of a key/value head) against a
// long context: the bound is the bytes of the context, and what decides the time of a usual one (a few thousand tokens, 3 us
// of HBM time) is latency.  So the keys are cut into as many pieces as there are CUs and the pieces are joined by a second launch.
#include "common.h"
#include "kernels.h"
#include <algorithm>
#include <mutex>

namespace cb {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int SA_TILE = 32;               // keys per tile
constexpr float kLazyMax = 8.f;           // a running maximum may lag behind by a factor 2^8

typedef __attribute__((ext_vector_type(4))) short s16x4;

template <int N> __device__ __forceinline__ void vm_wait() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// maximum over the four 16-lane groups of a wavefront (the lanes that hold one query), without LDS
__device__ __forceinline__ float group_max(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  const float w = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(w), __float_as_uint(w), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float group_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// What one workgroup does: a block of queries against a piece of one key range (a group's context or a tail).
struct Item {
  const char *k, *v;        // rows of the range, this key/value head's first channel
  int m0, m_end;            // its flattened queries m = row * g + head in group, numbered from row0
  int row0;                 // first row of the range's queries
  int limit;                // context: its length; tail: rows of a slab
  bool tail;
  size_t slot;              // slot of its first query in the partial results, and from one query to the next
  int slot_step;
};

__device__ __forceinline__ Item item_of(const SharedAttn &a, int es, int qpb, int kvh, unsigned w, int *piece, int *pieces) {
  Item it;
  const bool tail = w >= (unsigned)a.ctx_items;
  const FastDiv dp = tail ? a.by_tail_pieces : a.by_ctx_pieces, db = tail ? a.by_tail_blocks : a.by_ctx_blocks;
  if (tail) w -= a.ctx_items;
  const unsigned unit = dp.div(w), slab = db.div(unit), blk = unit - slab * db.d;
  const int slab_rows = tail ? a.n_q : a.n_seqs * a.n_q, stride = tail ? a.tail_stride : a.ctx_stride;
  *pieces = dp.d;
  *piece = w - unit * dp.d;
  it.tail = tail;
  it.row0 = slab * slab_rows;
  it.m0 = blk * qpb;
  it.m_end = min(it.m0 + qpb, slab_rows * a.g);
  const size_t off = ((size_t)slab * stride * a.hkv + kvh) * (size_t)(a.dh * es);
  it.k = (const char *)(tail ? a.kt : a.kc) + off;
  it.v = (const char *)(tail ? a.vt : a.vc) + off;
  it.limit = tail ? a.tail_stride : a.n_groups == 1 ? a.ctx_len[0] : a.ctx_len[slab];
  const size_t query = ((size_t)kvh * a.rows + it.row0) * a.g + it.m0;
  it.slot = (tail ? a.tail_slot0 : 0) + query * dp.d + *piece;
  it.slot_step = dp.d;
  return it;
}

// keys that flattened query m of the item sees (0 for padding rows; *real: whether its result is wanted)
__device__ __forceinline__ int visible(const SharedAttn &a, const Item &it, int m, bool *real) {
  const int seen = m < it.m_end ? a.row_tail[it.row0 + a.by_g.div(m)] : -1;
  *real = seen >= 0;
  return seen < 0 ? 0 : it.tail ? min(seen, it.limit) : it.limit;
}

__device__ __forceinline__ int min16(int v) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v = min(v, __shfl_xor(v, o, 64));
  return v;
}
__device__ __forceinline__ int max16(int v) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v = max(v, __shfl_xor(v, o, 64));
  return v;
}

// First slot of a query's context pieces in a wide launch, and how many pieces its group's context has
__device__ __forceinline__ size_t wide_slot(const SharedAttn &a, int row, int kvh, int j, int *n) {
  const int grp = (int)a.by_group_rows.div(row), r0 = row - grp * (int)a.by_group_rows.d;
  *n = ((a.ctx_len[grp] + 63) / 64 + a.split_tiles - 1) / a.split_tiles;
  return (((size_t)grp * a.hkv + kvh) * a.ctx_rows + (size_t)r0 * a.g + j) * a.ctx_pieces;
}

// The end of a query in a launch that folds: joins the context's pieces to the tail's part (top, l, acc: NC blocks of 4 channels from
// channel ch on, 16 apart) and writes the result.
template <int NC, int DH>
__device__ __forceinline__ void fold_and_store(const SharedAttn &a, int row, int kvh, int j, int ch, float top, float l, f32x4 *acc) {
  int n;
  const size_t slot0 = wide_slot(a, row, kvh, j, &n);
  if (a.row_tail[row] < 0) n = 0;
  for (int p = 0; p < n; ++p) {
    const float2 ml = *reinterpret_cast<const float2 *>(a.part_ml + (slot0 + p) * 2);
    const float nt = fmaxf(top, ml.x), ref = nt == -INFINITY ? 0.f : nt;
    const float w0 = __builtin_amdgcn_exp2f(top - ref), w1 = __builtin_amdgcn_exp2f(ml.x - ref);
    const float *src = a.part_o + (slot0 + p) * DH + ch;
    top = nt;
    l = l * w0 + w1 * ml.y;
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[c] = acc[c] * w0 + w1 * *reinterpret_cast<const f32x4 *>(src + 16 * c);
  }
  const bool none = l == 0.f || a.row_tail[row] < 0;
  const float inv = none ? 0.f : 1.f / l;
  bf16 *dst = (bf16 *)a.o + ((size_t)row * a.hq + kvh * a.g + j) * DH + ch;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const f32x4 v = none ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[c] * inv;
    store4<bf16>(dst + 16 * c, v[0], v[1], v[2], v[3]);
  }
}

// a piece without keys: the merge passes it over
__device__ __forceinline__ void store_empty(const SharedAttn &a, const Item &it, int tid) {
  for (int qi = tid; it.m0 + qi < it.m_end; qi += blockDim.x) {
    const size_t slot = it.slot + (size_t)qi * it.slot_step;
    *reinterpret_cast<float2 *>(a.part_ml + slot * 2) = make_float2(-INFINITY, 0.f);
  }
}

// ---------------------------------------------------------------------------
// bf16.  Both products are computed transposed, S^T[key, query] = K Q^T and O^T[channel, query] += V^T P^T with
// v_mfma_f32_16x16x32_bf16, so that a lane holds values of one query (lane % 16) only, and the exponentiated scores are the
// second product's operand as they are: its contraction slots 8h .. 8h+7 (h = lane / 16) stand for the keys 4h .. 4h+3 and
// 16+4h .. 16+4h+3 that the first product leaves in the lane, and V is fetched in that order by the transposing LDS read.
// A workgroup takes QB blocks of 16 queries and KS tiles of 32 keys at a time, one wavefront for each pair: the code is that of one
// block, whatever QB.  (With two blocks unrolled in one wavefront eight beams over 3136 keys took 10.0 us instead of 8.7: each
// instruction of a short piece is executed once, so the time is that of fetching them.)  The QB wavefronts of a tile share its loads;
// the KS tiles' results are joined in LDS.
// Eight beams, 32 query heads over 8: 3136 keys 8.8 us (their bytes at the copy rate: 2.6); 32896 keys 31 us = 4.4 TB/s, 65536
// keys 56 us = 4.8 TB/s.  Several tokens each: 8 x 5 over 3136 keys 18.5 us, 4 x 5 of 64 heads over 8000 28.2, 4 requests of 4 x 16 of 56 heads over
// 2300 84.
// ---------------------------------------------------------------------------
constexpr int shared_ring_bytes(int dh, int ks, int st) { return ks * st * 2 * SA_TILE * dh * 2; }
// RAGGED: several new tokens per continuation (n_q > 1), which see different tail rows and may be padding.  Else everything in the item's range
// is seen by all of its queries.
// NT: keys and values are loaded non-temporally.
// FOLD: the tails beside a wide launch, whose context pieces are joined here.
template <int DH, int QB, int KS, int ST, bool RAGGED, bool NT, bool FOLD>
__global__ __launch_bounds__(64 * QB * KS, RAGGED ? 2 : 4) void shared_attn_bf16_kernel(SharedAttn a) {
  constexpr int ROWB = DH * 2, CH = DH / 8, RPI = 1024 / ROWB, TB = SA_TILE * ROWB, LPT = SA_TILE / RPI, LPW = 2 * LPT / QB;
  constexpr int NKS = DH / 32, NCB = DH / 16, NQ = 16 * QB;
  static_assert(LPW >= 1 && ST >= 1 && ST <= 4 && NCB % KS == 0, "loads, waits and channels are shared out evenly");
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, ln = lane & 15, h = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), qb = wave % QB, ks = wave / QB;
  const unsigned work = a.by_hkv.div(blockIdx.x);
  const int kvh = (int)(blockIdx.x - work * a.hkv), g = a.g;
  int piece, pieces;
  const Item it = item_of(a, 2, NQ, kvh, work, &piece, &pieces);

  // A context is seen whole by every query; which tail rows are, and whether a block is all padding, has to be read.
  const int m = it.m0 + qb * 16 + ln, mc = min(m, it.m_end - 1), r = (int)a.by_g.div(mc);
  int vis = it.limit, kv_len = it.limit, min_vis = it.limit;
  if (!RAGGED && it.tail) kv_len = min_vis = min(max(a.row_tail[it.row0], 0), it.limit);
  if (RAGGED) {
    bool real;
    vis = visible(a, it, m, &real);
    kv_len = 0;
    min_vis = 0x7FFFFFFF;
#pragma unroll
    for (int i = 0; i < NQ; i += 64) {
      const int v = visible(a, it, it.m0 + i + min(lane, NQ - 1), &real);
      kv_len = max(kv_len, v);
      min_vis = min(min_vis, real ? v : 0x7FFFFFFF);
    }
    kv_len = max16(kv_len);
    kv_len = __builtin_amdgcn_readfirstlane(max(max(kv_len, __shfl_xor(kv_len, 16, 64)), max(__shfl_xor(kv_len, 32, 64), __shfl_xor(kv_len, 48, 64))));
    min_vis = min16(min_vis);
    min_vis = __builtin_amdgcn_readfirstlane(min(min(min_vis, __shfl_xor(min_vis, 16, 64)), min(__shfl_xor(min_vis, 32, 64), __shfl_xor(min_vis, 48, 64))));
  }
  const int n_tiles = (kv_len + SA_TILE - 1) / SA_TILE;
  const int per = (int)(it.tail ? a.by_tail_pieces : a.by_ctx_pieces).div(n_tiles + pieces - 1);
  const int t_begin = piece * per, t_end = min(n_tiles, t_begin + per);
  if (t_begin >= t_end && !FOLD) {
    store_empty(a, it, tid);
    return;
  }

  // slot of 16-byte chunk c of row r in LDS: c ^ f(r); the 16 rows of a K fragment, and the 8 keys x 32 bytes that half a
  // wavefront's transposing read takes, then lie in different banks
  auto fk = [](int r) { return DH == 128 ? (r & 15) : ((r >> 1) & 7); };
  auto fv = [](int r) { return DH == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3); };
  const unsigned row_bytes = (unsigned)a.hkv * ROWB;
  char *ring = smem + ks * (ST * 2 * TB);
  const unsigned ring0 = (unsigned)(size_t)smem + ks * (ST * 2 * TB);
  // A lane's row of load i is i RPI + its first one, and its chunk differs from the first load's by an exclusive or with f(i RPI).
  const unsigned lrow = lane / CH, kcol = ((lane % CH) ^ fk(lrow)) * 16, vcol = ((lane % CH) ^ fv(lrow)) * 16;
  auto issue = [&](int t, int stage) {
    const int last = kv_len - 1 - t * SA_TILE;            // rows past the end repeat the last one
    const size_t tile0 = (size_t)t * (SA_TILE * (size_t)row_bytes);
    unsigned lr = lrow, kc = kcol, vc = vcol;             // what follows is computed here, not kept in registers across the loop
    asm volatile("" : "+v"(lr), "+v"(kc), "+v"(vc));
#pragma unroll
    for (int j = 0; j < LPW; ++j) {
      const int l = qb * LPW + j, i = l & (LPT - 1);
      const bool is_v = l >= LPT;
      const unsigned col = is_v ? vc ^ (fv(i * RPI) * 16) : kc ^ (fk(i * RPI) * 16);
      const char *src = (is_v ? it.v : it.k) + tile0 + (unsigned)(min((int)(i * RPI + lr), last) * row_bytes + col);
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src,
                                       (__attribute__((address_space(3))) void *)(ring + stage * 2 * TB + l * 1024), 16, 0, NT ? 2 : 0);
    }
  };
  const int n_it = (t_end - t_begin + KS - 1) / KS, n_mine = (t_end - t_begin - ks + KS - 1) / KS;
#pragma unroll
  for (int i = 0; i < (ST > 1 ? ST - 1 : 1); ++i)
    if (i < n_mine) issue(t_begin + i * KS + ks, i);

  bf16x8 qf[NKS];
  {
    const bf16 *src = (const bf16 *)a.q + ((size_t)(it.row0 + r) * a.hq + kvh * g + (mc - r * g)) * DH + 8 * h;
#pragma unroll
    for (int k = 0; k < NKS; ++k) qf[k] = *reinterpret_cast<const bf16x8 *>(src + 32 * k);
  }
  // chunks 4 k + h and 2 c + x differ from their first in bits of their own, so the swizzled addresses do by an exclusive or
  const unsigned ka0 = ring0 + ln * ROWB + ((h ^ fk(ln)) << 4), vkey = 4 * h + (ln >> 2);
  const unsigned va0 = ring0 + TB + vkey * ROWB + ((((ln & 3) >> 1) ^ fv(vkey)) << 4) + (ln & 1) * 8;

  f32x4 oacc[NCB];
#pragma unroll
  for (int c = 0; c < NCB; ++c) oacc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float scale = a.scale_log2e, lazy = kLazyMax / scale;
  float ref = -INFINITY, thr = -INFINITY, neg_mc = 0.f, row_sum = 0.f;
#pragma unroll
  for (int k = 0; k < NKS; ++k) asm volatile("" : "+v"(qf[k]));       // the queries are waited for here, not in the loop

  int stage = 0;
#pragma unroll 1
  for (int i = 0; i < n_it; ++i, stage = stage + 1 == ST ? 0 : stage + 1) {
    // this wavefront's share of tile i has landed (younger: those of the next ST - 2 tiles), then everybody's
    const int younger = min(ST - 2, n_mine - 1 - i);
    if (ST > 3 && younger >= 2) vm_wait<2 * LPW>();
    else if (ST > 2 && younger >= 1) vm_wait<LPW>();
    else vm_wait<0>();
    if (QB > 1) asm volatile("s_barrier" ::: "memory");
    // the stage of tile i - 1, which everybody has read, takes tile i + ST - 1
    if (ST > 1 && i + ST - 1 < n_mine) issue(t_begin + (i + ST - 1) * KS + ks, stage == 0 ? ST - 1 : stage - 1);
    if (i >= n_mine) continue;           // (with one stage: only in the last iteration)
    const int t0 = (t_begin + i * KS + ks) * SA_TILE;
    const unsigned so = stage * 2 * TB;
    const bool masked = t0 + SA_TILE > min_vis;           // some key of the tile is hidden from some query
    f32x4 sc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {                       // 16 keys at a time: with all 32 the registers of two workgroups would not fit
      bf16x8 kf[NKS];
      if constexpr (NKS == 4)
        asm volatile(
            "ds_read_b128 %0, %4 offset:%8\n\tds_read_b128 %1, %5 offset:%8\n\tds_read_b128 %2, %6 offset:%8\n\t"
            "ds_read_b128 %3, %7 offset:%8\n\ts_waitcnt lgkmcnt(0)"
            : "=&v"(kf[0]), "=&v"(kf[1]), "=&v"(kf[2]), "=&v"(kf[3])
            : "v"(ka0 + so), "v"((ka0 + so) ^ 64), "v"((ka0 + so) ^ 128), "v"((ka0 + so) ^ 192), "n"(kb * 16 * ROWB)
            : "memory");
      else
        asm volatile("ds_read_b128 %0, %2 offset:%4\n\tds_read_b128 %1, %3 offset:%4\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(kf[0]), "=&v"(kf[1])
                     : "v"(ka0 + so), "v"((ka0 + so) ^ 64), "n"(kb * 16 * ROWB)
                     : "memory");
#pragma unroll
      for (int k = 0; k < NKS; ++k) sc[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[k], qf[k], sc[kb], 0, 0, 0);
    }
    if (masked) {
      const int seen = RAGGED ? vis : kv_len;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (t0 + 16 * kb + 4 * h + e >= seen) sc[kb][e] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 4; ++e) mx = fmaxf(fmaxf(mx, sc[0][e]), sc[1][e]);
    mx = group_max(mx);
    if (__any(mx > thr)) {
      // exponents are taken relative to a reference that only moves when a score exceeds it by 2^8: P and the sums carry a
      // common factor, which costs no precision
      const float nr = fmaxf(ref, mx);
      const float alpha = nr > ref ? __builtin_amdgcn_exp2f((ref - nr) * scale) : 1.f;
      ref = nr;
      thr = nr + lazy;
      neg_mc = nr == -INFINITY ? 0.f : -nr * scale;
      row_sum *= alpha;
#pragma unroll
      for (int c = 0; c < NCB; ++c) oacc[c] *= alpha;
    }
    bf16x8 pf;
    float psum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e >> 2][e & 3], scale, neg_mc));
      psum += p;
      pf[e] = (bf16)p;                                    // the matrix cores' operand type, as in the fusing pass; the sum keeps the float.  It
                                                          // adds a second error as large as the output's own rounding: 0.0017 -> 0.0024 (2-norm)
    }
    row_sum += psum;
#pragma unroll
    for (int c0 = 0; c0 < NCB; c0 += 4) {
      union VF { s16x4 s[2]; bf16x8 b; unsigned w[4]; } vf[4];
      asm volatile(
          "ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:%12\n\t"
          "ds_read_b64_tr_b16 %2, %9\n\tds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
          "ds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:%12\n\t"
          "ds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:%12\n\ts_waitcnt lgkmcnt(0)"
          : "=&v"(vf[0].s[0]), "=&v"(vf[0].s[1]), "=&v"(vf[1].s[0]), "=&v"(vf[1].s[1]), "=&v"(vf[2].s[0]), "=&v"(vf[2].s[1]),
            "=&v"(vf[3].s[0]), "=&v"(vf[3].s[1])
          : "v"((va0 + so) ^ (c0 * 32)), "v"((va0 + so) ^ (c0 * 32 + 32)), "v"((va0 + so) ^ (c0 * 32 + 64)),
            "v"((va0 + so) ^ (c0 * 32 + 96)), "n"(16 * ROWB)
          : "memory");
      // A hidden key has p = 0, but 0 times a value that is not finite is not 0.
      bool bad = false;
      if (masked) {
        // rows past the end repeat the last one: cleared, so that nothing is added for them
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = t0 + 16 * (e >> 1) + 4 * h + 2 * (e & 1);
          const unsigned keep = key + 1 < kv_len ? 0xFFFFFFFFu : key < kv_len ? 0xFFFFu : 0u;
#pragma unroll
          for (int c = 0; c < 4; ++c) vf[c].w[e] &= keep;
        }
        if (RAGGED) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {                 // two bf16 a word: an exponent of all ones is infinity or NaN
              const unsigned word = vf[c].w[e];
              bad |= (word & 0x7F80u) == 0x7F80u || (word & 0x7F800000u) == 0x7F800000u;
            }
          bad = __any(bad);
        }
      }
      if (!RAGGED || __builtin_expect(!bad, 1)) {
#pragma unroll
        for (int c = 0; c < 4; ++c) oacc[c0 + c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[c].b, pf, oacc[c0 + c], 0, 0, 0);
      } else {
        // the same sums key by key, over the keys that a query sees; key k of the tile is held by lane group (k % 16) / 4
        unsigned ch = 4 * h;
        asm volatile("" : "+v"(ch));
#pragma unroll 1
        for (int k = 0; k < SA_TILE; ++k) {
          const int slot = (k >> 4) * 4 + (k & 3), from = ((k & 15) >> 2) * 16 + ln;
          const char *vrow = it.v + (size_t)min(t0 + k, kv_len - 1) * row_bytes;
          float p = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (e == slot) p = (float)pf[e];
          p = __shfl(p, from, 64);
          if (t0 + k < vis) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const bf16x4 v4 = *reinterpret_cast<const bf16x4 *>(vrow + (16 * (c0 + c) + ch) * 2);
#pragma unroll
              for (int e = 0; e < 4; ++e) oacc[c0 + c][e] = __builtin_fmaf(p, (float)v4[e], oacc[c0 + c][e]);
            }
          }
        }
        // these loads and the ring's share a counter: with everything landed the waits that follow are met already
        vm_wait<0>();
      }
    }
    if (ST == 1 && i + 1 < n_it) {                        // everybody has read the tile: its place takes the next one
      if (QB > 1) asm volatile("s_barrier" ::: "memory");
      if (i + 1 < n_mine) issue(t_begin + (i + 1) * KS + ks, 0);
    }
  }
  row_sum = group_sum(row_sum);
  float top = ref * scale;
  const size_t slot = it.slot + (size_t)(qb * 16 + ln) * it.slot_step;
  float *dst = a.part_o + slot * DH + 4 * h;
  if constexpr (KS == 1) {
    if (m >= it.m_end) return;
    if constexpr (FOLD) return fold_and_store<NCB, DH>(a, it.row0 + r, kvh, m - r * g, 4 * h, top, row_sum, oacc);
    if (h == 0) *reinterpret_cast<float2 *>(a.part_ml + slot * 2) = make_float2(top, row_sum);
#pragma unroll
    for (int c = 0; c < NCB; ++c) *reinterpret_cast<f32x4 *>(dst + 16 * c) = oacc[c];
  } else {
    // Join the KS tiles' results in the rings' place, in a fixed order, each wavefront NCB / KS channel blocks of its queries.
    // Blocks lie in register order, 1 KB each, so neither side's access has a bank conflict.
    f32x4 *s_o = reinterpret_cast<f32x4 *>(smem);
    float2 *s_ml = reinterpret_cast<float2 *>(smem + shared_ring_bytes(DH, KS, ST));
    __syncthreads();
#pragma unroll
    for (int c = 0; c < NCB; ++c) s_o[(wave * NCB + c) * 64 + lane] = oacc[c];
    if (h == 0) s_ml[wave * 16 + ln] = make_float2(top, row_sum);
    __syncthreads();
    if (m >= it.m_end) return;
    constexpr int CPW = NCB / KS;
    float2 ml[KS];
    top = -INFINITY;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      ml[s] = s_ml[(s * QB + qb) * 16 + ln];
      top = fmaxf(top, ml[s].x);
    }
    const float base = top == -INFINITY ? 0.f : top;
    f32x4 acc[CPW];
    float l = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const float w = __builtin_amdgcn_exp2f(ml[s].x - base);             // 0 for a wavefront that saw no key of the query
      l += w * ml[s].y;
#pragma unroll
      for (int c = 0; c < CPW; ++c) {
        const f32x4 v = s_o[((s * QB + qb) * NCB + ks * CPW + c) * 64 + lane];
        acc[c] = s == 0 ? w * v : acc[c] + w * v;
      }
    }
    if constexpr (FOLD) return fold_and_store<CPW, DH>(a, it.row0 + r, kvh, m - r * g, 16 * ks * CPW + 4 * h, top, l, acc);
    if (h == 0 && ks == 0) *reinterpret_cast<float2 *>(a.part_ml + slot * 2) = make_float2(top, l);
#pragma unroll
    for (int c = 0; c < CPW; ++c) *reinterpret_cast<f32x4 *>(dst + 16 * (ks * CPW + c)) = acc[c];
  }
}

// Joins the wavefronts' results of CW channels from ch0 on in LDS, in a fixed order, and writes them as the item's partial result.
// s_o: [wavefronts][queries][CW + 4]
template <int NW, int NQ, int DH, int CW>
__device__ __forceinline__ void join_and_store(const SharedAttn &a, const Item &it, const float *s_o, const float (*s_m)[NQ],
                                               const float (*s_l)[NQ], int ch0, int tid) {
  constexpr int CG = CW / 4, LD = CW + 4;
  for (int e = tid; e < NQ * CG; e += 64 * NW) {
    const int qi = e / CG, c = e - qi * CG;
    if (it.m0 + qi >= it.m_end) break;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, s_m[w][qi]);
    const float ref = top == -INFINITY ? 0.f : top;
    float l = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float wt = __builtin_amdgcn_exp2f(s_m[w][qi] - ref);          // 0 for a wavefront that saw no key of the query
      l += wt * s_l[w][qi];
      acc += wt * *reinterpret_cast<const f32x4 *>(s_o + ((size_t)w * NQ + qi) * LD + c * 4);
    }
    const size_t slot = it.slot + (size_t)qi * it.slot_step;
    if (c == 0 && ch0 == 0) *reinterpret_cast<float2 *>(a.part_ml + slot * 2) = make_float2(top, l);
    *reinterpret_cast<f32x4 *>(a.part_o + slot * DH + ch0 + c * 4) = acc;
  }
}

// ---------------------------------------------------------------------------
// float, v_mfma_f32_16x16x4_f32: the same items with 16 queries per workgroup and K, V straight from memory (a float model's
// caches fit L2).  The contraction index a lane supplies in MFMA s is 4 (lane / 16) + s for both products.  Four beams over 544 keys
// of the 4 x 64 model 5.8 us, over 8000 6.1; 8 x 64 tokens over 2000 keys 38, with 8 heads of 128 74.
// ---------------------------------------------------------------------------
constexpr int SF_NW = 4;
template <int DH>
__global__ __launch_bounds__(64 * SF_NW) void shared_attn_f32_kernel(SharedAttn a) {
  constexpr int NC = DH / 16;
  __shared__ __attribute__((aligned(16))) float s_o[SF_NW * 16 * (DH + 4)];
  __shared__ float s_m[SF_NW][16], s_l[SF_NW][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ln = lane & 15, h = lane >> 4;
  const unsigned work = a.by_hkv.div(blockIdx.x);
  const int kvh = (int)(blockIdx.x - work * a.hkv), g = a.g;
  int piece, pieces;
  const Item it = item_of(a, 4, 16, kvh, work, &piece, &pieces);
  const int m = it.m0 + ln, mc = min(m, it.m_end - 1), r = (int)a.by_g.div(mc);
  bool real;
  const int vis = visible(a, it, m, &real);
  const float *qrow = (const float *)a.q + ((size_t)(it.row0 + r) * a.hq + kvh * g + (mc - r * g)) * DH + 4 * h;
  f32x4 qf[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) qf[c] = *reinterpret_cast<const f32x4 *>(qrow + 16 * c);
  const int kv_len = __builtin_amdgcn_readfirstlane(max16(vis));
  const int min_vis = __builtin_amdgcn_readfirstlane(min16(real ? vis : 0x7FFFFFFF));
  const int n_tiles = (kv_len + SA_TILE - 1) / SA_TILE;
  const int per = (int)(it.tail ? a.by_tail_pieces : a.by_ctx_pieces).div(n_tiles + pieces - 1);
  const int t_begin = piece * per, t_end = min(n_tiles, t_begin + per);
  if (t_begin >= t_end) {
    store_empty(a, it, tid);
    return;
  }
  const size_t row_bytes = (size_t)a.hkv * DH * 4;
  f32x4 oacc[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) oacc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  float run_max = -INFINITY, run_sum = 0.f;
  for (int t = t_begin + wave; t < t_end; t += SF_NW) {
    const int t0 = t * SA_TILE;
    f32x4 sc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}}, kf[2][NC];
    float vf[2][4][NC];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const char *krow = it.k + (size_t)min(t0 + 16 * b + ln, kv_len - 1) * row_bytes + 16 * h;
#pragma unroll
      for (int c = 0; c < NC; ++c) kf[b][c] = *reinterpret_cast<const f32x4 *>(krow + 64 * c);
    }
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const char *vrow = it.v + (size_t)min(t0 + 16 * b + 4 * h + i, kv_len - 1) * row_bytes + 4 * ln;
#pragma unroll
        for (int c = 0; c < NC; ++c) vf[b][i][c] = *reinterpret_cast<const float *>(vrow + 64 * c);
      }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int b = 0; b < 2; ++b) sc[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[b][c][i], qf[c][i], sc[b], 0, 0, 0);
    float mx = -INFINITY;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sc[b][i] = t0 + 16 * b + 4 * h + i < vis ? sc[b][i] * a.scale_log2e : -INFINITY;
        mx = fmaxf(mx, sc[b][i]);
      }
    const float new_max = fmaxf(run_max, group_max(mx));
    const float ref = new_max == -INFINITY ? 0.f : new_max;
    const float alpha = exp2f(run_max - ref);
    float psum = 0.f;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sc[b][i] = exp2f(sc[b][i] - ref);
        psum += sc[b][i];
      }
    run_sum = run_sum * alpha + psum;
    run_max = new_max;
#pragma unroll
    for (int c = 0; c < NC; ++c) oacc[c] *= alpha;
    bool bad = false;
    if (t0 + SA_TILE > min_vis) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int c = 0; c < NC; ++c) bad |= !(fabsf(vf[b][i][c]) < INFINITY);
    }
    if (!__any(bad)) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int c = 0; c < NC; ++c) oacc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[b][i][c], sc[b][i], oacc[c], 0, 0, 0);
      continue;
    }
    // a hidden key has p = 0, but 0 times a value that is not finite is not 0: key by key, over the keys that a query sees
#pragma unroll 1
    for (int k = 0; k < SA_TILE; ++k) {
      float p = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i == (k >> 4) * 4 + (k & 3)) p = sc[i >> 2][i & 3];
      p = __shfl(p, ((k & 15) >> 2) * 16 + ln, 64);
      const char *vrow = it.v + (size_t)min(t0 + k, kv_len - 1) * row_bytes + 16 * h;
      if (t0 + k < vis) {
#pragma unroll
        for (int c = 0; c < NC; ++c) oacc[c] += p * *reinterpret_cast<const f32x4 *>(vrow + 64 * c);
      }
    }
  }
  run_sum = group_sum(run_sum);
#pragma unroll
  for (int c = 0; c < NC; ++c) *reinterpret_cast<f32x4 *>(&s_o[(wave * 16 + ln) * (DH + 4) + 16 * c + 4 * h]) = oacc[c];
  if (h == 0) {
    s_m[wave][ln] = run_max;
    s_l[wave][ln] = run_sum;
  }
  __syncthreads();
  join_and_store<SF_NW, 16, DH, DH>(a, it, s_o, s_m, s_l, 0, tid);
}

// Joins a query's partial results: the context's pieces, then the tail's.  A row that sees no key, and a padding row, is zero.
// DH / 4 lanes hold a query's channels; SG groups of them share its pieces (many pieces are walked at the latency of one load after the
// other otherwise: 26 pieces of 256 queries 16.5 us, 3.6 with SG = 8) and add up through LDS.
template <typename T, int DH, int SG>
__global__ __launch_bounds__(256) void shared_merge_kernel(SharedAttn a) {
  constexpr int CG = DH / 4, QPB = 256 / (CG * SG);       // queries per workgroup
  __shared__ float2 s_ml[SG > 1 ? QPB * SG : 1];
  __shared__ f32x4 s_acc[SG > 1 ? 256 : 1];
  const int g = a.g, tid = threadIdx.x, c = tid % CG, sg = tid / CG % SG, qi = tid / (CG * SG);
  const long query = (long)blockIdx.x * QPB + qi, all = (long)a.rows * a.hq;
  const long qc = query < all ? query : all - 1;
  const int r = (int)a.by_hq.div((unsigned)qc), hd = (int)qc - r * a.hq, kvh = (int)a.by_g.div(hd);
  const bool real = a.row_tail[r] >= 0;
  const size_t m = ((size_t)kvh * a.rows + r) * g + (hd - kvh * g);
  size_t slot0 = m * a.ctx_pieces;
  int n_ctx = a.ctx_pieces;
  if (a.wide) {                            // slots by group, only as many pieces as the group's context has
    slot0 = wide_slot(a, r, kvh, hd - kvh * g, &n_ctx);
  }
  const int n = real ? n_ctx + a.tail_pieces : 0;
  float top = -INFINITY, l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  // pieces sg, sg + SG, ..: four at a time, loaded before the first is used
  constexpr int U = 4;
  for (int p0 = sg; p0 < n; p0 += SG * U) {
    float2 ml[U];
    f32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int p = p0 + u * SG;
      ml[u] = make_float2(-INFINITY, 0.f);
      if (p < n) {
        const size_t slot = p < n_ctx ? slot0 + p : a.tail_slot0 + m * a.tail_pieces + (p - n_ctx);
        ml[u] = *reinterpret_cast<const float2 *>(a.part_ml + slot * 2);
        v[u] = *reinterpret_cast<const f32x4 *>(a.part_o + slot * DH + c * 4);      // of a piece without keys: not used
      }
    }
    float nt = top;
#pragma unroll
    for (int u = 0; u < U; ++u) nt = fmaxf(nt, ml[u].x);
    const float ref = nt == -INFINITY ? 0.f : nt, w0 = __builtin_amdgcn_exp2f(top - ref);
    top = nt;
    l *= w0;
    acc *= w0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool none = ml[u].x == -INFINITY && ml[u].y == 0.f;       // a piece without keys left nothing else
      const float w = __builtin_amdgcn_exp2f(ml[u].x - ref);
      if (!none) {
        l += w * ml[u].y;
        acc += w * v[u];
      }
    }
  }
  if constexpr (SG > 1) {
    if (c == 0) s_ml[qi * SG + sg] = make_float2(top, l);
    s_acc[tid] = acc;
    __syncthreads();
    if (sg != 0) return;
    float nt = -INFINITY;
#pragma unroll
    for (int u = 0; u < SG; ++u) nt = fmaxf(nt, s_ml[qi * SG + u].x);
    const float ref = nt == -INFINITY ? 0.f : nt;
    l = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < SG; ++u) {
      const float2 ml = s_ml[qi * SG + u];
      const float w = __builtin_amdgcn_exp2f(ml.x - ref);
      l += w * ml.y;
      acc += w * s_acc[(qi * SG + u) * CG + c];
    }
  }
  if (query >= all) return;
  if (!real || l == 0.f) {
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
    l = 1.f;
  }
  const float inv = 1.f / l;
  store4<T>((T *)a.o + ((size_t)r * a.hq + hd) * DH + c * 4, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
}

template <int DH, int QB, int KS, int ST, bool RAGGED, bool NT, bool FOLD>
hipError_t launch_one(const SharedAttn &a, unsigned grid, hipStream_t s) {
  constexpr int smem = shared_ring_bytes(DH, KS, ST) + QB * KS * 16 * 8;
  static_assert(shared_ring_bytes(DH, KS, ST) >= QB * KS * (DH / 16) * 1024 || KS == 1, "the join fits in the rings' place");
  static std::once_flag once;
  std::call_once(once, [] {
    (void)hipFuncSetAttribute(reinterpret_cast<const void *>(&shared_attn_bf16_kernel<DH, QB, KS, ST, RAGGED, NT, FOLD>),
                              hipFuncAttributeMaxDynamicSharedMemorySize, smem);
  });
  hipLaunchKernelGGL((shared_attn_bf16_kernel<DH, QB, KS, ST, RAGGED, NT, FOLD>), dim3(grid), dim3(64 * QB * KS), smem, s, a);
  return hipGetLastError();
}
template <int DH, int QB, int KS, int ST, bool RAGGED>
hipError_t launch_bf16(const SharedAttn &a, unsigned grid, hipStream_t s) {
  return a.fold ? launch_one<DH, QB, KS, ST, RAGGED, false, true>(a, grid, s) : launch_one<DH, QB, KS, ST, RAGGED, false, false>(a, grid, s);
}
template <int DH>
hipError_t launch_bf16_qb(const SharedAttn &a, unsigned grid, hipStream_t s) {
  // as many tiles at a time as the wavefronts leave; one new token: two workgroups to a CU, which hide each other's loads
  if (a.stream) switch (a.qb) {
      case 1: return launch_one<DH, 1, 4, 1, false, true, false>(a, grid, s);
      case 2: return launch_one<DH, 2, 4, 1, false, true, false>(a, grid, s);
      case 4: return launch_one<DH, 4, 2, 2, false, true, false>(a, grid, s);
    }
  if (a.n_q == 1) switch (a.qb) {
      case 1: return launch_bf16<DH, 1, 4, 1, false>(a, grid, s);
      case 2: return launch_bf16<DH, 2, 4, 1, false>(a, grid, s);
      case 4: return launch_bf16<DH, 4, 2, 2, false>(a, grid, s);
      default: return launch_bf16<DH, 8, 1, 4, false>(a, grid, s);
    }
  switch (a.qb) {
    case 1: return launch_bf16<DH, 1, 4, 2, true>(a, grid, s);
    case 2: return launch_bf16<DH, 2, 4, 2, true>(a, grid, s);
    case 4: return launch_bf16<DH, 4, 2, 4, true>(a, grid, s);
    default: return launch_bf16<DH, 8, 1, 4, true>(a, grid, s);
  }
}

template <typename T, int DH>
hipError_t launch_merge(const SharedAttn &a, hipStream_t s) {
  constexpr int SG = 256 / (DH / 4) < 8 ? 256 / (DH / 4) : 8;
  const long queries = (long)a.rows * a.hq;
  auto grid = [&](int sg) { const long per = 256 / (DH / 4 * sg); return dim3((unsigned)((queries + per - 1) / per)); };
  if (a.ctx_pieces + a.tail_pieces > 4) hipLaunchKernelGGL((shared_merge_kernel<T, DH, SG>), grid(SG), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((shared_merge_kernel<T, DH, 1>), grid(1), dim3(256), 0, s, a);
  return hipGetLastError();
}

int query_blocks(int dtype, long queries) {   // blocks of 16 queries that a workgroup takes
  return dtype == 0 || queries <= 16 ? 1 : queries <= 32 ? 2 : queries <= 64 ? 4 : 8;
}
int tiles_at_a_time(int dtype, int qb) { return dtype == 0 ? SF_NW : qb <= 2 ? 4 : 8 / qb; }

}  // namespace

// Pieces: as many workgroups as the chip holds at a time, no piece shorter than the tiles a workgroup takes at a time.  Tails are
// short as a rule, and how long is not known here, only how long they can be: a piece per 512 rows, within half of the workgroups.
static void plan(SharedAttn &a, int max_ctx, bool may_wide, bool must_wide) {
  const int g = a.g = a.hq / a.hkv;
  const long ctx_q = (long)a.n_seqs * a.n_q * g, tail_q = (long)a.n_q * g;
  a.rows = a.n_groups * a.n_seqs * a.n_q;
  a.qb = query_blocks(a.dtype, ctx_q);
  // Many queries against a long context are bound by the matrix cores, or by how often a tile is read from LDS: wavefronts that take 32
  // queries each then pay for a launch of their own, as the tails go on in this file's kernel.  64 query heads, one new token, this
  // kernel's single launch against the two: 128 queries a key/value head over 8000 / 16000 / 28000 keys 23 / 37 / 58 us against
  // 23 / 27 / 37; 64 queries over 16000 / 28000 keys 20 / 30 against 23 / 35; 512 (8 tokens each) over 2000 / 8000 keys
  // 23 / 48 against 31 / 37.  Every group is a launch, so several groups have to be worth it each.
  a.wide = may_wide && a.dtype != 0 && max_ctx > 0 && ctx_q > 48 &&
           (must_wide || (double)ctx_q * max_ctx >= (a.n_groups == 1 ? 1.6e6 : 4e6));
  a.fold = 0;
  if (a.wide) a.qb = query_blocks(a.dtype, tail_q);
  const int qpb = 16 * a.qb, step = SA_TILE * tiles_at_a_time(a.dtype, a.qb);
  a.ctx_blocks = (int)((ctx_q + qpb - 1) / qpb);
  a.tail_blocks = (int)((tail_q + qpb - 1) / qpb);
  const long kSlots = a.dtype != 0 && a.n_q == 1 ? 512 : 256;
  const long ctx_units = (long)a.n_groups * a.hkv * a.ctx_blocks, tail_units = (long)a.n_groups * a.n_seqs * a.hkv * a.tail_blocks;
  a.tail_pieces = a.tail_stride == 0 ? 0 : (int)std::max<long>(1, std::min<long>((a.tail_stride + 511) / 512, kSlots / 2 / tail_units));
  if (a.wide) {
    a.split_tiles = 1;
    attention_context_plan(a.n_seqs * a.n_q, a.hq, a.hkv, max_ctx, &a.n_qwg, &a.ctx_pieces, &a.split_tiles, &a.most_pieces);
    a.ctx_rows = a.n_qwg * 256;
    a.ctx_items = 0;
    a.tail_slot0 = (size_t)a.n_groups * a.hkv * a.ctx_rows * a.ctx_pieces;
    a.fold = a.tail_pieces == 1 && a.ctx_pieces <= 2;    // 16 x 64 queries over 4064 tokens: 24 + 14 us for tails and merge -> 27
  } else {
    // A piece leaves 520 bytes per query for 512 bytes per key that it reads (dh = 128), written and read again: four keys to a query, up to 256.
    // 64 queries a key/value head over 3136 keys: 14.9 us without this, 10.8 with it; 128 queries 14.9 + 5.8 for the merge against 15.8 + 4.0
    // (with four keys to each of the 128: 18.8 + 4.0).
    const long least = std::max<long>(step, std::min<long>(4 * std::min<long>(ctx_q, qpb), 256));
    const long left = std::max(kSlots / 2, kSlots - tail_units * a.tail_pieces), most = (max_ctx + least - 1) / least;
    a.ctx_pieces = max_ctx == 0 ? 0 : (int)std::max<long>(1, std::min<long>(most, left / ctx_units));
    a.ctx_items = a.n_groups * a.ctx_blocks * a.ctx_pieces;
    a.tail_slot0 = (size_t)a.rows * a.hq * a.ctx_pieces;
  }
  a.by_group_rows = FastDiv(a.n_seqs * a.n_q);
  a.by_hq = FastDiv(a.hq);
  a.by_hkv = FastDiv(a.hkv);
  a.by_g = FastDiv(g);
  a.by_ctx_pieces = FastDiv(std::max(1, a.ctx_pieces));
  a.by_ctx_blocks = FastDiv(a.ctx_blocks);
  a.by_tail_pieces = FastDiv(std::max(1, a.tail_pieces));
  a.by_tail_blocks = FastDiv(a.tail_blocks);
}

// A launch numbers its threads with 32 bits.  Of the launches that contexts of any length take, the one that reads contexts and tails has the
// most (the tails beside a wide one take as many workgroups, of no more threads); the merge has at most 256 to a query and head.  Pieces beyond the
// first are made only within 512 and 256 workgroups.
bool shared_attention_plan(SharedAttn &a, int max_ctx) {
  const long seqs = (long)a.n_groups * a.n_seqs, most = 1 << 23;
  if (seqs > most || seqs * a.n_q > most || seqs * a.n_q * a.hq > most) return false;
  const long g = a.hq / a.hkv, ctx_q = (long)a.n_seqs * a.n_q * g, tail_q = a.n_q * g;
  const int qb = query_blocks(a.dtype, ctx_q), qpb = 16 * qb, threads = 64 * qb * tiles_at_a_time(a.dtype, qb);
  const long contexts = std::max(a.n_groups * a.hkv * ((ctx_q + qpb - 1) / qpb), 512l);
  const long tails = a.tail_stride == 0 ? 0 : std::max(seqs * a.hkv * ((tail_q + qpb - 1) / qpb), 256l);
  if ((contexts + tails) * threads >= 1l << 32) return false;
  plan(a, max_ctx, true, false);
  return true;
}

static size_t floats_of(const SharedAttn &a) {
  const size_t ctx = a.wide ? (size_t)a.n_groups * a.hkv * a.ctx_rows * a.most_pieces : a.tail_slot0;
  return (ctx + (size_t)a.rows * a.hq * a.tail_pieces) * (a.dh + 2);
}
// Neither kind of launch takes less for a longer context, but the longer one may be of the other kind: the larger of the two.
size_t shared_attention_floats(SharedAttn a, int max_ctx) {
  plan(a, max_ctx, false, false);
  const size_t narrow = floats_of(a);
  plan(a, max_ctx, true, true);
  return std::max(narrow, floats_of(a));
}

// One query block reads everything once, so contexts too large to be found in the caches by a later call need not be put there.  Where that begins
// depends on what is called in between.  Three contexts in turn, eight beams: 65536 keys (268 MB) 61 -> 56 us, 32896 keys 33.0 -> 31.7, 28000 keys
// 25.0 -> 23.6; 20000 keys (82 MB) 21.9 -> 22.3, 12000 keys 15.2 -> 17.1, which the bound of 96 MB follows.  One context again and again never
// gains (3136 keys 8.6 -> 8.7, 32896 keys 25.3 -> 29.8); contexts that always come from memory, as when a step reads one for each of many layers, gain at
// every length: 3136 keys 10.3 -> 10.0, 8000 14.6 -> 13.6, 16000 19.5 -> 17.6, 32896 32.7 -> 30.4.  The call does not know what is called in between;
// the bound is that of the first of these cases.
static bool past_the_caches(const SharedAttn &a) {
  double keys = 0;
  for (int grp = 0; grp < a.n_groups; ++grp) keys += a.ctx_len[grp];
  return !a.wide && a.n_q == 1 && a.qb <= 4 && a.ctx_blocks == 1 && keys * a.hkv * a.dh * 4 >= 96.0 * (1 << 20);
}

hipError_t launch_shared_attention(SharedAttn a, float *scratch, hipStream_t s) {
  a.part_o = scratch;
  a.part_ml = scratch + (a.tail_slot0 + (size_t)a.rows * a.hq * a.tail_pieces) * a.dh;
  a.scale_log2e = kLog2e / sqrtf((float)a.dh);
  a.stream = past_the_caches(a);
  if (a.wide) {
    const int rows = a.n_seqs * a.n_q;
    const size_t q_row = (size_t)a.hq * a.dh * 2, slab = (size_t)a.ctx_stride * a.hkv * a.dh * 2, slots = (size_t)a.hkv * a.ctx_rows * a.ctx_pieces;
    for (int grp = 0; grp < a.n_groups; ++grp) {
      if (a.ctx_len[grp] == 0) continue;
      hipError_t e = launch_attention_context((const char *)a.q + (size_t)grp * rows * q_row, a.row_tail + (size_t)grp * rows, rows,
                                              (const char *)a.kc + grp * slab, (const char *)a.vc + grp * slab, a.hq, a.hkv, a.dh, a.ctx_len[grp],
                                              a.n_qwg, a.ctx_pieces, a.split_tiles, a.part_o + grp * slots * a.dh, a.part_ml + grp * slots * 2, s);
      if (e != hipSuccess) return e;
    }
  }
  const long items = a.ctx_items + (long)a.n_groups * a.n_seqs * a.tail_blocks * a.tail_pieces;
  if (items > 0) {
    const unsigned grid = (unsigned)(items * a.hkv);
    hipError_t e;
    if (a.dtype == 0) {
      if (a.dh == 64) hipLaunchKernelGGL(shared_attn_f32_kernel<64>, dim3(grid), dim3(64 * SF_NW), 0, s, a);
      else hipLaunchKernelGGL(shared_attn_f32_kernel<128>, dim3(grid), dim3(64 * SF_NW), 0, s, a);
      e = hipGetLastError();
    } else {
      e = a.dh == 64 ? launch_bf16_qb<64>(a, grid, s) : launch_bf16_qb<128>(a, grid, s);
    }
    if (e != hipSuccess) return e;
  }
  if (a.fold) return hipSuccess;
  if (a.dtype == 0) return a.dh == 64 ? launch_merge<float, 64>(a, s) : launch_merge<float, 128>(a, s);
  return a.dh == 64 ? launch_merge<bf16, 64>(a, s) : launch_merge<bf16, 128>(a, s);
}

}  // namespace cb

// The plan of a call with contexts of max_ctx rows, for tests without a device: 1 and what follows, or 0 where it is refused
extern "C" int cb_internal_shared_plan(int dtype, int hq, int hkv, int dh, int n_groups, int n_seqs, int n_q, int max_ctx, int tail_stride, int *out) {
  cb::SharedAttn a = cb::SharedAttn();
  a.dtype = dtype; a.hq = hq; a.hkv = hkv; a.dh = dh;
  a.n_groups = n_groups; a.n_seqs = n_seqs; a.n_q = n_q; a.tail_stride = tail_stride;
  if (!cb::shared_attention_plan(a, max_ctx)) return 0;
  for (int grp = 0; grp < std::min(n_groups, cb::kSharedGroups); ++grp) a.ctx_len[grp] = max_ctx;
  const int v[] = {a.wide, a.fold, a.qb, a.ctx_blocks, a.ctx_pieces, a.tail_blocks, a.tail_pieces, dtype != 0 && cb::past_the_caches(a)};
  std::copy(v, v + 8, out);
  return 1;
}
