// Attention of several continuations of one fused context (beams, samples, questions about the same documents): every
// new token of a continuation sees the whole context, which is stored once, and its continuation's own tail.
//     o = softmax([q Kc^T, q Kt^T] / sqrt(dh)) [Vc; Vt]
// The two parts are computed apart and joined through the softmax statistics: with m the maximum and l the sum of the
// exponentials of a part, o = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s.  The context's part takes the queries of ALL
// continuations together, so its keys and values are read once for all of them; a tail meets its own queries only.
//
// A single new token per continuation leaves few queries (continuations x query heads of a key/value head) against a
// long context: the bound is the bytes of the context, and what decides the time of a usual one (a few thousand tokens, 2 us
// of HBM time) is latency.  So the keys are cut into as many pieces as there are CUs, every wavefront of a piece takes
// 32-key tiles of its own, and the pieces are joined by a second launch.
#include "common.h"
#include "kernels.h"
#include <algorithm>
#include <mutex>

namespace cb {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int SA_NW = 4;                  // wavefronts per workgroup, each with a ring of its own
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

__device__ __forceinline__ Item item_of(const SharedAttn &a, int es, int qpb, int kvh, int w, int *piece, int *pieces) {
  Item it;
  const int g = a.hq / a.hkv;
  const size_t row_bytes = (size_t)a.hkv * a.dh * es, head = (size_t)kvh * a.dh * es;
  const int rows_group = a.n_seqs * a.n_q;
  if (w < a.ctx_items) {
    *pieces = a.ctx_pieces;
    *piece = w % a.ctx_pieces;
    w /= a.ctx_pieces;
    const int grp = w / a.ctx_blocks, blk = w - grp * a.ctx_blocks;
    it.row0 = grp * rows_group;
    it.m0 = blk * qpb;
    it.m_end = min(it.m0 + qpb, rows_group * g);
    it.k = (const char *)a.kc + (size_t)grp * a.ctx_stride * row_bytes + head;
    it.v = (const char *)a.vc + (size_t)grp * a.ctx_stride * row_bytes + head;
    it.limit = a.ctx_len[grp];
    it.tail = false;
    it.slot = (((size_t)kvh * a.rows * g + (size_t)it.row0 * g + it.m0) * a.ctx_pieces) + *piece;
    it.slot_step = a.ctx_pieces;
  } else {
    w -= a.ctx_items;
    *pieces = a.tail_pieces;
    *piece = w % a.tail_pieces;
    w /= a.tail_pieces;
    const int seq = w / a.tail_blocks, blk = w - seq * a.tail_blocks;
    it.row0 = seq * a.n_q;
    it.m0 = blk * qpb;
    it.m_end = min(it.m0 + qpb, a.n_q * g);
    it.k = (const char *)a.kt + (size_t)seq * a.tail_stride * row_bytes + head;
    it.v = (const char *)a.vt + (size_t)seq * a.tail_stride * row_bytes + head;
    it.limit = a.tail_stride;
    it.tail = true;
    it.slot = a.tail_slot0 + (((size_t)kvh * a.rows * g + (size_t)it.row0 * g + it.m0) * a.tail_pieces) + *piece;
    it.slot_step = a.tail_pieces;
  }
  return it;
}

// keys that flattened query m of the item sees (0 for padding rows; *real: whether its result is wanted)
__device__ __forceinline__ int visible(const SharedAttn &a, const Item &it, int m, bool *real) {
  const int g = a.hq / a.hkv;
  const int seen = m < it.m_end ? a.row_tail[it.row0 + m / g] : -1;
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

// Joins the wavefronts' results in LDS, in a fixed order, and writes the item's partial result.  s_o: [SA waves][queries][DH + 4]
template <int NW, int NQ, int DH>
__device__ __forceinline__ void join_and_store(const SharedAttn &a, const Item &it, const float *s_o, const float (*s_m)[NQ],
                                               const float (*s_l)[NQ], int tid) {
  constexpr int CG = DH / 4, LD = DH + 4;
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
      const float wt = exp2f(s_m[w][qi] - ref);          // 0 for a wavefront that saw no key of the query
      l += wt * s_l[w][qi];
      acc += wt * *reinterpret_cast<const f32x4 *>(s_o + ((size_t)w * NQ + qi) * LD + c * 4);
    }
    const size_t slot = it.slot + (size_t)qi * it.slot_step;
    if (c == 0) {
      a.part_ml[slot * 2] = top;
      a.part_ml[slot * 2 + 1] = l;
    }
    *reinterpret_cast<f32x4 *>(a.part_o + slot * DH + c * 4) = acc;
  }
}

// a piece without keys: the merge passes it over
__device__ __forceinline__ void store_empty(const SharedAttn &a, const Item &it, int tid) {
  for (int qi = tid; it.m0 + qi < it.m_end; qi += blockDim.x) {
    const size_t slot = it.slot + (size_t)qi * it.slot_step;
    a.part_ml[slot * 2] = -INFINITY;
    a.part_ml[slot * 2 + 1] = 0.f;
  }
}

// ---------------------------------------------------------------------------
// bf16.  Both products are computed transposed, S^T[key, query] = K Q^T and O^T[channel, query] += V^T P^T with
// v_mfma_f32_16x16x32_bf16, so that a lane holds values of one query (lane % 16) only, and the exponentiated scores are the
// second product's operand as they are: its contraction slots 8h .. 8h+7 (h = lane / 16) stand for the keys 4h .. 4h+3 and
// 16+4h .. 16+4h+3 that the first product leaves in the lane, and V is fetched in that order by the transposing LDS read.
// Every wavefront has a two-stage ring of 32-key tiles of its own, filled by global->LDS loads, and needs no barrier.
// QB: blocks of 16 queries a workgroup takes; all of them use a tile's fragments.
// ---------------------------------------------------------------------------
template <int DH, int QB>
__global__ __launch_bounds__(64 * SA_NW, 1) void shared_attn_bf16_kernel(SharedAttn a) {
  constexpr int ROWB = DH * 2, CH = DH / 8, RPI = 1024 / ROWB, TB = SA_TILE * ROWB, LPT = SA_TILE / RPI;
  constexpr int NKS = DH / 32, NCB = DH / 16, NQ = 16 * QB;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ float s_m[SA_NW][NQ], s_l[SA_NW][NQ];
  const int tid = threadIdx.x, lane = tid & 63, ln = lane & 15, h = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = (int)(blockIdx.x % (unsigned)a.hkv), g = a.hq / a.hkv;
  int piece, pieces;
  const Item it = item_of(a, 2, NQ, kvh, (int)(blockIdx.x / (unsigned)a.hkv), &piece, &pieces);
  const int n_act = it.m_end - it.m0;

  int vis[QB], kv_len = 0, min_vis = 0x7FFFFFFF;
  bf16x8 qf[QB][NKS];
#pragma unroll
  for (int b = 0; b < QB; ++b) {
    const int m = it.m0 + b * 16 + ln;
    bool real;
    vis[b] = visible(a, it, m, &real);
    kv_len = max(kv_len, vis[b]);
    min_vis = min(min_vis, real ? vis[b] : 0x7FFFFFFF);
    const int mc = min(m, it.m_end - 1), r = mc / g;
    const bf16 *src = (const bf16 *)a.q + ((size_t)(it.row0 + r) * a.hq + kvh * g + (mc - r * g)) * DH + 8 * h;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qf[b][ks] = *reinterpret_cast<const bf16x8 *>(src + 32 * ks);
  }
  kv_len = __builtin_amdgcn_readfirstlane(max16(kv_len));
  min_vis = __builtin_amdgcn_readfirstlane(min16(min_vis));
  const int n_tiles = (kv_len + SA_TILE - 1) / SA_TILE, per = (n_tiles + pieces - 1) / pieces;
  const int t_begin = piece * per, t_end = min(n_tiles, t_begin + per);
  if (t_begin >= t_end) {
    store_empty(a, it, tid);
    return;
  }

  // slot of 16-byte chunk c of row r in LDS: c ^ f(r); the 16 rows of a K fragment, and the 8 keys x 32 bytes that half a
  // wavefront's transposing read takes, then lie in different banks
  auto fk = [](int r) { return DH == 128 ? (r & 15) : ((r >> 1) & 7); };
  auto fv = [](int r) { return DH == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3); };
  const size_t row_bytes = (size_t)a.hkv * ROWB;
  char *ring = smem + wave * (4 * TB);
  const unsigned ring0 = (unsigned)(size_t)smem + wave * (4 * TB);
  auto issue = [&](int t, int stage, bool is_v) {
#pragma unroll
    for (int i = 0; i < LPT; ++i) {
      const int r = i * RPI + lane / CH;
      const int chunk = (lane % CH) ^ (is_v ? fv(r) : fk(r));
      const char *src = (is_v ? it.v : it.k) + (size_t)min(t * SA_TILE + r, kv_len - 1) * row_bytes + chunk * 16;
      char *dst = ring + stage * 2 * TB + (is_v ? TB : 0) + i * 1024;
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src,
                                       (__attribute__((address_space(3))) void *)dst, 16, 0, 0);
    }
  };
  unsigned ka[NKS], va[NCB];
#pragma unroll
  for (int ks = 0; ks < NKS; ++ks) ka[ks] = ring0 + ln * ROWB + (((4 * ks + h) ^ fk(ln)) << 4);
  {
    const int key = 4 * h + (ln >> 2);
#pragma unroll
    for (int c = 0; c < NCB; ++c)
      va[c] = ring0 + TB + key * ROWB + (((2 * c + ((ln & 3) >> 1)) ^ fv(key)) << 4) + (ln & 1) * 8;
  }

  f32x4 oacc[QB][NCB];
  float ref[QB], thr[QB], neg_mc[QB], row_sum[QB];
#pragma unroll
  for (int b = 0; b < QB; ++b) {
    ref[b] = thr[b] = -INFINITY;
    neg_mc[b] = row_sum[b] = 0.f;
#pragma unroll
    for (int c = 0; c < NCB; ++c) oacc[b][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float scale = a.scale_log2e, lazy = kLazyMax / scale;

  int t = t_begin + wave, stage = 0;
  if (t < t_end) {
    issue(t, 0, false);
    issue(t, 0, true);
    if (t + SA_NW < t_end) {
      issue(t + SA_NW, 1, false);
      issue(t + SA_NW, 1, true);
    }
  }
  for (; t < t_end; t += SA_NW, stage ^= 1) {
    const bool n1 = t + SA_NW < t_end, n2 = t + 2 * SA_NW < t_end;
    const unsigned so = stage * 2 * TB;
    if (n1) vm_wait<3 * LPT>(); else vm_wait<LPT>();      // K of this tile has landed
    bf16x8 kf[2][NKS];
    if constexpr (NKS == 4) {
      asm volatile(
          "ds_read_b128 %0, %8\n\tds_read_b128 %1, %9\n\tds_read_b128 %2, %10\n\tds_read_b128 %3, %11\n\t"
          "ds_read_b128 %4, %8 offset:4096\n\tds_read_b128 %5, %9 offset:4096\n\t"
          "ds_read_b128 %6, %10 offset:4096\n\tds_read_b128 %7, %11 offset:4096\n\ts_waitcnt lgkmcnt(0)"
          : "=&v"(kf[0][0]), "=&v"(kf[0][1]), "=&v"(kf[0][2]), "=&v"(kf[0][3]), "=&v"(kf[1][0]), "=&v"(kf[1][1]),
            "=&v"(kf[1][2]), "=&v"(kf[1][3])
          : "v"(ka[0] + so), "v"(ka[1] + so), "v"(ka[2] + so), "v"(ka[3] + so)
          : "memory");
    } else {
      asm volatile(
          "ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %4 offset:2048\n\t"
          "ds_read_b128 %3, %5 offset:2048\n\ts_waitcnt lgkmcnt(0)"
          : "=&v"(kf[0][0]), "=&v"(kf[0][1]), "=&v"(kf[1][0]), "=&v"(kf[1][1])
          : "v"(ka[0] + so), "v"(ka[1] + so)
          : "memory");
    }
    if (n2) issue(t + 2 * SA_NW, stage, false);
    const int t0 = t * SA_TILE;
    const bool masked = t0 + SA_TILE > min_vis;           // some key of the tile is hidden from some query
    bf16x8 pf[QB];
#pragma unroll
    for (int b = 0; b < QB; ++b) {
      if (b * 16 >= n_act) continue;
      f32x4 sc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) sc[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kb][ks], qf[b][ks], sc[kb], 0, 0, 0);
      float mx = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (t0 + 16 * kb + 4 * h + i >= vis[b]) sc[kb][i] = -INFINITY;
          mx = fmaxf(mx, sc[kb][i]);
        }
      mx = group_max(mx);
      if (__any(mx > thr[b])) {
        // exponents are taken relative to a reference that only moves when a score exceeds it by 2^8: P and the sums carry a
        // common factor, which costs no precision
        const float nr = fmaxf(ref[b], mx);
        const float alpha = nr > ref[b] ? __builtin_amdgcn_exp2f((ref[b] - nr) * scale) : 1.f;
        ref[b] = nr;
        thr[b] = nr + lazy;
        neg_mc[b] = nr == -INFINITY ? 0.f : -nr * scale;
        row_sum[b] *= alpha;
#pragma unroll
        for (int c = 0; c < NCB; ++c) oacc[b][c] *= alpha;
      }
      float psum = 0.f;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[kb][i], scale, neg_mc[b]));
          psum += p;
          pf[b][4 * kb + i] = (bf16)p;                    // the matrix cores' operand type; the sum keeps the float
        }
      row_sum[b] += psum;
    }
    if (n2) vm_wait<3 * LPT>();                           // V of this tile has landed
    else if (n1) vm_wait<2 * LPT>();
    else vm_wait<0>();
    union VF { s16x4 s[2]; bf16x8 b; } vf[NCB];
#pragma unroll
    for (int c = 0; c < NCB; c += 4)
      asm volatile(
          "ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:%12\n\t"
          "ds_read_b64_tr_b16 %2, %9\n\tds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
          "ds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:%12\n\t"
          "ds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:%12\n\ts_waitcnt lgkmcnt(0)"
          : "=&v"(vf[c].s[0]), "=&v"(vf[c].s[1]), "=&v"(vf[c + 1].s[0]), "=&v"(vf[c + 1].s[1]), "=&v"(vf[c + 2].s[0]),
            "=&v"(vf[c + 2].s[1]), "=&v"(vf[c + 3].s[0]), "=&v"(vf[c + 3].s[1])
          : "v"(va[c] + so), "v"(va[c + 1] + so), "v"(va[c + 2] + so), "v"(va[c + 3] + so), "n"(16 * ROWB)
          : "memory");
    bool bad = false;
    if (masked) {
      // A hidden key has p = 0, but 0 times a value that is not finite is not 0 (rows past the end repeat the last one).
#pragma unroll
      for (int c = 0; c < NCB; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) bad |= !(fabsf((float)vf[c].b[i]) < INFINITY);
      bad = __any(bad);
    }
    if (!bad) {
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        if (b * 16 >= n_act) continue;
#pragma unroll
        for (int c = 0; c < NCB; ++c) oacc[b][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[c].b, pf[b], oacc[b][c], 0, 0, 0);
      }
    } else {
      // the same sums key by key, over the keys that a query sees; key k of the tile is held by lane group (k % 16) / 4
#pragma unroll 1
      for (int k = 0; k < SA_TILE; ++k) {
        const int slot = (k >> 4) * 4 + (k & 3), from = ((k & 15) >> 2) * 16 + ln;
        const char *vrow = it.v + (size_t)min(t0 + k, kv_len - 1) * row_bytes;
#pragma unroll
        for (int b = 0; b < QB; ++b) {
          if (b * 16 >= n_act) continue;
          float p = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (i == slot) p = (float)pf[b][i];
          p = __shfl(p, from, 64);
          if (t0 + k < vis[b]) {
#pragma unroll
            for (int c = 0; c < NCB; ++c) {
              const bf16x4 v4 = *reinterpret_cast<const bf16x4 *>(vrow + (16 * c + 4 * h) * 2);
#pragma unroll
              for (int i = 0; i < 4; ++i) oacc[b][c][i] = __builtin_fmaf(p, (float)v4[i], oacc[b][c][i]);
            }
          }
        }
      }
      // the loads above and the ring's share a counter: everything has landed here, the waits that follow are met already
      vm_wait<0>();
    }
    if (n2) issue(t + 2 * SA_NW, stage, true);
  }
  __syncthreads();                        // the rings become the join's buffer
  float *s_o = reinterpret_cast<float *>(smem);
#pragma unroll
  for (int b = 0; b < QB; ++b) {
    const float l = group_sum(row_sum[b]);
#pragma unroll
    for (int c = 0; c < NCB; ++c)
      *reinterpret_cast<f32x4 *>(s_o + ((size_t)wave * NQ + b * 16 + ln) * (DH + 4) + 16 * c + 4 * h) = oacc[b][c];
    if (h == 0) {
      s_m[wave][b * 16 + ln] = ref[b] * scale;
      s_l[wave][b * 16 + ln] = l;
    }
  }
  __syncthreads();
  join_and_store<SA_NW, NQ, DH>(a, it, s_o, s_m, s_l, tid);
}

// ---------------------------------------------------------------------------
// float, v_mfma_f32_16x16x4_f32: the same items with 16 queries per workgroup and K, V straight from memory (a float model's
// caches fit L2).  The contraction index a lane supplies in MFMA s is 4 (lane / 16) + s for both products.
// ---------------------------------------------------------------------------
constexpr int SF_NW = 4;
template <int DH>
__global__ __launch_bounds__(64 * SF_NW) void shared_attn_f32_kernel(SharedAttn a) {
  constexpr int NC = DH / 16;
  __shared__ __attribute__((aligned(16))) float s_o[SF_NW * 16 * (DH + 4)];
  __shared__ float s_m[SF_NW][16], s_l[SF_NW][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ln = lane & 15, h = lane >> 4;
  const int kvh = (int)(blockIdx.x % (unsigned)a.hkv), g = a.hq / a.hkv;
  int piece, pieces;
  const Item it = item_of(a, 4, 16, kvh, (int)(blockIdx.x / (unsigned)a.hkv), &piece, &pieces);
  const int m = it.m0 + ln, mc = min(m, it.m_end - 1), r = mc / g;
  bool real;
  const int vis = visible(a, it, m, &real);
  const float *qrow = (const float *)a.q + ((size_t)(it.row0 + r) * a.hq + kvh * g + (mc - r * g)) * DH + 4 * h;
  f32x4 qf[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) qf[c] = *reinterpret_cast<const f32x4 *>(qrow + 16 * c);
  const int kv_len = __builtin_amdgcn_readfirstlane(max16(vis));
  const int min_vis = __builtin_amdgcn_readfirstlane(min16(real ? vis : 0x7FFFFFFF));
  const int n_tiles = (kv_len + SA_TILE - 1) / SA_TILE, per = (n_tiles + pieces - 1) / pieces;
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
  join_and_store<SF_NW, 16, DH>(a, it, s_o, s_m, s_l, tid);
}

// Joins a query's partial results: the context's pieces, then the tail's.  A row that sees no key, and a padding row, is zero.
template <typename T, int DH>
__global__ __launch_bounds__(256) void shared_merge_kernel(SharedAttn a) {
  constexpr int CG = DH / 4;
  const int g = a.hq / a.hkv;
  const long idx = (long)blockIdx.x * 256 + threadIdx.x;
  if (idx >= (long)a.rows * a.hq * CG) return;
  const int c = (int)(idx % CG), hd = (int)(idx / CG % a.hq), r = (int)(idx / CG / a.hq);
  const int kvh = hd / g;
  const size_t m = (size_t)kvh * a.rows * g + (size_t)r * g + (hd - kvh * g);
  float top = -INFINITY, l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  auto part = [&](size_t slot0, int n) {
    const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + slot0;
    const f32x4 *src = reinterpret_cast<const f32x4 *>(a.part_o) + slot0 * CG + c;
    float pm = -INFINITY;
    for (int s = 0; s < n; ++s) pm = fmaxf(pm, ml[s].x);
    const float nt = fmaxf(top, pm), ref = nt == -INFINITY ? 0.f : nt, w0 = exp2f(top - ref);
    top = nt;
    l *= w0;
    acc *= w0;
    for (int s = 0; s < n; ++s) {
      const float2 v = ml[s];
      if (v.x == -INFINITY && v.y == 0.f) continue;      // a piece without keys left nothing else
      const float w = exp2f(v.x - ref);
      l += w * v.y;
      acc += w * src[(size_t)s * CG];
    }
  };
  if (a.row_tail[r] >= 0) {
    if (a.ctx_pieces) part(m * a.ctx_pieces, a.ctx_pieces);
    if (a.tail_pieces) part(a.tail_slot0 + m * a.tail_pieces, a.tail_pieces);
  }
  if (l == 0.f) acc = f32x4{0.f, 0.f, 0.f, 0.f};
  const float inv = l == 0.f ? 0.f : 1.f / l;
  store4<T>((T *)a.o + ((size_t)r * a.hq + hd) * DH + c * 4, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
}

template <int DH, int QB>
hipError_t launch_bf16(const SharedAttn &a, unsigned grid, hipStream_t s) {
  constexpr int ring = SA_NW * 4 * SA_TILE * DH * 2, join = SA_NW * 16 * QB * (DH + 4) * 4;
  constexpr int smem = ring > join ? ring : join;
  static std::once_flag once;
  std::call_once(once, [] {
    (void)hipFuncSetAttribute(reinterpret_cast<const void *>(&shared_attn_bf16_kernel<DH, QB>),
                              hipFuncAttributeMaxDynamicSharedMemorySize, smem);
  });
  hipLaunchKernelGGL((shared_attn_bf16_kernel<DH, QB>), dim3(grid), dim3(64 * SA_NW), smem, s, a);
  return hipGetLastError();
}

int query_blocks(int dtype, long queries) {   // blocks of 16 queries that a workgroup takes
  return dtype == 0 ? 1 : (int)std::min<long>(3, (queries + 15) / 16);
}

}  // namespace

// Pieces: about one workgroup per CU in all, no piece shorter than a tile for each wavefront.
void shared_attention_plan(SharedAttn &a, int max_ctx) {
  const int g = a.hq / a.hkv;
  const long ctx_q = (long)a.n_seqs * a.n_q * g, tail_q = (long)a.n_q * g;
  a.rows = a.n_groups * a.n_seqs * a.n_q;
  a.qb = query_blocks(a.dtype, ctx_q);
  const int qpb = 16 * a.qb;
  a.ctx_blocks = (int)((ctx_q + qpb - 1) / qpb);
  a.tail_blocks = (int)((tail_q + qpb - 1) / qpb);
  auto pieces = [&](long units, int keys) {
    const long most = (keys + SA_NW * SA_TILE - 1) / (SA_NW * SA_TILE);
    return (int)std::max<long>(1, std::min<long>(most, 256 / std::max<long>(1, units)));
  };
  a.ctx_pieces = max_ctx > 0 ? pieces((long)a.n_groups * a.hkv * a.ctx_blocks, max_ctx) : 0;
  a.tail_pieces = a.tail_stride > 0 ? pieces((long)a.n_groups * a.n_seqs * a.hkv * a.tail_blocks, a.tail_stride) : 0;
  a.ctx_items = a.n_groups * a.ctx_blocks * a.ctx_pieces;
  a.tail_slot0 = (size_t)a.rows * a.hq * a.ctx_pieces;
}

size_t shared_attention_floats(const SharedAttn &a) {
  return (size_t)a.rows * a.hq * (a.ctx_pieces + a.tail_pieces) * (a.dh + 2);
}

hipError_t launch_shared_attention(SharedAttn a, float *scratch, hipStream_t s) {
  a.part_o = scratch;
  a.part_ml = scratch + (size_t)a.rows * a.hq * (a.ctx_pieces + a.tail_pieces) * a.dh;
  a.scale_log2e = kLog2e / sqrtf((float)a.dh);
  const long items = a.ctx_items + (long)a.n_groups * a.n_seqs * a.tail_blocks * a.tail_pieces;
  if (items > 0) {
    const unsigned grid = (unsigned)(items * a.hkv);
    hipError_t e;
    if (a.dtype == 0) {
      if (a.dh == 64) hipLaunchKernelGGL(shared_attn_f32_kernel<64>, dim3(grid), dim3(64 * SF_NW), 0, s, a);
      else hipLaunchKernelGGL(shared_attn_f32_kernel<128>, dim3(grid), dim3(64 * SF_NW), 0, s, a);
      e = hipGetLastError();
    } else if (a.dh == 64) {
      e = a.qb == 1 ? launch_bf16<64, 1>(a, grid, s) : a.qb == 2 ? launch_bf16<64, 2>(a, grid, s)
        : launch_bf16<64, 3>(a, grid, s);
    } else {
      e = a.qb == 1 ? launch_bf16<128, 1>(a, grid, s) : a.qb == 2 ? launch_bf16<128, 2>(a, grid, s)
        : launch_bf16<128, 3>(a, grid, s);
    }
    if (e != hipSuccess) return e;
  }
  const dim3 mgrid((unsigned)(((long)a.rows * a.hq * (a.dh / 4) + 255) / 256));
  if (a.dtype == 0) {
    if (a.dh == 64) hipLaunchKernelGGL((shared_merge_kernel<float, 64>), mgrid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((shared_merge_kernel<float, 128>), mgrid, dim3(256), 0, s, a);
  } else {
    if (a.dh == 64) hipLaunchKernelGGL((shared_merge_kernel<bf16, 64>), mgrid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((shared_merge_kernel<bf16, 128>), mgrid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace cb
