"""References of the operators that carry several continuations of one fused context, in 64 bits and from their definitions,
with the error that the kernels' roundings can make of each output element."""
import math
from types import SimpleNamespace

import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}          # of a rounding, relative to the value


def model(hq, hkv, dh, dtype, layers=1, rope="adjacent", theta=1e4):
    return SimpleNamespace(n_layers=layers, d_model=hq * dh, n_q_heads=hq, n_kv_heads=hkv, head_dim=dh, d_ff=2 * hq * dh, rms_eps=1e-5,
                           rope_theta=theta, dtype=dtype, rope_layout=rope)


def normal(shape, seed, dtype=torch.float32, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return torch.empty(shape).normal_(0, std, generator=g).to(dtype)


def attention(q, kp, vp, plen, kt, vt, row_tail, n_seqs, n_q, dtype):
    """(out, bound) of cb_shared_prefix_attention, float64 on the inputs' device.  q [rows, Hq, dh]; kp [groups, stride, Hkv, dh];
    kt [groups * n_seqs, stride, Hkv, dh].  The bound adds up, with A = sum p |v| and n keys:
      - the probabilities' rounding to bf16 (A half steps; float models keep them) and the output's (|out| half steps);
      - a score's float sum of dh products, dh 2^-24 of the sum of their magnitudes S, its scaling and the reduced exponent
        (4 2^-24 of |score| <= S), on numerator and denominator: 2 A (dh + 4) 2^-24 max S;
      - the sums over n keys, the exponentials (2 units of 2^-23), the rescaling and joining (8 more): 2 A (n + 24) 2^-24."""
    rows, hq, dh = q.shape
    hkv = kp.shape[2] if kp.numel() else kt.shape[2]
    g = hq // hkv
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(out)
    for r in range(rows):
        seq = r // n_q
        group = seq // n_seqs
        seen = int(row_tail[r])
        if seen < 0:
            continue
        seen = min(seen, kt.shape[1])
        k = torch.cat((kp[group, :plen[group]], kt[seq, :seen])).double()
        v = torch.cat((vp[group, :plen[group]], vt[seq, :seen])).double()
        n = k.shape[0]
        if n == 0:
            continue
        qh = q[r].double().view(hkv, g, dh)
        s = torch.einsum("hgd,nhd->hgn", qh, k) / math.sqrt(dh)
        p = torch.softmax(s, -1)
        out[r] = torch.einsum("hgn,nhd->hgd", p, v).reshape(hq, dh)
        a = torch.einsum("hgn,nhd->hgd", p, v.abs()).reshape(hq, dh)
        size = torch.einsum("hgd,nhd->hgn", qh.abs(), k.abs()).amax(-1).reshape(hq, 1) / math.sqrt(dh)
        bound[r] = ((a if dtype == "bf16" else 0.0) + out[r].abs()) * HALF_STEP[dtype] * 1.01 + \
            2 * a * ((dh + 4) * 2.0 ** -24 * size + (n + 24) * 2.0 ** -24)
    return out, bound


def rope(x, pos, gain, m):
    """(out, bound) of the norm and rotation of x [rows, heads, dh] (gain None: no norm), float64.  Bound: the output's rounding, and for
    the float arithmetic before it: the table's rounding 1, two products and a sum 3, the norm's factor (the sum's 8 levels, the
    root 2, two products) 12: 16 units of 2^-24 of the magnitudes that are added."""
    x = x.double()
    half = m.head_dim // 2
    if gain is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + m.rms_eps) * gain.double()
    inv = m.rope_theta ** (-2.0 * torch.arange(half, dtype=torch.float64, device=x.device) / m.head_dim)
    ang = pos.double()[:, None, None] * inv
    i = torch.arange(half, device=x.device)
    a, b = (2 * i, 2 * i + 1) if m.rope_layout == "adjacent" else (i, i + half)
    out, size = torch.empty_like(x), torch.empty_like(x)
    out[..., a] = x[..., a] * ang.cos() - x[..., b] * ang.sin()
    out[..., b] = x[..., a] * ang.sin() + x[..., b] * ang.cos()
    size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return out, out.abs() * HALF_STEP[m.dtype] + size * 16 * 2.0 ** -24


def beam_scores(logits, scores, finished=None, end_token=0):
    """Scores of every continuation, float64 [rows, vocab], from the definition: NaN logits are -infinity, infinite ones share, a beam
    whose score is not finite is not there."""
    x = logits.double().nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    s = scores.double()
    out = torch.full_like(x, -math.inf)
    for r in range(x.shape[0]):
        if not math.isfinite(float(s[r])):
            continue
        if finished is not None and int(finished[r]) != 0:
            out[r, end_token] = s[r]
            continue
        m = float(x[r].max())
        if m == -math.inf:
            continue
        if m == math.inf:
            top = x[r] == math.inf
            out[r, top] = s[r] - math.log(int(top.sum()))
        else:
            out[r] = s[r] + (x[r] - (m + torch.exp(x[r] - m).sum().log()))
    return out


def best(all_scores, n_groups, n_keep):
    """(scores, beam, token) lists per group, best first; equal scores by lower beam, then lower token."""
    rows, vocab = all_scores.shape
    res = []
    for g in range(n_groups):
        flat = all_scores.view(n_groups, -1)[g]
        v, i = torch.sort(flat, descending=True, stable=True)
        v, i = v[:n_keep], i[:n_keep]
        res.append([(float(a), int(b) // vocab, int(b) % vocab) if a > -math.inf else (-math.inf, -1, -1) for a, b in zip(v, i)] +
                   [(-math.inf, -1, -1)] * (n_keep - len(v)))
    return res


def sum_error(vocab):
    """Of cb_beam_select's sums of exponentials, relative: 31 float additions of a lane's round, 6 levels of a wavefront twice, exponentials and
    joining factors of 2 units of 2^-24 each, 4 roundings; and for every unit of distance from the maximum up to 5 (3 for the exponent's subtraction,
    product and constant, 2 for the factor where a reference moves, which is by 1 at least).  The distances, weighted by the probabilities, average to
    at most ln vocab (sum p ln(max p / p) <= entropy), and a reference lags by at most 1 at two levels."""
    return (31 + 12 + 6 + 4 + 5 * (2 + math.log(vocab))) * 2.0 ** -24


def check_selection(got, logits, scores, n_groups, finished=None, end_token=0):
    """got: the three results.  Scores within the sums' error and one rounding; beams and tokens as the definition gives them wherever no other
    beam's score is nearer than twice the sums' error.  Beams of the same logits and score have the same sums; of the same logits in another order they
    do not, as float additions depend on it."""
    got = [t.cpu() for t in got]
    every, n_keep = beam_scores(logits, scores, finished, end_token), got[0].shape[1]
    vocab, beams = logits.shape[1], logits.shape[0] // n_groups
    wants = best(every, n_groups, min(n_keep + 1, beams * vocab))
    top = every.topk(min(n_keep + 1, vocab), -1).values.cpu()         # of each beam: what a neighbour can be
    every = every.cpu()
    ended = torch.zeros_like(scores) if finished is None else finished.to(scores)
    ids = {}
    kind = torch.tensor([ids.setdefault(row.tobytes(), len(ids)) for row in
                         torch.cat((logits.float() + 0.0, scores[:, None], ended[:, None]), 1).cpu().numpy()])
    for g in range(n_groups):
        want, seen = wants[g] + [(-math.inf, -1, -1)] * (n_keep + 1), set()
        for i in range(n_keep):
            s, b, t = float(got[0][g, i]), int(got[1][g, i]), int(got[2][g, i])
            ws, wb, wt = want[i]
            if ws == -math.inf:
                assert (s, b, t) == (-math.inf, -1, -1), (g, i, s, b, t)
                continue
            tol = sum_error(vocab)
            assert abs(s - ws) <= tol + abs(ws) * 2.0 ** -24, (g, i, s, ws)
            assert (b, t) not in seen and 0 <= b < beams and 0 <= t < vocab
            seen.add((b, t))
            mine = slice(g * beams, (g + 1) * beams)
            near = ((top[mine] - ws).abs() <= 2 * tol) & (kind[mine] != kind[g * beams + wb])[:, None]
            if bool(near.any()):
                assert abs(float(every[g * beams + b, t]) - ws) <= 2 * tol
            else:
                assert (b, t) == (wb, wt), (g, i, (s, b, t), want[i])


def attention_plan(m, n_groups, n_seqs, n_q, prefix, tail_stride):
    """The launches that cb_shared_prefix_attention chooses, asked of the library without a device; None: refused."""
    import ctypes
    from paper_2405_16444_amd.binding import _lib
    out = (ctypes.c_int * 8)()
    if not _lib.cb_internal_shared_plan(int(m.dtype == "bf16"), m.n_q_heads, m.n_kv_heads, m.head_dim, n_groups, n_seqs, n_q, prefix, tail_stride, out):
        return None
    return SimpleNamespace(**dict(zip(("wide", "fold", "qb", "ctx_blocks", "ctx_pieces", "tail_blocks", "tail_pieces", "stream"), out)))


# Shapes of attention that together reach every bf16 kernel: query heads, key/value heads, context rows, continuations, new tokens of each, and what the
# plan makes of them (query blocks, past the caches, folding).  Contexts past the caches have 96 MB and a little.
def plan_shapes(dh):
    far = (96 << 20) // (16 * dh * 4) + 457
    return [((16, 16, far, 3, 1), (1, 1, 0)), ((64, 16, far, 7, 1), (2, 1, 0)), ((64, 16, far, 12, 1), (4, 1, 0)),
            ((8, 2, 731, 3, 1), (1, 0, 0)), ((8, 2, 1999, 7, 1), (2, 0, 0)), ((8, 2, 2501, 12, 1), (4, 0, 0)), ((8, 2, 2999, 30, 1), (8, 0, 0)),
            ((64, 8, 611, 512, 1), (1, 0, 1)), ((32, 1, 437, 1024, 1), (2, 0, 1)), ((64, 1, 437, 512, 1), (4, 0, 1)), ((128, 1, 437, 256, 1), (8, 0, 1)),
            ((5, 5, 731, 2, 5), (1, 0, 0)), ((6, 3, 1999, 2, 7), (2, 0, 0)), ((4, 4, 1501, 3, 20), (4, 0, 0)), ((4, 2, 999, 3, 20), (8, 0, 0)),
            ((64, 8, 611, 256, 2), (1, 0, 1)), ((64, 8, 611, 128, 4), (2, 0, 1)), ((64, 8, 611, 64, 8), (4, 0, 1)), ((64, 8, 1003, 16, 64), (8, 0, 1))]


def coded_values(rows, heads, dh, first=0):
    """Values [rows, heads, dh] in which every tile of 32 rows has a channel of its own (the next tiles after dh of them take the same again): an output
    channel is the sum of a few tiles' probabilities, and a tile that is lost or taken twice changes it by its share of them."""
    row = torch.arange(rows)
    v = torch.zeros((rows, heads, dh))
    v[row, :, (first + row // 32) % dh] = (1 + (row * 37 % 61) / 128)[:, None]
    return v


def border_rows(prefix):
    return [0, 31, 32, 33, 63, 64, prefix // 2, prefix - 2, prefix - 1]


def towards_borders(q, kp, kt, prefix):
    """(q, kp, kt) in which the context's border rows and all tail rows have most of the probability: queries share a direction per key/value head, and
    these keys lie along it, for scores of 1.25 ln prefix beside the others' of less than 1.  Rows behind the context would take everything."""
    hkv, dh = kp.shape[2:]
    way = normal((hkv, dh), 97).sign().to(q.device)
    q = (way.repeat_interleave(q.shape[1] // hkv, 0) + 0.3 * q.float()).to(q.dtype)
    along = 1.25 * math.log(prefix) / dh ** 0.5 * way
    kp, kt = (0.3 * kp.float()).to(kp.dtype), (0.3 * kt.float() + along).to(kt.dtype)
    kp[0, border_rows(prefix)] = (kp[0, border_rows(prefix)].float() + along).to(kp.dtype)
    kp[0, prefix:] = (8 * way).to(kp.dtype)
    return q, kp, kt
