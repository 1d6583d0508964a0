"""Timing cases of the operators that carry several continuations of one fused context: a step of beam search, of sampling
several answers, or several questions about the same documents.

    op         one pass
    rope       cb_qkv_norm_rope: queries and keys of the new tokens normalised per head and rotated, K and V put into the cache
    attention  cb_shared_prefix_attention: every continuation's queries over the shared context and its own tail
    select     cb_beam_select: the best continuations over beams and vocabulary
    reorder    cb_beam_reorder: the tails of all layers follow the surviving beams

Where `own` is false a pass is the same arithmetic in elementary torch operations.  Models have the head layouts, depths and
vocabularies of workloads/configs.py.  Values are what the path meets: unit-variance activations, logits of a few units,
ragged lengths, padded query rows, cache rows behind a length that hold other data.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

# layers, query heads, key/value heads, head_dim, vocabulary, rotary base, storage type
MODELS = {
    "tiny": (2, 4, 2, 64, 32000, 1e4, "f32"),
    "mistral7b": (32, 32, 8, 128, 32000, 1e6, "bf16"),
    "yi34b": (60, 56, 8, 128, 64000, 5e6, "bf16"),
    "llama70b": (80, 64, 8, 128, 32000, 1e4, "bf16"),
}
POSITIONS = 36000                     # of the contexts: more than any position below
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _rope(model, rows, slots, far, norms, layout, name=None):
    """rows new tokens at positions up to far; a cache of `slots` rows receives their K and V"""
    c = {"name": name} if name else {}
    c.update(op="rope", model=model, rows=rows, slots=slots, far=far, norms=norms, layout=layout)
    return c


def _attention(model, groups, seqs, queries, prefix, tail, room, name=None):
    """groups x seqs continuations with up to `queries` new tokens each; contexts of 3/4 prefix .. prefix tokens (the first
    group's has all of them), tails of tail/2 .. tail tokens, the new ones among them, in slabs of `room` rows"""
    c = {"name": name} if name else {}
    c.update(op="attention", model=model, groups=groups, seqs=seqs, queries=queries, prefix=prefix, tail=tail, room=room)
    return c


def _select(model, groups, beams, keep, logits, vocab=0, pad=0, done=0.0, name=None):
    """done: share of the beams that have ended; pad: elements between two rows of the logits"""
    c = {"name": name} if name else {}
    c.update(op="select", model=model, groups=groups, beams=beams, keep=keep, logits=logits, vocab=vocab or MODELS[model][4],
             pad=pad, done=done)
    return c


def _reorder(model, layers, groups, beams, tail, room, name=None):
    c = {"name": name} if name else {}
    c.update(op="reorder", model=model, layers=layers, groups=groups, beams=beams, tail=tail, room=room)
    return c


def listed():
    return [
        # one decoding step of eight continuations: a few rows, bound by latency
        _rope("mistral7b", 8, 8 * 64, 3300, False, "half", name="rope_step"),
        # the prompts of a batch, heads with norms of their own, scattered into the cache
        _rope("llama70b", 4099, 5000, 9000, True, "adjacent", name="rope_prompt"),
        # a float model, four beams over a short context: the smallest attention call
        _attention("tiny", 1, 4, 1, 544, 16, 32, name="attention_tiny"),
        # eight beams over the usual retrieval request
        _attention("mistral7b", 1, 8, 1, 3136, 48, 128, name="attention_beams"),
        # four users' requests with five beams each, seven query heads per key/value head
        _attention("yi34b", 4, 5, 1, 2300, 90, 160, name="attention_requests"),
        # eight continuations of a 32 K context
        _attention("mistral7b", 1, 8, 1, 32896, 200, 256, name="attention_long"),
        # sixteen questions of up to 64 tokens about one set of documents
        _attention("llama70b", 1, 16, 64, 4064, 64, 64, name="attention_questions"),
        # one request with four beams
        _select("mistral7b", 1, 4, 8, "f32", name="select_one"),
        # many requests at once on the largest vocabulary
        _select("yi34b", 32, 8, 16, "f32", name="select_many"),
        # half-precision logits, an odd vocabulary, some beams at their end
        _select("yi34b", 6, 5, 10, "bf16", vocab=64007, done=0.15, name="select_odd"),
        # the tails of a short answer, four beams
        _reorder("mistral7b", 32, 1, 4, 24, 128, name="reorder_short"),
        # long answers of several requests on the deepest model
        _reorder("llama70b", 80, 4, 8, 80, 96, name="reorder_deep"),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["rope", "attention", "attention", "attention", "select", "select", "reorder"])
    model = rng.choice(["tiny", "mistral7b", "mistral7b", "yi34b", "llama70b"])
    if op == "rope":
        rows = _log(rng, 1, 4096)
        return _rope(model, rows, rows + rng.randint(0, 900), _log(rng, 100, 32000), rng.random() < 0.5,
                     rng.choice(["adjacent", "half"]))
    if op == "select":
        groups, beams = _log(rng, 1, 30), rng.randint(1, 8)
        vocab = MODELS[model][4] if rng.random() < 0.4 else _log(rng, 500, 64000)
        return _select(model, groups, beams, rng.randint(1, min(2 * beams, 16)), rng.choice(["f32", "bf16"]), vocab,
                       rng.choice([0, 0, rng.randint(1, 64)]), rng.choice([0.0, 0.0, 0.2]))
    if op == "reorder":
        room = _log(rng, 8, 96)
        return _reorder(model, rng.randint(1, MODELS[model][0]), rng.randint(1, 4), rng.randint(2, 8), rng.randint(1, room), room)
    kind = rng.random()
    if kind < 0.6:                     # decoding steps
        groups = rng.choice([1, 1, 1, rng.randint(2, 6)])
        prefix, queries, seqs = _log(rng, 100, 28000 // groups), 1, rng.randint(1, 16)
    elif kind < 0.8:                   # a few tokens at a time (drafts that are checked)
        groups, prefix, queries, seqs = 1, _log(rng, 100, 16000), rng.randint(2, 9), rng.randint(1, 8)
    else:                              # questions
        groups, prefix, queries, seqs = 1, _log(rng, 100, 3700), rng.randint(10, 64), rng.randint(2, 16)
    if model == "tiny":
        prefix = min(prefix, 2000)
    tail = queries + _log(rng, 1, 256)
    return _attention(model, groups, seqs, queries, prefix, tail, tail + rng.randint(0, 64))


def _lengths(case):
    """attention: (context length of every group, per continuation (tail length, new tokens))"""
    r = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    prefix = [case["prefix"]] + [r.randint(case["prefix"] * 3 // 4, case["prefix"]) for _ in range(case["groups"] - 1)]
    tails = []
    for _ in range(case["groups"] * case["seqs"]):
        n = r.randint(max(1, case["queries"] // 3), case["queries"])
        tails.append((r.randint(max(n, case["tail"] // 2), max(n, case["tail"])), n))
    return prefix, tails


def _parents(case):
    """reorder: (parent of every beam within its group, length of every tail)"""
    r = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    n = case["groups"] * case["beams"]
    return [r.randrange(case["beams"]) for _ in range(n)], [r.randint(max(1, case["tail"] * 3 // 4), case["tail"]) for _ in range(n)]


def _normal(shape, seed, dtype, std=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    layers, hq, hkv, dh, _, theta, dtype = MODELS[case["model"]]
    dt = TYPES[dtype]
    s = SimpleNamespace(op=case["op"], case=case, hq=hq, hkv=hkv, dh=dh, theta=theta, eps=1e-5)
    if s.op == "rope":
        n, slots = case["rows"], case["slots"]
        s.qkv = _normal((n, (hq + 2 * hkv) * dh), seed, dt)
        s.q_norm = 1 + _normal((dh,), seed + 1, torch.float32, 0.1).to(dt) if case["norms"] else None
        s.k_norm = 1 + _normal((dh,), seed + 2, torch.float32, 0.1).to(dt) if case["norms"] else None
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + 3)
        s.pos = torch.randint(0, case["far"], (n,), generator=g, device="cuda").to(torch.int32)
        s.row = torch.randperm(slots, generator=g, device="cuda")[:n].to(torch.int32)
        s.row[::17] = -1 if n > 16 else s.row[::17]      # rows of a padded batch: not kept
        s.k = _normal((slots, hkv, dh), seed + 4, dt)
        s.v = _normal((slots, hkv, dh), seed + 5, dt)
        s.q_out = torch.zeros((n, hq, dh), dtype=dt, device="cuda")
    elif s.op == "attention":
        prefix, tails = _lengths(case)
        s.prefix, s.n = prefix, (case["groups"], case["seqs"], case["queries"])
        s.longest = max(t for t, _ in tails)
        nseq, rows = case["groups"] * case["seqs"], case["groups"] * case["seqs"] * case["queries"]
        s.prefix_len = _ints(prefix)
        # new token i of a continuation sees the tail up to itself; rows past its new tokens are padding
        s.row_tail = _ints([t - n + 1 + i if i < n else -1 for t, n in tails for i in range(case["queries"])])
        s.q = _normal((rows, hq, dh), seed, dt)
        s.kp = _normal((case["groups"] * case["prefix"], hkv, dh), seed + 1, dt)
        s.vp = _normal((case["groups"] * case["prefix"], hkv, dh), seed + 2, dt)
        s.kt = _normal((nseq * case["room"], hkv, dh), seed + 3, dt)
        s.vt = _normal((nseq * case["room"], hkv, dh), seed + 4, dt)
        s.out = torch.empty((rows, hq, dh), dtype=dt, device="cuda")
    elif s.op == "select":
        rows = case["groups"] * case["beams"]
        wide = _normal((rows, case["vocab"] + case["pad"]), seed, TYPES[case["logits"]], 3.0)
        s.logits = wide[:, :case["vocab"]]
        s.scores = -20.0 + _normal((rows,), seed + 1, torch.float32, 2.0)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + 2)
        s.done = (torch.rand(rows, generator=g, device="cuda") < case["done"]).to(torch.int32) if case["done"] else None
    else:
        parents, lens = _parents(case)
        s.parent, s.len = _ints(parents), _ints(lens)
        s.tails = _normal((2, case["layers"], len(parents) * case["room"], hkv, dh), seed, dt)
        s.k, s.v = s.tails                    # every layer's keys, every layer's values
    return s


_CONTEXTS = {}


def _context(s, layout="adjacent"):
    """the program's context for a model: one for all of its calls"""
    key = (s.case["model"], layout)
    if key not in _CONTEXTS:
        import paper_2405_16444_amd as P
        m = SimpleNamespace(n_layers=MODELS[key[0]][0], d_model=s.hq * s.dh, n_q_heads=s.hq, n_kv_heads=s.hkv, head_dim=s.dh,
                            d_ff=4 * s.hq * s.dh, rms_eps=s.eps, rope_theta=s.theta, dtype=MODELS[key[0]][6], rope_layout=layout)
        _CONTEXTS[key] = P.cb_create(m, POSITIONS)
    return _CONTEXTS[key]


def _run_own(s):
    import paper_2405_16444_amd as P
    c = s.case
    if s.op == "rope":
        P.cb_qkv_norm_rope(_context(s, c["layout"]), s.qkv, s.pos, s.row, s.k, s.v, q_norm=s.q_norm, k_norm=s.k_norm, q_out=s.q_out)
        return {"q": s.q_out, "k": s.k, "v": s.v}
    if s.op == "attention":
        ctx = _context(s)
        if not hasattr(s, "ws"):
            s.ws = torch.empty(P.cb_shared_prefix_workspace_bytes(ctx, *s.n, c["prefix"], c["room"]), dtype=torch.uint8, device="cuda")
        return P.cb_shared_prefix_attention(ctx, s.q, *s.n, s.kp, s.vp, s.prefix, s.kt, s.vt, s.row_tail, out=s.out, workspace=s.ws)
    ctx = _context(s)
    if s.op == "select":
        if not hasattr(s, "ws"):
            s.ws = torch.empty(P.cb_beam_select_workspace_bytes(ctx, c["groups"], c["beams"], c["vocab"], c["keep"]), dtype=torch.uint8,
                               device="cuda")
        scores, beam, token = P.cb_beam_select(ctx, s.logits, s.scores, c["groups"], c["keep"], finished=s.done, end_token=2, workspace=s.ws)
        return {"scores": scores, "beam": beam, "token": token}
    P.cb_beam_reorder(ctx, s.k, s.v, c["groups"], s.parent, s.len)
    return s.tails


def _rotate(x, cos, sin, layout):
    """x [rows, heads, dh]; cos, sin [rows, 1, dh / 2]"""
    if layout == "adjacent":
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    a, b = x.chunk(2, -1)
    return torch.cat((a * cos - b * sin, a * sin + b * cos), -1)


def _run_rope(s):
    c, dt = s.case, s.qkv.dtype
    q, k, v = s.qkv.view(-1, s.hq + 2 * s.hkv, s.dh).split((s.hq, s.hkv, s.hkv), 1)
    i = torch.arange(s.dh // 2, dtype=torch.float64, device="cuda")
    angle = s.pos.double()[:, None, None] * s.theta ** (-2.0 * i / s.dh)
    cos, sin = angle.cos().float(), angle.sin().float()
    q, k = q.float(), k.float()
    if s.q_norm is not None:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + s.eps) * s.q_norm.float()
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + s.eps) * s.k_norm.float()
    s.q_out.copy_(_rotate(q, cos, sin, c["layout"]).to(dt))
    # rows without a place go to an extra one behind the cache
    at = torch.where(s.row >= 0, s.row, s.k.shape[0]).long()
    for cache, new in ((s.k, _rotate(k, cos, sin, c["layout"]).to(dt)), (s.v, v)):
        wide = torch.cat((cache, cache[:1]))
        wide[at] = new
        cache.copy_(wide[:-1])
    return {"q": s.q_out, "k": s.k, "v": s.v}


def _run_attention(s):
    G, S, Q = s.n
    hkv, g, dh, P, R, T = s.hkv, s.hq // s.hkv, s.dh, s.case["prefix"], s.case["room"], s.longest
    q = s.q.view(G, S, Q, hkv, g, dh).float() * dh ** -0.5
    kp, vp = (t.view(G, P, hkv, dh).transpose(1, 2).float() for t in (s.kp, s.vp))
    kt, vt = (t.view(G, S, R, hkv, dh)[:, :, :T].transpose(2, 3).float() for t in (s.kt, s.vt))
    seen = s.row_tail.view(G, S, 1, Q, 1, 1)
    qp = q.permute(0, 3, 1, 2, 4, 5).reshape(G, hkv, S * Q * g, dh)
    sp = torch.matmul(qp, kp.transpose(-1, -2)).view(G, hkv, S, Q, g, P).transpose(1, 2)
    sp = sp.masked_fill(torch.arange(P, device="cuda") >= s.prefix_len.view(G, 1, 1, 1, 1, 1), -math.inf)
    qt = q.permute(0, 1, 3, 2, 4, 5).reshape(G, S, hkv, Q * g, dh)
    st = torch.matmul(qt, kt.transpose(-1, -2)).view(G, S, hkv, Q, g, T)
    st = st.masked_fill(torch.arange(T, device="cuda") >= seen, -math.inf)
    top = torch.maximum(sp.amax(-1, keepdim=True), st.amax(-1, keepdim=True))
    sp, st = torch.exp(sp - top), torch.exp(st - top)
    total = sp.sum(-1, keepdim=True) + st.sum(-1, keepdim=True)
    op = torch.matmul(sp.transpose(1, 2).reshape(G, hkv, S * Q * g, P), vp).view(G, hkv, S, Q, g, dh).transpose(1, 2)
    ot = torch.matmul(st.view(G, S, hkv, Q * g, T), vt).view(G, S, hkv, Q, g, dh)
    out = torch.where(seen >= 0, (op + ot) / total, 0.0)
    return out.permute(0, 1, 3, 2, 4, 5).reshape(G * S * Q, s.hq, dh).to(s.q.dtype)


def _run_select(s):
    c = s.case
    x = s.logits.double()
    top = x.amax(-1, keepdim=True)
    lse = top + torch.exp(x - top).sum(-1, keepdim=True).log()
    cand = s.scores.double()[:, None] + (x - lse)
    if s.done is not None:             # a beam at its end goes on with its score and the end token alone
        ended = torch.where(torch.arange(c["vocab"], device="cuda") == 2, s.scores.double()[:, None], -math.inf)
        cand = torch.where(s.done[:, None] != 0, ended, cand)
    best, at = torch.sort(cand.view(c["groups"], -1), dim=-1, descending=True, stable=True)
    best, at = best[:, :c["keep"]], at[:, :c["keep"]]
    real = best > -math.inf
    return {"scores": best.float(), "beam": torch.where(real, at // c["vocab"], -1).to(torch.int32),
            "token": torch.where(real, at % c["vocab"], -1).to(torch.int32)}


def _run_reorder(s):
    c = s.case
    t = s.tails.view(2, c["layers"], c["groups"], c["beams"], c["room"], s.hkv * s.dh)
    p = s.parent.view(c["groups"], c["beams"]).long()
    moved = t[:, :, torch.arange(c["groups"], device="cuda")[:, None], p]
    rows = s.len.view(c["groups"], c["beams"]).gather(1, p)
    inside = torch.arange(c["room"], device="cuda") < rows[..., None]
    t.copy_(torch.where(inside[..., None], moved, t))
    return s.tails


def run(s):
    if own:
        return _run_own(s)
    return {"rope": _run_rope, "attention": _run_attention, "select": _run_select, "reorder": _run_reorder}[s.op](s)


def work(case):
    layers, hq, hkv, dh, _, _, dtype = MODELS[case["model"]]
    es, row = (4 if dtype == "f32" else 2), hkv * dh
    if case["op"] == "rope":
        n = case["rows"]
        kept = n - len(range(0, n, 17)) if n > 16 else n
        moved = n * hq * dh * es * 2 + kept * row * es * 4 + n * 8 + min(n, case["far"]) * dh * 4
        return {"bytes": moved, "flops": (6.0 * n + (10.0 * n if case["norms"] else 0)) * (hq + hkv) * dh / 2}
    if case["op"] == "attention":
        prefix, tails = _lengths(case)
        new = sum(n for _, n in tails)
        keys = sum(prefix) + sum(t for t, _ in tails)
        pairs = 0.0
        for i, (t, n) in enumerate(tails):
            pairs += n * (prefix[i // case["seqs"]] + t - (n - 1) / 2)
        rows = len(tails) * case["queries"]
        return {"bytes": (new + rows) * hq * dh * es + keys * row * es * 2 + rows * 4, "flops": 4.0 * hq * dh * pairs}
    if case["op"] == "select":
        rows, les = case["groups"] * case["beams"], 4 if case["logits"] == "f32" else 2
        return {"bytes": rows * (case["vocab"] * les + 8) + case["groups"] * case["keep"] * 12, "flops": 3.0 * rows * case["vocab"]}
    parents, lens = _parents(case)
    B, read, written = case["beams"], 0, 0
    for g in range(case["groups"]):
        p, n = parents[g * B:(g + 1) * B], lens[g * B:(g + 1) * B]
        out = [b for b in range(B) if p[b] != b]
        written += sum(n[p[b]] for b in out)
        read += sum(n[a] for a in {p[b] for b in out})
    return {"bytes": max(1, (read + written) * row * es * 2 * case["layers"]) + 8 * len(parents), "flops": 0.0}


def exact(case, seed):
    """From the definitions, in 64 bits, one continuation or one layout at a time."""
    s = prepare(case, seed)
    if s.op == "rope":
        x = s.qkv.double().reshape(case["rows"], -1, s.dh)
        half = s.dh // 2
        if case["layout"] == "adjacent":
            first = torch.arange(0, s.dh, 2, device="cuda")
            second = first + 1
        else:
            first = torch.arange(half, device="cuda")
            second = first + half
        turn = torch.pow(torch.tensor(float(s.theta), dtype=torch.float64, device="cuda"), -torch.arange(half, device="cuda").double() / half)
        z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s.pos.double()[:, None] * turn)
        heads = []
        for h in range(s.hq + s.hkv):
            y = x[:, h]
            if case["norms"]:
                y = y / (y.pow(2).sum(-1, keepdim=True) / s.dh + s.eps).sqrt() * (s.q_norm if h < s.hq else s.k_norm).double()
            y = torch.complex(y[:, first], y[:, second]) * z
            w = torch.empty((case["rows"], s.dh), dtype=torch.float64, device="cuda")
            w[:, first], w[:, second] = y.real, y.imag
            heads.append(w)
        kept = (s.row >= 0).nonzero().flatten()
        k, v = s.k.double(), s.v.double()
        for h in range(s.hkv):
            k[s.row[kept].long(), h] = heads[s.hq + h][kept]
            v[s.row[kept].long(), h] = x[kept, s.hq + s.hkv + h]
        return {"q": torch.stack(heads[:s.hq], 1), "k": k, "v": v}
    if s.op == "attention":
        prefix, tails = _lengths(case)
        Q, g = case["queries"], s.hq // s.hkv
        out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
        for b, (t, n) in enumerate(tails):
            group, p = b // case["seqs"], prefix[b // case["seqs"]]
            k, v = (torch.cat((c[group * case["prefix"]:group * case["prefix"] + p], own_[b * case["room"]:b * case["room"] + t])).double()
                    for c, own_ in ((s.kp, s.kt), (s.vp, s.vt)))
            future = torch.arange(p + t, device="cuda") > p + t - n + torch.arange(n, device="cuda")[:, None]
            for h in range(s.hq):
                a = s.q[b * Q:b * Q + n, h].double() @ k[:, h // g].T / math.sqrt(s.dh)
                out[b * Q:b * Q + n, h] = torch.softmax(a.masked_fill(future, -math.inf), -1) @ v[:, h // g]
        return out
    if s.op == "select":
        rows = []
        for r in range(case["groups"] * case["beams"]):
            if s.done is not None and int(s.done[r]):
                rows.append(s.scores[r:r + 1].double())
            else:
                rows.append((s.scores[r].double() + torch.log_softmax(s.logits[r].double(), -1)).topk(min(case["keep"], case["vocab"])).values)
        B, best = case["beams"], []
        for i in range(case["groups"]):
            pool = torch.cat(rows[i * B:(i + 1) * B]).sort(descending=True).values[:case["keep"]]
            best.append(torch.cat((pool, torch.full((case["keep"] - len(pool),), -math.inf, dtype=torch.float64, device="cuda"))))
        return {"scores": torch.stack(best), "beam": None, "token": None}
    new = s.tails.double()
    parents, lens, B, R = s.parent.tolist(), s.len.tolist(), case["beams"], case["room"]
    for b, p in enumerate(parents):
        a = b // B * B + p
        new[:, :, b * R:b * R + lens[a]] = s.tails[:, :, a * R:a * R + lens[a]].double()
    return new
