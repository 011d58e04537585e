"""Cases for the reader operators: what a program does with trained vectors once it has them.

A reader turns the static vector of every word of a token stream into a vector of the word in its
place: layer norm over the rows, attention over a window of the word's sentence (with the first words
of the sentence kept visible and a learned bias by distance), and, to answer with words, the product
of one vector with the whole output table held in 4 bits.  Training runs the first two backwards;
serving has a form of the attention for one new token per sequence.

`run` computes an operator in its plain form where `own` is false, and calls the library where it is
true; `exact` has the same results in 64 bits, from the definitions.
"""
import math

import numpy as np
import torch

own = False

VOCAB = 10_000                  # ids outside [0, VOCAB) are out of vocabulary; -1 ends a sentence
EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_model = None


def model():
    """The library's handle, as a program keeps one for its whole life."""
    global _model
    if _model is None:
        from paper_1606_08495_b200.binding import W2V
        _model = W2V(VOCAB, 100, seed=1)
    return _model


# ---- the cases -----------------------------------------------------------------------------
def listed():
    norm = dict(kind="norm", pad=0, train=True)
    att = dict(kind="attend", train=True, type="bf16", sinks=0, two_sided=True, buckets=32, reach=128)
    tok = dict(kind="token", type="bf16", sinks=4, buckets=32, reach=128)
    return [
        # one step of serving: a handful of vectors on their way to the next operator
        dict(norm, name="norm_step", rows=8, d=320, x="bf16", y="bf16", train=False),
        # the vectors of a 262,144-token minibatch, read out of the fp32 table with its 128-byte row grid
        dict(norm, name="norm_table_rows", rows=262_144, d=300, pad=20, x="f32", y="bf16"),
        # a wide model's activations, an odd number of rows
        dict(norm, name="norm_wide", rows=8_191, d=4_096, x="bf16", y="bf16"),
        # one short sentence, answered at once
        dict(att, name="attend_sentence", tokens=77, low=76, high=76, heads=5, kv=5, dim=64, left=10, right=10, train=False),
        # sessions of 5 to 40 words: a minibatch of 131,072 tokens, window 10, four attention heads of 80
        dict(att, name="attend_sessions", tokens=131_072, low=5, high=40, heads=4, kv=4, dim=80, left=10, right=10),
        # sentences of 1,000 words: a 65,536-token minibatch seen through 128 words either way
        dict(att, name="attend_sentences", tokens=65_536, low=1_000, high=1_000, heads=5, kv=5, dim=64, left=128, right=128, sinks=2),
        # long documents, read forwards, heads that share keys and values
        dict(att, name="attend_documents", tokens=16_381, low=2_000, high=9_000, heads=16, kv=4, dim=128, left=1_023, right=0, sinks=4,
             two_sided=False),
        # a long prompt before serving starts
        dict(att, name="attend_prompt", tokens=32_768, low=32_767, high=32_767, heads=8, kv=2, dim=64, left=4_095, right=0, sinks=4,
             two_sided=False, type="f16", train=False),
        # one user's next word
        dict(tok, name="token_one", batch=1, heads=5, kv=5, dim=64, left=1_000, low=0, high=5_000),
        # the next word of many conversations of all lengths, some of them empty places in the batch
        dict(tok, name="token_many", batch=96, heads=16, kv=4, dim=128, left=4_095, low=-1, high=20_000),
        # scores of one context vector against a 71,000-word table
        dict(kind="scores", name="scores_small", rows=71_000, d=200, m=1, group=32),
        # four context vectors against a table of four million words
        dict(kind="scores", name="scores_table", rows=4_000_001, d=300, m=4, group=32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "attend", "attend", "token", "scores"])
    if kind == "norm":
        d = rng.choice([100, 200, 300, 320, 64 * _log(rng, 1, 64), _log(rng, 8, 4096)])
        rows = _log(rng, 1, 70_000_000 // d if d <= 1024 else 33_000_000 // d)
        x = rng.choice(["f32", "bf16", "f16"])
        return dict(kind="norm", rows=rows, d=d, pad=rng.choice([0, 0, 4, 20]), x=x, y=rng.choice([x, "bf16"]) if x == "f32" else x,
                    train=rng.random() < 0.7)
    if kind == "attend":
        kv, dim = rng.choice([1, 2, 4, 5]), rng.choice([32, 64, 64, 80, 96, 128])
        heads = kv * rng.choice([1, 1, 2, 4])
        causal = rng.random() < 0.4
        left = _log(rng, 1, 2048)
        right = 0 if causal else min(left, 512)
        # tokens x heads x (keys seen) is held below the long documents' work
        tokens = _log(rng, 1, max(2, min(131_072, 200_000_000 // (heads * (left + right + 64)), 40_000_000 // (heads * dim))))
        high = max(1, min(tokens, _log(rng, 3, 10_000)))
        return dict(kind="attend", train=rng.random() < 0.7, type=rng.choice(["bf16", "f16"]), tokens=tokens, low=max(1, high // rng.choice([1, 2, 8])),
                    high=high, heads=heads, kv=kv, dim=dim, left=left, right=right, sinks=rng.choice([0, 1, 4, 7]), two_sided=not causal,
                    buckets=rng.choice([0, 16, 32, 32]), reach=rng.choice([128, 200, 512]))
    if kind == "token":
        kv, dim = rng.choice([1, 2, 4, 5, 8]), rng.choice([32, 64, 80, 128])
        left = _log(rng, 1, 8192)
        batch = _log(rng, 1, max(1, min(256, 96 * 4 * 128 * 4096 // (kv * dim * (left + 1)))))
        return dict(kind="token", type=rng.choice(["bf16", "f16"]), batch=batch, heads=kv * rng.choice([1, 2, 4]), kv=kv, dim=dim, left=left,
                    sinks=rng.choice([0, 1, 4, 7]), low=rng.choice([-1, 0]), high=_log(rng, 4, 30_000), buckets=rng.choice([0, 32]), reach=128)
    d = rng.choice([100, 200, 300, 320, 512, 1024, 4096, _log(rng, 8, 4096)])
    return dict(kind="scores", rows=_log(rng, 1, 4_000_000 * 300 // max(300, d)), d=d, m=rng.choice([1, 1, 2, 3, 4, 8]) if d <= 1024 else 1,
                group=rng.choice([32, 64, 128]))


# ---- the inputs ----------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + 11)
    rng = np.random.default_rng(seed)

    def normal(*shape, type=torch.float32, by=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * by).to(type)

    s = dict(case=dict(case))
    if case["kind"] == "norm":
        rows, d, pad = case["rows"], case["d"], case["pad"]
        by = 0.02 if case["x"] == "f32" else 1.0          # trained fp32 vectors are small; activations are not
        s["x"] = (normal(rows, d + pad) * by + by * normal(1, d + pad)).to(TYPES[case["x"]])[:, :d]
        s["gamma"], s["beta"] = 1 + normal(d, by=0.2), normal(d, by=0.2)
        if case["train"]:
            s["dy"] = normal(rows, d, type=TYPES[case["y"]])
    elif case["kind"] == "attend":
        n, h, kv, dim, t = case["tokens"], case["heads"], case["kv"], case["dim"], TYPES[case["type"]]
        lens = rng.integers(case["low"], case["high"] + 1, n // (case["low"] + 1) + 1)
        stream = rng.integers(0, VOCAB, n).astype(np.int32)
        stream[rng.random(n) < 0.01] = VOCAB + 5            # words that the vocabulary does not have
        ends = np.cumsum(lens + 1) - 1
        stream[ends[ends < n]] = -1
        s["tokens"] = torch.from_numpy(stream).cuda()
        s["qkv"] = normal(n, (h + 2 * kv) * dim, type=t)    # one projection's output, cut in three
        s["q"], s["k"], s["v"] = (x.view(n, -1, dim) for x in (s["qkv"][:, : h * dim], s["qkv"][:, h * dim: (h + kv) * dim], s["qkv"][:, (h + kv) * dim:]))
        s["bias"] = normal(case["buckets"], h, by=0.5) if case["buckets"] else None
        if case["train"]:
            s["do"] = normal(n, h, dim, type=t)
    elif case["kind"] == "token":
        b, h, kv, dim, t = case["batch"], case["heads"], case["kv"], case["dim"], TYPES[case["type"]]
        places = case["sinks"] + case["left"] + 1
        s["pos"] = torch.from_numpy(rng.integers(case["low"], case["high"] + 1, b).astype(np.int32)).cuda()
        s["q"], s["k"], s["v"] = normal(b, h, dim, type=t), normal(b, kv, dim, type=t), normal(b, kv, dim, type=t)
        s["cache_k"], s["cache_v"] = normal(b, places, kv, dim, type=t), normal(b, places, kv, dim, type=t)
        s["bias"] = normal(case["buckets"], h, by=0.5) if case["buckets"] else None
    else:
        rows, d, group = case["rows"], case["d"], case["group"]
        # the table as a program keeps it: two columns a byte (low half first, value + 8), bf16 scales by groups of
        # columns, both padded to whole words of 32 columns
        wide = -(-d // 32) * 32
        packed = torch.randint(0, 256, (rows, wide // 2), generator=g, device="cuda", dtype=torch.uint8)
        packed = torch.where((packed & 15) == 0, packed | 8, packed)            # stored values are 1..15
        packed = torch.where((packed >> 4) == 0, packed | 128, packed)
        s["packed"] = torch.where(torch.arange(wide // 2, device="cuda") * 2 < d, packed, torch.full_like(packed, 0x88))
        if d % 2:
            s["packed"][:, d // 2] = (s["packed"][:, d // 2] & 15) | 128
        s["scales"] = (0.002 + 0.004 * torch.rand(rows, -(-d // group), generator=g, device="cuda")).to(torch.bfloat16)
        s["x"] = normal(case["m"], d)
    return s


# ---- the plain forms -----------------------------------------------------------------------
def _plain_norm(s):
    c, x, w = s["case"], s["x"].float(), s["gamma"]
    mean = x.mean(1, keepdim=True)
    x = x - mean
    rstd = (x.square().mean(1, keepdim=True) + EPS).rsqrt()
    x = x * rstd
    out = {"y": (x * w + s["beta"]).to(TYPES[c["y"]])}
    if c["train"]:
        dy = s["dy"].float()
        out["dgamma"], out["dbeta"] = (dy * x).sum(0), dy.sum(0)
        dy = dy * w
        out["dx"] = (rstd * (dy - dy.mean(1, keepdim=True) - x * (dy * x).mean(1, keepdim=True))).to(s["x"].dtype)
    return out


def _buckets(rel, c):
    """Bucket of a key at distance `rel` after the query (before it: negative).  One side: the past only, a key after
    the query counts as distance 0.  Two sides: the second half of the buckets is for keys after the query.  Of a side's
    n buckets the first n/2 hold one distance each, bucket n/2 + k starts at ceil(n/2 (reach / (n/2))^(k / (n - n/2)))."""
    n = c["buckets"] // 2 if c["two_sided"] else c["buckets"]
    first = n // 2
    k = torch.arange(n - first, device=rel.device, dtype=torch.float64)
    starts = (first * (c["reach"] / first) ** (k / (n - first)) * (1 - 1e-12)).ceil().long()
    far = rel.abs() if c["two_sided"] else (-rel).clamp(min=0)
    b = torch.where(far < first, far, first - 1 + (torch.bucketize(far, starts, right=True)))
    return b + n * (rel > 0) if c["two_sided"] else b


def _plain_attend(s):
    c, q, k, v = s["case"], s["q"], s["k"], s["v"]
    n, h, dim = q.shape
    kv, left, right, sinks = c["kv"], c["left"], c["right"], c["sinks"]
    at, sep = torch.arange(n, device="cuda"), s["tokens"] == -1
    start = torch.where(sep, at + 1, 0).cummax(0).values
    end = torch.where(sep, at, n).flip(0).cummin(0).values.flip(0)
    seen = (s["tokens"] >= 0) & (s["tokens"] < VOCAB)
    size = min(512, max(32, (left + right) // 2))                 # queries that share a band of keys
    nb = -(-n // size)
    rows = torch.arange(nb * size, device="cuda").view(nb, size)
    real, ri = rows < n, rows.clamp(max=n - 1)
    band = (torch.arange(nb, device="cuda") * size - left)[:, None] + torch.arange(size + left + right, device="cuda")
    bi = band.clamp(0, n - 1)
    i, j = ri[:, :, None], band[:, None, :]
    a, e = start[ri][:, :, None], end[ri][:, :, None]
    ok = (j >= i - left) & (j <= i + right) & (j >= a) & (j < e) & seen[bi][:, None, :] & (seen[ri] & real)[:, :, None]
    first = a + torch.arange(sinks, device="cuda")                  # [nb, size, sinks]
    fi = first.clamp(max=n - 1)
    fok = (first < i - left) & (first < e) & seen[fi] & (seen[ri] & real)[:, :, None]
    qf = (q.float()[ri] * dim ** -0.5).view(nb, size, kv, h // kv, dim)
    kf, vf = k.float(), v.float()
    kb, vb, kfirst, vfirst = kf[bi], vf[bi], kf[fi], vf[fi]
    score = torch.cat([torch.einsum("bchgd,bwhd->bhgcw", qf, kb), torch.einsum("bchgd,bcshd->bhgcs", qf, kfirst)], -1)
    if s["bias"] is not None:
        near = _buckets((band[:1] - rows[:1].T), c)                 # [size, band]: the same for every block
        firstb = _buckets(first - i, c)
        bias = s["bias"].float().t().reshape(kv, h // kv, -1)
        score[..., : band.shape[1]] += bias[:, :, near]
        if sinks:
            score[..., band.shape[1]:] += bias[:, :, firstb].permute(2, 0, 1, 3, 4)
    score.masked_fill_(~torch.cat([ok, fok], -1)[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-1e30)
    p = score.sub_(top).exp_()
    del score
    p /= p.sum(-1, keepdim=True).clamp(min=1e-30)                # a row that sees nothing stays zero
    w = band.shape[1]
    o = torch.einsum("bhgcw,bwhd->bchgd", p[..., :w], vb) + torch.einsum("bhgcs,bcshd->bchgd", p[..., w:], vfirst)
    out = {"o": o.reshape(nb * size, h, dim)[:n].to(q.dtype)}
    if c["train"]:
        do = (s["do"].float()[ri] * real[:, :, None, None]).view(nb, size, kv, h // kv, dim)
        dv = torch.zeros_like(vf).index_add_(0, bi.reshape(-1), torch.einsum("bhgcw,bchgd->bwhd", p[..., :w], do).reshape(-1, kv, dim))
        if sinks:
            dv.index_add_(0, fi.reshape(-1), torch.einsum("bhgcs,bchgd->bcshd", p[..., w:], do).reshape(-1, kv, dim))
        ds = torch.cat([torch.einsum("bchgd,bwhd->bhgcw", do, vb), torch.einsum("bchgd,bcshd->bhgcs", do, vfirst)], -1)
        ds = (ds - (do * o).sum(-1).permute(0, 2, 3, 1)[..., None]).mul_(p)
        del p, vb, vfirst
        dq = torch.einsum("bhgcw,bwhd->bchgd", ds[..., :w], kb) + torch.einsum("bhgcs,bcshd->bchgd", ds[..., w:], kfirst)
        dk = torch.zeros_like(kf).index_add_(0, bi.reshape(-1), torch.einsum("bhgcw,bchgd->bwhd", ds[..., :w], qf).reshape(-1, kv, dim))
        if sinks:
            dk.index_add_(0, fi.reshape(-1), torch.einsum("bhgcs,bchgd->bcshd", ds[..., w:], qf).reshape(-1, kv, dim))
        out["dq"] = (dq.reshape(nb * size, h, dim)[:n] * dim ** -0.5).to(q.dtype)
        out["dk"], out["dv"] = dk.to(q.dtype), dv.to(q.dtype)
        if s["bias"] is not None:
            db = torch.zeros(c["buckets"], h, device="cuda").index_add_(0, near.reshape(-1), ds[..., :w].sum(0).reshape(h, -1).t())
            if sinks:
                db.index_add_(0, firstb.reshape(-1), ds[..., w:].permute(0, 3, 4, 1, 2).reshape(-1, h))
            out["dbias"] = db
    return out


def _plain_token(s):
    c, q, pos = s["case"], s["q"], s["pos"].long()
    b, h, dim = q.shape
    kv, left, sinks = c["kv"], c["left"], c["sinks"]
    ck, cv = s["cache_k"], s["cache_v"]
    ring = ck.shape[1] - sinks
    place = torch.where(pos < sinks, pos, sinks + (pos - sinks) % ring)
    live = pos >= 0
    each = torch.arange(b, device="cuda")
    place = place.clamp(min=0)
    ck[each, place] = torch.where(live[:, None, None], s["k"], ck[each, place])
    cv[each, place] = torch.where(live[:, None, None], s["v"], cv[each, place])
    slot = torch.arange(ck.shape[1], device="cuda")
    last = pos[:, None]
    held = torch.where(slot < sinks, slot, last - (last - slot) % ring)          # the position that a place holds now
    ok = (held <= last) & (held >= torch.where(slot < sinks, 0, sinks)) & ((held >= last - left) | (slot < sinks))
    score = torch.einsum("bhgd,bwhd->bhgw", (q.float() * dim ** -0.5).view(b, kv, h // kv, dim), ck.float())
    if s["bias"] is not None:
        score += s["bias"].float().t()[:, _buckets(held - last, dict(c, two_sided=False))].reshape(kv, h // kv, b, -1).permute(2, 0, 1, 3)
    score.masked_fill_(~ok[:, None, None], -math.inf)
    p = (score - score.amax(-1, keepdim=True).clamp(min=-1e30)).exp()
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    o = torch.einsum("bhgw,bwhd->bhgd", p, cv.float()).reshape(b, h, dim).to(q.dtype)
    return {"o": o, "cache_k": ck, "cache_v": cv}


def _plain_scores(s):
    d, group, packed = s["case"]["d"], s["case"]["group"], s["packed"]
    w = torch.stack([packed & 15, packed >> 4], -1).view(packed.shape[0], -1)[:, :d].float().sub_(8)
    w *= s["scales"].float().repeat_interleave(group, 1)[:, :d]
    return {"scores": s["x"] @ w.t()}


# ---- the operators -------------------------------------------------------------------------
def run(s):
    c = s["case"]
    if not own:
        return {"norm": _plain_norm, "attend": _plain_attend, "token": _plain_token, "scores": _plain_scores}[c["kind"]](s)
    m = model()
    if c["kind"] == "norm":
        y, saved = m.layer_norm(s["x"], s["gamma"], s["beta"], EPS, TYPES[c["y"]])
        if not c["train"]:
            return {"y": y}
        dx, dgamma, dbeta = m.layer_norm_backward(s["dy"], saved)
        return {"y": y, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if c["kind"] == "scores":
        return {"scores": m.fourbit_scores(s["x"], s["packed"], s["scales"], c["group"])}
    over = dict(left=c["left"], right=c.get("right", 0), sinks=c["sinks"], reach=c["reach"], two_sided=c.get("two_sided", False))
    if c["kind"] == "token":
        o = m.attend_token(s["q"], s["k"], s["v"], s["cache_k"], s["cache_v"], s["pos"], s["bias"], **over)
        return {"o": o, "cache_k": s["cache_k"], "cache_v": s["cache_v"]}
    spans = m.sentence_spans(s["tokens"])
    if not c["train"]:
        return {"o": m.attend(s["q"], s["k"], s["v"], spans, s["bias"], **over)}
    o, saved = m.attend(s["q"], s["k"], s["v"], spans, s["bias"], train=True, **over)
    dq, dk, dv, dbias = m.attend_backward(s["do"], saved)
    out = {"o": o, "dq": dq, "dk": dk, "dv": dv}
    return dict(out, dbias=dbias) if dbias is not None else out


# ---- what a pass cannot do without -----------------------------------------------------------
def _pairs(c):
    """Mean number of (query, key) pairs of a case's stream, sinks included."""
    total = words = 0.0
    for length in np.unique(np.linspace(c["low"], c["high"], 17).astype(int)):
        i = np.arange(length)
        total += float((np.minimum(i + c["right"], length - 1) - np.maximum(i - c["left"], 0) + 1 + np.minimum(c["sinks"], np.maximum(i - c["left"], 0))).sum())
        words += length + 1
    return total * c["tokens"] / words


def work(case):
    c, size = case, {"f32": 4, "bf16": 2, "f16": 2}
    if c["kind"] == "norm":
        n = c["rows"] * c["d"]
        fwd = n * (size[c["x"]] + size[c["y"]])
        return {"bytes": fwd + (n * (2 * size[c["x"]] + size[c["y"]]) if c["train"] else 0) + 16 * c["d"], "flops": n * (16 if c["train"] else 6)}
    if c["kind"] == "scores":
        wide = -(-c["d"] // 32) * 32
        return {"bytes": c["rows"] * (wide // 2 + 2 * -(-c["d"] // c["group"]) + 4 * c["m"]) + 4 * c["m"] * c["d"], "flops": 2 * c["rows"] * c["d"] * c["m"]}
    if c["kind"] == "token":
        low, high = max(0, c["low"]), max(0, c["high"])
        seen = float(np.minimum(np.linspace(low, high, 101) + 1, c["left"] + 1 + c["sinks"]).mean())
        return {"bytes": int(c["batch"] * (4 * c["kv"] * c["dim"] * (seen + 1) + 4 * c["heads"] * c["dim"])), "flops": int(4 * c["batch"] * c["heads"] * c["dim"] * seen)}
    wide = c["dim"] * c["tokens"] * 2
    fwd = wide * (2 * c["heads"] + 2 * c["kv"]) + 4 * c["tokens"]
    back = wide * (4 * c["heads"] + 4 * c["kv"]) if c["train"] else 0
    return {"bytes": int(fwd + back), "flops": int(_pairs(c) * c["heads"] * c["dim"] * (14 if c["train"] else 4))}


# ---- the definitions in 64 bits ----------------------------------------------------------------
def _exact_bucket_starts(n, reach):
    """The first distance of each of a side's n buckets, in whole numbers only: bucket n/2 + k starts at the least m
    with m^N >= e^(N - k) reach^k, e = n/2, N = n - e."""
    e = n // 2
    starts = list(range(e))
    for k in range(n - e):
        want, lo, hi = e ** (n - e - k) * reach ** k, e, reach
        while lo < hi:
            mid = (lo + hi) // 2
            lo, hi = (lo, mid) if mid ** (n - e) >= want else (mid + 1, hi)
        starts.append(lo)
    return starts


def _exact_bias(bias, rel, buckets, reach, two_sided):
    """(values [heads, ...], buckets) of the bias at the distances `rel`."""
    n = buckets // 2 if two_sided else buckets
    starts = torch.tensor(_exact_bucket_starts(n, reach), device=rel.device)
    far = rel.abs() if two_sided else (-rel).clamp(min=0)
    which = torch.searchsorted(starts, far.contiguous(), right=True) - 1
    if two_sided:
        which = which + n * (rel > 0).long()
    return bias.double()[which].movedim(-1, 0), which


def _exact_attend(s):
    c, toks = s["case"], s["tokens"].cpu().numpy()
    n, h, dim = s["q"].shape
    kv, group = c["kv"], h // c["kv"]
    start, end, begin = np.zeros(n, np.int64), np.zeros(n, np.int64), 0
    for stop in list(np.flatnonzero(toks == -1)) + [n]:
        start[begin: stop + 1], end[begin: stop + 1], begin = begin, stop, stop + 1
    seen = torch.from_numpy((toks >= 0) & (toks < VOCAB)).cuda()
    q, k, v = (s[x].double() for x in "qkv")
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    out = {"o": torch.zeros(n, h, dim, dtype=torch.float64, device="cuda")}
    if c["train"]:
        out |= {x: torch.zeros(n, h, dim, dtype=torch.float64, device="cuda") for x in ("dq", "dk", "dv")}
        if s["bias"] is not None:
            out["dbias"] = torch.zeros(c["buckets"], h, dtype=torch.float64, device="cuda")
    chunk = 512
    for i0 in range(0, n, chunk):
        i1 = min(n, i0 + chunk)
        band = np.arange(max(0, i0 - c["left"]), min(n, i1 + c["right"]))
        begins = np.unique(start[i0:i1])
        firsts = (begins[:, None] + np.arange(c["sinks"])).reshape(-1)
        j = torch.from_numpy(np.unique(np.concatenate([band, firsts[firsts < n]]))).cuda()
        i = torch.arange(i0, i1, device="cuda")[:, None]
        a, e = torch.from_numpy(start[i0:i1]).cuda()[:, None], torch.from_numpy(end[i0:i1]).cuda()[:, None]
        ok = seen[i] & seen[j] & (j >= a) & (j < e) & (((j >= i - c["left"]) & (j <= i + c["right"])) | ((j < a + c["sinks"]) & (j < i)))
        score = torch.einsum("chd,whd->hcw", q[i0:i1], k[j]) / math.sqrt(dim)
        if s["bias"] is not None:
            add, which = _exact_bias(s["bias"], j - i, c["buckets"], c["reach"], c["two_sided"])
            score += add
        score = torch.where(ok, score, torch.tensor(-math.inf, dtype=torch.float64, device="cuda"))
        p = torch.nan_to_num(torch.softmax(score, -1), nan=0.0)
        o = torch.einsum("hcw,whd->chd", p, v[j])
        out["o"][i0:i1] = o
        if c["train"]:
            do = s["do"][i0:i1].double()
            out["dv"].index_add_(0, j, torch.einsum("hcw,chd->whd", p, do))
            ds = p * (torch.einsum("chd,whd->hcw", do, v[j]) - torch.einsum("chd,chd->hc", do, o)[..., None])
            out["dq"][i0:i1] = torch.einsum("hcw,whd->chd", ds, k[j]) / math.sqrt(dim)
            out["dk"].index_add_(0, j, torch.einsum("hcw,chd->whd", ds, q[i0:i1]) / math.sqrt(dim))
            if s["bias"] is not None:
                out["dbias"].index_add_(0, which.reshape(-1), ds.reshape(h, -1).t())
    if c["train"]:
        out |= {x: out[x].view(n, kv, group, dim).sum(2) for x in ("dk", "dv")}
    return out


def _exact_token(s):
    c, q = s["case"], s["q"].double()
    b, h, dim = q.shape
    group, sinks = h // c["kv"], c["sinks"]
    ring = s["cache_k"].shape[1] - sinks
    ck, cv, o = s["cache_k"].double(), s["cache_v"].double(), torch.zeros(b, h, dim, dtype=torch.float64, device="cuda")
    for r, last in enumerate(s["pos"].tolist()):
        if last < 0:
            continue
        p = np.unique(np.concatenate([np.arange(min(sinks, last + 1)), np.arange(max(0, last - c["left"]), last + 1)]))
        at = torch.from_numpy(np.where(p < sinks, p, sinks + (p - sinks) % ring)).cuda()
        ck[r, at[-1]], cv[r, at[-1]] = s["k"][r].double(), s["v"][r].double()
        k, v = ck[r, at].repeat_interleave(group, 1), cv[r, at].repeat_interleave(group, 1)
        score = torch.einsum("hd,whd->hw", q[r], k) / math.sqrt(dim)
        if s["bias"] is not None:
            score = score + _exact_bias(s["bias"], torch.from_numpy(p).cuda() - last, c["buckets"], c["reach"], False)[0]
        o[r] = torch.einsum("hw,whd->hd", torch.softmax(score, -1), v)
    return {"o": o, "cache_k": ck, "cache_v": cv}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "attend":
        return _exact_attend(s)
    if case["kind"] == "token":
        return _exact_token(s)
    if case["kind"] == "scores":
        x, d, out = s["x"].double(), case["d"], torch.empty(case["m"], case["rows"], dtype=torch.float64, device="cuda")
        column = torch.arange(d, device="cuda")
        for r in range(0, case["rows"], 500_000):
            part = s["packed"][r: r + 500_000]
            value = (part[:, column // 2].int() >> (4 * (column % 2)).int()) % 16 - 8
            out[:, r: r + 500_000] = x @ (value.double() * s["scales"][r: r + 500_000].double()[:, column // case["group"]]).t()
        return {"scores": out}
    x, w, b = s["x"].double(), s["gamma"].double(), s["beta"].double()
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    inv = 1 / torch.sqrt(var + EPS)
    hat = (x - mean) * inv
    out = {"y": hat * w + b}
    if case["train"]:
        dy = s["dy"].double()
        out["dgamma"], out["dbeta"] = (dy * hat).sum(0), dy.sum(0)
        g = dy * w
        out["dx"] = inv * (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True))
    return out
