"""The reader operators against their definitions in 64 bits.

Bounds.  u is the unit roundoff of the arrays' type (2^-8 for bfloat16, 2^-11 for float16, 2^-24 for
float32).  Every result is rounded once to its type (u |result|); attention also rounds the softmax
weights and the score gradients once to that type before the matrix products (u times the sum of the
absolute products); what is left are fp32 sums and exponentials, for which 2^-18 of the sum of absolute
products is allowed (scores of magnitude below 32 lose 32 * 2^-24 each, the exponential passes that on).
"""
import math

import numpy as np
import pytest
import torch

from paper_1606_08495_b200 import binding

pytestmark = pytest.mark.gpu

VOCAB = 1000
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
F32 = 2.0 ** -18


@pytest.fixture(scope="module")
def model():
    m = binding.W2V(VOCAB, 64, seed=3)
    yield m
    m.close()


def randn(*shape, seed, dtype=torch.float32, by=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * by).to(dtype)


def inside(got, want, bound, what):
    err = (got.double() - want).abs()
    assert torch.isfinite(got.double()).all(), what
    bad = err > bound
    if bad.any():
        i = int((err - bound).flatten().argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {err.numel()} outside, worst {err.flatten()[i]:.3e} over {torch.as_tensor(bound).expand_as(err).flatten()[i]:.3e}")


# ---- layer norm -----------------------------------------------------------------------------------
NORM_SHAPES = [(1, 1), (3, 2), (5, 7), (257, 100), (64, 200), (1000, 300), (33, 320), (9, 512), (40, 513), (17, 1000), (700, 1024),
               (12, 1536), (5, 2047), (30, 4096), (2, 8192), (3, 8191)]
NORM_TYPES = [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.float32, torch.float16),
              (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16)]


def check_layer_norm(model, x, xt, yt):
    rows, d = x.shape
    g, b = 1 + randn(d, seed=1, by=0.3), randn(d, seed=2, by=0.3)
    dy = randn(rows, d, seed=5, dtype=yt)
    y, saved = model.layer_norm(x, g, b, 1e-5, yt)
    dx, dg, db = model.layer_norm_backward(dy, saved)
    X, G, B, D = x.double(), g.double(), b.double(), dy.double()
    mean = X.mean(1, keepdim=True)
    inv = 1 / torch.sqrt((X - mean).square().mean(1, keepdim=True) + 1e-5)
    hat = (X - mean) * inv
    # the subtraction of the mean loses 2^-24 (|x| + |mean|) times the row's 1/deviation
    lost = 8 * 2.0 ** -24 * (X.abs() + mean.abs()) * inv + F32 * hat.abs()
    inside(y, hat * G + B, U[yt] * (hat * G + B).abs() + lost * G.abs() + 2.0 ** -24 * (hat * G).abs() + 1e-7, "y")
    H = D * G
    dX = inv * (H - H.mean(1, keepdim=True) - hat * (H * hat).mean(1, keepdim=True))
    soft = inv * (H.abs() + H.abs().mean(1, keepdim=True) + hat.abs() * (H * hat).abs().mean(1, keepdim=True))
    shift = (lost * H.abs()).mean(1, keepdim=True)
    inside(dx, dX, U[xt] * dX.abs() + (F32 * soft + inv * (lost * (H * hat).abs().mean(1, keepdim=True) + hat.abs() * shift)) + 1e-7, "dx")
    inside(dg, (D * hat).sum(0), F32 * (D * hat).abs().sum(0) + (D.abs() * lost).sum(0) + 1e-7, "dgamma")
    inside(db, D.sum(0), F32 * D.abs().sum(0) + 1e-7, "dbeta")


@pytest.mark.parametrize("rows,d", NORM_SHAPES)
@pytest.mark.parametrize("xt,yt", NORM_TYPES)
def test_layer_norm(model, rows, d, xt, yt):
    for pad, lead in ((0, 0), (20, 0), (3, 1)):                 # dense, a padded table, rows that start anywhere
        x = randn(rows, d + pad, seed=d + pad, dtype=xt, by=0.7)[:, lead: lead + d] + torch.tensor(0.25, dtype=xt, device="cuda")
        if pad:
            wide = torch.zeros(rows, d + pad, dtype=xt, device="cuda")
            wide[:, lead: lead + d] = x
            x = wide[:, lead: lead + d]
            assert rows == 1 or d == 1 or not x.is_contiguous()
        check_layer_norm(model, x, xt, yt)


@pytest.mark.parametrize("rows,d,pad,xt,yt", [
    (5001, 300, 20, torch.float32, torch.bfloat16),      # a padded table, an odd number of rows of 600 bytes
    (4999, 300, 0, torch.bfloat16, torch.bfloat16),      # rows of 600 bytes without gaps: accesses of 8 bytes
    (2999, 1000, 0, torch.float16, torch.float16),
    (3001, 4096, 0, torch.bfloat16, torch.bfloat16),
    (2500, 2048, 8, torch.float32, torch.float32),
    (4001, 100, 0, torch.float32, torch.float16),        # dy in rows of 200 bytes
    (9001, 36, 4, torch.float32, torch.float32),
    (2401, 8192, 0, torch.bfloat16, torch.bfloat16),
    (2400, 1536, 0, torch.float32, torch.bfloat16),
])
def test_layer_norm_of_many_rows(model, rows, d, pad, xt, yt):
    """Enough rows for those that go through shared memory; the same bounds."""
    wide = randn(rows, d + pad, seed=d + pad, dtype=xt, by=0.7) + torch.tensor(0.25, dtype=xt, device="cuda")
    check_layer_norm(model, wide[:, :d], xt, yt)


def test_layer_norm_rows_of_one_value_and_no_rows(model):
    g, b = torch.ones(300, device="cuda"), torch.full((300,), 0.5, device="cuda")
    y, saved = model.layer_norm(torch.full((4, 300), 3.0, device="cuda"), g, b)
    assert (y == 0.5).all()
    dx, dg, db = model.layer_norm_backward(torch.ones(4, 300, device="cuda"), saved)
    assert (dx == 0).all() and (dg == 0).all() and (db == 4).all()
    y, saved = model.layer_norm(torch.empty(0, 300, device="cuda"), g, b)
    dx, dg, db = model.layer_norm_backward(torch.empty(0, 300, device="cuda"), saved)
    assert y.shape == (0, 300) and dx.shape == (0, 300) and (dg == 0).all() and (db == 0).all()


def test_layer_norm_gradient_against_differences(model):
    x, g, b = randn(3, 36, seed=1).requires_grad_(False), 1 + randn(36, seed=2, by=0.2), randn(36, seed=3)
    dy = randn(3, 36, seed=4)
    y, saved = model.layer_norm(x, g, b, 1e-5)
    dx, dg, _ = model.layer_norm_backward(dy, saved)
    step = 2.0 ** -6                    # the difference quotient is off by step^2 (third derivative), its noise 2^-24 / step per term

    def loss(x, g):
        return float((model.layer_norm(x, g, b, 1e-5)[0].double() * dy.double()).sum())
    for i, j in ((0, 0), (1, 17), (2, 35)):
        e = torch.zeros_like(x)
        e[i, j] = step
        assert abs((loss(x + e, g) - loss(x - e, g)) / (2 * step) - float(dx[i, j])) < 5e-3
        assert abs((loss(x, g + e[i]) - loss(x, g - e[i])) / (2 * step) - float(dg[j])) < 5e-3


# ---- sentence bounds --------------------------------------------------------------------------------
def spans_by_hand(toks):
    out, begin = np.zeros((len(toks), 2), np.int32), 0
    for stop in list(np.flatnonzero(toks == -1)) + [len(toks)]:
        for t in range(begin, min(stop + 1, len(toks))):
            out[t] = (begin, stop) if 0 <= toks[t] < VOCAB else (t, t)
        begin = stop + 1
    return out


@pytest.mark.parametrize("n,share", [(0, 0.1), (1, 0.0), (1, 1.0), (7, 0.3), (2048, 0.02), (2049, 0.0005), (20_001, 0.03), (600_000, 0.0), (700_001, 1e-5)])
def test_sentence_spans(model, n, share):
    rng = np.random.default_rng(n + 1)
    toks = rng.integers(0, VOCAB, n).astype(np.int32)
    toks[rng.random(n) < 0.05] = VOCAB + 3
    toks[rng.random(n) < 0.02] = -7
    toks[rng.random(n) < share] = -1
    got = model.sentence_spans(torch.from_numpy(toks).cuda()).cpu().numpy()
    assert np.array_equal(got, spans_by_hand(toks))


# ---- attention --------------------------------------------------------------------------------------
def bucket(rel, n, reach, two):
    starts = torch.from_numpy(binding.w2v_bucket_starts(2 * n if two else n, reach, two)).cuda().long()
    far = rel.abs() if two else (-rel).clamp(min=0)
    b = torch.searchsorted(starts, far.contiguous(), right=True) - 1
    return b + n * (rel > 0).long() if two else b


def attend_by_hand(q, k, v, toks, bias, left, right, sinks, reach, two, d_o, rest):
    """Dense 64-bit attention: (results, their bounds) as dicts."""
    n, h, dim = q.shape
    u, group, scale = U[q.dtype], h // k.shape[1], dim ** -0.5
    sp = torch.from_numpy(spans_by_hand(toks)).cuda().long()
    seen = sp[:, 1] > sp[:, 0]
    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
    ok = (j >= sp[:, :1]) & (j < sp[:, 1:]) & seen[None] & (((j >= i - left) & (j <= i + right)) | ((j < sp[:, :1] + sinks) & (j < i)))
    Q, K, V, D = q.double(), k.double().repeat_interleave(group, 1), v.double().repeat_interleave(group, 1), d_o.double()
    S = torch.einsum("ihd,jhd->hij", Q, K) * scale
    if bias is not None:
        which = bucket(j - i, bias.shape[0] // 2 if two else bias.shape[0], reach, two)
        S = S + bias.double()[which].permute(2, 0, 1)
    S = S.masked_fill(~ok, -math.inf)
    P = torch.nan_to_num(torch.softmax(S, -1), nan=0.0)
    o = torch.einsum("hij,jhd->ihd", P, V)
    dP, delta = torch.einsum("ihd,jhd->hij", D, V), (D * o).sum(-1).t()
    dS = P * (dP - delta[..., None])
    aP, aD = torch.einsum("ihd,jhd->hij", D.abs(), V.abs()), (D * o).abs().sum(-1).t()
    # rounding of the weights, then of the result; fp16 weights below 2^-14 of the row's largest keep 2^-25 of it
    small = 2.0 ** -25 if q.dtype == torch.float16 else 0.0
    keys = ok.sum(1).double()
    out = {"o": o}
    bound = {"o": u * o.abs() + (u + F32) * torch.einsum("hij,jhd->ihd", P, V.abs()) + small * keys[:, None, None] * V.abs().amax() + 1e-6}
    # a score gradient: fp32 products, and the row's delta (exact for dbias, from the rounded output otherwise)
    eS = P * (F32 * (aP + aD[..., None]) + (0 if rest else u) * aD[..., None])
    shared = lambda x: x.view(n, h // group, group, dim).sum(2)  # noqa: E731
    out["dq"] = torch.einsum("hij,jhd->ihd", dS, K) * scale
    bound["dq"] = u * out["dq"].abs() + scale * torch.einsum("hij,jhd->ihd", u * dS.abs() + eS + small, K.abs()) + 1e-6
    out["dk"] = shared(torch.einsum("hij,ihd->jhd", dS, Q)) * scale
    bound["dk"] = u * out["dk"].abs() + scale * shared(torch.einsum("hij,ihd->jhd", u * dS.abs() + eS + small, Q.abs())) + 1e-6
    out["dv"] = shared(torch.einsum("hij,ihd->jhd", P, D))
    bound["dv"] = u * out["dv"].abs() + shared(torch.einsum("hij,ihd->jhd", (u + F32) * P + small * ok, D.abs())) + 1e-6
    if bias is not None:
        add = lambda x: torch.zeros(bias.shape[0], h, dtype=torch.float64, device="cuda").index_add_(0, which.reshape(-1), x.reshape(h, -1).t())  # noqa: E731
        out["dbias"], bound["dbias"] = add(dS), add(eS) + 1e-6
    return out, bound


def stream(n, lens, seed, oov=0.03):
    rng = np.random.default_rng(seed)
    toks = rng.integers(0, VOCAB, n).astype(np.int32)
    if oov:
        toks[rng.random(n) < oov] = VOCAB
    at = 0
    while at < n:
        at += int(rng.integers(lens[0], lens[1] + 1))
        if at < n:
            toks[at] = -1
        at += 1
    return toks


#        n, sentence lengths, heads, kv, dim, left, right, sinks, buckets, reach, two-sided
ATTEND = [
    (1, (1, 1), 1, 1, 64, 0, 0, 0, 0, 128, False),
    (1, (1, 1), 2, 1, 8, 3, 3, 1, 4, 16, True),
    (5, (0, 1), 3, 3, 16, 2, 2, 2, 8, 32, True),            # sentences of no and of one word
    (77, (76, 76), 5, 5, 64, 10, 10, 0, 32, 128, True),
    (300, (5, 40), 4, 4, 80, 10, 10, 0, 32, 128, True),
    (300, (5, 40), 4, 4, 80, 3, 0, 2, 16, 64, False),       # many sentences with sinks of their own in a tile
    (257, (257, 257), 5, 1, 64, 128, 128, 2, 32, 128, True),
    (900, (400, 800), 4, 2, 64, 60, 0, 4, 32, 128, False),  # sinks far before the window
    (900, (900, 900), 2, 2, 128, 100, 0, 64, 0, 128, False),
    (1000, (300, 900), 8, 2, 128, 511, 0, 4, 32, 128, False),
    (700, (100, 700), 4, 1, 96, 300, 300, 3, 64, 1024, True),
    (640, (640, 640), 1, 1, 32, 0, 0, 0, 2, 7, False),      # only itself
    (640, (640, 640), 2, 1, 72, 0, 130, 0, 6, 9, True),     # only after
    (513, (513, 513), 1, 1, 64, 100_000, 100_000, 0, 16, 200, True),
    (1290, (1290, 1290), 3, 1, 120, 40, 5, 17, 32, 300, True),
    (512, (3, 3), 2, 2, 64, 1, 1, 1, 4, 3, True),
]


@pytest.mark.parametrize("case", range(len(ATTEND)))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attend(model, case, dtype):
    n, lens, h, kv, dim, left, right, sinks, buckets, reach, two = ATTEND[case]
    toks = stream(n, lens, case)
    qkv = randn(n, (h + 2 * kv) * dim, seed=case, dtype=dtype)
    q, k, v = (t.view(n, -1, dim) for t in (qkv[:, : h * dim], qkv[:, h * dim: (h + kv) * dim], qkv[:, (h + kv) * dim:]))
    bias = randn(buckets, h, seed=9, by=0.5) if buckets else None
    d_o = randn(n, h, dim, seed=77, dtype=dtype)
    over = dict(left=left, right=right, sinks=sinks, reach=reach, two_sided=two)
    spans = model.sentence_spans(torch.from_numpy(toks).cuda())
    o, saved = model.attend(q, k, v, spans, bias, train=True, **over)
    dq, dk, dv, dbias = model.attend_backward(d_o, saved)
    model.sync()
    want, bound = attend_by_hand(q, k, v, toks, bias, left, right, sinks, reach, two, d_o, bias is not None)
    got = {"o": o, "dq": dq, "dk": dk, "dv": dv}
    if bias is not None:
        got["dbias"] = dbias
    for name, x in got.items():
        inside(x, want[name], bound[name], name)
    empty = torch.from_numpy(~((toks >= 0) & (toks < VOCAB))).cuda()
    for x in (o, dq, dk, dv):
        assert (x[empty] == 0).all()
    # the same bits again, and without what training keeps
    o2, saved2 = model.attend(q, k, v, spans, bias, train=True, **over)
    again = model.attend_backward(d_o, saved2)
    assert torch.equal(o, o2) and all(torch.equal(a, b) for a, b in zip((dq, dk, dv, dbias), again) if a is not None)
    assert torch.equal(o, model.attend(q, k, v, spans, bias, **over))


def test_attend_large_scores_and_nonfinite_values_where_nothing_looks(model):
    """Scores of some hundreds do not overflow, a bias of the lowest float hides a bucket, and infinities or NaN
    in rows that the vocabulary does not have, or in other sentences, reach nobody."""
    n, dim = 400, 64
    toks = stream(n, (150, 190), 1)
    q, k, v = (randn(n, 2, dim, seed=s, dtype=torch.bfloat16, by=b) for s, b in ((1, 6.0), (2, 6.0), (3, 1.0)))
    d_o = randn(n, 2, dim, seed=4, dtype=torch.bfloat16)
    bias = randn(8, 2, seed=5)
    bias[2] = torch.finfo(torch.float32).min
    over = dict(left=30, right=30, sinks=2, reach=16, two_sided=True)
    spans = model.sentence_spans(torch.from_numpy(toks).cuda())
    o, saved = model.attend(q, k, v, spans, bias, train=True, **over)
    g = model.attend_backward(d_o, saved)
    assert all(torch.isfinite(t).all() for t in (o, *g))
    assert (g[3][2] == 0).all()
    hidden = torch.from_numpy(~((toks >= 0) & (toks < VOCAB))).cuda()
    assert hidden.any()
    q2, k2, v2, d2 = q.clone(), k.clone(), v.clone(), d_o.clone()
    q2[hidden], k2[hidden], v2[hidden], d2[hidden] = math.nan, math.inf, math.nan, -math.inf
    o2, saved2 = model.attend(q2, k2, v2, spans, bias, train=True, **over)
    g2 = model.attend_backward(d2, saved2)
    assert torch.equal(o, o2) and all(torch.equal(a, b) for a, b in zip(g, g2))


SPOILED = [(300, (5, 40), 4, 2, 80, 10, 10, 0, 32, 128, True), (900, (400, 800), 4, 2, 64, 60, 0, 4, 32, 128, False),
           (700, (3, 90), 4, 2, 128, 511, 0, 4, 16, 64, False), (700, (100, 700), 4, 1, 96, 30, 30, 3, 64, 1024, True),
           (513, (513, 513), 2, 2, 128, 40, 0, 20, 8, 16, False)]


@pytest.mark.parametrize("case", range(len(SPOILED)))
@pytest.mark.parametrize("which", ["q", "k", "v", "d_o"])
def test_attend_nonfinite_words_reach_who_sees_them_only(model, case, which):
    """A word that holds NaN spoils every row that its value enters by the formulas, and nothing else: not the other
    sentences of its tile, nor what lies outside of the window."""
    n, lens, h, kv, dim, left, right, sinks, buckets, reach, two = SPOILED[case]
    toks = stream(n, lens, case)
    clean = {"q": randn(n, h, dim, seed=1, dtype=torch.bfloat16), "k": randn(n, kv, dim, seed=2, dtype=torch.bfloat16),
             "v": randn(n, kv, dim, seed=3, dtype=torch.bfloat16), "d_o": randn(n, h, dim, seed=4, dtype=torch.bfloat16)}
    bias = randn(buckets, h, seed=9, by=0.5)
    want, bound = attend_by_hand(clean["q"], clean["k"], clean["v"], toks, bias, left, right, sinks, reach, two, clean["d_o"], True)
    sp = torch.from_numpy(spans_by_hand(toks)).cuda().long()
    seen = sp[:, 1] > sp[:, 0]
    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
    ok = (j >= sp[:, :1]) & (j < sp[:, 1:]) & seen[None] & (((j >= i - left) & (j <= i + right)) | ((j < sp[:, :1] + sinks) & (j < i)))
    buckets_of = bucket(j - i, buckets // 2 if two else buckets, reach, two)
    spans = model.sentence_spans(torch.from_numpy(toks).cuda())
    words = torch.nonzero(seen).flatten()
    # one in the middle, and the first word of the last sentence that has 3 of them (a sink where there are some)
    starts = [int(w) for w in words if sp[w, 0] == w and sp[w, 1] - w >= 3]
    for x in (int(words[len(words) // 2]), starts[-1]):
        for value in (math.nan, math.inf):
            t = {name: u.clone() for name, u in clean.items()}
            t[which][x] = value
            o, saved = model.attend(t["q"], t["k"], t["v"], spans, bias, train=True, left=left, right=right, sinks=sinks, reach=reach, two_sided=two)
            dq, dk, dv, dbias = model.attend_backward(t["d_o"], saved)
            model.sync()
            rows = ok[:, x] if which in "kv" else torch.arange(n, device="cuda") == x       # queries whose weights or dS it enters
            keys = (rows[:, None] & ok).any(0)
            none = torch.zeros_like(rows)
            hit = {"o": none if which == "d_o" else rows, "dq": rows, "dk": keys, "dv": none if which == "v" else keys}
            for name, got in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
                inside(got[~hit[name]], want[name][~hit[name]], bound[name][~hit[name]], name)
                if value != value:
                    assert torch.isnan(got[hit[name]]).all(), name
            spoilt = torch.zeros(buckets, dtype=torch.bool, device="cuda")
            spoilt[buckets_of[rows[:, None] & ok]] = True
            inside(dbias[~spoilt], want["dbias"][~spoilt], bound["dbias"][~spoilt], "dbias")
            if value != value:
                assert torch.isnan(dbias[spoilt]).all()


def test_attend_alone_with_nan(model):
    q = torch.full((1, 1, 64), math.nan, dtype=torch.float16, device="cuda")
    one = torch.ones_like(q)
    spans = model.sentence_spans(torch.ones(1, dtype=torch.int32, device="cuda"))
    for a, b, c in ((q, one, one), (one, q, one), (one, one, q)):
        assert torch.isnan(model.attend(a, b, c, spans, left=3)).all()
        cache = torch.zeros(2, 1, 4, 1, 64, dtype=torch.float16, device="cuda")
        assert torch.isnan(model.attend_token(a, b, c, cache[0], cache[1], torch.zeros(1, dtype=torch.int32, device="cuda"), left=3)).all()


def test_attend_token_nonfinite_places(model):
    """NaN at a place that a sequence sees spoils that sequence, all of its heads of that key/value head, and nothing else."""
    batch, h, kv, dim, left = 3, 4, 2, 64, 600
    q, k, v = (randn(batch, x, dim, seed=x + s, dtype=torch.bfloat16) for s, x in ((0, h), (1, kv), (2, kv)))
    cache = [randn(batch, left + 1, kv, dim, seed=s, dtype=torch.bfloat16) for s in (5, 6)]
    pos = torch.tensor([500, 590, 31], dtype=torch.int32, device="cuda")
    want = model.attend_token(q, k, v, cache[0].clone(), cache[1].clone(), pos, left=left)
    for which in (0, 1):
        c = [x.clone() for x in cache]
        c[which][1, 200, 1] = math.nan
        c[which][2, 32:] = math.nan                                  # beyond what sequence 2 sees
        got = model.attend_token(q, k, v, *c, pos, left=left)
        assert torch.isnan(got[1, 2:]).all() and torch.equal(got[1, :2], want[1, :2])
        assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])


def test_attend_gradient_against_differences(model):
    """Along a random direction, in float16: the loss moves by its gradient's product with the direction."""
    n, h, kv, dim, dtype = 150, 4, 2, 64, torch.float16
    toks = stream(n, (60, 80), 3)
    q, k, v = randn(n, h, dim, seed=1, dtype=dtype), randn(n, kv, dim, seed=2, dtype=dtype), randn(n, kv, dim, seed=3, dtype=dtype)
    bias, d_o = randn(16, h, seed=4), randn(n, h, dim, seed=5, dtype=dtype)
    over = dict(left=20, right=20, sinks=2, reach=32, two_sided=True)
    spans = model.sentence_spans(torch.from_numpy(toks).cuda())
    _, saved = model.attend(q, k, v, spans, bias, train=True, **over)
    grads = model.attend_backward(d_o, saved)
    step = 2.0 ** -4                 # exact in float16 for these magnitudes; third-order terms are step^2 = 0.4 %

    def loss(*args):
        return float((model.attend(*args[:3], spans, args[3], **over).double() * d_o.double()).sum())
    args = [q, k, v, bias]
    for which in range(4):
        e = randn(*args[which].shape, seed=20 + which).sign().to(args[which].dtype) * step
        up, down = list(args), list(args)
        up[which], down[which] = args[which] + e, args[which] - e
        real = ((up[which].double() - down[which].double()) / 2)                     # what the additions really moved
        slope = float((grads[which].double() * real).sum())
        # each o is off by u |o|: noise of the difference is u sqrt(sum (o d_o)^2), once for each side
        o = model.attend(*args[:3], spans, bias, **over).double()
        noise = 2.0 ** -11 * float((o * d_o.double()).square().sum().sqrt()) * 8
        size = float((grads[which].double() * real).square().sum().sqrt())
        assert abs((loss(*up) - loss(*down)) / 2 - slope) < 0.05 * size + noise


def test_attend_no_rows_and_views(model):
    spans = model.sentence_spans(torch.empty(0, dtype=torch.int32, device="cuda"))
    q = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    o, saved = model.attend(q, q, q, spans, train=True)
    assert o.shape == q.shape and all(g.shape == q.shape for g in model.attend_backward(q, saved)[:3])
    bias = randn(8, 4, seed=1)
    _, saved = model.attend(q, q, q, spans, bias, reach=16, train=True)
    assert (model.attend_backward(q, saved)[3] == 0).all()
    # heads that are not side by side are brought together first
    n = 50
    base = randn(4, n, 64, seed=2, dtype=torch.bfloat16)
    spans = model.sentence_spans(torch.ones(n, dtype=torch.int32, device="cuda"))
    a = model.attend(base.transpose(0, 1), base.transpose(0, 1), base.transpose(0, 1), spans, left=9)
    c = base.transpose(0, 1).contiguous()
    assert torch.equal(a, model.attend(c, c, c, spans, left=9))


def test_attend_on_a_stream_of_its_own():
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        m = binding.W2V(VOCAB, 64, seed=3)
        q = randn(333, 2, 64, seed=1, dtype=torch.bfloat16)
        spans = m.sentence_spans(torch.ones(333, dtype=torch.int32, device="cuda"))
        a = m.attend(q, q, q, spans, left=40, right=7)
        m.sync()
    side.synchronize()
    want = m.attend(q, q, q, spans, left=40, right=7)
    m.sync()
    assert torch.equal(a, want)
    m.close()


# ---- one new token per sequence -----------------------------------------------------------------------
#        batch, heads, kv, dim, left, sinks, buckets, extra places
TOKEN = [(1, 1, 1, 64, 0, 0, 0, 0), (3, 5, 5, 64, 10, 2, 8, 0), (2, 8, 2, 128, 100, 4, 32, 5), (5, 4, 1, 80, 1000, 0, 32, 0), (4, 6, 2, 32, 37, 7, 0, 3),
         (2, 40, 2, 64, 64, 1, 16, 0), (1, 2, 1, 8, 5000, 64, 32, 1), (7, 7, 1, 120, 33, 3, 32, 0)]


@pytest.mark.parametrize("case", range(len(TOKEN)))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attend_token_walks_like_attend(model, case, dtype):
    """Positions -1, 0, 1, ... of sequences of different ages against the definition, over a ring that wraps."""
    batch, h, kv, dim, left, sinks, buckets, extra = TOKEN[case]
    places = sinks + left + 1 + extra
    ages = [(-1, 0, 1, sinks, left, places, places + 3, 3 * places + 7)[(b + case) % 8] for b in range(batch)]
    longest = max(ages) + 1
    rng = torch.Generator(device="cuda").manual_seed(case)
    K, V = (torch.randn(batch, longest + 1, kv, dim, generator=rng, device="cuda").to(dtype) for _ in range(2))
    q = torch.randn(batch, h, dim, generator=rng, device="cuda").to(dtype)
    bias = randn(buckets, h, seed=6, by=0.5) if buckets else None
    ck, cv = torch.full((batch, places, kv, dim), math.nan, dtype=dtype, device="cuda"), torch.full((batch, places, kv, dim), math.nan, dtype=dtype, device="cuda")
    place = lambda p: p if p < sinks else sinks + (p - sinks) % (places - sinks)  # noqa: E731
    want, bound, wk, wv = [], [], ck, cv
    for b, age in enumerate(ages):
        for p in range(max(0, age - places), age):                 # what earlier calls left behind
            if p >= sinks:
                ck[b, place(p)], cv[b, place(p)] = K[b, p], V[b, p]
        for p in range(min(sinks, age)):
            ck[b, p], cv[b, p] = K[b, p], V[b, p]
    wk, wv = ck.clone(), cv.clone()
    for b, age in enumerate(ages):
        if age < 0:
            want.append(torch.zeros(h, dim, dtype=torch.float64, device="cuda"))
            bound.append(torch.zeros(h, dim, dtype=torch.float64, device="cuda"))
            continue
        wk[b, place(age)], wv[b, place(age)] = K[b, age], V[b, age]
        p = torch.tensor(sorted(set(range(min(sinks, age + 1))) | set(range(max(0, age - left), age + 1))), device="cuda")
        kk, vv = (t[b, p].double().repeat_interleave(h // kv, 1) for t in (K, V))
        s = torch.einsum("hd,phd->hp", q[b].double(), kk) * dim ** -0.5
        if buckets:
            s = s + bias.double()[bucket(p - age, buckets, 128, False)].t()
        P = torch.softmax(s, -1)
        o = torch.einsum("hp,phd->hd", P, vv)
        want.append(o)
        bound.append(U[dtype] * o.abs() + F32 * torch.einsum("hp,phd->hd", P, vv.abs()) + 1e-6)
    pos = torch.tensor(ages, dtype=torch.int32, device="cuda")
    at = pos.long().clamp(min=0)
    each = torch.arange(batch, device="cuda")
    o = model.attend_token(q, K[each, at], V[each, at], ck, cv, pos, bias, left=left, sinks=sinks, reach=128)
    inside(o, torch.stack(want), torch.stack(bound), "o")
    assert torch.equal(torch.nan_to_num(ck, 7.0), torch.nan_to_num(wk, 7.0)) and torch.equal(torch.nan_to_num(cv, 7.0), torch.nan_to_num(wv, 7.0))


def test_attend_token_matches_attend_word_by_word(model):
    n, h, kv, dim, left, sinks = 90, 4, 2, 64, 20, 3
    q, k, v = (randn(n, x, dim, seed=x + s, dtype=torch.bfloat16) for s, x in ((0, h), (1, kv), (2, kv)))
    bias = randn(16, h, seed=8)
    spans = model.sentence_spans(torch.ones(n, dtype=torch.int32, device="cuda"))
    o = model.attend(q, k, v, spans, bias, left=left, sinks=sinks, reach=64).float()
    ck, cv = (torch.zeros(1, sinks + left + 1, kv, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in range(n):
        pos = torch.tensor([t], dtype=torch.int32, device="cuda")
        one = model.attend_token(q[t: t + 1], k[t: t + 1], v[t: t + 1], ck, cv, pos, bias, left=left, sinks=sinks, reach=64)
        # both round once, and the first also rounds its weights: 3 u of a mean of values below max |v|
        assert (one[0].float() - o[t]).abs().max() <= 3 * 2.0 ** -8 * v[: t + 1].float().abs().max()


def test_attend_token_long_cache_passes_32_bit_offsets(model):
    """Places beyond 2^31 elements into the cache (4.3 GB and more a side)."""
    batch, kv, dim, left, dtype = 3, 8, 128, 1_000_000, torch.float16
    places = left + 1
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    ck = torch.zeros(batch, places, kv, dim, dtype=dtype, device="cuda")
    cv = torch.zeros(batch, places, kv, dim, dtype=dtype, device="cuda")
    assert ck.numel() > 2 ** 31
    q = torch.zeros(batch, kv, dim, dtype=dtype, device="cuda")
    q[..., 0] = 16.0 * dim ** 0.5
    k, v = torch.zeros_like(q), torch.zeros_like(q)
    pos = torch.full((batch,), left, dtype=torch.int32, device="cuda")
    at = left - 1
    ck[2, at, :, 0] = 4.0                                          # one key with a score of 64 against a million of 0
    cv[2, at] = 3.0
    o = model.attend_token(q, k, v, ck, cv, pos, left=left)
    assert (o[:2] == 0).all() and (o[2] == 3.0).all()


# ---- tables in 4 bits ------------------------------------------------------------------------------------
def unpack(packed, scales, d, group):
    w = torch.stack([packed & 15, packed >> 4], -1).view(packed.shape[0], -1).int() - 8
    assert (w[:, d:] == 0).all()
    return w[:, :d].double() * scales.double().repeat_interleave(group, 1)[:, :d]


@pytest.mark.parametrize("n,d", [(1, 1), (2, 31), (100, 32), (33, 100), (1000, 300), (17, 129), (64, 320), (129, 1024), (7, 4099)])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_fourbit_table(model, n, d, group):
    rows = randn(n, d + 5, seed=d, by=0.01)[:, :d]
    if n > 1:
        rows[1] = 0
    packed, scales = model.fourbit_pack(rows, group)
    w = unpack(packed, scales, d, group)
    groups = -(-d // group)
    padded = torch.nn.functional.pad(rows, (0, groups * group - d)).view(n, groups, group)
    scale = (padded.abs().amax(-1) / torch.full((), 7.0, device="cuda")).to(torch.bfloat16)     # a tensor: a true division
    assert torch.equal(scales, scale)
    wide = scale.float().repeat_interleave(group, 1)[:, :d]
    value = torch.where(wide > 0, (rows / wide.clamp(min=1e-30)).round().clamp(-7, 7), torch.zeros_like(rows))
    assert torch.equal(w, value.double() * wide.double())
    for m in (1, 2, 3, 4, 7, 8):
        x = randn(m, d + 1, seed=m)[:, 1:]
        out = model.fourbit_scores(x, packed, scales, group)
        inside(out, x.double() @ w.t(), F32 * (x.double().abs() @ w.abs().t()) + 1e-12, f"scores of {m}")


def test_fourbit_scores_of_the_models_own_table(model):
    """Rows of a padded table, straight from the handle, and an empty call."""
    m = binding.W2V(500, 300, seed=1, row_stride=320)
    table = m.U.view(500, 320)[:, :300]
    packed, scales = m.fourbit_pack(table)
    x = randn(2, 300, seed=1)
    out = m.fourbit_scores(x, packed, scales)
    inside(out, x.double() @ unpack(packed, scales, 300, 32).t(), F32 * (x.double().abs() @ unpack(packed, scales, 300, 32).abs().t()), "scores")
    assert m.fourbit_scores(x[:0], packed, scales).shape == (0, 500)
    assert m.fourbit_scores(x, packed[:0], scales[:0]).shape == (2, 0)
    m.close()


# ---- refusals ---------------------------------------------------------------------------------------------
def refused(call, *words):
    with pytest.raises((binding.W2VError, ValueError, TypeError)) as e:
        call()
    if isinstance(e.value, binding.W2VError):
        assert e.value.code == binding.W2V_ERR_ARG
    for w in words:
        assert w in str(e.value), str(e.value)


def test_refusals(model):
    f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    b = lambda *s: torch.zeros(*s, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    refused(lambda: model.layer_norm(f(2, 8193), f(8193), f(8193)), "8192")
    refused(lambda: model.layer_norm(f(2, 8), f(7), f(8)), "weights")
    refused(lambda: model.layer_norm(b(2, 8), f(8), f(8), out_dtype=torch.float32), "type of x")
    refused(lambda: model.layer_norm(f(2, 8), f(8), f(8), eps=-1.0), "eps")
    refused(lambda: model.layer_norm(f(2, 8), f(8), f(8), eps=math.nan), "eps")
    refused(lambda: model.layer_norm(f(2, 8).double(), f(8), f(8)), "float64")
    refused(lambda: model.layer_norm(torch.zeros(2, 8), f(8), f(8)), "cpu")
    _, saved = model.layer_norm(f(2, 8), f(8), f(8))
    refused(lambda: model.layer_norm_backward(b(2, 8), saved), "dy")
    spans = model.sentence_spans(torch.ones(4, dtype=torch.int32, device="cuda"))
    q = b(4, 4, 64)
    refused(lambda: model.attend(f(4, 4, 64), f(4, 4, 64), f(4, 4, 64), spans), "float16")
    refused(lambda: model.attend(q, b(4, 3, 64), b(4, 3, 64), spans), "multiple")
    refused(lambda: model.attend(b(4, 4, 12), b(4, 4, 12), b(4, 4, 12), spans), "head_dim")
    refused(lambda: model.attend(b(4, 4, 136), b(4, 4, 136), b(4, 4, 136), spans), "head_dim")
    refused(lambda: model.attend(q, q, q, spans[:3]), "spans")
    refused(lambda: model.attend(q, q, q, spans, sinks=65), "sinks")
    refused(lambda: model.attend(q, q, q, spans, left=1 << 30), "left")
    refused(lambda: model.attend(q, q, q, spans, f(66, 4)), "buckets")
    refused(lambda: model.attend(q, q, q, spans, f(7, 4), two_sided=True), "even")
    refused(lambda: model.attend(q, q, q, spans, f(32, 4), reach=16), "reach")
    refused(lambda: model.attend(q, q, q, spans, f(32, 4), reach=1025), "reach")
    refused(lambda: model.attend(q, q, q, spans, f(32, 3)), "bias")
    refused(lambda: model.attend(q, q, q, spans, scale=math.inf), "scale")
    cache, pos = b(4, 8, 4, 64), torch.zeros(4, dtype=torch.int32, device="cuda")
    refused(lambda: model.attend_token(q, q, q, cache, cache, pos, left=8), "places")
    refused(lambda: model.attend_token(q, q, q, cache, cache, pos, left=4, right=1), "right")
    refused(lambda: model.attend_token(q, q, q, cache[:3], cache[:3], pos, left=4), "caches")
    refused(lambda: model.attend_token(q, q, q, cache, cache, pos.long(), left=4), "int32")
    refused(lambda: model.fourbit_pack(f(3, 10), 48), "group")
    packed, scales = model.fourbit_pack(f(3, 10))
    refused(lambda: model.fourbit_scores(f(9, 10), packed, scales), "m must")
    refused(lambda: model.fourbit_scores(f(1, 33), packed, scales), "packed")
    refused(lambda: binding.w2v_attend(model.h, binding.Window(1, 4, 4, 64, 0, 0, 0, 0, 0, 0, 1.0), 4, spans.data_ptr(), q.data_ptr() + 2, 256,
                                       q.data_ptr(), 256, q.data_ptr(), 256, None, q.data_ptr(), 256, None), "16-byte")
    refused(lambda: binding.w2v_attend(model.h, binding.Window(1, 4, 4, 64, 0, 0, 0, 0, 0, 0, 1.0), 4, spans.data_ptr(), q.data_ptr(), 255,
                                       q.data_ptr(), 256, q.data_ptr(), 256, None, q.data_ptr(), 256, None), "16-byte")
    model.sync()
