"""The reader operators where layouts end: many sinks, tiles without words, rows that hold anything.

Definitions and bounds are those of test_gpu_reader.py.
"""
import pytest
import torch

from paper_1606_08495_b200 import binding
from test_gpu_reader import F32, U, VOCAB, attend_by_hand, check_layer_norm, inside, randn, stream

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def model():
    m = binding.W2V(VOCAB, 64, seed=3)
    yield m
    m.close()


def both_ways(model, toks, h, kv, dim, dtype, bias, seed, left, right=0, sinks=0, reach=128, two_sided=False, change=None):
    """Attention and its gradient against the definition; `change` alters what rows hold that nobody may see."""
    n = len(toks)
    q, k, v, d_o = (randn(n, x, dim, seed=seed + s, dtype=dtype) for s, x in ((0, h), (1, kv), (2, kv), (3, h)))
    want, bound = attend_by_hand(q, k, v, toks, bias, left, right, sinks, reach, two_sided, d_o, bias is not None)
    if change:
        change(q, k, v, d_o)
    over = dict(left=left, right=right, sinks=sinks, reach=reach, two_sided=two_sided)
    spans = model.sentence_spans(torch.from_numpy(toks).cuda())
    o, saved = model.attend(q, k, v, spans, bias, train=True, **over)
    dq, dk, dv, dbias = model.attend_backward(d_o, saved)
    model.sync()
    for name, x in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv), ("dbias", dbias)):
        if x is not None:
            inside(x, want[name], bound[name], name)
    return (o, dq, dk, dv), saved


# ---- sinks that take more than one tile ------------------------------------------------------------
@pytest.mark.parametrize("dim", [64, 72, 80, 96, 128])
@pytest.mark.parametrize("sinks", [31, 32, 33, 40, 64])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attend_many_sinks(model, dim, sinks, dtype):
    """A sentence much longer than the window, with words among the sinks that the vocabulary does not have."""
    toks = stream(900, (900, 900), sinks + dim)
    toks[[1, sinks // 2, sinks - 1, 33]] = VOCAB + 1
    both_ways(model, toks, 4, 2, dim, dtype, randn(16, 4, seed=9, by=0.5), sinks, left=30, sinks=sinks, reach=64)


# ---- 128 positions without a word -------------------------------------------------------------------
@pytest.mark.parametrize("dim", [8, 64, 80, 128])
@pytest.mark.parametrize("n,first,last", [(1, 0, 1), (129, 128, 129), (128, 0, 128), (700, 100, 430), (512, 128, 512), (40_000, 0, 40_000)])
def test_attend_tiles_without_words(model, dim, n, first, last):
    """Separators and words that the vocabulary does not have in [first, last), which holds whole tiles: zeros, whatever q holds."""
    toks = stream(n, (20, 90), n + dim)
    toks[first: last: 2] = VOCAB
    toks[first + 1: last: 2] = -1
    toks[last - 1] = -1
    if n <= 1000:
        got, saved = both_ways(model, toks, 4, 2, dim, torch.bfloat16, randn(16, 4, seed=9, by=0.5), n, left=30, right=30, sinks=3, two_sided=True)
        assert all((t[first: last] == 0).all() for t in got)
        assert (saved[-1][:, first: last] == float("inf")).all()
        return
    # many blocks, one after the other on the same SMs
    q, k, d_o = randn(n, 4, dim, seed=1, dtype=torch.bfloat16), randn(n, 2, dim, seed=2, dtype=torch.bfloat16), randn(n, 4, dim, seed=3, dtype=torch.bfloat16)
    spans = model.sentence_spans(torch.from_numpy(toks).cuda())
    for _ in range(5):
        o, saved = model.attend(q, k, k, spans, left=30, right=30, train=True)
        grads = model.attend_backward(d_o, saved)[:3]
        assert all((t == 0).all() for t in (o, *grads))
    model.sync()


# ---- what words outside the vocabulary hold -----------------------------------------------------------
@pytest.mark.parametrize("dim", [64, 80, 128])
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), 3e38, float("nan")])
@pytest.mark.parametrize("biased", [False, True])
def test_attend_hidden_rows_hold_anything(model, dim, value, biased):
    """One element, or a whole row, of q, k, v and d_o of words that the vocabulary does not have: zeros and +infinity come out
    there, and nobody else changes.  Windows well past the bias' reach, so that tiles without masks are among them."""
    toks = stream(900, (900, 900), 5, oov=0.004)
    bias = randn(16, 4, seed=9, by=0.5) if biased else None
    over = dict(left=400, right=300, sinks=2, reach=64, two_sided=True)
    plain, _ = both_ways(model, toks, 4, 2, dim, torch.bfloat16, bias, 1, **over)
    hidden = torch.from_numpy(~((toks >= 0) & (toks < VOCAB))).cuda()
    assert 2 <= int(hidden.sum()) <= 12
    for columns in (slice(3, 4), slice(None)):
        def change(q, k, v, d_o):
            for t in (q, k, v, d_o):
                t[..., columns][hidden] = value
        got, saved = both_ways(model, toks, 4, 2, dim, torch.bfloat16, bias, 1, change=change, **over)
        assert all(torch.equal(a, b) for a, b in zip(got, plain))
        assert all((t[hidden] == 0).all() for t in got) and (saved[-1][:, hidden] == float("inf")).all()


@pytest.mark.parametrize("dim", [64, 128])
def test_attend_key_that_no_query_likes(model, dim):
    """A key with an infinity that every query's score turns into -infinity has weight zero everywhere; a query in its
    reach that is not a word must not make it NaN."""
    toks = stream(300, (300, 300), 6, oov=0.0)
    toks[[90, 171, 202]] = VOCAB
    bias = randn(16, 2, seed=9, by=0.5)

    def run(change):
        q, k, v, d_o = (randn(300, 2, dim, seed=s, dtype=torch.bfloat16) for s in (1, 2, 3, 4))
        q[..., 0] = q[..., 0].abs() + 0.25
        k[150, :, 0] = -change
        spans = model.sentence_spans(torch.from_numpy(toks).cuda())
        o, saved = model.attend(q, k, v, spans, bias, left=120, right=120, reach=32, two_sided=True, train=True)
        return (o, *model.attend_backward(d_o, saved))
    hidden, clean = run(float("inf")), run(1e30)                    # both weights are zero; 0 * dS keeps dq finite in the second
    for a, b, name in zip(hidden, clean, ("o", "dq", "dk", "dv", "dbias")):
        if name == "dq":                                             # zero weights times an infinite key: NaN by the formula
            continue
        assert torch.equal(a, b), name


# ---- calls from another stream than the model's ---------------------------------------------------------
def every_operator(m, x, spans_of, rows, pos):
    """All operators once, from tensors that make the calls copy some of them first."""
    n = x.shape[0]
    g, b = x.new_ones(64), x.new_zeros(64)
    wide = x.repeat(1, 2)[:, ::2]                                    # columns two apart: brought together in the call
    y, saved = m.layer_norm(wide, g, b)
    out = [y, *m.layer_norm_backward(wide * 0.5, saved)]
    q = x.bfloat16().view(n, 2, 32).transpose(0, 1).contiguous().transpose(0, 1)
    spans = m.sentence_spans(spans_of.long())
    o, kept = m.attend(q, q, q, spans, left=20, right=3, train=True)
    out += [spans, o, *m.attend_backward(q, kept)[:3]]
    cache = torch.zeros(2, 4, 9, 2, 32, dtype=torch.bfloat16, device="cuda")
    out += [m.attend_token(q[:4], q[:4], q[:4], cache[0], cache[1], pos, left=8), cache]
    packed, scales = m.fourbit_pack(rows.t())
    return out + [packed, scales, m.fourbit_scores(wide[:3], packed, scales)]


def test_operators_on_another_stream(model):
    """Inputs that are written late on a side stream, results that are read there, and memory that is handed out again."""
    data = [randn(500, 64, seed=1), torch.from_numpy(stream(500, (20, 60), 1)).cuda(), randn(64, 300, seed=2),
            torch.tensor([0, 1, 2, -1], dtype=torch.int32, device="cuda")]
    want = [t.clone() for t in every_operator(model, *data)]
    model.sync()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(20):
            late = [torch.zeros_like(t) for t in data]
            torch.cuda._sleep(3_000_000)                             # some milliseconds
            for a, b in zip(late, data):
                a.copy_(b)
            got = every_operator(model, *late)
            same = torch.stack([(a == b).all() for a, b in zip(got, want)])
            del late, got
            torch.full((4_000_000,), float("nan"), device="cuda")    # over memory that calls have given back
            assert same.all()


def test_reader_on_another_stream(model):
    """A reader's step while the model's stream is busy writing the tables it reads."""
    from paper_1606_08495_b200.reader import Reader
    m = binding.W2V(VOCAB, 64, seed=4)
    tables = [randn(VOCAB * m.row_stride, seed=s, by=0.5) for s in (1, 2)]
    toks = torch.from_numpy(stream(300, (20, 60), 2)).cuda()
    drawn = torch.randint(0, VOCAB, (300, 3), device="cuda")
    words = torch.arange(3, dtype=torch.int32, device="cuda")

    def step():
        r = Reader(m, left=20)
        h, saved = r.read(toks, train=True)
        loss, dh = r.loss(h, toks, drawn)
        grads = r.gradients(dh, saved)
        state = r.start(3)
        return [h, loss, grads["qkv"], grads["x"], *r.next(state, words)]
    for t, table in zip((m.U, m.V), tables):
        t.copy_(table)
    want = step()
    m.sync()
    for t in (m.U, m.V):
        t.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        with torch.cuda.stream(m.stream):
            torch.cuda._sleep(10_000_000)
            for t, table in zip((m.U, m.V), tables):
                t.copy_(table)
        got = step()
        with torch.cuda.stream(m.stream):
            m.U.zero_()
            m.V.zero_()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    m.close()


# ---- the reader's ends ------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def reader():
    from paper_1606_08495_b200.reader import Reader
    m = binding.W2V(VOCAB, 96, seed=4)
    for s, t in enumerate((m.U, m.V)):
        t.copy_(randn(t.numel(), seed=s, by=0.5))
    r = Reader(m, left=20)
    r.p["out"].copy_(randn(*r.p["out"].shape, seed=3, by=0.1))
    r.p["beta_h"].copy_(randn(96, seed=4))
    yield r
    m.close()


def test_reader_next_takes_words_that_the_vocabulary_lacks(reader):
    """They move nothing and fault nothing; the other sentences go on as they would."""
    words = torch.randint(0, VOCAB, (6, 5), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    some, all_known = reader.start(5), reader.start(2)
    for t in range(6):
        w = words[t].clone()
        for at, unknown in ((1, VOCAB), (2, VOCAB + 12_345), (3, 2 ** 31 - 1), (4, -7)):
            if t != 2:
                w[at] = unknown
        h, scores = reader.next(some, w)
        if t == 2:
            h2, s2 = reader.next(all_known, w[:2].contiguous())
            assert torch.equal(h[1:2], h2[1:2])                      # the first word that sentence 1 has moved
        else:
            h2, s2 = reader.next(all_known, torch.stack([w[0], w.new_tensor(-1)]))
            nothing, _ = reader.m.layer_norm(torch.zeros(1, 96, device="cuda"), reader.p["gamma_h"], reader.p["beta_h"])
            assert torch.equal(h[1:], nothing.expand(4, -1))
        assert torch.equal(h[0], h2[0]) and torch.isfinite(scores).all()
    assert some["pos"].tolist() == [6, 1, 1, 1, 1]
    torch.cuda.synchronize()


def test_reader_answers_from_the_table_as_it_is_at_start(reader):
    words = torch.tensor([3, 4], dtype=torch.int32, device="cuda")
    reader.next(reader.start(2), words)
    keep = reader.m.V.clone()
    reader.m.V.mul_(-3.0)
    h, scores = reader.next(reader.start(2), words)
    want = h @ reader.answers.t()
    reader.m.V.copy_(keep)
    # 4 bits a column: half a step of a group's largest / 7 each, a tenth of the vectors' own size at the most
    assert (scores - want).abs().max() <= 0.1 * h.norm(dim=1).max() * 3 * keep.view(VOCAB, -1).norm(dim=1).max()
    again = reader.next(reader.start(2), words)[1]
    assert (torch.nn.functional.cosine_similarity(again, scores) < -0.99).all()


@pytest.mark.parametrize("n", [0, 1])
def test_reader_of_no_words_and_one(reader, n):
    keep = {name: t.clone() for name, t in reader.p.items()}
    toks = torch.full((n,), 7, dtype=torch.int32, device="cuda")
    h, saved = reader.read(toks, train=True)
    assert h.shape == (n, 96) and torch.equal(reader.read(toks), h)
    grads = reader.gradients(torch.ones_like(h), saved)
    assert all(grads[name].shape == t.shape and torch.isfinite(grads[name]).all() for name, t in reader.p.items())
    loss = reader.train_step(toks, torch.zeros(n, 3, dtype=torch.int64, device="cuda"), 0.1)       # nothing follows: no loss, no step
    assert float(loss) == 0 and all(torch.equal(t, keep[name]) for name, t in reader.p.items())
    h, scores = reader.next(reader.start(n), toks)
    assert h.shape == (n, 96) and scores.shape == (n, VOCAB)


def test_reader_loss_leaves_out_drawn_words_that_the_vocabulary_lacks(reader):
    toks = torch.from_numpy(stream(200, (20, 60), 3)).cuda()
    h = randn(200, 96, seed=1)
    drawn = torch.randint(0, VOCAB, (200, 4), generator=torch.Generator().manual_seed(2)).cuda()
    want = reader.loss(h, toks, drawn)
    wider = torch.cat([drawn, drawn.new_tensor([-1, VOCAB, 2 ** 40]).expand(200, -1)], 1)
    got = reader.loss(h, toks, wider)
    # sums of the same terms, and zeros, in another order
    assert abs(float(got[0] - want[0])) <= 1e-5 * float(want[0]) and (got[1] - want[1]).abs().max() <= 1e-5 * want[1].abs().max()
    torch.cuda.synchronize()


# ---- layer norm in place -----------------------------------------------------------------------------------
def norm_raw(m, x, y, g, b, stats, x_stride, y_stride, rows=None):
    from paper_1606_08495_b200.binding import _TYPES
    rows, d = x.shape[0] if rows is None else rows, g.numel()
    binding.w2v_layer_norm(m.h, rows, d, x.data_ptr(), x_stride, _TYPES[x.dtype], g.data_ptr(), b.data_ptr(), 1e-5, y.data_ptr(), y_stride,
                           _TYPES[y.dtype], stats.data_ptr(), stats.data_ptr() + 4 * rows)


def norm_back_raw(m, dy, x, dx, g, stats, dw, dy_stride, x_stride, dx_stride):
    from paper_1606_08495_b200.binding import _TYPES
    rows, d = x.shape[0], g.numel()
    binding.w2v_layer_norm_backward(m.h, rows, d, dy.data_ptr(), dy_stride, _TYPES[dy.dtype], x.data_ptr(), x_stride, _TYPES[x.dtype], g.data_ptr(),
                                    stats.data_ptr(), stats.data_ptr() + 4 * rows, dx.data_ptr(), dx_stride, dw.data_ptr(), dw.data_ptr() + 4 * d)


@pytest.mark.parametrize("rows,d,pad", [(1, 300, 0), (77, 300, 4), (5001, 300, 20), (3001, 4096, 0), (4999, 101, 3)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_layer_norm_in_place(model, rows, d, pad, dtype):
    """y over x, dx over dy and dx over x, with few rows and with enough for the ring: the same bits as side by side."""
    x, dy = randn(rows, d + pad, seed=1, dtype=dtype), randn(rows, d + pad, seed=2, dtype=dtype)
    g, b, ld = 1 + randn(d, seed=3, by=0.2), randn(d, seed=4), d + pad
    stats, dw = torch.empty(2, rows, device="cuda"), torch.empty(2, d, device="cuda")
    y, dx = torch.zeros_like(x), torch.zeros_like(x)
    norm_raw(model, x, y, g, b, stats, ld, ld)
    norm_back_raw(model, dy, x, dx, g, stats, dw, ld, ld, ld)
    for over in (0, 1):
        t, dw2 = (dy, x)[over].clone(), torch.empty_like(dw)
        norm_back_raw(model, (t, dy)[over], (x, t)[over], t, g, stats, dw2, ld, ld, ld)
        assert torch.equal(t[:, :d], dx[:, :d]) and torch.equal(t[:, d:], (dy, x)[over][:, d:]) and torch.equal(dw, dw2)
    t, stats2 = x.clone(), torch.empty_like(stats)
    norm_raw(model, t, t, g, b, stats2, ld, ld)
    assert torch.equal(t[:, :d], y[:, :d]) and torch.equal(t[:, d:], x[:, d:]) and torch.equal(stats, stats2)


def test_layer_norm_in_place_refusals(model):
    x, g, b = randn(4, 64, seed=1), torch.ones(32, device="cuda"), torch.zeros(32, device="cuda")
    half, stats, dw, other = x.view(torch.bfloat16), torch.zeros(2, 4, device="cuda"), torch.zeros(2, 32, device="cuda"), randn(4, 64, seed=2)
    keep = x.clone()

    def refused(*call):
        with pytest.raises(binding.W2VError, match="same type and stride") as e:
            call[0](*call[1:])
        assert e.value.code == binding.W2V_ERR_ARG
    refused(norm_raw, model, x, x, g, b, stats, 64, 32)
    refused(norm_raw, model, x, half, g, b, stats, 64, 64)
    refused(norm_raw, model, x, half, g, b, stats, 64, 64, 1)
    refused(norm_back_raw, model, x, other, x, g, stats, dw, 64, 64, 32)
    refused(norm_back_raw, model, other, x, x, g, stats, dw, 64, 64, 32)
    refused(norm_back_raw, model, half, other, x, g, stats, dw, 64, 64, 64)
    model.sync()
    assert torch.equal(x, keep)
    norm_raw(model, x, x, g, b, stats, 64, 32, 1)                    # a single row has no stride


# ---- numbers that do not fit ----------------------------------------------------------------------------------
def test_numbers_beyond_32_bits_are_refused(model):
    """Not taken modulo 2^32: a group of 2^32 + 32 would have written 32-column scales into one scale a row."""
    big = 1 << 32
    q = randn(4, 4, 64, seed=1, dtype=torch.bfloat16)
    spans = model.sentence_spans(torch.ones(4, dtype=torch.int32, device="cuda"))
    bias = randn(8, 4, seed=2)
    for name, value in (("left", big), ("left", big + 3), ("left", -1), ("right", big), ("sinks", big + 1), ("sinks", -big), ("reach", big + 16)):
        with pytest.raises(ValueError, match=name):
            model.attend(q, q, q, spans, bias, **{"reach": 16, name: value})
    cache = torch.zeros(4, 8, 4, 64, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="left"):
        model.attend_token(q, q, q, cache, cache.clone(), pos, left=big)
    rows = randn(40, 300, seed=3)
    packed, scales = model.fourbit_pack(rows)
    for group in (big + 32, big, -32, 0, 33):
        with pytest.raises(ValueError, match="group"):
            model.fourbit_pack(rows, group)
        with pytest.raises(ValueError, match="group"):
            model.fourbit_scores(rows[:1], packed, scales, group)
    with pytest.raises(ValueError, match="m must"):
        model.fourbit_scores(rows[:9], packed, scales)
    model.sync()


def test_misaligned_small_arrays_are_refused(model):
    """Addresses of lse, bias, dbias, pos, mean and rstd that are not multiples of their elements' size end in an error, not in a fault."""
    q, bias, f = randn(4, 4, 64, seed=1, dtype=torch.bfloat16), randn(8, 4, seed=2), torch.zeros(64, device="cuda")
    spans, pos = model.sentence_spans(torch.ones(4, dtype=torch.int32, device="cuda")), torch.zeros(4, dtype=torch.int32, device="cuda")
    cache = torch.zeros(4, 8, 4, 64, dtype=torch.bfloat16, device="cuda")
    w = binding.Window(binding.TYPE_BF16, 4, 4, 64, 3, 0, 0, 8, 16, 0, 0.125)
    a, s, b, e, h = q.data_ptr(), spans.data_ptr(), bias.data_ptr(), f.data_ptr(), model.h
    attend = lambda bias, lse: binding.w2v_attend(h, w, 4, s, a, 256, a, 256, a, 256, bias, a, 256, lse)  # noqa: E731
    back = lambda bias, lse, dbias: binding.w2v_attend_backward(h, w, 4, s, a, 256, a, 256, a, 256, bias, a, 256, lse, a, 256, a, 256, a, 256, a, 256, dbias)  # noqa: E731
    token = lambda pos, bias: binding.w2v_attend_token(h, w, 4, pos, a, a, a, cache.data_ptr(), cache.data_ptr(), 8, bias, a)  # noqa: E731
    norm = lambda mean, rstd: binding.w2v_layer_norm(h, 4, 16, e, 16, 0, b, b, 1e-5, e, 16, 0, mean, rstd)  # noqa: E731
    for call in (lambda: attend(b + 1, None), lambda: attend(b, e + 2), lambda: back(b + 2, e, e), lambda: back(b, e + 1, e), lambda: back(b, e, e + 3),
                 lambda: token(pos.data_ptr() + 2, b), lambda: token(pos.data_ptr(), b + 2), lambda: norm(e + 2, None), lambda: norm(None, e + 1)):
        with pytest.raises(binding.W2VError, match="aligned") as err:
            call()
        assert err.value.code == binding.W2V_ERR_ARG
    model.sync()


# ---- spans that are not this stream's -----------------------------------------------------------------------------
@pytest.mark.parametrize("dim", [64, 80, 128])
def test_attend_with_spans_of_another_stream(model, dim):
    """Pairs that do not lie around their position count as empty: zeros there, and no index is formed from them."""
    n, h, kv = 700, 4, 2
    q, k, v, d_o = (randn(n, x, dim, seed=s, dtype=torch.bfloat16) for s, x in ((1, h), (2, kv), (3, kv), (4, h)))
    bias = randn(16, h, seed=5)
    longer = model.sentence_spans(torch.from_numpy(stream(5000, (300, 2000), 1)).cuda())
    at = torch.arange(n, device="cuda")
    wild = torch.randint(-2 ** 31, 2 ** 31 - 1, (n, 2), generator=torch.Generator().manual_seed(1), dtype=torch.int64).to(torch.int32).cuda()
    near = torch.randint(-40, 40, (n, 2), generator=torch.Generator().manual_seed(2)).to(torch.int32).cuda() + at[:, None].int()
    o = model.attend(q, k, v, longer[:n].contiguous(), bias, left=90, right=20, sinks=40, reach=64)
    cut = model.sentence_spans(torch.from_numpy(stream(5000, (300, 2000), 1)[:n].copy()).cuda())
    assert not torch.equal(cut, longer[:n]) and torch.equal(o, model.attend(q, k, v, cut, bias, left=90, right=20, sinks=40, reach=64))
    for spans in (longer[3000: 3000 + n].contiguous(), longer[:n].contiguous(), wild, near, torch.full_like(wild, 2 ** 31 - 1)):
        o, saved = model.attend(q, k, v, spans, bias, left=90, right=20, sinks=40, reach=64, train=True)
        got = (o, *model.attend_backward(d_o, saved))
        model.sync()
        empty = ~((spans[:, 0] >= 0) & (spans[:, 0] <= at) & (spans[:, 1] > at))
        assert all(torch.isfinite(t).all() for t in got) and all((t[empty] == 0).all() for t in got[:4])


# ---- rows whose every bias is far from zero -----------------------------------------------------------------------------
@pytest.mark.parametrize("dim", [64, 80, 128])
@pytest.mark.parametrize("low", [-1e5, -1e9, torch.finfo(torch.float32).min, 1e5])
def test_attend_bias_that_swallows_scores(model, dim, low):
    """Keys are alike, so that softmax is a mean whatever the bias: tiles with and without masks must lose the same digits."""
    toks = stream(900, (900, 900), 8, oov=0.002)
    bias = torch.full((16, 4), low, device="cuda")
    q, v = randn(900, 4, dim, seed=1, dtype=torch.bfloat16), randn(900, 2, dim, seed=3, dtype=torch.bfloat16)
    k = randn(1, 2, dim, seed=12, dtype=torch.bfloat16).expand(900, -1, -1)
    want, bound = attend_by_hand(q, k, v, toks, bias, 500, 0, 40, 64, False, q, True)
    o = model.attend(q, k, v, model.sentence_spans(torch.from_numpy(toks).cuda()), bias, left=500, sinks=40, reach=64)
    inside(o, want["o"], bound["o"], "o")


@pytest.mark.parametrize("dim", [64, 80, 128])
@pytest.mark.parametrize("low", [-1e3, -1e5, -1e9, torch.finfo(torch.float32).min, 1e5])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attend_rows_of_nothing_but_low_biases(model, dim, low, dtype):
    """A head without any other bias, and words that see hidden buckets only (the first ones of their sentence): softmax does not
    know a constant, forwards and backwards.  Keys are alike, so that the scores' digits, which a bias of 1e9 swallows in 32
    bits, do not matter; the bounds are the usual ones."""
    n, h, kv = 700, 4, 2
    toks = stream(n, (1, 300), 8)
    bias = randn(16, h, seed=9, by=0.5)
    bias[:, 1] = low                                                 # a whole head
    bias[:4, 2] = low                                                # distances 0 to 3
    one = randn(1, kv, dim, seed=12, dtype=dtype)
    q, k, v, d_o = randn(n, h, dim, seed=1, dtype=dtype), one.expand(n, -1, -1), randn(n, kv, dim, seed=3, dtype=dtype), randn(n, h, dim, seed=4, dtype=dtype)
    for left, right, sinks, two in ((60, 0, 4, False), (500, 90, 0, True), (100, 5, 40, False)):
        want, bound = attend_by_hand(q, k, v, toks, bias, left, right, sinks, 64, two, d_o, True)
        spans = model.sentence_spans(torch.from_numpy(toks).cuda())
        o, saved = model.attend(q, k, v, spans, bias, left=left, right=right, sinks=sinks, reach=64, two_sided=two, train=True)
        for name, x in zip(("o", "dq", "dk", "dv", "dbias"), (o, *model.attend_backward(d_o, saved))):
            inside(x, want[name], bound[name], name)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("low", [-float("inf"), torch.finfo(torch.float32).min, -1e5, 2e3])
def test_attend_far_buckets_hidden(model, dim, low):
    """The last bucket, which whole tiles without masks lie in, and sinks beyond it; with -infinity in every bucket of a head its rows
    are empty."""
    toks = stream(1200, (1200, 1200), 8, oov=0.002)
    bias = randn(16, 4, seed=9, by=0.5)
    bias[15, :2] = low
    if low == -float("inf"):
        bias[:, 3] = low
    q, k, v, d_o = (randn(1200, x, dim, seed=s, dtype=torch.bfloat16) for s, x in ((1, 4), (2, 2), (3, 2), (4, 4)))
    if low > 0:
        k[:] = k[:1].clone()                                         # scores alike: what a bias of thousands swallows of them does not matter
    want, bound = attend_by_hand(q, k, v, toks, bias, 700, 0, 8, 64, False, d_o, True)
    spans = model.sentence_spans(torch.from_numpy(toks).cuda())
    o, saved = model.attend(q, k, v, spans, bias, left=700, sinks=8, reach=64, train=True)
    for name, x in zip(("o", "dq", "dk", "dv", "dbias"), (o, *model.attend_backward(d_o, saved))):
        inside(x, want[name], bound[name], name)
    if low == -float("inf"):
        assert (o[:, 3] == 0).all() and (saved[-1][3] == float("inf")).all()


@pytest.mark.parametrize("dim", [64, 128])
def test_attend_very_low_biases_keep_their_order(model, dim):
    """A bias of -1e32 outweighs one of the lowest float, in every kernel."""
    toks, bias = stream(600, (600, 600), 3, oov=0.0), torch.full((16, 4), torch.finfo(torch.float32).min, device="cuda")
    bias[2], bias[15, 1] = -1e32, -1e31
    q, v, d_o = (randn(600, x, dim, seed=s, dtype=torch.bfloat16) for s, x in ((1, 4), (3, 2), (4, 4)))
    k = randn(1, 2, dim, seed=12, dtype=torch.bfloat16).expand(600, -1, -1)
    want, bound = attend_by_hand(q, k, v, toks, bias, 300, 0, 4, 64, False, d_o, True)
    spans = model.sentence_spans(torch.from_numpy(toks).cuda())
    o, saved = model.attend(q, k, v, spans, bias, left=300, sinks=4, reach=64, train=True)
    for name, x in zip(("o", "dq", "dk", "dv", "dbias"), (o, *model.attend_backward(d_o, saved))):
        inside(x, want[name], bound[name], name)
    cache = torch.zeros(2, 1, 305, 2, dim, dtype=torch.bfloat16, device="cuda")
    for t in range(5):
        one = model.attend_token(q[t: t + 1], k[t: t + 1].contiguous(), v[t: t + 1], cache[0], cache[1], torch.tensor([t], dtype=torch.int32, device="cuda"), bias,
                                 left=300, sinks=4, reach=64)
        inside(one[0], want["o"][t], bound["o"][t], f"word {t}")


# ---- sinks of sentences with long stretches that nobody sees -----------------------------------------------------------------
@pytest.mark.parametrize("left", [30, 300, 700])
@pytest.mark.parametrize("kv", [1, 4])
def test_attend_sinks_across_empty_tiles(model, left, kv):
    """Words that the vocabulary does not have fill whole tiles within a sentence, at its beginning and between sentences; the sinks'
    gradients come from the tiles behind them."""
    n = 2000
    toks = stream(n, (n, n), 4, oov=0.02)
    toks[[0, 100, 101, 1300]] = -1
    toks[102: 110] = 5                                               # sinks, and then nothing for three tiles
    for a, b in ((110, 560), (700, 980), (1301, 1600), (1900, 2000)):
        toks[a: b] = VOCAB + 9
    both_ways(model, toks, 4, kv, 64, torch.bfloat16, randn(16, 4, seed=9, by=0.5), left, left=left, right=3, sinks=6, reach=64, two_sided=True)


def test_attend_backward_of_a_padded_stream(model):
    """A short stream in a long buffer of separators or unknown words: the gradient's time goes with the words."""
    n, words = 2_000_000, 2000
    toks = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    toks[:words] = torch.from_numpy(stream(words, (400, 900), 4)).cuda()
    q, k = randn(n, 1, 64, seed=1, dtype=torch.bfloat16), randn(n, 1, 64, seed=2, dtype=torch.bfloat16)
    times = {}
    for sinks in (0, 4):
        for pad in (-1, VOCAB):
            toks[words:] = pad
            spans = model.sentence_spans(toks)
            _, saved = model.attend(q, k, k, spans, left=60, sinks=sinks, train=True)
            for _ in range(3):
                begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
                begin.record()
                grads = model.attend_backward(q, saved)
                end.record()
                torch.cuda.synchronize()
                times[sinks, pad] = min(times.get((sinks, pad), 1e9), begin.elapsed_time(end))
            assert all((g[words:] == 0).all() for g in grads[:3])
    assert max(times.values()) < 10 * min(times.values())            # sinks cost a small part; looking for them from every tile on cost 170 times the rest


# ---- layer norm: rows enough for the kernels with a ring ------------------------------------------------------------------------
@pytest.mark.parametrize("rows,d,pad,xt,yt", [
    (7001, 300, 20, torch.float32, torch.bfloat16),       # 3 accesses a lane, forwards
    (30_001, 400, 0, torch.float32, torch.float32),       # 4 accesses a lane, both ways
    (155_001, 256, 0, torch.bfloat16, torch.bfloat16),    # 1 access a lane, both ways
    (19_001, 64, 8, torch.float16, torch.float16),        # backwards
    (11_001, 320, 0, torch.bfloat16, torch.bfloat16),
    (140_001, 200, 0, torch.float32, torch.bfloat16),     # backwards
    (90_001, 300, 20, torch.float32, torch.float16),      # dy in rows of 600 bytes without gaps, an odd number of them
    (5001, 404, 0, torch.float32, torch.bfloat16),        # dy in rows of 808 bytes
    (299, 8192, 8, torch.bfloat16, torch.bfloat16),
])
def test_layer_norm_of_rows_for_the_ring(model, rows, d, pad, xt, yt):
    wide = randn(rows, d + pad, seed=d + pad, dtype=xt, by=0.7) + torch.tensor(0.25, dtype=xt, device="cuda")
    check_layer_norm(model, wide[:, :d], xt, yt)


# ---- single tokens over long windows ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("score", [-12.5, -17.6875, -19.0])
def test_attend_token_many_small_weights(model, dtype, score):
    """One key ahead of 200,000 that are alike: together they matter, each of them is less than the smallest float16."""
    left, dim = 200_000, 64
    ck = torch.zeros(1, left + 1, 1, dim, dtype=dtype, device="cuda")
    cv = torch.ones_like(ck)
    ck[..., 0] = score
    ck[:, 0], cv[:, 0] = 0, 0                                        # the first key seen, with score 0 and value 0
    q, k, v = torch.zeros(1, 1, dim, dtype=dtype, device="cuda"), ck[:, 1].clone(), cv[:, 1].clone()
    q[..., 0] = 8.0                                                  # dim ** -0.5 * 8 = 1
    pos = torch.full((1,), left, dtype=torch.int32, device="cuda")
    o = model.attend_token(q, k, v, ck, cv, pos, left=left)
    w = left * torch.tensor(float(torch.tensor(score, dtype=dtype)), dtype=torch.float64, device="cuda").exp()
    want = (w / (1 + w)).expand_as(o)
    inside(o, want, U[dtype] * want + F32 * want + 1e-6, "o")


def test_sentence_spans_of_wide_ids(model):
    """Ids beyond 32 bits are words that the vocabulary does not have, not what is left of them modulo 2^32."""
    toks = torch.tensor([3, 2 ** 32 + 5, 4, 2 ** 32 - 1, -2 ** 32 - 1, 2 ** 40, -1, 7, -2 ** 63, 2 ** 63 - 1], device="cuda")
    want = torch.tensor([[0, 6], [1, 1], [0, 6], [3, 3], [4, 4], [5, 5], [6, 6], [7, 10], [8, 8], [9, 9]], dtype=torch.int32, device="cuda")
    assert torch.equal(model.sentence_spans(toks), want)
    assert torch.equal(model.sentence_spans(toks[::3].to(torch.int16)), model.sentence_spans(torch.tensor([3, -1, -1, -1], dtype=torch.int32, device="cuda")))
    with pytest.raises(TypeError, match="whole numbers"):
        model.sentence_spans(toks.float())


@pytest.mark.parametrize("dim", [64, 80, 128])
@pytest.mark.parametrize("which", ["q", "k", "v", "d_o"])
def test_attend_nonfinite_words_and_sinks_that_are_no_words(model, dim, which):
    """A word that holds NaN spoils the bias' gradient at the distances of pairs that are seen, not at those to a sink that
    the vocabulary does not have."""
    toks = stream(300, (300, 300), 2, oov=0.0)
    toks[:30] = VOCAB                                                # of forty sinks
    t = {"q": randn(300, 2, dim, seed=1, dtype=torch.bfloat16), "k": randn(300, 1, dim, seed=2, dtype=torch.bfloat16),
         "v": randn(300, 1, dim, seed=3, dtype=torch.bfloat16), "d_o": randn(300, 2, dim, seed=4, dtype=torch.bfloat16)}
    bias, over = randn(64, 2, seed=5, by=0.5), dict(left=1, sinks=40, reach=1024)
    want, bound = attend_by_hand(t["q"], t["k"], t["v"], toks, bias, 1, 0, 40, 1024, False, t["d_o"], True)
    spans = model.sentence_spans(torch.from_numpy(toks).cuda())
    starts = torch.from_numpy(binding.w2v_bucket_starts(64, 1024, False)).cuda().long()
    for x in (50, 140, 270):
        spoilt = {name: u.clone() for name, u in t.items()}
        spoilt[which][x] = float("nan")
        _, saved = model.attend(spoilt["q"], spoilt["k"], spoilt["v"], spans, bias, train=True, **over)
        dbias = model.attend_backward(spoilt["d_o"], saved)[3]
        rows = [x] if which in ("q", "d_o") else [x, x + 1]
        seen = torch.tensor([i - j for i in rows for j in (*range(30, 40), i - 1, i)], device="cuda")
        hit = torch.zeros(64, dtype=torch.bool, device="cuda")
        hit[torch.searchsorted(starts, seen, right=True) - 1] = True
        assert torch.isnan(dbias[hit]).all()
        inside(dbias[~hit], want["dbias"][~hit], bound["dbias"][~hit], "dbias")
