"""The reader over trained rows: its gradients against a plain 64-bit layer, its words against its streams."""
import numpy as np
import pytest
import torch

from paper_1606_08495_b200 import binding

pytestmark = pytest.mark.gpu
VOCAB, D = 700, 96


@pytest.fixture(scope="module")
def reader():
    from paper_1606_08495_b200.reader import Reader
    m = binding.W2V(VOCAB, D, seed=5, row_stride=binding.aligned_row_stride(D))
    gen = torch.Generator(device="cuda").manual_seed(3)
    for t in (m.U, m.V):
        t.view(VOCAB, m.row_stride)[:, :D].normal_(std=0.5, generator=gen)
    r = Reader(m, heads=4, kv_heads=2, head_dim=64, left=20, sinks=2, buckets=16, reach=32)
    r.p["bias"].normal_(std=0.3, generator=gen)
    r.p["out"].normal_(std=(4 * 64) ** -0.5, generator=gen)        # zeros at first, which hide all that lies behind them
    r.p["gamma"].normal_(mean=1.0, std=0.1, generator=gen)
    yield r
    m.close()


def stream(n, seed):
    rng = np.random.default_rng(seed)
    toks = rng.integers(0, VOCAB, n).astype(np.int32)
    toks[rng.random(n) < 0.03] = -1
    toks[rng.random(n) < 0.02] = VOCAB + 1
    return torch.from_numpy(toks).cuda()


def plain(r, toks, p, x):
    """h in 64 bits, differentiable."""
    n, h, kv, dim, over = len(toks), r.heads, r.kv, r.dim, r.over
    norm = lambda t, g, b: torch.nn.functional.layer_norm(t, (D,), g, b, 1e-5)  # noqa: E731
    qkv = (norm(x, p["gamma"], p["beta"]) @ p["qkv"]).view(n, -1, dim)
    q, k, v = qkv.split([h, kv, kv], 1)
    k, v = (t.repeat_interleave(h // kv, 1) for t in (k, v))
    word = (toks >= 0) & (toks < VOCAB)
    sentence = (toks == -1).cumsum(0)
    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
    start = torch.cummax(torch.where(toks == -1, i[:, 0] + 1, 0), 0).values
    ok = (sentence[:, None] == sentence[None]) & word[:, None] & word[None] & (j <= i) & ((j >= i - over["left"]) | (j < start[:, None] + over["sinks"]))
    starts = torch.from_numpy(binding.w2v_bucket_starts(p["bias"].shape[0], over["reach"], False)).cuda().long()
    which = torch.searchsorted(starts, (i - j).clamp(min=0), right=True) - 1
    s = torch.einsum("ihd,jhd->hij", q, k) * dim ** -0.5 + p["bias"][which].permute(2, 0, 1)
    w = torch.softmax(s.masked_fill(~ok, -1e300), -1) * ok
    o = torch.einsum("hij,jhd->ihd", w, v)
    return norm(x + o.flatten(1) @ p["out"], p["gamma_h"], p["beta_h"])


def test_gradients(reader):
    toks = stream(330, 1)
    dh = torch.randn(330, D, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    h, saved = reader.read(toks, train=True)
    got = reader.gradients(dh, saved)
    p = {name: t.double().requires_grad_() for name, t in reader.p.items()}
    word = (toks >= 0) & (toks < VOCAB)
    x = (reader.table[torch.where(word, toks, 0).long()] * word[:, None]).double().requires_grad_()
    want = plain(reader, toks, p, x)
    (want * dh.double()).sum().backward()
    # activations and their gradients are rounded to 8 bits some four times on the way, each 2^-9 of its size on average;
    # a sum of such is off by some 2^-7 of its norm, 2^-5 leaves room
    close = lambda a, b: float((a.double() - b).detach().norm() / b.detach().norm()) < 2.0 ** -5  # noqa: E731
    assert close(h[word], want[word])
    seen = word[:, None].expand_as(x)                              # rows of zeros have a layer norm of no use
    assert close(got.pop("x")[seen], x.grad[seen])
    for name, g in got.items():
        assert close(g, p[name].grad), name


def test_words_one_by_one_like_a_stream(reader):
    toks = torch.from_numpy(np.random.default_rng(4).integers(0, VOCAB, (3, 60)).astype(np.int32)).cuda()
    whole = [reader.read(t.contiguous()) for t in toks]
    state = reader.start(3)
    reader.next(state, torch.full((3,), -1, dtype=torch.int32, device="cuda"))             # nobody moves
    packed, scales = reader.packed
    nib = torch.stack([packed & 15, packed >> 4], -1).flatten(1)[:, :D].float() - 8
    table = nib * scales.float().repeat_interleave(32, 1)[:, :D]
    for t in range(60):
        h, scores = reader.next(state, toks[:, t].contiguous())
        for b in range(3):
            # the same roundings in another order: four of 2^-8, of values up to the largest
            assert (h[b] - whole[b][t]).abs().max() <= 2.0 ** -6 * whole[b][t].abs().max()
        assert (scores - h @ table.t()).abs().max() <= 1e-3 * (h.abs() @ table.abs().t()).max()
    assert state["pos"].tolist() == [60] * 3


def test_training_lowers_the_loss(reader):
    toks = stream(2000, 6)
    keep = {name: t.clone() for name, t in reader.p.items()}
    gen = torch.Generator(device="cuda").manual_seed(1)
    drawn = torch.randint(0, VOCAB, (2000, 5), generator=gen, device="cuda")
    losses = [float(reader.train_step(toks, drawn, 0.05)) for _ in range(15)]
    reader.p.update(keep)
    assert losses[-1] < 0.9 * losses[0] and all(b < a * 1.02 for a, b in zip(losses, losses[1:]))
