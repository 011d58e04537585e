"""A small reader over trained rows: a word's vector in its place, from one layer of attention over the sentence.

The tables of a `W2V` model stay as they are: input rows come from U, words are answered from V.  Between them lie
layer norm, attention over a window of the sentence with a bias by distance, and a second layer norm, trained by their
gradients to tell a sentence's next word from drawn ones, served word by word from a ring cache, with scores from a copy
of V in 4 bits:

    x = U[w]    z = x + attend(norm(x) Wqkv) Wo    h = norm(z)    score(w') = h . V[w']

The products with Wqkv and Wo are library products.  `python -m paper_1606_08495_b200.reader` trains both parts on
a stream of made-up sentences and then continues one.  On another stream than the model's, calls are ordered with
the model's (`W2V.join_streams`).
"""
from __future__ import annotations

import numpy as np
import torch

from . import binding


class Reader:
    """One layer of `heads` attention heads of `head_dim` (`kv_heads` of keys and values), windows of `left` words before
    and the first `sinks` words of the sentence; `buckets` distances up to `reach` have a bias of their own."""

    def __init__(self, model, heads=4, kv_heads=2, head_dim=64, left=63, sinks=1, buckets=32, reach=64, seed=1):
        self.m, self.heads, self.kv, self.dim = model, heads, kv_heads, head_dim
        self.over = dict(left=left, sinks=sinks, reach=reach)
        self.table, self.answers = (t.view(model.vocab, model.row_stride)[:, : model.d] for t in (model.U, model.V))
        gen = torch.Generator(device=self.table.device).manual_seed(seed)
        f = lambda *s: torch.zeros(*s, device=self.table.device)  # noqa: E731
        d, wide = model.d, (heads + 2 * kv_heads) * head_dim
        self.p = {"gamma": f(d) + 1, "beta": f(d), "qkv": f(d, wide).normal_(std=d ** -0.5, generator=gen), "bias": f(buckets, heads),
                  "out": f(heads * head_dim, d), "gamma_h": f(d) + 1, "beta_h": f(d)}
        self.packed = None

    # ---- a stream of sentences ----------------------------------------------------------------------
    def read(self, tokens, train=False):
        """h [n, d] of every position of a token stream (int32, -1 between sentences, words that the vocabulary does not
        have are seen by nobody); with train=True (h, what `gradients` needs)."""
        m, p = self.m, self.p
        m.join_streams()                                             # the tables' rows are read here
        word = (tokens >= 0) & (tokens < m.vocab)
        x = self.table[torch.where(word, tokens, 0).long()] * word[:, None]
        y, norm = m.layer_norm(x, p["gamma"], p["beta"], out_dtype=torch.bfloat16)
        qkv = (y @ p["qkv"].bfloat16()).view(len(tokens), self.heads + 2 * self.kv, self.dim)
        q, k, v = qkv.split([self.heads, self.kv, self.kv], 1)
        spans = m.sentence_spans(tokens)
        o = m.attend(q, k, v, spans, p["bias"], train=train, **self.over)
        o, kept = o if train else (o, None)
        z = x + (o.flatten(1) @ p["out"].bfloat16()).float()
        h, norm_h = m.layer_norm(z, p["gamma_h"], p["beta_h"])
        return (h, (y, norm, o, kept, norm_h)) if train else h

    def gradients(self, dh, saved):
        """Gradients of the parameters by name, and of the input rows as "x"."""
        m, p, g = self.m, self.p, {}
        y, norm, o, kept, norm_h = saved
        dz, g["gamma_h"], g["beta_h"] = m.layer_norm_backward(dh, norm_h)
        da = dz.bfloat16()
        g["out"] = (o.flatten(1).t() @ da).float()
        do = (da @ p["out"].bfloat16().t()).view(o.shape)
        dq, dk, dv, g["bias"] = m.attend_backward(do, kept)
        dqkv = torch.cat([dq, dk, dv], 1).flatten(1)
        g["qkv"] = (y.t() @ dqkv).float()
        dx, g["gamma"], g["beta"] = m.layer_norm_backward(dqkv @ p["qkv"].bfloat16().t(), norm)
        g["x"] = dz + dx
        return g

    def loss(self, h, tokens, drawn):
        """(mean loss, its gradient in h): logistic, the next word of the sentence against the words drawn [n, k]; a drawn
        word that the vocabulary does not have takes no part."""
        here, after, drawn = tokens[:-1], tokens[1:], drawn[:-1]
        in_v = lambda t: (t >= 0) & (t < self.m.vocab)  # noqa: E731
        use = (in_v(here) & in_v(after)).float()[:, None]
        ids = torch.cat([torch.where(use[:, 0] > 0, after, 0)[:, None], torch.where(in_v(drawn), drawn, 0)], 1).long()
        self.m.join_streams()
        rows = self.answers[ids]
        self.m.join_streams()                                        # the model may go on writing its rows
        score = torch.einsum("nd,nkd->nk", h[:-1], rows)
        sign = torch.ones_like(score)
        sign[:, 1:] = -1.0
        count = use.sum().clamp(min=1)
        use = torch.cat([use, use * in_v(drawn)], 1)
        loss = (torch.nn.functional.softplus(-sign * score) * use).sum() / count
        dh = torch.zeros_like(h)
        dh[:-1] = torch.einsum("nk,nkd->nd", -sign * torch.sigmoid(-sign * score) * use / count, rows)
        return loss, dh

    def train_step(self, tokens, drawn, lr):
        """One step of gradient descent; the loss before it (a tensor on the device)."""
        h, saved = self.read(tokens, train=True)
        loss, dh = self.loss(h, tokens, drawn)
        for name, g in self.gradients(dh, saved).items():
            if name != "x":
                self.p[name] -= lr * g
        return loss

    # ---- word by word ---------------------------------------------------------------------------------
    def start(self, batch):
        """Caches for `batch` sentences that grow one word at a time.  Packs the table of answers as it is now: `next` scores with
        the copy of the last `start`, whatever training has done to V since."""
        places = self.over["sinks"] + self.over["left"] + 1
        make = lambda: torch.zeros(batch, places, self.kv, self.dim, dtype=torch.bfloat16, device=self.table.device)  # noqa: E731
        self.packed = self.m.fourbit_pack(self.answers)
        return {"k": make(), "v": make(), "pos": torch.zeros(batch, dtype=torch.int32, device=self.table.device)}

    def next(self, state, words):
        """(h [batch, d], scores [batch, vocab]) after one more word per sentence.  A sentence waits at -1 and at every other
        word that the vocabulary does not have: its cache and position stay, as if the word were not there (`read` counts
        such a word's position), and h is that of a word that holds and sees nothing."""
        m, p = self.m, self.p
        m.join_streams()
        goes = (words >= 0) & (words < m.vocab)
        x = self.table[torch.where(goes, words, 0).long()] * goes[:, None]
        y, _ = m.layer_norm(x, p["gamma"], p["beta"], out_dtype=torch.bfloat16)
        qkv = (y @ p["qkv"].bfloat16()).view(len(words), self.heads + 2 * self.kv, self.dim)
        q, k, v = qkv.split([self.heads, self.kv, self.kv], 1)
        pos = torch.where(goes, state["pos"], -1)
        o = m.attend_token(q, k, v, state["k"], state["v"], pos, p["bias"], **self.over)
        state["pos"] += goes
        h, _ = m.layer_norm(x + (o.flatten(1) @ p["out"].bfloat16()).float(), p["gamma_h"], p["beta_h"])
        return h, torch.cat([m.fourbit_scores(h[i: i + 8], *self.packed) for i in range(0, max(len(words), 1), 8)])


def main():
    vocab, d, words = 2000, 128, 20_000
    gen = torch.Generator(device="cuda").manual_seed(7)
    # sentences that walk through the vocabulary in steps of 1 to 3
    step = torch.randint(1, 4, (words // 20, 20), generator=gen, device="cuda")
    walk = (torch.randint(0, vocab, (words // 20, 1), generator=gen, device="cuda") + step.cumsum(1)) % vocab
    tokens = torch.cat([walk, torch.full_like(walk[:, :1], -1)], 1).flatten().to(torch.int32)
    model = binding.W2V(vocab, d, seed=1)
    model.build_alias(np.full(vocab, words // vocab, np.uint64), 0.0)
    for i in range(60):
        model.set_step(i)
        model.sgns_step(tokens, 5, 5, 0.05, binding.MODE_HOGWILD, want_stats=False)
    reader = Reader(model)
    for i in range(200):
        drawn = torch.randint(0, vocab, (len(tokens), 5), generator=gen, device="cuda")
        loss = reader.train_step(tokens, drawn, 0.01)
        if i % 40 == 0 or i == 199:
            print(f"step {i:3d}  loss {float(loss):.4f}")
    state, word, line = reader.start(1), tokens[:1], []
    for _ in range(12):
        line.append(int(word))
        _, scores = reader.next(state, word)
        scores[0, line] = -float("inf")                             # no word twice
        word = scores.argmax(1).to(torch.int32)
    print("continued:", *line)
    model.close()


if __name__ == "__main__":
    main()
