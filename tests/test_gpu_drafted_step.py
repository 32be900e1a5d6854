"""A step of drafted tokens as a served model takes it: the layer with group steps, norm and rotation where the heads lie, the cache, the
tree's attention, the layer behind it, and the log probabilities of the drafts -- then the tokens that are kept go into the cache in a
row, and the next token sees them."""
import numpy as np
import pytest

from oracle import drafts
from test_gpu_kv import Pair, tables
from test_gpu_parity import host, mpq
from test_gpu_tokens import dev, full, rng

pytestmark = pytest.mark.gpu

HEADS, KV, DIM, WIDTH, VOCAB, GROUP = 4, 2, 64, 256, 1000, 64


class Model:
    """One layer and its head: what the device computes from, and the same numbers on the host."""

    def __init__(self, r):
        self.w = {n: mpq.group_quant(dev(r.standard_normal((rows, cols)) * cols ** -0.5), GROUP)
                  for n, rows, cols in (("qkv", (HEADS + 2 * KV) * DIM, WIDTH), ("out", WIDTH, HEADS * DIM), ("head", VOCAB, WIDTH))}
        self.host = {n: (drafts.nibbles(host(w)), host(s)) for n, (w, s) in self.w.items()}
        self.freq = (10000.0 ** (-np.arange(DIM // 2) / (DIM // 2))).astype(np.float32)
        self.weights = [(1 + 0.2 * r.standard_normal(DIM)).astype(np.float32) for _ in range(2)]

    def linear(self, name, x):
        return mpq.linear_groups(x, *self.w[name])

    def linear_host(self, name, x):
        return drafts.linear_groups(x, *self.host[name], GROUP)

    def heads(self, x, positions):
        """(queries, keys, values) on the device: views of one tensor, queries and keys turned in place."""
        qkv = self.linear("qkv", x).view(x.shape[0], -1, DIM)
        q, k, v = qkv[:, :HEADS], qkv[:, HEADS:HEADS + KV], qkv[:, HEADS + KV:]
        mpq.rotate_heads(q, k, dev(positions, "int32"), dev(self.freq), dev(self.weights[0]), dev(self.weights[1]), q_out=q, k_out=k)
        return q, k, v

    def heads_host(self, x, positions):
        qkv = self.linear_host("qkv", x).reshape(x.shape[0], -1, DIM)
        q, _ = drafts.rotate_heads(qkv[:, :HEADS], positions, self.freq, self.weights[0], 1e-6, False)
        k, _ = drafts.rotate_heads(qkv[:, HEADS:HEADS + KV], positions, self.freq, self.weights[1], 1e-6, False)
        return q, k, qkv[:, HEADS + KV:]


def test_a_step_of_drafted_tokens():
    """In fp32.  The cache rounds to 8 bits, and its codes may fall to either side where a key lies near the middle: the host's cache takes
    the device's keys and values, and these are compared with the host's own beforehand."""
    r = rng(42)
    model = Model(r)
    held, trees = [37, 90], [[-1, 0, 0, 1, -1, 3], [-1, -1, 1, 1]]
    new = [len(t) for t in trees]
    depth = [np.array([bin(int(b)).count("1") - 1 for b in mpq.tree_bits(t)[:, 0]]) for t in trees]
    positions = np.concatenate([h + d for h, d in zip(held, depth)]).astype(np.int32)
    pages, table = tables(r, 2, 8)
    c = Pair(pages, KV, 16, DIM, 8)
    before = np.concatenate([np.arange(h) for h in held]).astype(np.int32)
    q, k, v = model.heads(dev(r.standard_normal((sum(held), WIDTH))), before)
    c.append(c.batch(held, held, table), k, v)

    x = r.standard_normal((sum(new), WIDTH)).astype(np.float32)
    q, k, v = model.heads(dev(x), positions)
    for a, b in zip((q, k, v), model.heads_host(x, positions)):
        # the layer: 55 * 2 * 64 u of its terms' magnitude (test_gpu_groups), below 2^-11 of the largest output; norm and rotation add units
        assert np.abs(host(a) - b).max() <= 2.0 ** -11 * np.abs(b).max()
    b = c.batch(new, [h + n for h, n in zip(held, new)], table)
    c.append(b, k, v)
    c.check_codes()
    import torch
    tree = torch.cat([mpq.tree_bits(t) for t in trees]).cuda()
    o = mpq.kv_attention_tree(c.dev, b, q, tree)
    seen = [int(w) for w in tree[:, 0].tolist()]
    want_o, _, _ = drafts.attention_tree(c.host, c.starts, c.length, c.table, host(q), seen, DIM ** -0.5)
    assert np.abs(host(o) - want_o).max() <= 2.0 ** -17 * np.abs(want_o).max()     # logits below 64: 64 ((DIM + 4) u + 2^-21) and terms
    y = model.linear("out", o.view(sum(new), -1))
    logits = model.linear("head", y)
    ids = r.integers(0, VOCAB, sum(new)).astype(np.int32)
    logprob, entropy, best, index = mpq.token_logprobs(logits, dev(ids, "int32"), 5)
    want_logits = model.linear_host("head", model.linear_host("out", want_o.reshape(sum(new), -1)))
    want, want_h, want_best, _, _, _ = drafts.token_logprobs(want_logits, ids, 5, 1.0)
    near = 2.0 ** -9 * max(np.abs(want_logits).max(), 1)
    assert np.abs(host(logprob) - want).max() <= near and np.abs(host(best) - want_best).max() <= near
    assert np.abs(host(entropy) - want_h).max() <= near * 8
    np.testing.assert_array_equal(host(index), drafts.token_logprobs(host(logits), ids, 5, 1.0)[3])

    # a branch of each sequence is kept: drafts 0, 1, 3, 5 and 1, 2
    kept = [[0, 1, 3, 5], [1, 2]]
    rows = np.concatenate([np.array(p) + s for p, s in zip(kept, (0, new[0]))])
    at = torch.from_numpy(rows).cuda()
    length = [h + len(p) for h, p in zip(held, kept)]
    b = c.batch([len(p) for p in kept], length, table)
    c.append(b, k[at].contiguous(), v[at].contiguous())
    c.check_codes()
    gk, gv = mpq.kv_gather(c.dev, b)
    wk, wv = c.host.gather(c.starts, c.length, c.table, b.rows)
    np.testing.assert_array_equal(host(gk), wk)
    np.testing.assert_array_equal(host(gv), wv)
    # and the next token of each, a draft of one, sees them as attention of single tokens does
    x = dev(r.standard_normal((2, WIDTH)))
    q, k, v = model.heads(x, np.array(length, np.int32))
    b = c.batch([1, 1], [n + 1 for n in length], table)
    c.append(b, k, v)
    one = torch.ones((2, 1), dtype=torch.int64, device="cuda")
    a, t = host(mpq.kv_attention(c.dev, b, q)), host(mpq.kv_attention_tree(c.dev, b, q, one))
    assert np.abs(a - t).max() <= 2.0 ** -19 * np.abs(a).max()


def test_a_captured_step():
    """The whole step as one graph, replayed with new inputs, positions, lengths and trees, against the calls one by one."""
    import torch
    r = rng(43)
    model = Model(r)
    held, new = [100, 60], [4, 3]
    pages, table = tables(r, 2, 8)
    c = Pair(pages, KV, 16, DIM, 8)
    _, k, v = model.heads(dev(r.standard_normal((sum(held), WIDTH))), np.concatenate([np.arange(h) for h in held]).astype(np.int32))
    c.append(c.batch(held, held, table), k, v)
    b = c.batch(new, [h + n for h, n in zip(held, new)], table)
    x, positions = torch.empty((7, WIDTH), device="cuda"), torch.empty(7, dtype=torch.int32, device="cuda")
    tree, ids = torch.empty((7, 1), dtype=torch.int64, device="cuda"), torch.empty(7, dtype=torch.int32, device="cuda")
    freq, qw, kw = dev(model.freq), dev(model.weights[0]), dev(model.weights[1])

    def fill():
        lists = [[int(r.integers(-1, i)) for i in range(n)] for n in new]
        tree.copy_(torch.cat([mpq.tree_bits(p) for p in lists]))
        x.copy_(dev(r.standard_normal((7, WIDTH))))
        positions.copy_(dev(r.integers(60, 110, 7), "int32"))
        ids.copy_(dev(r.integers(0, VOCAB, 7), "int32"))

    def step():
        qkv = model.linear("qkv", x).view(7, -1, DIM)
        q, k, v = qkv[:, :HEADS], qkv[:, HEADS:HEADS + KV], qkv[:, HEADS + KV:]
        mpq.rotate_heads(q, k, positions, freq, qw, kw, q_out=q, k_out=k)
        mpq.kv_append(c.dev, b, k, v)
        o = mpq.kv_attention_tree(c.dev, b, q, tree)
        return mpq.token_logprobs(model.linear("head", model.linear("out", o.view(7, -1))), ids, 3)

    fill()
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    # (a page's maximum grows with what was ever drafted onto it: both runs of a step start from the same cache)
    parts = (c.dev.k_codes, c.dev.v_codes, c.dev.k_absmax, c.dev.v_absmax)
    for _ in range(3):
        fill()
        saved = [t.clone() for t in parts]
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for t, s in zip(parts, saved):
            t.copy_(s)
        assert all(torch.equal(p, q) for p, q in zip(got, step()))
