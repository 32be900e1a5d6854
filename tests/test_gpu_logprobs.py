"""Log probabilities, entropy and the most probable tokens against a plain reference in 64 bits."""
import numpy as np
import pytest

from oracle import drafts
from test_gpu_parity import host, mpq
from test_gpu_tokens import dev, full, rng

pytestmark = pytest.mark.gpu

DTYPES = ("float32", "bfloat16", "float16")
U = 2.0 ** -24
INF = float("inf")


def check(got, x, tokens, top, scale):
    """With u = 2^-24, d = scale (x - max) and p the probabilities: an exponent is off by 3 u |d| (a difference and two products), its
    exponential by 2 u more, a sum of a chain of 64, then 14, then at most 32 more by 110 u; pieces' factors bring 4 u |d| + 3 u:
    the sum l by rel = 7 u spread + 115 u, spread = sum p |d|.  sum p |d| itself by u (7 bend + 120), relative, bend = sum p d^2 / spread.  So
      log p = d - log l: rel + 3 u |d| + 3 u |log l| + u;   entropy = log l + spread: rel (1 + spread) + spread u (7 bend + 123) + 3 u |log l|."""
    want, want_h, want_top, want_index, spread, bend = drafts.token_logprobs(x, tokens, top, scale)
    with np.errstate(over="ignore"):
        want, want_top = want.astype(np.float32).astype(np.float64), want_top.astype(np.float32).astype(np.float64)   # (u more)
    logprob, entropy, best, index = (host(t) for t in got)
    log_l = np.maximum(want_h - spread, 0)
    rel = U * (7 * spread + 115)

    def close(a, b, bound, what):
        with np.errstate(invalid="ignore"):
            bad = ~((np.abs(a - b) <= bound) | (a == b))
        assert not bad.any(), (what, np.argwhere(bad)[:5], a[bad][:3], b[bad][:3], np.broadcast_to(bound, a.shape)[bad][:3])

    def of(lp):
        with np.errstate(invalid="ignore"):
            d = np.where(np.isfinite(lp), np.abs(lp), 0)
        return d

    close(logprob, want, rel + 3 * U * (of(want) + log_l) + 3 * U * log_l + U, "logprob")
    close(entropy, want_h, rel * (1 + spread) + spread * U * (7 * bend + 123) + 3 * U * (log_l + want_h) + U, "entropy")
    np.testing.assert_array_equal(index, want_index)
    close(best, want_top, rel[:, None] + 3 * U * (of(want_top) + log_l[:, None]) + 3 * U * log_l[:, None] + U, "top")


def rows(r, n, vocab, dtype, peak=10.0):
    x = r.standard_normal((n, vocab)) * 2
    x[np.arange(n), r.integers(0, vocab, n)] += peak * r.random(n)
    return dev(x, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,vocab,top", [(1, 1, 1), (3, 7, 32), (1, 2048, 5), (5, 2049, 5), (2, 32768, 20), (1, 100003, 32), (40, 4099, 1),
                                         (600, 1000, 8), (700, 16390, 20), (300, 33000, 3), (7, 65, 0)])
def test_logprobs(dtype, n, vocab, top):
    r = rng(vocab + n)
    x = rows(r, n, vocab, dtype)
    tokens = r.integers(0, vocab, n).astype(np.int32)
    for scale in (1.0, 0.7, 3.0):
        got = mpq.token_logprobs(x, dev(tokens, "int32"), top, scale)
        if top == 0:
            assert got[2] is None and got[3] is None
            got = got[:2] + tuple(dev(np.zeros((n, 0)), t) for t in ("float32", "int32"))
        check(got, full(x), tokens, top, scale)


@pytest.mark.parametrize("n,vocab", [(1, 16384), (2, 16385), (3, 32768), (2, 32769), (3, 65535), (2, 65536), (2, 65537), (257, 33001), (513, 17001)])
def test_where_a_row_is_cut(n, vocab):
    """The sizes at which a row goes from one workgroup's hold to the next, and the rows at which it is cut after all."""
    r = rng(n * vocab)
    for dtype, top in (("float32", 32), ("bfloat16", 7)):
        x = rows(r, n, vocab, dtype)
        tokens = np.concatenate(([vocab - 1], r.integers(0, vocab, n - 1))).astype(np.int32)
        check(mpq.token_logprobs(x, dev(tokens, "int32"), top), full(x), tokens, top, 1.0)
    x = np.zeros((n, vocab), np.float32)
    check(mpq.token_logprobs(dev(x), dev(tokens, "int32"), 32), x, tokens, 32, 1.0)


@pytest.mark.parametrize("n,vocab", [(1, 5000), (600, 5000), (2, 70000)])
def test_equal_logits(n, vocab):
    """All equal, two values, ties across pieces: the lowest index first."""
    r = rng(n)
    x = np.zeros((n, vocab), np.float32)
    tokens = r.integers(0, vocab, n).astype(np.int32)
    check(mpq.token_logprobs(dev(x), dev(tokens, "int32"), 32), x, tokens, 32, 1.0)
    x[:, r.random(vocab) < 0.5] = 1.0
    check(mpq.token_logprobs(dev(x), dev(tokens, "int32"), 32), x, tokens, 32, 1.0)
    x = np.round(r.standard_normal((n, vocab))).astype(np.float32)
    check(mpq.token_logprobs(dev(x), dev(tokens, "int32"), 20), x, tokens, 20, 1.0)
    for x in (np.sort(r.standard_normal((n, vocab)).astype(np.float32), 1), -np.sort(r.standard_normal((n, vocab)).astype(np.float32), 1)):
        check(mpq.token_logprobs(dev(x), dev(tokens, "int32"), 32), x, tokens, 32, 1.0)


def test_equal_logits_of_many_pieces():
    """More equal alternatives than the join lists at once."""
    x = np.zeros((1, 2 ** 21 + 9), np.float32)
    x[0, 12345] = 1.0
    tokens = np.array([2 ** 21], np.int32)
    check(mpq.token_logprobs(dev(x), dev(tokens, "int32"), 32), x, tokens, 32, 1.0)


@pytest.mark.parametrize("n,vocab", [(3, 500), (1, 40000), (530, 9000)])
def test_tokens_that_are_ruled_out(n, vocab):
    r = rng(vocab)
    x = host(rows(r, n, vocab, "float32")).copy()
    x[r.random((n, vocab)) < 0.5] = -INF
    x[0] = -INF
    x[0, vocab // 2] = -3.5                # a row of one
    x[-1, 7:] = -INF                       # fewer than are asked for
    x[-1, :7] = np.arange(7)
    tokens = r.integers(0, vocab, n).astype(np.int32)
    got = mpq.token_logprobs(dev(x), dev(tokens, "int32"), 20)
    check(got, x, tokens, 20, 1.0)
    if n > 1:
        assert host(got[1])[0] == 0 and host(got[2])[0, 0] == 0 and (host(got[3])[0, 1:] == -1).all()
    # tokens outside of the vocabulary have no probability
    tokens[0], tokens[-1] = -1, vocab
    check(mpq.token_logprobs(dev(x), dev(tokens, "int32"), 3), x, tokens, 3, 1.0)


@pytest.mark.parametrize("n,vocab", [(4, 900), (4, 50000)])
def test_rows_without_a_distribution(n, vocab):
    r = rng(vocab)
    x = host(rows(r, n, vocab, "float32")).copy()
    clean = x.copy()
    x[0] = -INF
    x[1, vocab - 1] = float("nan")
    x[2, 3] = INF
    tokens = r.integers(0, vocab, n).astype(np.int32)
    logprob, entropy, best, index = (host(t) for t in mpq.token_logprobs(dev(x), dev(tokens, "int32"), 4))
    assert np.isnan(logprob[:3]).all() and np.isnan(entropy[:3]).all()
    assert np.isneginf(best[0]).all() and (index[0] == -1).all() and np.isnan(best[1]).all()
    x[1, vocab - 1] = -INF
    np.testing.assert_array_equal(index[1], np.argsort(-x[1], kind="stable")[:4])
    assert index[2, 0] == 3
    want = drafts.token_logprobs(clean[3:], tokens[3:], 4, 1.0)
    assert abs(logprob[3] - want[0][0]) < 1e-4 and (index[3] == want[3][0]).all()


def test_large_values_and_scales():
    r = rng(2)
    tokens = r.integers(0, 3000, 6).astype(np.int32)
    x = r.standard_normal((6, 3000)).astype(np.float32)
    for size, scale in ((1e30, 1e-30), (1e-30, 1e30), (3e38, 1e-38), (1.0, 1e-6), (1.0, 1000.0)):
        y = np.clip(x * np.float32(size), -3.4e38, 3.4e38).astype(np.float32)
        if size == 3e38:
            y = np.clip(y, -1.6e38, 1.6e38)      # (differences stay within the range)
        check(mpq.token_logprobs(dev(y), dev(tokens, "int32"), 4, scale), y, tokens, 4, scale)


@pytest.mark.parametrize("dtype", ("float32", "bfloat16"))
@pytest.mark.parametrize("vocab", (3000, 40000, 90000))
def test_logits_of_the_whole_range(dtype, vocab):
    """Logits up to twice the type's largest apart, and scales that bring them together, down to the least ones that there are."""
    r = rng(vocab + 1)
    top = 3.3e38
    x = dev(np.clip(r.standard_normal((4, vocab)) * 2e38, -top, top), dtype)
    x[1, ::2], x[1, 1::2] = top, -top
    x[2, 5] = -INF
    tokens = r.integers(0, vocab, 4).astype(np.int32)
    for scale in (1e-38, 3e-38, 2.0 ** -126, 1e-40, 2.0 ** -149, 0.7e-37, 0.3):
        check(mpq.token_logprobs(x, dev(tokens, "int32"), 7, scale), full(x), tokens, 7, scale)


def test_the_largest_scale():
    """Up to the one whose product with log2 e is the last finite number; the rest is refused."""
    r = rng(12)
    for size in (1e-38, 1e-3):
        x = (r.standard_normal((3, 5000)) * size).astype(np.float32)
        x[2] = 0
        tokens = r.integers(0, 5000, 3).astype(np.int32)
        for scale in (1e38, 2.35e38):
            check(mpq.token_logprobs(dev(x), dev(tokens, "int32"), 4, scale), x, tokens, 4, scale)
    for scale in (2.4e38, 3.4e38):
        with pytest.raises(mpq.MpqError):
            mpq.token_logprobs(dev(x), dev(tokens, "int32"), 4, scale)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", (700, 30000))
def test_rows_of_the_lowest_value(dtype, vocab):
    """Masks of the type's lowest value: behind them a row of nothing else is even, and one of a few others is those."""
    import torch
    r = rng(vocab)
    low = torch.finfo(getattr(torch, dtype)).min
    x = rows(r, 5, vocab, dtype)
    x[0] = low
    x[1, 5:] = low
    x[2] = -low
    x[3, ::2] = -INF
    x[3, 1::2] = low
    tokens = r.integers(0, vocab, 5).astype(np.int32)
    for scale in (1.0, 0.5, 2.0):
        # (with scale 2 an exponent of the lowest value passes the range: none of it is left, as in the reference)
        check(mpq.token_logprobs(x, dev(tokens, "int32"), 7, scale), full(x), tokens, 7, scale)


def test_strides_outputs_and_the_last_vocabulary():
    import torch
    r = rng(3)
    for dtype in DTYPES:
        wide = torch.empty(5 * 3011 + 1, dtype=getattr(torch, dtype), device="cuda")[1:].view(5, 3011)[:, :3001]
        wide.copy_(rows(r, 5, 3001, dtype))
        tokens = r.integers(0, 3001, 5).astype(np.int32)
        check(mpq.token_logprobs(wide, dev(tokens, "int32"), 6), full(wide), tokens, 6, 1.0)
    x = rows(r, 2, 2 ** 22, "bfloat16")
    tokens = r.integers(0, 2 ** 22, 2).astype(np.int32)
    check(mpq.token_logprobs(x, dev(tokens, "int32"), 32), full(x), tokens, 32, 1.0)
    none, entropy, best, index = mpq.token_logprobs(wide, None, 2)
    assert none is None and torch.equal(entropy, mpq.token_logprobs(wide)[1])
    only = mpq.token_logprobs(wide, dev(tokens[:1].repeat(5) % 3001, "int32"), 0, want_entropy=False)
    assert only[0].shape == (5,) and only[1] is None
    empty = mpq.token_logprobs(wide[:0], dev(np.zeros(0), "int32"), 3)
    assert [t.shape for t in empty] == [(0,), (0,), (0, 3), (0, 3)]


@pytest.mark.parametrize("vocab", (1000, 40000, 70000))
def test_offsets_past_32_bits(vocab):
    """Rows that lie 2^31 bytes apart."""
    import torch
    r = rng(8)
    x = rows(r, 6, vocab, "bfloat16")
    far = torch.empty((5 << 30) + vocab, dtype=torch.bfloat16, device="cuda").as_strided((6, vocab), (1 << 30, 1))
    far.copy_(x)
    t = dev(r.integers(0, vocab, 6), "int32")
    for a, z in zip(mpq.token_logprobs(far, t, 9), mpq.token_logprobs(x, t, 9)):
        assert torch.equal(a, z)


def test_graphs_that_bring_scratch_of_their_own():
    """Rows of several pieces: two captured graphs, and eager calls with one workspace, in turn."""
    import torch
    r = rng(9)
    n, vocab = 5, 90001
    x, t, ws = rows(r, n, vocab, "float16"), dev(r.integers(0, vocab, n), "int32"), mpq.Workspace()
    assert mpq.token_logprobs_workspace_bytes(n, vocab, x.dtype, 6) > 0
    graphs = []
    mpq.token_logprobs(x, t, 6, ws=ws)
    torch.cuda.synchronize()
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = mpq.token_logprobs(x, t, 6)
        graphs.append((g, out))
    for i in range(4):
        x.copy_(rows(r, n, vocab, "float16"))
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        want = mpq.token_logprobs(x, t, 6, ws=ws)
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refusals_of_the_binding():
    r = rng(4)
    x = rows(r, 3, 100, "float32")
    t = dev(np.zeros(3), "int32")
    for bad in ((x[0], t), (x.t(), t), (x, t[:2]), (x, t.long()), (x.double(), t), (x.cpu(), t)):
        with pytest.raises(ValueError):
            mpq.token_logprobs(*bad)
    for bad in ((x, t, 33), (x, t, -1), (x, t, 3, 0.0), (x, t, 3, INF)):
        with pytest.raises((mpq.MpqError, ValueError)):
            mpq.token_logprobs(*bad)
    with pytest.raises(mpq.MpqError):
        mpq.token_logprobs(x, want_entropy=False)


def test_graphs_and_streams():
    """Two captured graphs of one call each, replayed in turn with eager calls between them."""
    import torch
    r = rng(5)
    x = rows(r, 3, 50000, "bfloat16")
    t = dev(r.integers(0, 50000, 3), "int32")
    want = [a.clone() for a in mpq.token_logprobs(x, t, 5)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = mpq.token_logprobs(x, t, 5)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = mpq.token_logprobs(x, t, 5)
        graphs.append((g, out))
    for i in range(4):
        x.copy_(rows(r, 3, 50000, "bfloat16"))
        g, out = graphs[i % 2]
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, mpq.token_logprobs(x, t, 5)))
