"""The cache of quantized pages -- append, gather, attention -- against plain references on the host."""
import numpy as np
import pytest

from oracle import serving
from test_gpu_parity import host, mpq
from test_gpu_tokens import dev, full, rng

pytestmark = pytest.mark.gpu

DTYPES = ("float32", "bfloat16", "float16")
NAN = float("nan")


class Pair:
    """The same cache on the device and on the host.  The device's starts as garbage: nothing that no token of a call
    reaches may matter."""

    def __init__(self, pages, heads, page, dim, bits, seed=0):
        import torch
        self.dev = mpq.KvCache.empty(pages, heads, page, dim, bits)
        g = torch.Generator(device="cuda").manual_seed(seed)
        for t in (self.dev.k_codes, self.dev.v_codes):
            t.copy_(torch.randint(-128, 128, t.shape, dtype=torch.int8, device="cuda", generator=g))
        self.dev.k_absmax.fill_(NAN)
        self.dev.v_absmax.fill_(NAN)
        self.host = serving.Cache(pages, heads, page, dim, bits)

    def batch(self, new, length, table, max_new=None, max_len=None, behind=0):
        starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.starts, self.length, self.table = starts, np.asarray(length, np.int32), np.asarray(table, np.int32)
        return mpq.KvBatch(dev(starts, "int32"), dev(self.length, "int32"), dev(self.table, "int32"), int(starts[-1]) + behind, max_new, max_len)

    def append(self, batch, k, v):
        """k, v: device tensors [rows, heads, dim]"""
        mpq.kv_append(self.dev, batch, k, v)
        self.host.append(self.starts, self.length, self.table, full(k), full(v))

    def check_codes(self):
        """Codes of every token that was written and maxima of every page that has one, bit for bit."""
        for name, codes, absmax in (("k", host(self.dev.k_codes), host(self.dev.k_absmax)), ("v", host(self.dev.v_codes), host(self.dev.v_absmax))):
            if name == "v":
                p, h, g, d, _ = codes.shape
                codes = codes.transpose(0, 1, 2, 4, 3).reshape(p, h, 4 * g, d)
            used = self.host.used[name]
            np.testing.assert_array_equal(codes.transpose(0, 2, 1, 3)[used], self.host.codes[name].transpose(0, 2, 1, 3)[used])
            some = used.any(1)
            np.testing.assert_array_equal(absmax[some], self.host.absmax[name][some])


def tables(r, seqs, per_seq, spare=3):
    pages = seqs * per_seq + spare
    return pages, r.permutation(pages)[:seqs * per_seq].reshape(seqs, per_seq).astype(np.int32)


def tokens(r, rows, heads, dim, dtype, spread=1.0):
    """Two views [rows, heads, dim] into one tensor, as a layer leaves keys and values; sizes grow from row to row."""
    both = r.standard_normal((rows, 2, heads, dim)) * np.exp(spread * r.standard_normal((rows, 1, heads, 1)))
    both = dev(both, dtype)
    return both[:, 0], both[:, 1]


@pytest.mark.parametrize("page", (16, 32, 64, 128))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,dim,bits", [(1, 16, 8), (3, 80, 6), (2, 128, 8), (2, 256, 2)])
def test_append_and_gather(page, dtype, heads, dim, bits):
    """Prompts, then single tokens one after the other across a page's end, several at once, a token twice."""
    r = rng(page + dim)
    seqs = 4
    pages, table = tables(r, seqs, 300 // page + 2)
    c = Pair(pages, heads, page, dim, bits, seed=page)
    length = np.zeros(seqs, int)

    def step(new):
        nonlocal length
        length = length + np.asarray(new)
        b = c.batch(new, length, table)
        k, v = tokens(r, b.rows, heads, dim, dtype)
        c.append(b, k, v)
        c.check_codes()
        return b, k, v

    step([0, 1, page - 1, 2 * page + 5])
    for _ in range(3):
        b, k, v = step([1, 1, 1, 1])
    mpq.kv_append(c.dev, b, k, v)  # the same rows again: nothing changes
    c.check_codes()
    step([5, 0, 2, 70])
    b = c.batch(length, length, table)  # whole sequences back
    for out in DTYPES:
        gk, gv = mpq.kv_gather(c.dev, b, dtype=getattr(__import__("torch"), out))
        wk, wv = c.host.gather(c.starts, c.length, c.table, b.rows)
        np.testing.assert_array_equal(full(gk), full(dev(wk, out)))
        np.testing.assert_array_equal(full(gv), full(dev(wv, out)))
    only, none = mpq.kv_gather(c.dev, b, want_v=False)
    assert none is None
    np.testing.assert_array_equal(host(only), wk)


def test_rows_of_no_sequence_and_pages_that_do_not_exist():
    import torch
    r = rng(5)
    heads, dim, page = 2, 32, 16
    pages, table = tables(r, 3, 3)
    c = Pair(pages, heads, page, dim, 8)
    table[1, 1] = pages + 7
    table[2, 0] = -1
    # sequence 2 is longer than its table; rows 90.. belong to nobody
    b = c.batch([20, 40, 30], [20, 40, 60], table, behind=6)
    k, v = tokens(r, b.rows, heads, dim, "float32")
    before = [t.clone() for t in (c.dev.k_codes, c.dev.v_codes)]
    # (the first half of sequence 2 has to be in the cache before its second half is)
    first = c.batch([0, 0, 30], [0, 0, 30], table)
    c.append(first, k[:30], v[:30])
    b = c.batch([20, 40, 30], [20, 40, 60], table, behind=6)
    c.append(b, k, v)
    c.check_codes()
    touched = torch.from_numpy(c.host.used["k"].any(1)).cuda()
    for old, t in zip(before, (c.dev.k_codes, c.dev.v_codes)):
        assert torch.equal(old[~touched], t[~touched])
    assert torch.isnan(c.dev.k_absmax[~touched]).all()
    gk = torch.full((b.rows, heads, dim), 5.0, device="cuda")
    gv = gk.clone()
    mpq.kv_gather(c.dev, b, k=gk, v=gv)
    wk, wv = c.host.gather(c.starts, c.length, c.table, b.rows)
    for g, w in ((gk, wk), (gv, wv)):
        np.testing.assert_array_equal(host(g)[:90], w[:90])
        assert torch.all(g[90:] == 5.0)
    q = dev(r.standard_normal((b.rows, 4, dim)))
    out = torch.full((b.rows, 4, dim), 5.0, device="cuda")
    mpq.kv_attention(c.dev, b, q, out=out)
    assert torch.all(out[90:] == 5.0)
    check_attention(c, host(out)[:90], host(q)[:90], True, 0, dim ** -0.5, "float32")


def test_starts_and_lengths_that_make_no_sense_stay_inside():
    """Ranges out of order, beyond the rows, negative lengths: cut, whatever comes out of it."""
    import torch
    r = rng(6)
    pages, table = tables(r, 3, 2)
    c = Pair(pages, 1, 16, 16, 8)
    batch = mpq.KvBatch(dev([5, 2, 2000, -7], "int32"), dev([-3, 2 ** 31 - 1, 10], "int32"), dev(table, "int32"), 12)
    k, v = tokens(r, 12, 1, 16, "float32")
    mpq.kv_append(c.dev, batch, k, v)
    gk, gv = mpq.kv_gather(c.dev, batch)
    out = mpq.kv_attention(c.dev, batch, dev(r.standard_normal((12, 1, 16))))
    torch.cuda.synchronize()
    assert gk.shape == gv.shape == out.shape


def check_attention(c, got, q, causal, window, scale, dtype, q_true=None):
    """Bound of |got - exact| for a row and head, with L the largest sum of |q_d K_d| scale over its tokens (so |logit| <= L),
    V its largest |value|, n its tokens, u = 2^-24:
      a logit is off by at most e = L ((dim + 4) u + 2^-21): dim additions and four scalings in fp32, q in two terms of fp16
      (or in one, exact);  its exponential by that and 2^-21 more (e * ln 2 units, the subtraction of a maximum below L);
      numerator and sum are chains of at most n / 4 + 64 additions in fp32; probabilities as fp16 are off by 2^-11 (fp32: two
      terms, 2^-22), in the numerator alone, p below being half of that, and by 2^-39 absolutely;
    so a weighted mean of values is off by at most 2 V (2 e + 2^-21 + (n / 4 + 64) u + p) and n 2^-38 V, and the output's type
    rounds by half a step (fp16: at least 2^-25)."""
    want, logit, big = c.host.attention(c.starts, c.length, c.table, q, causal, window, scale)
    rows = want.shape[0]
    n = max(int(c.length.max()), 1)
    u, dim = 2.0 ** -24, want.shape[2]
    p = 2.0 ** -22 if dtype == "float32" else 2.0 ** -12
    e = logit * ((dim + 4) * u + 2.0 ** -21)
    off = 2 * big * (2 * e + 2.0 ** -21 + (n / 4 + 64) * u + p) + n * 2.0 ** -38 * big
    half = {"float32": u, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}[dtype]
    bound = off[..., None] + half * (np.abs(want) + off[..., None]) + (2.0 ** -25 if dtype == "float16" else 0.0)
    bad = np.abs(got[:rows] - want) > bound
    assert not bad.any(), (np.argwhere(bad)[:5], np.abs(got - want).max(), bound.min())


def filled(r, seqs, lengths, heads, dim, page, bits, dtype, spread=0.7):
    pages, table = tables(r, seqs, (max(lengths) + page - 1) // page + 1)
    c = Pair(pages, heads, page, dim, bits)
    b = c.batch(lengths, lengths, table)
    k, v = tokens(r, b.rows, heads, dim, dtype, spread)
    c.append(b, k, v)
    return c, table


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", (16, 32, 64, 128))
@pytest.mark.parametrize("heads,group,dim", [(1, 1, 64), (2, 3, 128), (1, 16, 96), (3, 1, 16), (1, 5, 256), (2, 2, 144)])
def test_single_tokens(dtype, page, heads, group, dim):
    """Lengths from none to several steps of every wave, in one batch."""
    r = rng(page * 3 + dim)
    lengths = [1, 15, 16, 17, 63, 64, 65, 129, 0, 300, 777]
    c, table = filled(r, len(lengths), lengths, heads, dim, page, 8, dtype)
    new = [1] * len(lengths)
    b = c.batch(new, lengths, table)
    q = dev(r.standard_normal((b.rows, heads * group, dim)) * 2, dtype)
    for causal in (True, False):
        out = mpq.kv_attention(c.dev, b, q, causal=causal)
        check_attention(c, full(out), full(q), causal, 0, dim ** -0.5, dtype)
    assert not full(out)[8].any()      # the sequence without a token


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 37)])
@pytest.mark.parametrize("heads,group,dim,page,new,held", [
    (2, 2, 64, 16, [7, 40, 1], [0, 13, 90]), (1, 3, 128, 64, [130, 65], [0, 61]), (1, 1, 80, 32, [64, 33], [100, 3]),
    (1, 7, 256, 128, [20, 5], [130, 0]), (1, 4, 128, 16, [200], [77])])
def test_several_rows(dtype, causal, window, heads, group, dim, page, new, held):
    r = rng(sum(new) + dim + window)
    lengths = [a + b for a, b in zip(new, held)]
    c, table = filled(r, len(new), lengths, heads, dim, page, 8, dtype)
    b = c.batch(new, lengths, table, max(new), max(lengths))
    wide = dev(r.standard_normal((b.rows, heads * group + 3, dim + 8)) * 2, dtype)
    q = wide[:, 1:1 + heads * group, 3:3 + dim]     # strided, at any element
    scale = 0.3 / dim ** 0.5
    store = __import__("torch").full((b.rows, heads * group, 2, dim), 9.0, dtype=q.dtype, device="cuda")
    out = mpq.kv_attention(c.dev, b, q, causal=causal, window=window, softmax_scale=scale, out=store[:, :, 1])
    assert (store[:, :, 0] == 9.0).all()
    check_attention(c, full(out), full(q), causal, window, scale, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_in_front_of_the_first_token_see_nothing(dtype):
    """More rows than tokens under a causal mask: the first ones lie at negative positions."""
    r = rng(11)
    c, table = filled(r, 2, [40, 5], 1, 64, 16, 8, dtype)
    b = c.batch([60, 5], [40, 5], table)
    q = dev(r.standard_normal((65, 2, 64)), dtype)
    out = full(mpq.kv_attention(c.dev, b, q))
    assert not out[:20].any() and out[20:].any(axis=(1, 2)).all()
    check_attention(c, out, full(q), True, 0, 0.125, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bits", (8, 4, 2))
def test_peaked_and_flat_rows_and_uneven_pages(dtype, bits):
    """Logits up to several hundred, a row of zeros (a plain mean), keys and values whose maxima differ by orders from page
    to page, a page of zeros."""
    r = rng(bits)
    heads, dim, page, n = 2, 64, 16, 500
    pages, table = tables(r, 1, 33)
    c = Pair(pages, heads, page, dim, bits)
    b = c.batch([n], [n], table)
    k, v = tokens(r, n, heads, dim, dtype, 0.3)
    size = np.exp(r.uniform(-6, 3, n // page + 1)).repeat(page)[:n, None, None]
    size[48:64] = 0
    k, v = k * dev(np.minimum(size, 4), dtype), v * dev(size, dtype)
    c.append(b, k, v)
    b = c.batch([4], [n], table)
    q = dev(r.standard_normal((4, 4, dim)) * np.array([0, 1, 8, 40])[:, None, None], dtype)
    for scale in (0.125, -0.125):
        out = mpq.kv_attention(c.dev, b, q, causal=False, softmax_scale=scale)
        check_attention(c, full(out), full(q), False, 0, scale, dtype)
    # tiny and huge tensors: exponents far from 0 on either side
    small = Pair(pages, heads, page, dim, bits)
    b = small.batch([n], [n], table)
    small.append(b, dev(r.standard_normal((n, heads, dim)) * 1e-30), dev(r.standard_normal((n, heads, dim)) * 1e-33))
    b = small.batch([2], [n], table)
    q = dev(r.standard_normal((2, 4, dim)) * 1e30)
    out = mpq.kv_attention(small.dev, b, q, causal=False)
    check_attention(small, full(out), full(q), False, 0, 0.125, "float32")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("seqs,held,group", [(1, 5000, 4), (2, 3000, 1), (1, 9001, 16)])
def test_long_sequences_are_split(dtype, seqs, held, group):
    r = rng(held)
    heads, dim, page = 1, 128, 64
    lengths = [held] + [held // 3] * (seqs - 1)
    c, table = filled(r, seqs, lengths, heads, dim, page, 8, dtype)
    for new in (1, 3):
        b = c.batch([new] * seqs, lengths, table, new, held)
        assert mpq.kv_attention_workspace_bytes(c.dev, b, getattr(__import__("torch"), dtype), heads * group) > 0
        q = dev(r.standard_normal((b.rows, heads * group, dim)) * 2, dtype)
        out = mpq.kv_attention(c.dev, b, q)
        check_attention(c, full(out), full(q), True, 0, dim ** -0.5, dtype)
        out = mpq.kv_attention(c.dev, b, q, window=700)
        check_attention(c, full(out), full(q), True, 700, dim ** -0.5, dtype)


def test_results_do_not_depend_on_the_run():
    """The same call twice, on another stream, and with its own scratch: the same bits."""
    import torch
    r = rng(12)
    c, table = filled(r, 3, [2000, 100, 1], 2, 128, 32, 8, "bfloat16")
    b = c.batch([1, 1, 1], [2000, 100, 1], table)
    q = dev(r.standard_normal((3, 8, 128)), "bfloat16")
    a = mpq.kv_attention(c.dev, b, q)
    assert torch.equal(a, mpq.kv_attention(c.dev, b, q))
    assert torch.equal(a, mpq.kv_attention(c.dev, b, q, ws=mpq.Workspace()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o = mpq.kv_attention(c.dev, b, q)
    side.synchronize()
    assert torch.equal(a, o)


def test_a_shared_page_is_read_by_both_sequences():
    import torch
    r = rng(13)
    c, table = filled(r, 1, [100], 2, 64, 16, 8, "float32")
    both = np.concatenate([table, table])
    b = c.batch([1, 1], [100, 100], both)
    q = dev(r.standard_normal((1, 4, 64))).repeat(2, 1, 1)
    out = mpq.kv_attention(c.dev, b, q)
    assert torch.equal(out[0], out[1])
    check_attention(c, full(out), full(q), True, 0, 0.125, "float32")


def test_offsets_past_32_bits():
    """A cache of more than 2^32 bytes of key codes: its last pages."""
    import torch
    r = rng(14)
    heads, dim, page = 8, 128, 128
    pages = (1 << 32) // (heads * dim * page) + 40
    c = mpq.KvCache.empty(pages, heads, page, dim)
    small = Pair(40, heads, page, dim, 8)
    table = r.permutation(40)[:6].reshape(2, 3).astype(np.int32)
    new = [300, 200]
    b = small.batch(new, new, table)
    far = mpq.KvBatch(b.starts, b.kv_len, b.table + (pages - 40), b.rows)
    k, v = tokens(r, b.rows, heads, dim, "bfloat16")
    small.append(b, k, v)
    mpq.kv_append(c, far, k, v)
    for x, y in zip(mpq.kv_gather(c, far), mpq.kv_gather(small.dev, b)):
        assert torch.equal(x, y)
    q = dev(r.standard_normal((b.rows, 8, dim)), "bfloat16")
    assert torch.equal(mpq.kv_attention(c, far, q), mpq.kv_attention(small.dev, b, q))


def test_decode_steps_from_a_replayed_graph():
    """Append and attention of a step captured once; the program writes new lengths and inputs between the replays."""
    import torch
    mpq.init()
    r = rng(15)
    heads, group, dim, page, seqs, steps = 2, 4, 64, 16, 3, 6
    lengths = np.array([14, 700, 31])
    c, table = filled(r, seqs, list(lengths), heads, dim, page, 8, "bfloat16")
    twin = mpq.KvCache(*(t.clone() for t in (c.dev.k_codes, c.dev.v_codes, c.dev.k_absmax, c.dev.v_absmax)), 8)
    starts, kv_len, dtable = dev(np.arange(seqs + 1), "int32"), dev(lengths, "int32"), dev(table, "int32")
    b = mpq.KvBatch(starts, kv_len, dtable, seqs, 1, page * table.shape[1])
    k, v = (torch.zeros(seqs, heads, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros(seqs, heads * group, dim, dtype=torch.bfloat16, device="cuda")
    g = torch.cuda.CUDAGraph()
    kept = [t.clone() for t in (twin.k_codes, twin.v_codes, twin.k_absmax, twin.v_absmax)]
    with torch.cuda.graph(g):
        mpq.kv_append(twin, b, k, v)
        out = mpq.kv_attention(twin, b, q)
    for t, o in zip((twin.k_codes, twin.v_codes, twin.k_absmax, twin.v_absmax), kept):
        t.copy_(o)
    for _ in range(steps):
        kv_len += 1
        for t in (k, v, q):
            t.copy_(dev(r.standard_normal(tuple(t.shape)) * 2, "bfloat16"))
        g.replay()
        mpq.kv_append(c.dev, b, k, v)
        want = mpq.kv_attention(c.dev, b, q)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    np.testing.assert_array_equal(host(twin.k_codes), host(c.dev.k_codes))
    np.testing.assert_array_equal(host(twin.v_codes), host(c.dev.v_codes))
    np.testing.assert_array_equal(host(twin.k_absmax), host(c.dev.k_absmax))


def test_no_probability_of_fp32_is_off_by_a_step_of_fp16():
    """Probabilities are multiplied as two fp16 terms, which together have about 22 bits.  With a value of its own channel for each
    of 64 tokens an output is a token's probability.  Products of whole numbers are exact here, so that a logit below 8 is
    off by its scalings alone (8 * 4 * 2^-24 = 2^-19) and a probability by that, its exponential, its terms and the sum (2^-21,
    2^-21, 64 * 2^-24): below 2^-17 together; a step of fp16 is 2^-11."""
    r = rng(21)
    heads, dim, page = 16, 64, 16
    for seed in range(12):
        pages, table = tables(r, 1, 4)
        c = Pair(pages, heads, page, dim, 8)
        b = c.batch([64], [64], table)
        k = r.integers(-127, 128, (64, heads, dim)).astype(np.float64)
        k[::page] = 127.0                      # a page's maximum, so that codes are the numbers
        v = np.broadcast_to(np.eye(64)[:, None, :] * (1 + seed / 16), (64, heads, dim))
        c.append(b, dev(k), dev(v))
        b = c.batch([1], [64], table)
        q = r.integers(-3, 4, (1, heads, dim)).astype(np.float64)
        scale = 1 / 1024
        got = full(mpq.kv_attention(c.dev, b, dev(q), causal=False, softmax_scale=scale)).astype(np.float64)
        x = np.einsum("jhd,hd->hj", k, q[0]) * scale
        p = np.exp(x - x.max(1, keepdims=True))
        p = p / p.sum(1, keepdims=True) * (1 + seed / 16)
        assert np.abs(x).max() < 8 and (np.abs(got[0] / p - 1) < 2.0 ** -16).all(), np.abs(got[0] / p - 1).max()
