"""The cache and its attention where device arrays and tensors hold what a program rarely gives them: lengths beyond the table,
windows and values at the end of their ranges.  Bounds: check_attention's."""
import numpy as np
import pytest

from test_gpu_kv import DTYPES, check_attention, filled
from test_gpu_parity import mpq
from test_gpu_tokens import dev, full, rng

pytestmark = pytest.mark.gpu


def check(c, got, *args):
    """check_attention compares with >, which a NaN never is: outputs have to be numbers as well."""
    assert np.isfinite(got).all(), np.argwhere(~np.isfinite(got))[:5]
    check_attention(c, got, *args)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new,group", [(1, 1), (1, 16), (12, 3), (70, 2)])
@pytest.mark.parametrize("dim,page", [(64, 64), (128, 16), (256, 32)])
def test_a_window_behind_the_tables_end_sees_nothing(dtype, new, group, dim, page):
    """A length beyond what the table holds, and a window that ends short of it: rows see nothing and give 0, those of a sequence
    whose window reaches back into the table see its end.  The table lies inside a larger tensor of valid page numbers."""
    r = rng(dim + page + new)
    room, window = 192, 75
    lengths = [room, room, room, 150]
    c, table = filled(r, 4, lengths, 1, dim, page, 8, dtype)
    table = table[:, :room // page]
    wide = np.zeros((40, room // page), np.int32)
    wide[:4] = table
    whole = dev(wide, "int32")
    said = [1000, room + 40, room + window + new, 150]
    b = c.batch([new] * 4, said, table)
    b = mpq.KvBatch(b.starts, b.kv_len, whole[:4], b.rows, new, 1024)
    q = dev(r.standard_normal((b.rows, group, dim)) * 2, dtype)
    out = full(mpq.kv_attention(c.dev, b, q, window=window))
    assert not out[:new].any() and out[new:2 * new].any(axis=(1, 2)).all() and not out[3 * new - 1].any()
    check(c, out, full(q), True, window, dim ** -0.5, dtype)


@pytest.mark.parametrize("window", (2 ** 31, 2 ** 62, 2 ** 63 - 1))
@pytest.mark.parametrize("new,heads", [(200, 1), (128, 16)])
def test_a_window_of_any_size_is_none_when_it_reaches_everything(window, new, heads):
    """Rows in front of the first token among them, in calls that either kernel takes."""
    import torch
    r = rng(new)
    lengths = [40, new, 130, 5, 70, 300, 1, 2]
    c, table = filled(r, 8, lengths, heads, 64, 16, 8, "bfloat16")
    b = c.batch([new] * 8, lengths, table, new, 300)
    q = dev(r.standard_normal((b.rows, heads, 64)), "bfloat16")
    want = mpq.kv_attention(c.dev, b, q)
    assert torch.equal(mpq.kv_attention(c.dev, b, q, window=window), want)
    check(c, full(want), full(q), True, 0, 0.125, "bfloat16")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", (16, 64))
@pytest.mark.parametrize("new", (1, 128))
def test_pages_whose_maximum_is_zero_whatever_their_codes(dtype, page, new):
    """A caller's own cache, or one whose maxima were cleared: codes under a maximum of 0 are zeros (code * 0 / qmax), for
    values as for keys, and their tokens keep their weight.  A sequence whose value maxima are all 0 gives 0."""
    r = rng(page + new)
    lengths = [256, 200, 300, 130, 128, 140, 257, 190]
    c, table = filled(r, 8, lengths, 4, 64, page, 8, dtype)
    for s, at, name in ((0, 0, "v"), (0, 128 // page, "v"), (1, 64 // page, "k"), (2, 192 // page, "v"), (2, 192 // page, "k"), (3, 0, "v")):
        (c.dev.v_absmax if name == "v" else c.dev.k_absmax)[int(table[s, at])] = 0
        c.host.absmax[name][table[s, at]] = 0
    for on in table[4]:
        c.dev.v_absmax[int(on)] = 0
        c.host.absmax["v"][on] = 0
    assert c.host.codes["v"][table[4, 0]].any()
    b = c.batch([new] * 8, lengths, table, new, 300)
    q = dev(r.standard_normal((b.rows, 8, 64)) * 2, dtype)
    out = full(mpq.kv_attention(c.dev, b, q))
    assert not out[4 * new:5 * new].any()
    check(c, out, full(q), True, 0, 0.125, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", "kv")
@pytest.mark.parametrize("page", (16, 64))
@pytest.mark.parametrize("new,window", [(1, 0), (1, 40), (7, 0), (7, 40), (128, 0), (128, 40)])
def test_an_infinite_page_spoils_the_rows_that_see_it(dtype, name, page, new, window):
    """A token with an infinity leaves an infinite maximum on its page.  Rows that see the page become NaN; rows in front of it,
    behind the window or of other heads keep their values, whatever tile or step they share with it."""
    import torch
    r = rng(page + new + window)
    lengths = [256, 200, 300, 130, 128, 140, 257, 190]
    c, table = filled(r, 8, lengths, 4, 64, page, 8, dtype)
    b = c.batch([new] * 8, lengths, table, new, 300)
    q = dev(r.standard_normal((b.rows, 8, 64)), dtype)
    clean = mpq.kv_attention(c.dev, b, q, window=window)
    bad = np.zeros((b.rows, 8), bool)
    for s, at, h in ((0, 192 // page, 1), (1, 0, 0), (2, 2, 3), (4, 64 // page, 2), (6, 256 // page, 0), (7, 176 // page, 3)):
        (c.dev.k_absmax if name == "k" else c.dev.v_absmax)[int(table[s, at]), h] = float("inf")
        codes = c.dev.k_codes if name == "k" else c.dev.v_codes      # what append leaves under such a maximum
        codes[int(table[s, at]), h] = 0
        for i in range(new):
            p = lengths[s] - new + i
            if p >= at * page and (window == 0 or (at + 1) * page > p - window + 1):
                bad[s * new + i, 2 * h:2 * h + 2] = True
    got = mpq.kv_attention(c.dev, b, q, window=window)
    t = torch.from_numpy(bad).cuda()
    assert bad.any() and not bad.all() and got[t].isnan().all()
    got[t] = clean[t]
    check(c, full(got), full(q), True, window, 0.125, dtype)


def half_step(x, dtype):
    """Half a step of the type at x."""
    half, least = {"float32": (2.0 ** -24, 0.0), "bfloat16": (2.0 ** -8, 0.0), "float16": (2.0 ** -11, 2.0 ** -25)}[dtype]
    return np.maximum(half * 2.0 ** np.floor(np.log2(np.maximum(x, 1e-30))), least)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", (16, 64))
@pytest.mark.parametrize("rows", (1, 512))
def test_probabilities_keep_their_bits(dtype, page, rows):
    """With a value of its own channel for each of 64 tokens an output is a token's probability.  Products of whole numbers are exact
    here, so that a logit below 9 is off by its scalings alone (9 * 4 * 2^-24 = 1.125 * 2^-19) and a probability by that, its exponential
    and the value factor that it takes along (2^-20), its two fp16 terms and the sum (2^-21, 64 * 2^-24): 1.94 * 2^-18 together.
    The terms end at 2^-25 of a scale that holds the largest one at 2^8 or more: 2^-33, of values below 2.  bf16 prompts (512 rows of
    16 key heads) have one term: 2^-11 more.  Beyond that an output is off by the half step that it is rounded by."""
    r = rng(page + rows)
    heads = 16
    for seed in range(6):
        c, table = filled(r, 1, [64], heads, 64, page, 8, dtype)
        k = r.integers(-127, 128, (64, heads, 64)).astype(np.float64)
        k[::page] = 127.0                      # a page's maximum, so that codes are the numbers
        size = 1 + seed / 16
        v = np.broadcast_to(np.eye(64)[:, None, :] * size, (64, heads, 64))
        b = c.batch([64], [64], table)
        mpq.kv_append(c.dev, b, dev(k, dtype), dev(v, dtype))
        b = c.batch([rows], [64], table)
        q = r.integers(-3, 4, (rows, heads, 64)).astype(np.float64)
        scale = 1 / 1024
        got = full(mpq.kv_attention(c.dev, b, dev(q, dtype), causal=False, softmax_scale=scale)).astype(np.float64)
        x = np.einsum("jhd,rhd->rhj", k, q) * scale
        e = np.exp(x - x.max(2, keepdims=True))
        p = e / e.sum(2, keepdims=True) * size
        off = p * (2.0 ** -17 + (2.0 ** -11 if dtype == "bfloat16" and rows > 1 else 0)) + 2.0 ** -32
        assert np.abs(x).max() < 9 and np.isfinite(got).all()
        over = np.abs(got - p) - off - half_step(p + off, dtype)
        assert (over <= 0).all(), (over.max(), (over > 0).sum())


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 90)])
@pytest.mark.parametrize("seqs,heads,group,dim,page,new,held", [
    (3, 1, 2, 64, 16, 1, 700), (2, 2, 4, 128, 64, 1, 300), (1, 1, 4, 128, 64, 1, 5000), (2, 1, 1, 256, 128, 20, 200),
    (8, 4, 2, 64, 16, 128, 70), (8, 4, 2, 128, 64, 128, 30), (8, 4, 2, 80, 128, 64, 1500), (8, 16, 1, 256, 32, 128, 9)])
def test_fp16_keeps_the_bits_of_its_type(causal, window, seqs, heads, group, dim, page, new, held):
    """check_attention's bound with the two terms of an fp16 call's probabilities: 2^-22 of each, and 2^-33 absolutely (prompts; single
    tokens 2^-39), so that the values' mean is off by 2 V 2^-22 and n 2^-32 V in place of 2 V 2^-12 and n 2^-38 V."""
    r = rng(dim + page + new + window)
    lengths = [new + held - 3 * s for s in range(seqs)]
    c, table = filled(r, seqs, lengths, heads, dim, page, 8, "float16")
    b = c.batch([new] * seqs, lengths, table, new, max(lengths))
    q = dev(r.standard_normal((b.rows, heads * group, dim)) * 2, "float16")
    got = full(mpq.kv_attention(c.dev, b, q, causal=causal, window=window))
    want, logit, big = c.host.attention(c.starts, c.length, c.table, full(q), causal, window, dim ** -0.5)
    n, u = max(lengths), 2.0 ** -24
    e = logit * ((dim + 4) * u + 2.0 ** -21)
    off = (2 * big * (2 * e + 2.0 ** -21 + (n / 4 + 64) * u + 2.0 ** -22) + n * 2.0 ** -32 * big)[..., None]
    over = np.abs(got - want) - off - half_step(np.abs(want) + off, "float16")
    assert np.isfinite(got).all() and (over <= 0).all(), over.max()


@pytest.mark.parametrize("dtype", ("float32", "bfloat16"))
@pytest.mark.parametrize("size", (3e38, 1e-30, 1e-33, 2e-36))
@pytest.mark.parametrize("seqs,heads,dim,page,new,held", [
    (3, 1, 64, 16, 1, 700), (1, 1, 128, 64, 1, 5000), (2, 1, 256, 128, 20, 200), (8, 4, 64, 64, 128, 70), (8, 4, 128, 16, 64, 1500)])
def test_values_at_the_ends_of_their_range(dtype, size, seqs, heads, dim, page, new, held):
    """Single tokens and prompts, split and not: a weighted mean of values is no larger than they are and as precise, next to the
    largest number of the type (sums pass it) and next to the smallest (a factor of the sums passes that).  An output of a bf16 call
    may be one of its subnormals, of 2^-133, and an fp32 one of 2^-149: a half step of those more, 2^-134."""
    import torch
    r = rng(dim + page + new)
    lengths = [new + held - 3 * s for s in range(seqs)]
    c, table = filled(r, seqs, lengths, heads, dim, page, 8, dtype)
    b = c.batch(lengths, lengths, table)
    k = r.standard_normal((b.rows, heads, dim))
    v = r.uniform(-1, 1, (b.rows, heads, dim)) + 0.5 * np.sign(r.standard_normal((1, heads, dim)))   # channels with a mean
    v = (torch.from_numpy(v / 1.5).double() * size).to(getattr(torch, dtype)).cuda()
    c.append(b, dev(k, dtype), v)
    b = c.batch([new] * seqs, lengths, table, new, max(lengths))
    q = dev(r.standard_normal((b.rows, heads * 2, dim)), dtype)
    got = full(mpq.kv_attention(c.dev, b, q)).astype(np.float64)
    want, logit, big = c.host.attention(c.starts, c.length, c.table, full(q), True, 0, dim ** -0.5)
    n, u = max(lengths), 2.0 ** -24
    e = logit * ((dim + 4) * u + 2.0 ** -21)
    p = 2.0 ** -22 if dtype == "float32" else 2.0 ** -12
    off = (2 * big * (2 * e + 2.0 ** -21 + (n / 4 + 64) * u + p) + n * 2.0 ** -32 * big)[..., None]
    over = np.abs(got - want) - off - (2.0 ** -24 if dtype == "float32" else 2.0 ** -8) * (np.abs(want) + off) - 2.0 ** -134
    assert np.isfinite(got).all() and (over <= 0).all(), (over / size).max()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", (16, 64, 128))
@pytest.mark.parametrize("new", (1, 9, 128))
def test_pages_behind_the_window_may_hold_anything(dtype, page, new):
    """A server gives the pages that a window has left behind to other sequences, or never wrote them: their codes and maxima
    (a NaN here) reach no row, also where a step's tokens lie on both sides of the window's beginning."""
    import torch
    r = rng(page + new)
    window = 70
    lengths = [256, 200, 300, 150, 141, 140, 257, 190]
    c, table = filled(r, 8, lengths, 4, 64, page, 8, dtype)
    b = c.batch([new] * 8, lengths, table, new, 300)
    for s, n in enumerate(lengths):
        for on in table[s, :max(n - new - window + 1, 0) // page]:
            for t in (c.dev.k_absmax, c.dev.v_absmax):
                t[int(on)] = float("nan")
            for t in (c.dev.k_codes, c.dev.v_codes):
                t[int(on)] = torch.randint(-128, 128, t[int(on)].shape, dtype=torch.int8, device="cuda")
    assert c.dev.k_absmax[torch.from_numpy(table[2, :2]).cuda().long()].isnan().any() or page == 128 or new == 128
    q = dev(r.standard_normal((b.rows, 8, 64)), dtype)
    check(c, full(mpq.kv_attention(c.dev, b, q, window=window)), full(q), True, window, 0.125, dtype)
