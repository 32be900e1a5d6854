"""Attention of a tree of drafted tokens over the cache of quantized pages, against a plain reference in 64 bits."""
import numpy as np
import pytest

from oracle import drafts
from test_gpu_kv import DTYPES, NAN, Pair, tables, tokens
from test_gpu_kv_edges import half_step
from test_gpu_parity import host, mpq
from test_gpu_tokens import dev, full, rng

pytestmark = pytest.mark.gpu


def parents(r, n, reach=8):
    return [int(r.integers(max(-1, i - reach), i)) for i in range(n)]


def bits_of(lists, words=None):
    """(Python integers per row, the call's tensor): lists of parents, a sequence each."""
    import torch
    parts = [mpq.tree_bits(p) for p in lists]
    words = words or max(t.shape[1] for t in parts)
    t = torch.cat([torch.nn.functional.pad(t, (0, words - t.shape[1])) for t in parts]) if parts else torch.zeros((0, words), dtype=torch.int64)
    seen = [sum((int(w) & (1 << 64) - 1) << 64 * i for i, w in enumerate(row)) for row in t.tolist()]
    return seen, t.cuda()


def check(c, got, q, seen, scale, dtype, lengths=None):
    """The bound of test_gpu_kv.check_attention: the same products and sums, fp16 terms of a probability two, or one (bf16 calls of many
    rows)."""
    want, logit, big = drafts.attention_tree(c.host, c.starts, c.length, c.table, q, seen, scale)
    n = max(int(c.length.max()), 1)
    u, dim = 2.0 ** -24, want.shape[2]
    p = 2.0 ** -22 if dtype == "float32" else 2.0 ** -12
    e = logit * ((dim + 4) * u + 2.0 ** -21)
    off = 2 * big * (2 * e + 2.0 ** -21 + (n / 4 + 64) * u + p) + n * 2.0 ** -38 * big
    half = {"float32": u, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}[dtype]
    bound = off[..., None] + half * (np.abs(want) + off[..., None]) + (2.0 ** -25 if dtype == "float16" else 0.0)
    bad = ~(np.abs(got[:want.shape[0]] - want) <= bound)
    assert not bad.any(), (np.argwhere(bad)[:5], np.abs(got - want).max(), bound.min())


def drafted(r, lengths, new, heads, dim, page, bits, dtype):
    """A cache with `lengths` tokens of each sequence, and the batch of its last `new`."""
    pages, table = tables(r, len(lengths), (max(lengths) + page - 1) // page + 1)
    c = Pair(pages, heads, page, dim, bits)
    b = c.batch(lengths, lengths, table)
    k, v = tokens(r, b.rows, heads, dim, dtype, 0.7)
    c.append(b, k, v)
    return c, c.batch(new, lengths, table)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", (16, 32, 64, 128))
@pytest.mark.parametrize("heads,group,dim", [(1, 1, 64), (2, 3, 128), (1, 8, 96), (3, 1, 16), (1, 5, 256), (2, 2, 144)])
def test_small_trees(dtype, page, heads, group, dim):
    """One to three tiles of rows, sequences from the drafted tokens alone to several steps of every wave."""
    r = rng(page * 3 + dim)
    lengths = [1, 5, 17, 64, 65, 130, 300, 700]
    for new in ([1] * 8, [1, 5, 3, 7, 2, 7, 1, 6], [0, 5, 0, 7, 2, 0, 1, 6]):
        c, b = drafted(r, lengths, new, heads, dim, page, 8, dtype)
        seen, tree = bits_of([parents(r, n) for n in new])
        q = dev(r.standard_normal((b.rows, heads * group, dim)) * 2, dtype)
        check(c, full(mpq.kv_attention_tree(c.dev, b, q, tree)), full(q), seen, dim ** -0.5, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", (16, 64, 128))
@pytest.mark.parametrize("heads,group,dim,new,lengths", [(2, 4, 128, [63, 64, 9], [63, 200, 1000]), (1, 2, 64, [65, 130, 1], [70, 700, 300]),
                                                         (1, 1, 256, [100, 33], [133, 900]), (3, 1, 80, [128, 20], [128, 260]),
                                                         (1, 7, 128, [40, 13], [1500, 3000])])
def test_wide_trees(dtype, page, heads, group, dim, new, lengths):
    """More rows than a wave takes, more drafted tokens than a word has bits, splits along long sequences."""
    r = rng(page + dim + len(new))
    c, b = drafted(r, lengths, new, heads, dim, page, 6, dtype)
    seen, tree = bits_of([parents(r, n, 20) for n in new])
    q = dev(r.standard_normal((b.rows, heads * group, dim)) * 2, dtype)
    check(c, full(mpq.kv_attention_tree(c.dev, b, q, tree)), full(q), seen, dim ** -0.5, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", (4, 24, 140))
def test_any_bits(dtype, rows):
    """Bits that are no tree: nothing of the drafted tokens, all of them, later ones, some; more words than needed, bits behind the last
    token; a sequence of nothing but drafted tokens whose row sees none gives 0."""
    r = rng(rows)
    heads, group, dim, page = 2, 2, 64, 16
    lengths, new = [rows, rows + 37, rows], [rows, rows, rows // 2]
    c, b = drafted(r, lengths, new, heads, dim, page, 8, dtype)
    words = (rows + 63) // 64 + 1
    import torch
    tree = torch.from_numpy(r.integers(-2 ** 63, 2 ** 63, (b.rows, words), dtype=np.int64)).cuda()
    tree[0] = 0
    tree[1] = -1
    tree[rows] = 0
    seen = [sum((int(w) & (1 << 64) - 1) << 64 * i for i, w in enumerate(row)) for row in tree.tolist()]
    q = dev(r.standard_normal((b.rows, heads * group, dim)), dtype)
    out = full(mpq.kv_attention_tree(c.dev, b, q, tree, softmax_scale=-0.3))
    check(c, out, full(q), seen, -0.3, dtype)
    assert not out[0].any()


def test_a_chain_is_causal_attention():
    """A tree without branches sees what a causal mask leaves."""
    r = rng(1)
    for dtype in DTYPES:
        for new, heads, group, dim in (([1, 3, 8], 2, 2, 128), ([60, 17, 33], 1, 4, 64)):
            c, b = drafted(r, [70, 500, 40], new, heads, dim, 32, 8, dtype)
            _, tree = bits_of([range(-1, n - 1) for n in new])
            q = dev(r.standard_normal((b.rows, heads * group, dim)), dtype)
            a, t = full(mpq.kv_attention(c.dev, b, q)), full(mpq.kv_attention_tree(c.dev, b, q, tree))
            off = {"float32": 2.0 ** -19, "bfloat16": 2.0 ** -7, "float16": 2.0 ** -10}[dtype]   # two roundings, and p below 2^-11
            assert np.abs(a - t).max() <= off * np.abs(a).max()


@pytest.mark.parametrize("new", (3, 40))
def test_pages_that_are_not_there_and_rows_of_nobody(new):
    import torch
    r = rng(new)
    heads, group, dim, page = 2, 2, 32, 16
    lengths, news = [100, 90, 200, 64], [new, 0, new, min(new, 64)]
    pages, table = tables(r, 4, 13)
    c = Pair(pages, heads, page, dim, 8)
    table[0, 2] = pages + 7
    table[2, 0] = -1
    table[2, -1] = -5
    table[3, :] = -1                 # nothing there at all
    b = c.batch(lengths, lengths, table)
    k, v = tokens(r, b.rows, heads, dim, "float32")
    c.append(b, k, v)
    b = c.batch(news, lengths, table, behind=5)
    seen, tree = bits_of([parents(r, n) for n in news] + [[-1] * 5])
    q = dev(r.standard_normal((b.rows, heads * group, dim)))
    q[-5:] = NAN
    out = torch.full((b.rows, heads * group, dim), 5.0, device="cuda")
    assert mpq.kv_attention_tree(c.dev, b, q, tree, out=out) is out
    assert (out[-5:] == 5).all()
    n = b.rows - 5
    check(c, host(out)[:n], host(q)[:n], seen, dim ** -0.5, "float32")
    assert not out[n - min(new, 64):n].any()


@pytest.mark.parametrize("new", (2, 50))
def test_a_sequence_longer_than_its_table(new):
    """Tokens behind the table's places are absent, drafted ones among them."""
    r = rng(new)
    heads, dim, page = 1, 64, 16
    pages, table = tables(r, 2, 4)
    c = Pair(pages, heads, page, dim, 8)
    first = c.batch([64, 60], [64, 60], table)
    k, v = tokens(r, first.rows, heads, dim, "float32")
    c.append(first, k, v)
    b = c.batch([new, new], [70, 60], table)
    seen, tree = bits_of([parents(r, new), parents(r, new)])
    q = dev(r.standard_normal((b.rows, 3, dim)))
    check(c, host(mpq.kv_attention_tree(c.dev, b, q, tree)), host(q), seen, dim ** -0.5, "float32")


def test_batches_that_make_no_sense_stay_inside():
    """Ranges out of order, beyond the rows, negative lengths, more rows than max_new or than the length: cut, whatever comes out of it."""
    import torch
    r = rng(6)
    pages, table = tables(r, 3, 2)
    c = Pair(pages, 1, 16, 16, 8)
    c.dev.k_absmax.fill_(1)
    c.dev.v_absmax.fill_(1)
    for group in (1, 16):
        for max_new in (None, 2):
            batch = mpq.KvBatch(dev([5, 2, 2000, -7], "int32"), dev([-3, 2 ** 31 - 1, 10], "int32"), dev(table, "int32"), 12, max_new)
            tree = torch.full((12, 1), -1, dtype=torch.int64, device="cuda")
            out = mpq.kv_attention_tree(c.dev, batch, dev(r.standard_normal((12, group, 16))), tree)
            torch.cuda.synchronize()
            assert out.shape == (12, group, 16)
    # five rows of a sequence of three tokens: the first two rows' own tokens are absent
    c = Pair(pages, 1, 16, 16, 8)
    b = c.batch([3], [3], table[:1])
    k, v = tokens(r, 3, 1, 16, "float32")
    c.append(b, k, v)
    b = c.batch([5], [3], table[:1])
    seen, tree = bits_of([[-1, 0, 1, 0, 3]])
    q = dev(r.standard_normal((5, 2, 16)))
    out = host(mpq.kv_attention_tree(c.dev, b, q, tree))
    check(c, out, host(q), seen, 0.25, "float32")
    assert not out[:2].any() and out[2:].any(2).all()


@pytest.mark.parametrize("new", (3, 64))
def test_values_at_the_ends(new):
    """NaN in one row of q and an infinite page that only some rows see spoil those rows alone."""
    r = rng(new + 1)
    heads, dim, page = 1, 64, 16
    c, b = drafted(r, [80 + new], [new], heads, dim, page, 8, "float32")
    seen, tree = bits_of([[-1] * new])
    q = dev(r.standard_normal((new, 4, dim)))
    q[1, 2, 7] = NAN
    out = mpq.kv_attention_tree(c.dev, b, q, tree)
    bad = np.isnan(host(out)).any(2)
    want = np.zeros((new, 4), bool)
    want[1, 2] = True
    np.testing.assert_array_equal(bad, want)
    # the first drafted tokens' page: rows that see none of its tokens keep their numbers
    q = dev(r.standard_normal((new, 4, dim)))
    tree[1:] = 0
    tree[0] = 1
    clean = host(mpq.kv_attention_tree(c.dev, b, q, tree))
    c.dev.v_absmax[int(c.table[0, 5])] = float("inf")        # tokens 80 .. 95: the first is row 0's
    out = host(mpq.kv_attention_tree(c.dev, b, q, tree))
    assert np.isnan(out[0]).any(1).all()
    np.testing.assert_array_equal(out[1:], clean[1:])


def test_strides():
    import torch
    r = rng(9)
    for dtype in DTYPES:
        for new in ([3, 7], [40, 64]):
            heads, group, dim = 2, 2, 80
            c, b = drafted(r, [100, 300], new, heads, dim, 32, 8, dtype)
            _, tree = bits_of([parents(r, n) for n in new])
            q = dev(r.standard_normal((b.rows, heads * group, dim)), dtype)
            want = mpq.kv_attention_tree(c.dev, b, q, tree)
            t = getattr(torch, dtype)
            inside = torch.empty(b.rows * 7 * 90 + 1, dtype=t, device="cuda")[1:].view(b.rows, 7, 90)[:, 1:5, 5:85]
            inside.copy_(q)
            out = torch.full((4, b.rows, 84), 9.0, dtype=t, device="cuda")
            mpq.kv_attention_tree(c.dev, b, inside, tree, out=out[:, :, 2:82].transpose(0, 1))
            assert torch.equal(out[:, :, 2:82].transpose(0, 1), want) and (out[:, :, :2] == 9).all() and (out[:, :, 82:] == 9).all()


@pytest.mark.parametrize("new", ([3, 5], [40, 30], [130, 200]))
def test_offsets_past_32_bits(new):
    """A cache of more than 2^32 bytes of key codes: its last pages."""
    import torch
    r = rng(14)
    heads, dim, page = 8, 128, 128
    pages = (1 << 32) // (heads * dim * page) + 40
    c = mpq.KvCache.empty(pages, heads, page, dim)
    small = Pair(40, heads, page, dim, 8)
    table = r.permutation(40)[:6].reshape(2, 3).astype(np.int32)
    length = [300, 200]
    b = small.batch(length, length, table)
    far = mpq.KvBatch(b.starts, b.kv_len, b.table + (pages - 40), b.rows)
    k, v = tokens(r, b.rows, heads, dim, "bfloat16")
    small.append(b, k, v)
    mpq.kv_append(c, far, k, v)
    b = small.batch(new, length, table)
    far = mpq.KvBatch(b.starts, b.kv_len, b.table + (pages - 40), b.rows)
    seen, tree = bits_of([parents(r, n) for n in new])
    q = dev(r.standard_normal((b.rows, heads, dim)), "bfloat16")
    got = mpq.kv_attention_tree(c, far, q, tree)
    assert torch.equal(got, mpq.kv_attention_tree(small.dev, b, q, tree))
    check(small, full(got), full(q), seen, dim ** -0.5, "bfloat16")


@pytest.mark.parametrize("dtype,page,heads,group,dim,new", [("bfloat16", 64, 8, 2, 64, 5), ("float32", 16, 8, 1, 16, 20), ("float16", 32, 16, 2, 64, 30),
                                                            ("bfloat16", 64, 16, 3, 16, 61), ("float32", 128, 4, 1, 128, 40), ("bfloat16", 16, 8, 2, 144, 9),
                                                            ("float16", 64, 16, 1, 80, 150)])
def test_sequences_of_many_lengths(dtype, page, heads, group, dim, new):
    """One long one, some short, one of its drafted tokens alone, one that brings none."""
    import torch
    r = rng(16)
    length = [5000, 200, 2600, 4999, 151, 3, 700, 64]
    rows = [min(new, n) for n in length]
    rows[4], rows[6] = min(151, new), 0
    c, b = drafted(r, length, rows, heads, dim, page, 8, dtype)
    seen, tree = bits_of([parents(r, n) for n in rows], (new + 63) // 64)
    q = dev(r.standard_normal((b.rows, heads * group, dim)), dtype)
    got = mpq.kv_attention_tree(c.dev, b, q, tree)
    check(c, full(got), full(q), seen, dim ** -0.5, dtype)
    # shorter than the bound that the call was planned for
    b.kv_len.copy_(dev([max(n, m) for n, m in zip([900, 200, 1, 64, 151, 3, 700, 64], rows)], "int32"))
    c.length = full(b.kv_len).astype(np.int32)
    check(c, full(mpq.kv_attention_tree(c.dev, b, q, tree)), full(q), seen, dim ** -0.5, dtype)
    assert torch.equal(mpq.kv_attention_tree(c.dev, b, q, tree), mpq.kv_attention_tree(c.dev, b, q, tree))


@pytest.mark.parametrize("new", (6, 70))
def test_a_bound_of_rows_too_low(new):
    """max_new below a sequence's rows: the others' rows are right, and those of every row within the bound."""
    import torch
    r = rng(15)
    length = [2000, 900, 1500]
    c, b = drafted(r, length, [new, 3, 2], 2, 64, 64, 8, "float16")
    seen, tree = bits_of([parents(r, n) for n in (new, 3, 2)])
    q = dev(r.standard_normal((b.rows, 4, 64)), "float16")
    want = mpq.kv_attention_tree(c.dev, b, q, tree)
    most = new - 2
    low = mpq.KvBatch(b.starts, b.kv_len, b.table, b.rows, most, 2000)
    got = mpq.kv_attention_tree(c.dev, low, q, tree)
    near = lambda a, z: (full(a) - full(z)).__abs__().max() <= 2.0 ** -9 * abs(full(z)).max()  # noqa: E731  (two roundings of fp16, splits)
    assert near(got[new:], want[new:]) and near(got[:most], want[:most])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", (16, 64))
@pytest.mark.parametrize("new,group,dim", [(2, 1, 64), (5, 4, 64), (5, 6, 128), (3, 5, 256), (40, 1, 64), (33, 2, 128), (40, 1, 256), (64, 3, 64),
                                           (64, 4, 128), (64, 3, 256)])
def test_probabilities_keep_their_bits(dtype, page, new, group, dim):
    """With a value of its own channel for each of 64 tokens an output is a token's probability.  Products of whole numbers are exact
    here, so that a logit below 9 is off by its scalings alone (9 * 4 * 2^-24 = 1.125 * 2^-19) and a probability by that, its exponential
    and the value factor that it takes along (2^-20), its two fp16 terms and the sum (2^-21, 64 * 2^-24): 1.94 * 2^-18 together.
    The terms end at 2^-25 of a scale that holds the largest one at 2^8 or more: 2^-33, of values below 2.  Beyond that an output is off by
    the half step that it is rounded by, however many rows the call has."""
    import torch
    r = rng(page + new + dim)
    heads = 4
    pages, table = tables(r, 1, 900 // page)          # (places for more than short sequences, so that many rows go to the kernel for many)
    c = Pair(pages, heads, page, dim, 8)
    scale = 1 / 128 / dim ** 0.5
    for seed in range(4):
        k = r.integers(-127, 128, (64, heads, dim)).astype(np.float64)
        k[::page] = 127.0                              # a page's maximum, so that codes are the numbers
        v = np.broadcast_to(np.eye(64, dim)[:, None, :] * (1 + seed / 16), (64, heads, dim))
        mpq.kv_append(c.dev, c.batch([64], [64], table), dev(k, dtype), dev(v, dtype))
        b = c.batch([new], [64], table, new, 900)
        bits = r.integers(0, 2 ** 63, new, dtype=np.int64) | 1 << np.arange(new, dtype=np.int64) % 63
        tree = torch.from_numpy(bits[:, None]).cuda()
        q = r.integers(-3, 4, (new, heads * group, dim)).astype(np.float64)
        got = full(mpq.kv_attention_tree(c.dev, b, dev(q, dtype), tree, softmax_scale=scale)).astype(np.float64)
        x = np.einsum("jhd,rhgd->rhgj", k, q.reshape(new, heads, group, dim)).reshape(new, heads * group, 64) * scale
        j = np.arange(64)
        sees = (j < 64 - new) | (bits[:, None] >> np.maximum(j - (64 - new), 0) & 1 != 0)
        assert np.abs(x).max() < 9 and sees.any(1).all()
        x = np.where(sees[:, None, :], x, -np.inf)
        e = np.exp(x - x.max(2, keepdims=True))
        p = e / e.sum(2, keepdims=True) * (1 + seed / 16)
        off = p * 2.0 ** -17 + 2.0 ** -32
        assert np.isfinite(got).all() and not got[..., 64:].any()
        over = np.abs(got[..., :64] - p) - off - half_step(p + off, dtype)
        assert (over <= 0).all(), (over.max(), (over > 0).sum())


@pytest.mark.parametrize("new", (6, 70, 75))
def test_rows_behind_a_low_bound_are_nobodys(new):
    """max_new below a sequence's rows: those behind it are left as they were or are what the full call gives, whatever the scratch held."""
    import torch
    r = rng(17)
    length = [2000, 900, 1500]
    c, b = drafted(r, length, [new, 3, 2], 2, 64, 64, 8, "float16")
    seen, tree = bits_of([parents(r, n) for n in (new, 3, 2)])
    q = dev(r.standard_normal((b.rows, 4, 64)), "float16")
    for most in (new - 1, new - 2, new - 5):
        low = mpq.KvBatch(b.starts, b.kv_len, b.table, b.rows, most, 2000)
        need = mpq.kv_attention_tree_workspace_bytes(c.dev, low, q.dtype, 4)
        assert need > 0
        ws = mpq.Workspace()
        ws.get(need)
        ws.buf.fill_(255)
        out = torch.full((b.rows, 4, 64), 9.0, dtype=torch.float16, device="cuda")
        mpq.kv_attention_tree(c.dev, low, q, tree, out=out, ws=ws)
        left = (full(out) == 9).all((1, 2))
        assert not left[:most].any() and not left[new:new + min(most, 3)].any() and not left[new + 3:new + 3 + min(most, 2)].any()
        check(c, np.where(left[:, None, None], full(mpq.kv_attention_tree(c.dev, b, q, tree)), full(out)), full(q), seen, 0.125, "float16")


def splits_of(c, b, dtype, q_heads, most):
    """Of a call, from the scratch that it asks for: partial results of 16 rows x (dim + 3) floats per tile and split."""
    import torch
    rows = most * q_heads // c.dev.heads
    tiles = (rows + 15) // 16 * c.dev.heads * len(c.length)
    return mpq.kv_attention_tree_workspace_bytes(c.dev, b, getattr(torch, dtype), q_heads) / (tiles * 16 * (c.dev.dim + 3) * 4)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,group,dim,new,length", [(1, 2, 64, 5, 9100), (2, 4, 64, 5, 9100), (1, 3, 256, 5, 9100), (2, 1, 64, 40, 12100),
                                                        (1, 1, 128, 150, 12100), (1, 1, 64, 150, 12100), (1, 2, 256, 30, 12100)])
def test_many_splits(dtype, heads, group, dim, new, length):
    """One long sequence in more than 16 pieces, in every kernel: one and two tiles of 16 rows, pieces of 64 and of 128."""
    r = rng(dim + new)
    c, b = drafted(r, [length], [new], heads, dim, 64, 8, dtype)
    b = mpq.KvBatch(b.starts, b.kv_len, b.table, new, new, length)
    assert splits_of(c, b, dtype, heads * group, new) > 16
    seen, tree = bits_of([parents(r, new)])
    q = dev(r.standard_normal((new, heads * group, dim)), dtype)
    check(c, full(mpq.kv_attention_tree(c.dev, b, q, tree)), full(q), seen, dim ** -0.5, dtype)


@pytest.mark.parametrize("dtype,page,heads,group,dim,new", [("bfloat16", 64, 8, 2, 64, 5), ("float32", 16, 2, 1, 16, 20), ("float16", 32, 4, 2, 64, 14),
                                                            ("bfloat16", 64, 2, 3, 128, 10), ("float32", 128, 4, 1, 128, 4), ("bfloat16", 16, 2, 2, 144, 9)])
def test_few_rows_of_many_lengths(dtype, page, heads, group, dim, new):
    """The bounds that a serving program knows: the most rows of a sequence, and the longest."""
    r = rng(18)
    length = [5000, 200, 2600, 4999, 151, 3, 700, 64]
    rows = [min(new, n) for n in length]
    rows[6] = 0
    c, b = drafted(r, length, rows, heads, dim, page, 8, dtype)
    b = mpq.KvBatch(b.starts, b.kv_len, b.table, b.rows, max(rows), max(length))
    assert new * group <= 32 and splits_of(c, b, dtype, heads * group, max(rows)) >= 1
    seen, tree = bits_of([parents(r, n) for n in rows], 1)
    q = dev(r.standard_normal((b.rows, heads * group, dim)), dtype)
    check(c, full(mpq.kv_attention_tree(c.dev, b, q, tree)), full(q), seen, dim ** -0.5, dtype)


def test_graphs_streams_and_workspace():
    """Two captured graphs, each with scratch of its own, replayed in turn while lengths and bits change."""
    import torch
    r = rng(10)
    heads, group, dim, page = 2, 4, 128, 64
    lengths, new = [3000, 2500], [5, 9]
    c, b = drafted(r, lengths, new, heads, dim, page, 8, "bfloat16")
    seen, tree = bits_of([parents(r, n) for n in new])
    q = dev(r.standard_normal((b.rows, heads * group, dim)), "bfloat16")
    assert mpq.kv_attention_tree_workspace_bytes(c.dev, b, q.dtype, heads * group) > 0
    ws = mpq.Workspace()
    want = mpq.kv_attention_tree(c.dev, b, q, tree)
    assert torch.equal(mpq.kv_attention_tree(c.dev, b, q, tree, ws=ws), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = mpq.kv_attention_tree(c.dev, b, q, tree)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = mpq.kv_attention_tree(c.dev, b, q, tree)
        graphs.append((g, out))
    for i in range(4):
        q.copy_(dev(r.standard_normal(q.shape), "bfloat16"))
        tree.copy_(bits_of([parents(r, n) for n in new])[1])
        b.kv_len.copy_(dev([3000 - 7 * i, 2500 - i], "int32"))
        g, out = graphs[i % 2]
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, mpq.kv_attention_tree(c.dev, b, q, tree))


def test_refusals_of_the_binding():
    import torch
    r = rng(11)
    c, b = drafted(r, [20, 30], [2, 3], 2, 64, 16, 8, "float32")
    q = dev(r.standard_normal((5, 4, 64)))
    _, tree = bits_of([parents(r, 2), parents(r, 3)])
    for bad_q, bad_tree in ((q[:4], tree), (q[:, :, :32], tree), (q.double(), tree), (q, tree[:4]), (q, tree.int()), (q, tree[:, 0]),
                            (q, tree.cpu()), (q.cpu(), tree), (q, tree.repeat(1, 2)[:, ::2])):
        with pytest.raises(ValueError):
            mpq.kv_attention_tree(c.dev, b, bad_q, bad_tree)
    with pytest.raises(ValueError):
        mpq.kv_attention_tree(c.dev, b, q, tree, out=torch.empty((5, 4, 64), dtype=torch.half, device="cuda"))
    with pytest.raises(mpq.MpqError):
        mpq.kv_attention_tree(c.dev, b, q[:, :3], tree)
    with pytest.raises(mpq.MpqError):
        mpq.kv_attention_tree(c.dev, b, q, tree[:, :0])
