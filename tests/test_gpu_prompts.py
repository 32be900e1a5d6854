"""Attention of prompts over the cache of quantized pages: calls of enough rows that a kernel of their own takes them, in pieces
of 64 rows of a key head, of 128, and split along the tokens.  Bounds: check_attention's."""
import numpy as np
import pytest

from test_gpu_kv import DTYPES, NAN, check_attention, filled, tables, tokens, Pair
from test_gpu_parity import mpq
from test_gpu_tokens import dev, full, rng

pytestmark = pytest.mark.gpu

NEW = [128, 1, 0, 77, 126, 65, 3, 100]
HELD = [0, 13, 40, 64, 2, 15, 129, 1]


def queries(r, rows, heads, dim, dtype, size=2.0):
    return dev(r.standard_normal((rows, heads, dim)) * size, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim,page,causal,window", [
    (16, 16, True, 0), (64, 32, False, 0), (64, 128, True, 0), (80, 64, True, 37), (128, 128, True, 0), (128, 16, False, 0),
    (144, 32, True, 70), (256, 64, True, 0), (256, 16, False, 0)])
def test_ragged_prompts(dtype, dim, page, causal, window):
    """Eight sequences, one without a row: 32 pairs of sequence and key head, 64-row pieces (128 for dim > 128)."""
    r = rng(dim + page + window)
    lengths = [a + b for a, b in zip(NEW, HELD)]
    c, table = filled(r, 8, lengths, 4, dim, page, 8, dtype)
    b = c.batch(NEW, lengths, table, max(NEW), max(lengths), behind=2)
    q = queries(r, b.rows, 8, dim, dtype)
    out = dev(np.full((b.rows, 8, dim), 9.0), dtype)
    mpq.kv_attention(c.dev, b, q, causal=causal, window=window, out=out)
    got = full(out)
    assert (got[-2:] == 9.0).all()     # rows behind the last sequence
    check_attention(c, got[:-2], full(q)[:-2], causal, window, dim ** -0.5, dtype)


@pytest.mark.parametrize("dtype,dim,page", [("bfloat16", 64, 32), ("bfloat16", 128, 64), ("float16", 128, 16), ("float32", 64, 64),
                                            ("float32", 128, 128), ("float16", 64, 128)])
def test_many_pairs(dtype, dim, page):
    """264 pairs of 129 rows: pieces of 128 rows and one more."""
    r = rng(dim)
    new, held = [43] * 8, [5, 0, 60, 21, 64, 1, 30, 9]
    lengths = [a + b for a, b in zip(new, held)]
    c, table = filled(r, 8, lengths, 33, dim, page, 8, dtype)
    b = c.batch(new, lengths, table, 43, max(lengths))
    q = queries(r, b.rows, 99, dim, dtype)
    check_attention(c, full(mpq.kv_attention(c.dev, b, q, softmax_scale=-0.4 * dim ** -0.5)), full(q), True, 0, -0.4 * dim ** -0.5, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim,page,window", [(64, 64, 0), (128, 32, 900), (128, 128, 0), (256, 64, 0)])
def test_prompts_split_along_the_tokens(dtype, dim, page, window):
    import torch
    r = rng(dim + window)
    new, held = [64, 64, 1, 30, 64, 50, 64, 20], [1500, 1499, 1000, 3, 0, 800, 1409, 700]
    lengths = [a + b for a, b in zip(new, held)]
    c, table = filled(r, 8, lengths, 4, dim, page, 8, dtype)
    b = c.batch(new, lengths, table, 64, max(lengths))
    assert mpq.kv_attention_workspace_bytes(c.dev, b, getattr(torch, dtype), 8) > 0
    q = queries(r, b.rows, 8, dim, dtype)
    check_attention(c, full(mpq.kv_attention(c.dev, b, q, window=window)), full(q), True, window, dim ** -0.5, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", (16, 64))
def test_pages_that_do_not_exist(dtype, page):
    """The first page of one sequence, one in the middle, all of another's: their tokens are absent, rows that see nothing else
    give 0.  More rows than tokens: the first ones see nothing."""
    r = rng(page)
    new = [128] * 8
    lengths = [128, 200, 300, 100, 128, 140, 128, 1]
    c, table = filled(r, 8, lengths, 4, 64, page, 8, dtype)
    table = table.copy()
    table[0, 0], table[1, 128 // page], table[2, :], table[4, 64 // page:] = -1, c.dev.pages, 2 ** 31 - 1, -2 ** 31
    b = c.batch(new, lengths, table, 128, max(lengths))
    q = queries(r, b.rows, 8, 64, dtype)
    got = full(mpq.kv_attention(c.dev, b, q))
    assert not got[:page].any() and not got[256:384].any() and not got[384:384 + 28].any() and not got[-128:-1].any()
    assert got[-1].any() and got[page:128].any(axis=(1, 2)).all()
    check_attention(c, got, full(q), True, 0, 0.125, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", (16, 64))
@pytest.mark.parametrize("bits", (8, 3))
def test_logits_that_grow_and_uneven_pages(dtype, page, bits):
    """Keys whose logits rise along the sequence, so that maxima are passed again and again by little and by much; pages whose
    maxima differ by orders, a page of zeros; a row of zeros; logits up to hundreds."""
    r = rng(bits + page)
    n, heads, dim, seqs = 256, 8, 64, 8
    pages, table = tables(r, seqs, n // page)
    c = Pair(pages, heads, page, dim, bits)
    b = c.batch([n] * seqs, [n] * seqs, table)
    k, v = tokens(r, seqs * n, heads, dim, dtype, 0.3)
    rise = np.tile(np.linspace(0.05, 4, n), seqs)[:, None, None]
    size = np.exp(r.uniform(-6, 3, (seqs, n // page))).repeat(page, 1)
    size[:, page:2 * page] = 0
    k = (k.double() * dev(rise, "float64")).to(k.dtype)
    v = (v.double() * dev(size.reshape(-1, 1, 1), "float64")).to(v.dtype)
    c.append(b, k, v)
    b = c.batch([32] * seqs, [n] * seqs, table, 32, n)
    q = queries(r, b.rows, heads * 4, dim, dtype) * dev(np.tile([0, 1, 8, 40], 8 * heads).reshape(1, -1, 1)[:, :heads * 4], dtype)
    for causal in (True, False):
        check_attention(c, full(mpq.kv_attention(c.dev, b, q, causal=causal)), full(q), causal, 0, 0.125, dtype)


def test_prompts_from_a_replayed_graph_on_another_stream_and_twice():
    """The same call eagerly, on another stream and from a graph, whose replays follow other work and new queries: the same bits.
    Two graphs of calls with workspaces, replayed at once."""
    import torch
    mpq.init()
    r = rng(5)
    new, lengths = [64] * 8, [1564] * 8
    c, table = filled(r, 8, lengths, 4, 64, 64, 8, "bfloat16")
    b = c.batch(new, lengths, table, 64, 1564)
    q = queries(r, b.rows, 8, 64, "bfloat16")
    want = mpq.kv_attention(c.dev, b, q)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs, graphs = [], []
    for s in streams:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(mpq.kv_attention(c.dev, b, q))
        graphs.append(g)
    for _ in range(3):
        q.copy_(queries(r, b.rows, 8, 64, "bfloat16"))
        want = mpq.kv_attention(c.dev, b, q)
        torch.cuda.synchronize()
        for s, g, o in zip(streams, graphs, outs):
            o.zero_()
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        with torch.cuda.stream(streams[0]):
            other = mpq.kv_attention(c.dev, b, q)
        torch.cuda.synchronize()
        assert torch.equal(other, want) and torch.equal(outs[0], want) and torch.equal(outs[1], want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new,held", [(1, 90), (1, 5000), (128, 20), (64, 1600)])
def test_a_row_with_nan_or_inf_spoils_itself_alone(dtype, new, held):
    """Single tokens and prompts, split and not."""
    import torch
    r = rng(new + held)
    lengths = [new + held] * 8
    c, table = filled(r, 8, lengths, 4, 64, 64, 8, dtype)
    b = c.batch([new] * 8, lengths, table, new, new + held)
    q = queries(r, b.rows, 8, 64, dtype)
    clean = mpq.kv_attention(c.dev, b, q)
    spoilt = q.clone()
    spoilt[3, 2, 5], spoilt[b.rows - 1, 7, :], spoilt[0, 0, 63] = NAN, NAN, float("inf")
    got = mpq.kv_attention(c.dev, b, spoilt)
    bad = torch.zeros(b.rows, 8, dtype=torch.bool, device="cuda")
    bad[3, 2] = bad[b.rows - 1, 7] = bad[0, 0] = True
    assert got[bad].isnan().all() and torch.equal(got[~bad], clean[~bad])


def test_more_rows_than_the_call_was_told_of_stay_inside():
    """Device arrays that name more rows of a sequence than max_new: a part is processed, and nothing is written outside the
    workspace or to rows that were not."""
    import ctypes
    import torch
    r = rng(77)
    new, lengths, group = 128, [1628] * 8, 2
    c, table = filled(r, 8, lengths, 4, 64, 64, 8, "bfloat16")
    b = c.batch([new] * 8, lengths, table, 65, 1628)
    q = queries(r, b.rows, 4 * group, 64, "bfloat16")
    size = mpq.kv_attention_workspace_bytes(c.dev, b, torch.bfloat16, 4 * group)
    assert size > 0
    ws = torch.full((size + (1 << 20),), 85, dtype=torch.uint8, device="cuda")
    out = torch.full_like(q, 9.0)
    rc = mpq.lib().mpq_kv_attention(c.dev.ref, b.ref, mpq.BF16, q.data_ptr(), 512, 64, 8, 0.125, 1, 0, out.data_ptr(), 512, 64,
                                    ws.data_ptr(), size, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    assert rc == 0 and (ws[size:] == 85).all()
    got = out.view(8, new, 8, 64)
    assert (got[:, 72:] == 9.0).all()      # (65 rows of two heads end in the ninth tile of 16)
    whole = c.batch([new] * 8, lengths, table, new, 1628)
    got[:, 65:] = mpq.kv_attention(c.dev, whole, q).view(8, new, 8, 64)[:, 65:]
    check_attention(c, full(out), full(q), True, 0, 0.125, "bfloat16")


@pytest.mark.parametrize("most", (149, 146))
def test_rows_behind_a_low_bound_are_nobodys(most):
    """Rows behind max_new of a split prompt: left as they were or what the full call gives, whatever the scratch held."""
    import torch
    r = rng(78)
    new, length, group = 150, 16000, 2
    c = mpq.KvCache.empty(length // 64 + 1, 2, 64, 64)
    g = torch.Generator(device="cuda").manual_seed(3)
    for t in (c.k_codes, c.v_codes):
        t.copy_(torch.randint(-127, 128, t.shape, dtype=torch.int8, device="cuda", generator=g))
    c.k_absmax.fill_(0.3)
    c.v_absmax.fill_(1.0)
    arrays = dev([0, new], "int32"), dev([length], "int32"), dev(np.arange(251)[None], "int32")
    q = queries(r, new, 2 * group, 64, "bfloat16")
    want = mpq.kv_attention(c, mpq.KvBatch(*arrays, new, new, length), q)
    low = mpq.KvBatch(*arrays, new, most, length)
    need = mpq.kv_attention_workspace_bytes(c, low, torch.bfloat16, 2 * group)
    assert need > 0
    ws = mpq.Workspace()
    ws.get(need)
    ws.buf.fill_(255)
    out = torch.full_like(q, 9.0)
    mpq.kv_attention(c, low, q, out=out, ws=ws)
    left = (full(out) == 9).all((1, 2))
    assert not left[:most].any()
    # (both are off by 2 V (2^-12 + n / 4 2^-24 + ...) < 2^-9 V and a rounding of 2^-8 of themselves, V = 1)
    got, want = full(out)[~left], full(want)[~left]
    assert (np.abs(got - want) <= 2.0 ** -8 + 2.0 ** -7 * np.abs(want)).all()


def test_offsets_past_32_bits_of_a_prompt():
    """Pages behind the first 4 GiB of codes."""
    import torch
    heads, dim, page = 4, 256, 128
    pages = 2 ** 32 // (heads * dim * page) + 100
    r = rng(8)
    small = Pair(12, heads, page, dim, 8)
    table = r.permutation(12)[:8].reshape(8, 1).astype(np.int32)
    lengths = [128, 100, 65, 1, 64, 127, 33, 90]
    b = small.batch(lengths, lengths, table)
    k, v = tokens(r, b.rows, heads, dim, "bfloat16")
    small.append(b, k, v)
    c = mpq.KvCache.empty(pages, heads, page, dim, 8)
    far = mpq.KvBatch(b.starts, b.kv_len, dev(table + pages - 12, "int32"), b.rows, 128, 128)
    mpq.kv_append(c, far, k, v)
    q = queries(r, b.rows, 8, dim, "bfloat16")
    near = mpq.KvBatch(b.starts, b.kv_len, dev(table, "int32"), b.rows, 128, 128)
    assert torch.equal(mpq.kv_attention(c, far, q), mpq.kv_attention(small.dev, near, q))
    for a, z in zip(mpq.kv_gather(c, far, torch.bfloat16), mpq.kv_gather(small.dev, near, torch.bfloat16)):
        assert torch.equal(a, z)
    check_attention(small, full(mpq.kv_attention(c, far, q)), full(q), True, 0, 1 / 16, "bfloat16")
