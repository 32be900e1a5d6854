"""The self-attention layer served from quantized weights and cache: the calls together, as a generating model runs them."""
import numpy as np
import pytest

import oracle
from oracle import search as osearch
from oracle import serving
from paper_2302_01382_amd.attention import QuantAttention
from test_gpu_kv import DTYPES, Pair, check_attention
from test_gpu_parity import host, mpq
from test_gpu_tokens import dev, full, rng, rounded

pytestmark = pytest.mark.gpu

LENGTHS = [70, 3, 1, 150, 34]


def layer(dtype, q_heads, kv_heads, dim, K, N, widths=(8, 4, 2), single_tokens=3, lengths=LENGTHS, page=16, seed=0):
    r = rng(seed)
    w_qkv = r.standard_normal(((q_heads + 2 * kv_heads) * dim, K), dtype=np.float32) / np.float32(np.sqrt(K) / 2)
    w_out = r.standard_normal((N, q_heads * dim), dtype=np.float32)
    x = dev(r.standard_normal((sum(lengths), K)), dtype)
    att = QuantAttention(x, lengths, dev(w_qkv), dev(w_out), kv_heads, dim, widths, single_tokens, page=page)
    return att, w_qkv, w_out


def plain_linear(x, w, w_bits, a_bits):
    """The quantized layer with the oracle's functions; exact up to the output's type."""
    a_q, a_scale = serving.token_quant(x, a_bits)
    absmax = oracle.absmax(w, oracle.PER_ROW)
    _, codes, _ = oracle.fake_quant(w, absmax, w_bits, oracle.PER_ROW)
    return serving.qgemm_tokens(a_q, codes, a_scale, oracle.scale_from_absmax(absmax, w_bits))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("q_heads,kv_heads,dim,K,N,bits", [(8, 2, 64, 96, 80, (8, 4, 8)), (3, 3, 80, 250, 33, (4, 8, 4)),
                                                           (4, 4, 16, 64, 64, (2, 2, 2))])
def test_every_call_of_a_run(dtype, q_heads, kv_heads, dim, K, N, bits):
    """Prompts and single tokens of five sequences, call by call, each call against the oracle on what the one before it left:
    linear layers and cache bit for bit, attention within its bound; run() gives the same outputs."""
    att, w_qkv, w_out = layer(dtype, q_heads, kv_heads, dim, K, N, seed=K)
    c = Pair(att.pages, kv_heads, att.page, dim, bits[2])
    whole = np.zeros((sum(LENGTHS), N), np.float32)
    seen = 0
    for rows, batch in att.calls:
        x = att.x[rows]
        wq, sq, store = att.w_qkv[bits[0]]
        qkv = mpq.linear_tokens(x, wq, sq, store)
        np.testing.assert_array_equal(full(qkv), rounded(plain_linear(full(x), w_qkv, bits[0], 8), dtype))
        qkv = qkv.view(len(rows), -1, dim)
        q, k, v = qkv[:, :q_heads], qkv[:, q_heads:q_heads + kv_heads], qkv[:, q_heads + kv_heads:]
        c.starts, c.length, c.table = host(batch.starts), host(batch.kv_len), host(batch.table)
        c.append(batch, k, v)
        c.check_codes()
        o = mpq.kv_attention(c.dev, batch, q)
        check_attention(c, full(o), full(q), True, 0, dim ** -0.5, dtype)
        wo, so, store = att.w_out[bits[1]]
        y = mpq.linear_tokens(o.view(len(rows), -1), wo, so, store)
        np.testing.assert_array_equal(full(y), rounded(plain_linear(full(o).reshape(len(rows), -1), w_out, bits[1], 8), dtype))
        whole[host(rows)] = full(y)
        seen += len(rows)
    assert seen == sum(LENGTHS)      # every token came once
    np.testing.assert_array_equal(full(att.run(bits)), whole)
    # the score: sums of squares in 64 bits against the same outputs
    want = 1.0 - ((whole.astype(np.float64) - host(att.y_ref)) ** 2).sum() / (host(att.y_ref).astype(np.float64) ** 2).sum()
    assert att.evaluate(bits) == pytest.approx(want, abs=1e-6 * (1 + abs(1 - want)))


def test_one_by_one_or_all_at_once():
    """Prompts alone, and every token by itself: a run covers all tokens either way, and a sequence of one token, whose page's
    maximum is its own in both, gives the same bits."""
    att, _, _ = layer("float32", 2, 1, 64, 64, 64, single_tokens=0)
    single, _, _ = layer("float32", 2, 1, 64, 64, 64, single_tokens=max(LENGTHS))
    assert len(att.calls) == 1 and len(single.calls) == max(LENGTHS)
    assert [b.max_new for _, b in single.calls] == [1] * max(LENGTHS)
    one, other = full(att.run([8, 8, 8])), full(single.run([8, 8, 8]))
    assert np.isfinite(one).all() and np.isfinite(other).all()
    at = LENGTHS.index(1)
    np.testing.assert_array_equal(one[sum(LENGTHS[:at])], other[sum(LENGTHS[:at])])


def test_searches_over_weights_and_cache():
    """Both searches, driven by the library and by the oracle's code, over the same scores."""
    att, _, _ = layer("bfloat16", 4, 2, 32, 64, 48, seed=4)
    top = att.evaluate_once([8, 8, 8])
    lost = att.sensitivity(4)
    assert lost == [top - att.evaluate([4, 8, 8]), top - att.evaluate([8, 4, 8]), top - att.evaluate([8, 8, 4])]
    order = att.order_by(lost)
    assert sorted(order) == [0, 1, 2] and sorted(lost) == [lost[i] for i in order]
    for share in (0.999, 0.97, 0.8):
        target = share * top
        bits, asked = att.greedy(order, target)
        assert (bits, asked) == osearch.greedy(order, [8, 4, 2], target, att.evaluate_once)
        bits, asked = att.bisection(order, target)
        assert (bits, asked) == osearch.bisection(order, [8, 4, 2], target, att.evaluate_once, True)
        assert att.evaluate_once(bits) >= target or bits == [8, 8, 8]


def test_a_generating_loop_from_one_graph():
    """A token of each sequence per replay: one captured step, whose lengths and inputs the program rewrites, against the steps
    called one by one."""
    import torch
    mpq.init()
    att, _, _ = layer("bfloat16", 8, 2, 64, 96, 80, single_tokens=8, lengths=[40, 9, 8, 100], seed=7)
    bits = [8, 4, 8]
    want = att.run(bits)
    cache = mpq.KvCache.empty(att.pages, 2, att.page, 64, 8)
    y = torch.zeros_like(want)
    (rows, prompts), steps = att.calls[0], att.calls[1:]
    y[rows] = att.step(att.x[rows], prompts, cache, bits)
    first = steps[0][1]
    lengths = first.kv_len.clone()
    batch = mpq.KvBatch(first.starts, lengths, first.table, 4, 1, 100)
    x = torch.zeros_like(att.x[:4])
    kept = [t.clone() for t in (cache.k_codes, cache.v_codes, cache.k_absmax, cache.v_absmax)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = att.step(x, batch, cache, bits)
    for t, o in zip((cache.k_codes, cache.v_codes, cache.k_absmax, cache.v_absmax), kept):
        t.copy_(o)
    for rows, b in steps:
        assert len(rows) == 4
        x.copy_(att.x[rows])
        lengths.copy_(b.kv_len)
        g.replay()
        y[rows] = out
    torch.cuda.synchronize()
    assert torch.equal(y, want)


def test_refusals():
    import torch
    w = torch.randn(96, 32, device="cuda")
    x = torch.randn(10, 32, device="cuda")
    for x_, lengths, w_qkv, w_out in ((x, [4, 5], w, w[:, :32]), (x, [10], w, w[:, :24]), (x, [10], w[:80], w[:, :32]),
                                      (x[:, :16], [10], w, w[:, :32])):
        with pytest.raises(ValueError):
            QuantAttention(x_, lengths, w_qkv, w_out, 2, 16, [8])
