"""Norm and rotation of heads against a plain reference in 64 bits."""
import numpy as np
import pytest

from oracle import drafts
from test_gpu_parity import host, mpq
from test_gpu_tokens import dev, full, rng

pytestmark = pytest.mark.gpu

DTYPES = ("float32", "bfloat16", "float16")
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
U = 2.0 ** -24
LAYOUTS = (0, 1)   # halves, neighbouring pairs


def frequencies(pairs, base=10000.0):
    return (base ** (-np.arange(pairs) / max(pairs, 1))).astype(np.float32)


def check(got, x, positions, freq, weight, eps, layout, dtype):
    """y is off by the norm's dim / 8 + 8 roundings of sums (a square root halves them), those of the mean, its root and two products: at most
    dim / 16 + 12 units of |y|; cosine and sine by 4 units, the angle by the rounding of half a turn at most to 2^-25, 2 pi 2^-26 < 2
    units, and of the product in 64 bits, 2^-51 of 2^31 / 2 pi turns at most, < 16 units of a turn's 2 pi; a product and a fused sum
    are two more: together below dim / 16 + 36 units of |a| + |b|.  Then half a step of the type (fp16: at least 2^-25)."""
    want, size = drafts.rotate_heads(x, positions, freq, weight, eps, bool(layout))
    off = (x.shape[2] / 16 + 36) * U * size
    bound = off + HALF[dtype] * (np.abs(want) + off) + (2.0 ** -25 if dtype == "float16" else 2.0 ** -149)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (np.argwhere(bad)[:5], np.abs(got - want).max(), bound.min())


def heads(r, rows, n, dim, dtype):
    return dev(r.standard_normal((rows, n, dim)) * np.exp(r.standard_normal((1, n, 1))), dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("rows,q_heads,k_heads,dim,pairs", [(1, 1, 1, 16, 8), (1, 16, 16, 64, 32), (3, 5, 2, 80, 40), (7, 32, 8, 128, 64),
                                                           (2, 3, 1, 96, 24), (5, 4, 4, 256, 128), (300, 7, 1, 48, 4), (9, 2, 2, 32, 0),
                                                           (700, 12, 12, 64, 16), (3000, 1, 1, 144, 72)])
def test_rotate(dtype, layout, rows, q_heads, k_heads, dim, pairs):
    r = rng(rows + dim + pairs)
    q, k = heads(r, rows, q_heads, dim, dtype), heads(r, rows, k_heads, dim, dtype)
    pos = r.integers(0, 5000, rows).astype(np.int32)
    f = frequencies(pairs)
    qw, kw = ((1 + 0.3 * r.standard_normal(dim)).astype(np.float32) for _ in range(2))
    qo, ko = mpq.rotate_heads(q, k, dev(pos, "int32"), dev(f), dev(qw), dev(kw), 1e-5, layout)
    assert qo.dtype == q.dtype and qo.is_contiguous() and ko.is_contiguous()
    check(full(qo), full(q), pos, f, qw, 1e-5, layout, dtype)
    check(full(ko), full(k), pos, f, kw, 1e-5, layout, dtype)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_far_and_negative_positions(layout):
    """The last positions that 32 bits have, where an angle in fp32 would be off by a hundred radians."""
    r = rng(4)
    pos = np.array([0, 1, -1, 1000003, -999999, 2 ** 31 - 1, -2 ** 31, 123456789], np.int32)
    x = heads(r, len(pos), 3, 64, "float32")
    f = frequencies(32)
    out, none = mpq.rotate_heads(x, None, dev(pos, "int32"), dev(f), layout=layout)
    assert none is None
    check(host(out), host(x), pos, f, None, 1e-6, layout, "float32")
    np.testing.assert_array_equal(host(out)[0], host(x)[0])      # position 0 turns nothing, no weight scales nothing
    _, back = mpq.rotate_heads(None, out, dev(np.where(pos == -2 ** 31, 0, -pos).astype(np.int32), "int32"), dev(f), layout=layout)
    keep = pos != -2 ** 31
    assert np.abs(host(back) - host(x))[keep].max() < 120 * U * np.abs(host(x)).max()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
def test_views_in_place(dtype, layout):
    """Queries and keys inside the layer's output, turned where they lie; the values beside them stay."""
    import torch
    r = rng(5)
    rows, qh, kh, dim = 41, 6, 2, 96
    qkv = heads(r, rows, qh + 2 * kh, dim, dtype)
    was = qkv.clone()
    pos, f = r.integers(0, 100000, rows).astype(np.int32), frequencies(48)
    w = (1 + 0.1 * r.standard_normal(dim)).astype(np.float32)
    q, k = qkv[:, :qh], qkv[:, qh:qh + kh]
    qo, ko = mpq.rotate_heads(q, k, dev(pos, "int32"), dev(f), dev(w), None, layout=layout, q_out=q, k_out=k)
    assert qo is q and ko is k
    check(full(q), full(was[:, :qh]), pos, f, w, 1e-6, layout, dtype)
    check(full(k), full(was[:, qh:qh + kh]), pos, f, None, 1e-6, layout, dtype)
    assert torch.equal(qkv[:, qh + kh:], was[:, qh + kh:])
    # heads before rows, at an odd element, into a wider output
    t = getattr(torch, dtype)
    x = torch.empty(qh * rows * dim + 1, dtype=t, device="cuda")[1:].view(qh, rows, dim).transpose(0, 1)
    x.copy_(was[:, :qh])
    out = torch.full((rows, qh, dim + 5), 3.0, dtype=t, device="cuda")
    mpq.rotate_heads(x, None, dev(pos, "int32"), dev(f), dev(w), layout=layout, q_out=out[:, :, 2:2 + dim])
    assert torch.equal(out[:, :, 2:2 + dim], q) and (out[:, :, :2] == 3).all() and (out[:, :, 2 + dim:] == 3).all()


def test_norm_alone_and_ends_of_the_range():
    r = rng(6)
    x = heads(r, 5, 3, 64, "float32")
    w = np.ones(64, np.float32)
    x[1, 1] = 0
    x[2] *= 1e16
    x[3] *= 1e-18
    out, _ = mpq.rotate_heads(x, None, None, None, dev(w), eps=1e-6)
    check(host(out), host(x), np.zeros(5, np.int32), frequencies(0), w, 1e-6, 0, "float32")
    assert not host(out)[1, 1].any()
    x[2, 0, 5] = 1e30      # its square passes the range: that head alone is no number
    x[4, 2, 0] = float("nan")
    y = host(mpq.rotate_heads(x, None, None, None, dev(w))[0])
    bad = np.zeros((5, 3), bool)
    bad[2, 0] = bad[4, 2] = True
    np.testing.assert_array_equal(np.isnan(y).all(2), bad)
    np.testing.assert_array_equal(np.isnan(y).any(2), bad)


def test_offsets_past_32_bits():
    """Rows, and heads, that lie more than 2^32 bytes apart."""
    import torch
    r = rng(30)
    q, k = heads(r, 34, 2, 64, "bfloat16"), heads(r, 34, 3, 64, "bfloat16")
    far = torch.empty(34 << 26, dtype=torch.bfloat16, device="cuda")
    wide = far.as_strided((34, 2, 64), (1 << 26, 100, 1))
    wide.copy_(q)
    tall = torch.empty(5 << 30, dtype=torch.bfloat16, device="cuda").as_strided((34, 3, 64), (64, 1 << 31, 1))
    tall.copy_(k)
    pos, f = dev(r.integers(0, 5000, 34), "int32"), dev(frequencies(32))
    want = mpq.rotate_heads(q, k, pos, f)
    for got, w in zip(mpq.rotate_heads(wide, tall, pos, f, q_out=wide, k_out=tall), want):
        assert torch.equal(got, w)


def test_nothing_is_looked_at_of_no_heads():
    """In C: a weight, strides and pointers of the one that has no heads."""
    import ctypes as C
    import torch
    r = rng(31)
    x = heads(r, 9, 4, 64, "float32")
    pos, f, out = dev(r.integers(0, 5000, 9), "int32"), dev(frequencies(32)), torch.empty_like(x)
    odd = C.c_void_p(x.data_ptr() + 1)
    want = mpq.rotate_heads(x, None, pos, f)[0]
    for q, k in (((x.data_ptr(), 256, 64, 4), (odd, -1, -1, 0)), ((odd, -1, -1, 0), (x.data_ptr(), 256, 64, 4))):
        out.zero_()
        weights = (None, odd) if q[3] else (odd, None)
        outs = [(out.data_ptr(), 256, 64) if n[3] else (odd, -1, -1) for n in (q, k)]
        rc = mpq.lib().mpq_rotate_heads(0, 9, 64, *q, *k, pos.data_ptr(), f.data_ptr(), 32, 0, *weights, 1e-6, *outs[0], *outs[1],
                                        C.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert rc == mpq.OK and torch.equal(out, want)


def test_outputs_in_one_place_are_refused():
    """Both outputs, or an output and the other's input; heads in turn in one buffer are neither."""
    import torch
    r = rng(32)
    q, k = heads(r, 6, 4, 64, "bfloat16"), heads(r, 6, 4, 64, "bfloat16")
    pos, f = dev(r.integers(0, 900, 6), "int32"), dev(frequencies(32))
    want = mpq.rotate_heads(q, k, pos, f)
    out = torch.zeros((6, 8, 64), dtype=q.dtype, device="cuda")
    for qo, ko in ((out[:, :4], out[:, :4]), (out[:, :4], out[:, 3:7]), (k, None), (None, q), (q, q)):
        with pytest.raises(mpq.MpqError):
            mpq.rotate_heads(q, k, pos, f, q_out=qo, k_out=ko)
    for qo, ko in ((out[:, ::2], out[:, 1::2]), (out[:, 4:], out[:, :4]), (out.view(12, 4, 64)[:6], out.view(12, 4, 64)[6:]),
                   (out.view(8, 6, 64)[:4].transpose(0, 1), out.view(8, 6, 64)[4:].transpose(0, 1))):
        out.zero_()
        mpq.rotate_heads(q, k, pos, f, q_out=qo, k_out=ko)
        assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])


def test_refusals_of_the_binding():
    import torch
    r = rng(7)
    q, k = heads(r, 4, 3, 64, "float32"), heads(r, 4, 1, 64, "float32")
    pos, f, w = dev(np.arange(4), "int32"), dev(frequencies(32)), dev(np.ones(64))
    for bad in ((None, None, pos, f), (q[0], k, pos, f), (q, k[:3], pos, f), (q, k[:, :, :32], pos, f), (q, k.half(), pos, f),
                (q, k, pos[:3], f), (q, k, pos.long(), f), (q, k, pos, f.double()), (q, k, pos, f, w[:32]), (q, k, pos, f, w, w.half()),
                (q.transpose(1, 2), k, pos, f), (q, k.cpu(), pos, f), (q, None, pos, f, w, w)):
        with pytest.raises(ValueError):
            mpq.rotate_heads(*bad)
    with pytest.raises(ValueError):
        mpq.rotate_heads(q, k, pos, f, q_out=torch.empty_like(k))
    with pytest.raises(ValueError):
        mpq.rotate_heads(q, k, None, f)
    with pytest.raises(mpq.MpqError):
        mpq.rotate_heads(q, k, pos, dev(frequencies(30)))
    with pytest.raises(mpq.MpqError):
        mpq.rotate_heads(q, k, pos, f, eps=0.0)
    with pytest.raises(mpq.MpqError):
        mpq.rotate_heads(q, k, pos, f, q_out=q[:, :1].expand(4, 3, 64))
    empty, _ = mpq.rotate_heads(q[:0], k[:0], pos[:0], f)
    assert empty.shape == (0, 3, 64)


def test_graphs_and_streams():
    import torch
    r = rng(8)
    q, k = heads(r, 20, 8, 128, "bfloat16"), heads(r, 20, 2, 128, "bfloat16")
    pos, f, w = dev(r.integers(0, 9000, 20), "int32"), dev(frequencies(64)), dev(np.ones(128))
    want = [t.clone() for t in mpq.rotate_heads(q, k, pos, f, w, w)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = mpq.rotate_heads(q, k, pos, f, w, w)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = mpq.rotate_heads(q, k, pos, f, w, w)
    for i in range(3):
        pos.copy_(dev(r.integers(0, 9000, 20), "int32"))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, mpq.rotate_heads(q, k, pos, f, w, w)))
