"""The quantizer and the linear layer with a step per token, against plain references."""
import numpy as np
import pytest

from oracle import serving
from test_gpu_parity import host, mpq

pytestmark = pytest.mark.gpu

DTYPES = ("float32", "bfloat16", "float16")


def dev(a, dtype="float32"):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(getattr(torch, dtype))


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def full(t):
    """A 16-bit tensor's values as float32 on the host."""
    return host(t.float())


def weights(r, N, K, w_bits):
    """(codes int8 [N, K], the layer's tensor, steps)"""
    q = 2 ** (w_bits - 1) - 1
    codes = r.integers(-q, q + 1, (N, K)).astype(np.int8)
    held = codes
    if w_bits == 4:
        u = codes.astype(np.uint8) & 15
        held = (u[:, ::2] | u[:, 1::2] << 4).astype(np.uint8)
    import torch
    return codes, torch.from_numpy(held).cuda(), (r.random(N, dtype=np.float32) + 0.5) * 0.01


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K", [(1, 1), (1, 7), (3, 8), (5, 65), (2, 1023), (17, 4096), (700, 64), (513, 4096), (1, 20001),
                                 (515, 4097), (600, 1000), (2, 16392)])
def test_token_quant(M, K, dtype):
    r = rng(M * 7919 + K)
    x = dev(np.clip(r.standard_normal((M, K)) * np.exp(r.standard_normal((M, 1)) * 3), -6e4, 6e4), dtype)
    x[M // 2] = 0
    for bits in (8, 5, 2):
        codes, scale = mpq.token_quant(x, bits)
        want, step = serving.token_quant(full(x), bits)
        np.testing.assert_array_equal(host(codes), want)
        np.testing.assert_array_equal(host(scale), step)


@pytest.mark.parametrize("dtype", DTYPES)
def test_token_quant_of_a_strided_view_at_an_odd_address(dtype):
    r = rng(3)
    for rows, cols, off in ((9, 100, 3), (600, 257, 1)):
        big = dev(r.standard_normal((rows, cols + 40)), dtype)
        x = big[:, off:off + cols]
        codes, scale = mpq.token_quant(x, 8)
        want, step = serving.token_quant(full(x), 8)
        np.testing.assert_array_equal(host(codes), want)
        np.testing.assert_array_equal(host(scale), step)


def test_codes_at_midpoints_and_extremes():
    """Products that lie on a tie or next to the clamp: ties go to the even code."""
    m = np.float32(127.0)
    x = np.concatenate([np.arange(-126.5, 127.5, 0.5), [127.0, -127.0]]).astype(np.float32)[None]
    assert np.abs(x).max() == m
    codes, _ = mpq.token_quant(dev(x), 8)
    np.testing.assert_array_equal(host(codes)[0], np.rint(x[0]).astype(np.int8))
    tiny = dev(np.array([[1e-38, -3e-39, 0, 2e-45]], np.float32))      # subnormal entries and step
    codes, scale = mpq.token_quant(tiny, 8)
    want, step = serving.token_quant(host(tiny), 8)
    np.testing.assert_array_equal(host(codes), want)
    np.testing.assert_array_equal(host(scale), step)


def layer(M, N, K, w_bits, dtype, act, seed, a_view=0):
    import torch
    r = rng(seed)
    a = r.integers(-127, 128, (M, K)).astype(np.int8)
    codes, w, w_scale = weights(r, N, K, w_bits)
    a_scale = (r.random(M, dtype=np.float32) + 0.01) * 0.1
    flat = torch.empty(M * K + a_view, dtype=torch.int8, device="cuda")
    da = flat[a_view:].view(M, K)
    da.copy_(torch.from_numpy(a))
    t = getattr(torch, dtype)
    y = torch.full((M + 2, N), 77.0, dtype=t, device="cuda")
    got = mpq.qgemm_tokens(da, w, dev(a_scale), dev(w_scale), w_bits, mpq.PER_ROW, act, y=y[:M])
    assert got.data_ptr() == y.data_ptr()
    assert torch.all(y[M:] == 77.0)       # rows behind the last one are left alone
    return full(got), serving.qgemm_tokens(a, codes, a_scale, w_scale)


def rounded(want, dtype):
    import torch
    return torch.from_numpy(want).to(getattr(torch, dtype)).float().numpy()


FEW = [(1, 1, 1), (1, 16, 16), (1, 130, 257), (3, 31, 33), (15, 64, 128), (16, 5000, 100), (17, 4100, 1024), (33, 48, 4096),
       (64, 258, 130), (49, 4096, 2050), (64, 33, 14)]
MANY = [(65, 17, 30), (65, 64, 128), (130, 258, 257), (300, 130, 1000), (517, 771, 1001), (130, 66, 14), (129, 128, 1040),
        (1000, 1000, 512), (2000, 258, 2000)]


@pytest.mark.parametrize("M,N,K", FEW + MANY)
@pytest.mark.parametrize("w_bits", (8, 4))
def test_layer_is_exact(M, N, K, w_bits):
    if w_bits == 4 and K % 2:
        K += 1
    for i, dtype in enumerate(DTYPES):
        got, want = layer(M, N, K, w_bits, dtype, mpq.ACT_NONE, M + N + K + i, a_view=i)
        np.testing.assert_array_equal(got, rounded(want, dtype))
        got, want = layer(M, N, K, w_bits, dtype, mpq.ACT_RELU, M * 3 + N + K + i)
        np.testing.assert_array_equal(got, rounded(np.maximum(want, 0), dtype))


# each tile of the fast kernels, whole and ragged, several output tiles per workgroup
@pytest.mark.parametrize("M,N,K", [(3585, 3600, 256), (12288, 768, 128), (12200, 768, 1040), (6272, 256, 160), (1408, 2048, 2048),
                                   (24001, 128, 528), (9000, 64, 64), (20011, 320, 96), (70000, 512, 64)])
@pytest.mark.parametrize("w_bits", (8, 4))
def test_layer_is_exact_in_every_tile(M, N, K, w_bits):
    import torch
    if w_bits == 4:
        K = (K + 31) // 32 * 32
    r = rng(M + N + K)
    g = torch.Generator(device="cuda").manual_seed(M)
    a = torch.randint(-127, 128, (M, K), dtype=torch.int8, device="cuda", generator=g)
    codes, w, w_scale = weights(r, N, K, w_bits)
    a_scale = torch.rand(M, device="cuda", generator=g) + 0.5
    ws = dev(w_scale)
    acc = a.double() @ torch.from_numpy(codes).cuda().double().t().contiguous()
    want = (acc.float() * a_scale[:, None]) * ws
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        y = mpq.qgemm_tokens(a, w, a_scale, ws, w_bits, dtype=dtype)
        assert torch.equal(y, want.to(dtype))
    one = ws[:1].contiguous()
    y = mpq.qgemm_tokens(a, w, a_scale, one, w_bits, mpq.PER_TENSOR, mpq.ACT_RELU)
    assert torch.equal(y, ((acc.float() * a_scale[:, None]) * one).clamp(min=0))


@pytest.mark.parametrize("M,N,K", [(5, 100, 64), (130, 100, 250), (1000, 1024, 256), (4096, 4096, 64)])
def test_gelu(M, N, K):
    """GELU is evaluated within 1e-5 relative of its value, or 4e-7 |Y| where that is larger; a 16-bit output adds half a
    step, eps / 2 of the value (fp16: at least half of its smallest step, 2^-25)."""
    import torch
    for dtype, half, least in (("float32", 2.0 ** -24, 0.0), ("bfloat16", 2.0 ** -8, 0.0), ("float16", 2.0 ** -11, 2.0 ** -25)):
        r = rng(K)
        a = r.integers(-127, 128, (M, K)).astype(np.int8)
        codes, w, w_scale = weights(r, N, K, 8)
        a_scale = (r.random(M, dtype=np.float32) + 0.1) * 0.01
        y = serving.qgemm_tokens(a, codes, a_scale, w_scale).astype(np.float64)
        got = full(mpq.qgemm_tokens(dev(a, "int8"), w, dev(a_scale), dev(w_scale), act=mpq.ACT_GELU, dtype=getattr(torch, dtype)))
        want = (torch.from_numpy(y) * torch.special.ndtr(torch.from_numpy(y))).numpy()
        bound = np.maximum(1e-5 * np.abs(want), 4e-7 * np.abs(y))
        bound = bound + half * (np.abs(want) + bound) + least
        assert np.all(np.abs(got - want) <= bound)


@pytest.mark.parametrize("M,N,K,w_bits", [(1, 1024, 1024, 8), (4, 65, 100, 8), (19, 4100, 512, 4), (64, 128, 1000, 4), (333, 300, 257, 8),
                                          (1531, 640, 768, 8)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_is_the_two_calls(M, N, K, w_bits, dtype):
    import torch
    r = rng(M)
    x = dev(r.standard_normal((M, K + 8)), dtype)[:, 3:3 + K]
    x[0] = 0
    _, w, w_scale = weights(r, N, K, w_bits)
    ws = dev(w_scale)
    for bits, act, out in ((8, mpq.ACT_NONE, None), (6, mpq.ACT_GELU, torch.float32), (4, mpq.ACT_RELU, torch.float16)):
        a, s = mpq.token_quant(x, bits)
        two = mpq.qgemm_tokens(a, w, s, ws, w_bits, act=act, dtype=out or x.dtype)
        one = mpq.linear_tokens(x, w, ws, w_bits, mpq.PER_ROW, bits, act, dtype=out)
        assert one.dtype == (out or x.dtype) and torch.equal(one, two)
        own = mpq.Workspace()
        again = mpq.linear_tokens(x, w, ws, w_bits, mpq.PER_ROW, bits, act, y=torch.empty_like(one), ws=own)
        assert torch.equal(again, two)


def test_no_tokens():
    import torch
    x = torch.empty(0, 64, device="cuda")
    codes, scale = mpq.token_quant(x)
    assert codes.shape == (0, 64) and scale.shape == (0,)
    _, w, w_scale = weights(rng(1), 8, 64, 8)
    assert mpq.qgemm_tokens(codes, w, scale, dev(w_scale)).shape == (0, 8)
    assert mpq.linear_tokens(x, w, dev(w_scale)).shape == (0, 8)


def test_replayed_graphs_and_other_streams_give_the_eager_results():
    """Two captured graphs of the same layers, replayed in turn with eager work between: none of them shares scratch."""
    import torch
    mpq.init()
    r = rng(9)
    xs = [dev(r.standard_normal((m, 512)), "bfloat16") for m in (3, 200)]
    _, w, w_scale = weights(r, 384, 512, 8)
    ws = dev(w_scale)
    want = [mpq.linear_tokens(x, w, ws) for x in xs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = [mpq.linear_tokens(x, w, ws) for x in xs]
    side.synchronize()
    graphs, outs = [], []
    for x in xs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(mpq.linear_tokens(x, w, ws))
        graphs.append(g)
    for _ in range(3):
        for o in outs:
            o.zero_()
        for g in graphs:
            g.replay()
        eager = [mpq.linear_tokens(x, w, ws) for x in xs]
        torch.cuda.synchronize()
        for a, b, c, d in zip(want, other, outs, eager):
            assert torch.equal(a, b) and torch.equal(a, c) and torch.equal(a, d)


@pytest.mark.parametrize("M,N,K,w_bits", [(16, 100, 4096, 8), (16, 100, 4112, 8), (9, 257, 2064, 4), (1, 33, 16, 8), (2, 5, 32, 4), (15, 300, 48, 8),
                                          (16, 12, 4096, 4), (5, 40, 13104, 8), (1, 20, 65536, 8), (1, 20, 65552, 4)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_one_kernel_or_two_are_the_same(M, N, K, w_bits, dtype):
    """Rows that the product's kernel quantizes itself, and the first sizes that it does not."""
    import torch
    r = rng(M + K)
    x = dev(r.standard_normal((M, K + 5)) * np.exp(3 * r.standard_normal((M, 1))), dtype)[:, 2:2 + K]
    x[M // 2] = 0
    _, w, w_scale = weights(r, N, K, w_bits)
    ws = dev(w_scale)
    fused = M * K <= 65536
    assert (mpq.linear_tokens_workspace_bytes(M, N, K, w_bits) == 0) == fused
    for bits, out in ((8, None), (3, torch.float32)):
        a, s = mpq.token_quant(x, bits)
        two = mpq.qgemm_tokens(a, w, s, ws, w_bits, dtype=out or x.dtype)
        assert torch.equal(mpq.linear_tokens(x, w, ws, w_bits, mpq.PER_ROW, bits, dtype=out), two)
