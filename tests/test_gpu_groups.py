"""The linear layer whose 4-bit weights have a step per group, against a plain reference in 64 bits."""
import numpy as np
import pytest

from oracle import drafts
from test_gpu_parity import host, mpq
from test_gpu_tokens import dev, full, rng

pytestmark = pytest.mark.gpu

DTYPES = ("float32", "bfloat16", "float16")
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
U = 2.0 ** -24


def layer(r, N, K, group, dtype="float32"):
    """(codes, packed on the device, steps on the host as the device has them, on the device)"""
    import torch
    codes = r.integers(-8, 8, (N, K))
    u = codes.astype(np.uint8) & 15
    steps = dev((r.random((N, K // group)) + 0.5) * 0.01, dtype)
    return codes, torch.from_numpy((u[:, ::2] | u[:, 1::2] << 4).astype(np.uint8)).cuda(), full(steps), steps


def check(got, x, codes, steps, group, out, act=None):
    """A group's sum is a chain of at most 2 group fp32 additions of terms of at most 24 |x| and 31 |x|, so that no partial sum passes
    55 sum |x|; chains of 8 waves and of the groups follow, of numbers that are at most 8 |x| step each.  GELU's slope is below 1.13, its
    own error below 4e-7 of |y|; outputs round by half a step (fp16: at least 2^-25)."""
    K = x.shape[1]
    want = drafts.linear_groups(x, codes, steps, group)
    size = np.abs(x).astype(np.float64) @ np.repeat(np.abs(steps).astype(np.float64), group, 1).T
    off = U * size * (55 * 2 * group + 8 * (K // group + 16))
    if act == "relu":
        want = np.maximum(want, 0)
    elif act == "gelu":
        want, off = drafts.gelu(want), 1.13 * off + 4e-7 * np.abs(want)
    bound = off + HALF[out] * (np.abs(want) + off) + (2.0 ** -25 if out == "float16" else 0.0)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (np.argwhere(bad)[:5], np.abs(got - want).max(), bound.min())
    return want


@pytest.mark.parametrize("group", (32, 64, 128))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N,K", [(1, 1, 128), (1, 17, 384), (2, 33, 256), (3, 64, 2048), (16, 100, 640), (17, 31, 512), (33, 47, 896),
                                   (64, 130, 4096), (65, 16, 128), (150, 5, 1152)])
def test_linear(group, dtype, M, N, K):
    r = rng(M * 7 + N + K)
    codes, w, steps, steps_dev = layer(r, N, K, group)
    x = r.standard_normal((M, K))
    x[:, r.integers(0, K, 4)] *= 20
    x = dev(x, dtype)
    y = mpq.linear_groups(x, w, steps_dev)
    assert y.dtype == x.dtype and y.shape == (M, N)
    check(full(y), full(x), codes, steps, group, dtype)


@pytest.mark.parametrize("group,K", [(32, 32), (32, 96), (32, 160), (32, 1056), (64, 64), (64, 192), (64, 2112), (128, 2176)])
def test_rows_that_end_inside_a_step(group, K):
    """k ends 32, 64 or 96 channels into the 128 that a lane's quarter of a load covers."""
    r = rng(K)
    codes, w, steps, steps_dev = layer(r, 21, K, group)
    for dtype in DTYPES:
        x = dev(r.standard_normal((5, K)), dtype)
        check(full(mpq.linear_groups(x, w, steps_dev)), full(x), codes, steps, group, dtype)


@pytest.mark.parametrize("group", (32, 64, 128))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N,K", [(9, 4200, 256), (40, 8300, 384), (64, 8333, 128), (100, 4111, 256), (1, 40, 131072), (8, 21, 14336), (5, 6, 65536)])
def test_channel_tiles_and_long_rows(group, dtype, M, N, K):
    """More channels than one tile to a workgroup fills the chip with; rows and steps that LDS holds no longer, or just."""
    test_linear(group, dtype, M, N, K)


@pytest.mark.parametrize("M,N,K", [(1, 2_200_000, 4096), (3, 140_000, 65536), (20, 140_000, 65536)])
def test_offsets_past_32_bits(M, N, K):
    """More than 2^32 bytes of codes: the last channels' are those of a small layer."""
    import torch
    r = rng(K)
    codes, w, steps, steps_dev = layer(r, 70, K, 128, "bfloat16")
    big_w = torch.zeros((N, K // 2), dtype=torch.uint8, device="cuda")
    big_s = torch.zeros((N, K // 128), dtype=torch.bfloat16, device="cuda")
    big_w[-70:] = w
    big_s[-70:] = steps_dev
    x = dev(r.standard_normal((M, K)), "bfloat16")
    y = mpq.linear_groups(x, big_w, big_s)
    check(full(y[:, -70:]), full(x), codes, steps, 128, "bfloat16")
    assert not y[:, :-70].any()


def test_offsets_past_32_bits_of_x():
    import torch
    r = rng(6)
    codes, w, steps, steps_dev = layer(r, 20, 256, 64)
    x = dev(r.standard_normal((30, 256)), "float16")
    far = torch.empty(29 * (1 << 27) + 256, dtype=torch.float16, device="cuda").as_strided((30, 256), (1 << 27, 1))
    far.copy_(x)
    for rows in (30, 20, 5):   # (5: the last row at 2^30 bytes; its stride is a long one all the same)
        assert torch.equal(mpq.linear_groups(far[:rows], w, steps_dev), mpq.linear_groups(x[:rows], w, steps_dev))
    check(full(mpq.linear_groups(far, w, steps_dev)), full(x), codes, steps, 64, "float16")


@pytest.mark.parametrize("steps_type", DTYPES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", (None, "relu", "gelu"))
def test_types_and_activations(steps_type, dtype, act):
    import torch
    r = rng(3)
    codes, w, steps, steps_dev = layer(r, 77, 512, 64, steps_type)
    x = dev(r.standard_normal((9, 512)) * 3, dtype)
    code = {None: mpq.ACT_NONE, "relu": mpq.ACT_RELU, "gelu": mpq.ACT_GELU}[act]
    for out in DTYPES:
        y = mpq.linear_groups(x, w, steps_dev, code, dtype=getattr(torch, out))
        check(full(y), full(x), codes, steps, 64, out, act)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("group", (32, 64, 128))
def test_every_channel_and_code(dtype, group):
    """One channel of x at a time: each product by itself, 24 bits of x.  The sums of such a row have two terms other than 0, 24 |x| and
    31 |x| at most, each rounded to 2^-24 of what is there: 2 (24 + 31) |x| steps."""
    r = rng(group)
    K, N = 256, 16
    codes, w, steps, steps_dev = layer(r, N, K, group)
    value = (r.random(K) + 1) * np.exp2(r.integers(-20, 20, K))
    x = dev(np.diag(value), dtype)
    y = mpq.linear_groups(x, w, steps_dev, dtype=__import__("torch").float32)
    v = np.diag(full(x)).astype(np.float64)      # (fp16 holds some of them as infinities, whose rows are not numbers)
    fine = np.isfinite(v)
    assert not np.isfinite(host(y)[~fine]).any() and fine.sum() > 150
    v, y = v[fine], host(y)[fine]
    codes, steps = codes[:, fine], np.repeat(steps, group, 1)[:, fine]
    want = v[:, None] * (codes * steps.astype(np.float64)).T
    bound = (110 * U + 4 * U * 8) * np.abs(v)[:, None] * steps.T
    assert (np.abs(y - want) <= bound).all(), np.abs(y - want).max()


def test_strides_alignment_and_outputs():
    """Rows far apart, weights at any byte, steps, rows and outputs at any element."""
    import torch
    r = rng(8)
    M, N, K, group = 7, 19, 320, 64
    codes, w, steps, steps_dev = layer(r, N, K, group)
    for dtype in DTYPES:
        t = getattr(torch, dtype)
        wide = torch.zeros(M * 400 + 1, dtype=t, device="cuda")[1:].view(M, 400)[:, 3:3 + K]
        wide.copy_(dev(r.standard_normal((M, K)), dtype))
        moved = torch.empty(N * K // 2 + 5, dtype=torch.uint8, device="cuda")[5:].view(N, K // 2)
        moved.copy_(w)
        s = torch.empty(N * K // group + 1, dtype=torch.float32, device="cuda")[1:].view(N, K // group)
        s.copy_(steps_dev)
        out = torch.full((M * N + 2,), 7.0, dtype=t, device="cuda")
        y = out[1:1 + M * N].view(M, N)
        assert mpq.linear_groups(wide, moved, s, y=y) is y
        check(full(y), full(wide), codes, steps, group, dtype)
        assert out[0] == 7 and out[-1] == 7
    assert mpq.linear_groups(dev(np.zeros((0, K))), w, steps_dev).shape == (0, N)


def test_rows_do_not_depend_on_their_neighbours():
    """A row alone gives the bits that it gives in a batch (its tile's sums are the same)."""
    import torch
    r = rng(9)
    codes, w, steps, steps_dev = layer(r, 48, 1024, 32)
    x = dev(r.standard_normal((40, 1024)), "bfloat16")
    y = mpq.linear_groups(x, w, steps_dev)
    for m in (0, 15, 16, 39):
        assert torch.equal(mpq.linear_groups(x[m:m + 1], w, steps_dev)[0], y[m])
    again = mpq.linear_groups(x, w, steps_dev)
    assert torch.equal(again, y)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("group", (32, 64, 128))
@pytest.mark.parametrize("M", (2, 8, 40))
def test_one_sided_rows(dtype, group, M):
    """Rows behind a ReLU, or all positive, steps of either sign, fp32 outputs: relative to the outputs' norm as near to 64 bits as products of the
    codes themselves.  Roundings are independent, u / sqrt(3) of a partial sum each.  32 k in three terms bring at most 24 (one per four products),
    a group of 128 then 96, of partial sums whose mean square is half of the group's at most: u sqrt(96 / 6) = 4 u of a group's sum, and of the outputs'
    norm, since groups' sums are independent as well.  The 32 to 128 groups and 8 waves bring u sqrt(136 / 6) = 4.8 u.  Together 6.3 u = 3.7e-7."""
    r = rng(group + M)
    K, N = 4096, 96
    import torch
    codes, w, steps, _ = layer(r, N, K, group)
    steps = steps * r.choice([-1, 1], steps.shape).astype(np.float32)
    steps_dev = dev(steps)
    for x in (np.maximum(r.standard_normal((M, K)), 0), r.random((M, K)) + 0.5):
        x = dev(x, dtype)
        y = host(mpq.linear_groups(x, w, steps_dev, dtype=torch.float32)).astype(np.float64)
        want = drafts.linear_groups(full(x), codes, steps, group)
        assert np.linalg.norm(y - want) <= 1e-6 * np.linalg.norm(want), np.linalg.norm(y - want) / np.linalg.norm(want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("group", (32, 64, 128))
@pytest.mark.parametrize("steps_type", ("float32", "float16"))
def test_every_channel_and_code_in_few_rows(dtype, group, steps_type):
    """One channel of x at a time, in calls of up to 8 rows: each product by itself, 24 bits of x.  x's terms times a code are exact, their sum is
    rounded at most twice and its product with the step once: 3 u of |x c step|, and u of it for the bits that three terms leave."""
    import torch
    r = rng(group + 7)
    K, N = 256, 21
    codes, w, steps, steps_dev = layer(r, N, K, group, steps_type)
    value = (r.random(K) + 1) * np.exp2(r.integers(-12, 12, K)) * r.choice([-1, 1], K)
    x = dev(np.diag(value), dtype)
    v = np.diag(full(x)).astype(np.float64)
    wide = np.repeat(steps.astype(np.float64), group, 1)
    at = 0
    for rows in [1, 2, 3, 5, 7, 8] * 12:
        if at >= K:
            break
        m = slice(at, min(at + rows, K))
        y = host(mpq.linear_groups(x[m], w, steps_dev, dtype=torch.float32))
        want = v[m, None] * (codes * wide)[:, m].T
        assert (np.abs(y - want) <= 4 * U * np.abs(want)).all(), (at, np.abs(y - want).max())
        at += rows
    assert at >= K
    y = host(mpq.linear_groups(x, w, steps_dev, dtype=torch.float32))
    want = v[:, None] * (codes * wide).T
    assert (np.abs(y - want) <= 4 * U * np.abs(want)).all()


@pytest.mark.parametrize("group,K", [(32, 4096), (64, 4224), (128, 11008), (32, 1120), (64, 8256)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_row_alone_and_in_a_batch(dtype, group, K):
    """The same bits, in fp32, however many rows there are: one order of k for all of them."""
    import torch
    r = rng(K)
    codes, w, steps, steps_dev = layer(r, 70, K, group)
    x = dev(r.standard_normal((70, K)), dtype)
    y = mpq.linear_groups(x, w, steps_dev, dtype=torch.float32)
    for rows in (1, 2, 8, 9, 16, 17, 33, 64, 65):
        for at in (0, 70 - rows):
            assert torch.equal(mpq.linear_groups(x[at:at + rows], w, steps_dev, dtype=torch.float32), y[at:at + rows]), rows


@pytest.mark.parametrize("dtype", DTYPES)
def test_an_output_in_the_inputs_place(dtype):
    """Refused: workgroups would read what others have written.  An output between x's rows is none of them."""
    import torch
    r = rng(14)
    K = N = 128
    codes, w, steps, steps_dev = layer(r, N, K, 32, dtype)
    x = dev(r.standard_normal((4, K)), dtype)
    with pytest.raises(mpq.MpqError):
        mpq.linear_groups(x, w, steps_dev, y=x)
    both = torch.zeros(2, 2 * K, dtype=x.dtype, device="cuda")
    both[:, :K] = x[:2]
    got = mpq.linear_groups(both[:, :K], w[:64], steps_dev[:64], y=both[0, K:].view(2, 64))
    assert torch.equal(got, mpq.linear_groups(x[:2], w[:64], steps_dev[:64]))
    with pytest.raises(mpq.MpqError):
        mpq.linear_groups(both[:, :K], w[:64], steps_dev[:64], y=both.view(-1)[K + 1:K + 129].view(2, 64))


def test_group_quant_and_its_layer():
    import torch
    r = rng(10)
    N, K = 33, 512
    for group in (32, 64, 128):
        w = dev(r.standard_normal((N, K)))
        packed, steps = mpq.group_quant(w, group)
        codes = drafts.nibbles(host(packed))
        parts = host(w).reshape(N, K // group, group)
        top = np.abs(parts).max(2)
        np.testing.assert_array_equal(host(steps), (top / np.float32(7)).astype(np.float32))
        inv = (np.float32(7) / top).astype(np.float32)
        np.testing.assert_array_equal(codes, np.rint(parts.astype(np.float64) * inv[..., None].astype(np.float64)).reshape(N, K))
        x = dev(r.standard_normal((3, K)))
        check(host(mpq.linear_groups(x, packed, steps)), host(x), codes, host(steps), group, "float32")
    for bad in ((w, 16), (w, 96), (w[0], 32)):
        with pytest.raises(ValueError):
            mpq.group_quant(*bad)


def test_values_at_the_ends():
    """Rows that are not finite give no numbers, and only themselves; a step of 0 is a group of zeros; large and small rows."""
    import torch
    r = rng(11)
    codes, w, steps, steps_dev = layer(r, 20, 256, 32)
    x = dev(r.standard_normal((4, 256)), "bfloat16")
    x[1, 77] = float("inf")
    x[2, 3] = float("nan")
    y = full(mpq.linear_groups(x, w, steps_dev))
    assert np.isfinite(y[[0, 3]]).all() and not np.isfinite(y[1]).any() and np.isnan(y[2]).all()
    steps_dev[:, 2] = 0
    x = dev(r.standard_normal((4, 256)))
    check(host(mpq.linear_groups(x, w, steps_dev)), host(x), codes, host(steps_dev), 32, "float32")
    for size in (2.0 ** 100, 2.0 ** -80):
        x = dev(r.standard_normal((4, 256)) * size)
        check(host(mpq.linear_groups(x, w, steps_dev)), host(x), codes, host(steps_dev), 32, "float32")


def test_refusals_of_the_binding():
    import torch
    r = rng(12)
    codes, w, steps, s = layer(r, 20, 256, 32)
    x = dev(r.standard_normal((4, 256)))
    for bad in ((x[0], w, s), (x.t(), w, s), (x, w[:, :64], s), (x, w.t(), s), (x, w, s[:10]), (x, w, s.t()), (x, w, s[:, 0]), (x.int(), w, s),
                (x, w, s.int()), (x.cpu(), w, s)):
        with pytest.raises(ValueError):
            mpq.linear_groups(*bad)
    with pytest.raises(ValueError):
        mpq.linear_groups(x, w, s, y=torch.empty((4, 19), device="cuda"))
    with pytest.raises(mpq.MpqError):
        mpq.linear_groups(x, w, s[:, :1].contiguous())                       # a group of 256
    with pytest.raises(mpq.MpqError):
        mpq.linear_groups(x, w, s, 7)


def test_graphs_and_streams():
    import torch
    r = rng(13)
    codes, w, steps, s = layer(r, 64, 512, 64)
    x = dev(r.standard_normal((6, 512)), "float16")
    want = mpq.linear_groups(x, w, s).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        on_side = mpq.linear_groups(x, w, s)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(on_side, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = mpq.linear_groups(x, w, s)
    for i in range(3):
        x.copy_(dev(r.standard_normal((6, 512)), "float16"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, mpq.linear_groups(x, w, s))
