"""The layer with a step per token on few rows and wide weights: workgroups of two, three and four tiles of 16 output channels, on
codes and with the rows quantized in the product's kernel."""
import pytest

from test_gpu_parity import mpq
from test_gpu_tokens import DTYPES, dev, rng, weights

pytestmark = pytest.mark.gpu

WIDE = (4117, 8209, 8212, 12301, 14352)      # tiles per workgroup: 2, 3, 3, 4, 4 for up to 32 rows, 2 for more


def exact(a, codes, a_scale, w_scale):
    """fl32(fl32(acc a_scale) w_scale), acc a whole number far below 2^53."""
    acc = a.double() @ codes.double().t().contiguous()
    return (acc.float() * a_scale[:, None]) * w_scale


@pytest.mark.parametrize("N", WIDE)
@pytest.mark.parametrize("M,K", [(8, 80), (16, 1042), (17, 512), (24, 1042), (33, 64), (48, 1042), (64, 512)])
@pytest.mark.parametrize("w_bits", (8, 4))
def test_layer_of_few_rows_is_exact(M, N, K, w_bits):
    import torch
    r = rng(M + N + K)
    codes, w, w_scale = weights(r, N, K, w_bits)
    g = torch.Generator(device="cuda").manual_seed(M + N)
    a = torch.randint(-127, 128, (M, K), dtype=torch.int8, device="cuda", generator=g)
    a_scale, ws = torch.rand(M, device="cuda", generator=g) * 0.01 + 1e-4, dev(w_scale)
    want = exact(a, dev(codes, "int8"), a_scale, ws)
    for dtype in DTYPES:
        t = getattr(torch, dtype)
        y = torch.full((M + 1, N), 77.0, dtype=t, device="cuda")
        mpq.qgemm_tokens(a, w, a_scale, ws, w_bits, y=y[:M])
        assert torch.equal(y[:M], want.to(t)) and (y[M] == 77.0).all()
        one = ws[:1].contiguous()
        y = mpq.qgemm_tokens(a, w, a_scale, one, w_bits, mpq.PER_TENSOR, mpq.ACT_RELU, dtype=t)
        assert torch.equal(y, exact(a, dev(codes, "int8"), a_scale, one).clamp(min=0).to(t))


@pytest.mark.parametrize("N", (17,) + WIDE)
@pytest.mark.parametrize("M,K", [(1, 16), (8, 80), (9, 4128), (16, 4096)])
@pytest.mark.parametrize("w_bits", (8, 4))
@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_quantized_in_the_products_kernel(M, N, K, w_bits, dtype):
    """Against the two calls, and their product against whole numbers."""
    import torch
    if w_bits == 4:
        K = max(K, 32)
    r = rng(M + N + K)
    codes, w, w_scale = weights(r, N, K, w_bits)
    g = torch.Generator(device="cuda").manual_seed(M + N)
    x = torch.randn(M, K + 3, device="cuda", generator=g).to(getattr(torch, dtype))[:, 1:1 + K]
    x[M // 2] *= 30
    ws = dev(w_scale)
    assert mpq.linear_tokens_workspace_bytes(M, N, K, w_bits) == 0
    a, s = mpq.token_quant(x)
    for out in (None, torch.float32):
        t = out or x.dtype
        want = exact(a, dev(codes, "int8"), s, ws).to(t)
        assert torch.equal(mpq.linear_tokens(x, w, ws, w_bits, dtype=out), want)
        assert torch.equal(mpq.qgemm_tokens(a, w, s, ws, w_bits, dtype=t), want)
