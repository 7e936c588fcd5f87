"""The operators between the blocks at the edges of what they take: far strides, sizes that a call cannot carry, values next to what
fp32 holds.  Definitions and tolerances as in test_operators.py."""
import pytest
import torch

from tests.test_operators import BF16, F8, assert_linear, eight_bits, generator, rand, toma, tuning  # noqa: F401 (fixtures)


@pytest.mark.gpu
@pytest.mark.parametrize("m", [2, 9, 16, 40])
@pytest.mark.parametrize("far", [2 ** 28, 2 ** 29], ids=["2^28", "2^29"])
def test_q8_weights_with_rows_far_apart(toma, far, m):  # noqa: F811
    """Rows of w whose distance times eight passes 32 bits: the same as of a dense copy."""
    n, k = 16, 328
    g = generator(far, m)
    a, a_scale = eight_bits(rand(g, m, k))
    w, w_scale = eight_bits(rand(g, n, k))
    r = rand(g, m, n, dtype=BF16)
    buf = torch.empty((n - 1) * far + 336, dtype=torch.uint8, device="cuda")
    apart = buf.view(F8).as_strided((n, k), (far, 1))
    apart.copy_(w)
    near, c = torch.empty_like(r), torch.empty_like(r)
    toma.toma_linear_q8(a, a_scale, w, w_scale, near, act="silu", residual=r)
    toma.toma_linear_q8(a, a_scale, apart, w_scale, c, act="silu", residual=r)
    torch.cuda.synchronize()
    assert_linear(near, a.float(), w.float().t(), None, "silu", r, a_scale, w_scale)
    assert torch.equal(c, near)


@pytest.mark.gpu
@pytest.mark.parametrize("m", [2, 16])
def test_few_rows_far_apart(toma, m):  # noqa: F811
    """Rows of the activations, the residual and the result beyond 32 bits of bytes, in each type."""
    n, k, far = 40, 72, 2 ** 28
    g = generator(m)
    for dtype in (BF16, torch.float32):
        buf = torch.empty((m - 1) * far + 4096, dtype=dtype, device="cuda")
        a, c, r = (buf[at:].as_strided((m, cols), (far, 1)) for at, cols in ((0, k), (1024, n), (2048, n)))
        a.copy_(rand(g, m, k)), r.copy_(rand(g, m, n))
        w = rand(g, k, n, dtype=dtype)
        toma.toma_linear_act(a, w, c, act="gelu", residual=r)
        torch.cuda.synchronize()
        assert_linear(c, a, w, None, "gelu", r)
        del buf, a, c, r
    q, a_scale = eight_bits(rand(g, m, k))
    w, w_scale = eight_bits(rand(g, n, k))
    buf = torch.empty((m - 1) * far + 4096, dtype=torch.uint8, device="cuda")
    a = buf.view(F8).as_strided((m, k), (far, 1))
    a.copy_(q)
    c = torch.empty(m, n, dtype=BF16, device="cuda")
    toma.toma_linear_q8(a, a_scale, w, w_scale, c)
    torch.cuda.synchronize()
    assert_linear(c, a.float(), w.float().t(), a_scale=a_scale, w_scale=w_scale)
