"""The operators between the blocks at the edges of what they take: far strides, sizes that a call cannot carry, values next to what
fp32 holds.  Definitions and tolerances as in test_operators.py."""
import math

import pytest
import torch

from tests.test_operators import BF16, F8, assert_linear, eight_bits, generator, norm, rand, run_linear, run_linear_q8, to_e4m3, toma, tuning  # noqa: F401 (fixtures)


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


# ---- what a call cannot carry: sizes and strides beyond 32 bits ----

def meta(shape, stride, dtype):
    return torch.empty_strided(shape, stride, dtype=dtype, device="meta")


@pytest.fixture
def no_device(toma, monkeypatch):  # noqa: F811
    """The binding with tensors that have no memory taken for the current device's: what it refuses, it refuses before the library's
    call, which fails the test."""
    from paper_2509_10918_b200 import binding

    def called(*args):
        raise AssertionError("reached the library")

    at = meta((1,), (1,), BF16).get_device()
    monkeypatch.setattr(binding, "_current_device", lambda: at)
    for name in ("toma_rms_norm", "toma_rms_norm_q8", "toma_linear_act", "toma_linear_q8", "toma_quantise_weight", "toma_mlp_layer"):
        monkeypatch.setattr(binding.lib, name, called)
    monkeypatch.setattr(binding, "_stream", lambda: None)
    return binding


FAR = [2 ** 31, 2 ** 32 + 64, 2 ** 33]


@pytest.mark.parametrize("far", FAR)
def test_strides_beyond_32_bits_are_refused(no_device, far):
    b = no_device
    f32, one = torch.float32, meta((64,), (1,), BF16)
    x, wide = meta((2, 64), (64, 1), BF16), meta((2, 64), (far, 1), BF16)
    q, q_wide, scale = meta((2, 64), (64, 1), F8), meta((2, 64), (far, 1), F8), meta((2,), (1,), f32)
    w = meta((64, 64), (64, 1), BF16)
    w8, w8_wide, scales = meta((64, 64), (64, 1), F8), meta((64, 64), (far, 1), F8), meta((64,), (1,), f32)
    for call in (
            lambda: b.toma_rms_norm(wide, one, x), lambda: b.toma_rms_norm(x, one, wide), lambda: b.toma_rms_norm(x, one, x, delta=wide),
            lambda: b.toma_rms_norm(x, one, x, delta=x, sum_out=wide), lambda: b.toma_rms_norm_q8(x, one, q_wide, scale),
            lambda: b.toma_rms_norm_q8(wide, one, q, scale), lambda: b.toma_linear_act(wide, w, x), lambda: b.toma_linear_act(x, w, wide),
            lambda: b.toma_linear_act(x, w, x, residual=wide), lambda: b.toma_linear_q8(q_wide, scale, w8, scales, x),
            lambda: b.toma_linear_q8(q, scale, w8_wide, scales, x), lambda: b.toma_linear_q8(q, scale, w8, scales, wide),
            lambda: b.toma_quantise_weight(w, w8_wide, scales)):
        with pytest.raises(ValueError, match="apart"):
            call()
    with pytest.raises(AssertionError, match="reached"):  # the stride of a single row is no one's
        b.toma_rms_norm(meta((1, 64), (far, 1), BF16), one, meta((1, 64), (64, 1), BF16))


@pytest.mark.parametrize("rows", [2 ** 31, 2 ** 32 + 2])
def test_sizes_beyond_32_bits_are_refused(no_device, rows):
    b = no_device
    x, y = meta((rows, 8), (8, 1), BF16), meta((rows, 8), (8, 1), BF16)
    q, scale, w8, s8 = meta((rows, 16), (16, 1), F8), meta((rows,), (1,), torch.float32), meta((8, 16), (16, 1), F8), meta((8,), (1,), torch.float32)
    w, wide = meta((8, 8), (8, 1), BF16), meta((8, rows), (rows, 1), BF16)
    for call in (lambda: b.toma_rms_norm(x, None, y), lambda: b.toma_rms_norm_q8(x, None, q, scale), lambda: b.toma_linear_act(x, w, y),
                 lambda: b.toma_linear_act(w, wide, wide), lambda: b.toma_linear_q8(q, scale, w8, s8, y), lambda: b.toma_quantise_weight(wide, q, scale),
                 lambda: b.toma_mlp_layer_workspace_bytes(rows, 8, 8, "bf16"), lambda: b.toma_mlp_layer_workspace_bytes(8, 8, rows, "f32"),
                 lambda: b.toma_mlp_layer(x, None, w, None, w, None, y, w), lambda: b.toma_mlp_layer(w, None, wide, None, w, None, w, w)):
        with pytest.raises(ValueError, match="at most"):
            call()


@pytest.mark.gpu
def test_rows_more_than_32_bits_apart_are_refused(toma):  # noqa: F811
    buf = torch.zeros(2 ** 32 + 256, dtype=torch.uint8, device="cuda").view(F8)
    a, scale = buf.as_strided((2, 64), (2 ** 32 + 64, 1)), torch.ones(2, device="cuda")
    w, w_scale, c = torch.zeros(64, 64, device="cuda").to(F8), torch.ones(64, device="cuda"), torch.zeros(2, 64, dtype=BF16, device="cuda")
    with pytest.raises(ValueError):
        toma.toma_linear_q8(a, scale, w, w_scale, c)
    with pytest.raises(ValueError):
        toma.toma_rms_norm_q8(c, None, a, scale)


# ---- a single column ----

def test_a_single_column_has_no_step(no_device):
    """[rows, 1] is contiguous whatever the second stride says; a transposed row has the row's length there."""
    x, w, c = meta((5, 1), (1, 5), torch.float32), meta((1, 1), (1, 1), torch.float32), meta((5, 1), (1, 5), torch.float32)
    assert x.is_contiguous()
    with pytest.raises(AssertionError, match="reached"):
        no_device.toma_linear_act(x, w, c, residual=c)
    with pytest.raises(ValueError):
        no_device.toma_linear_act(meta((5, 2), (1, 5), torch.float32), meta((2, 1), (1, 1), torch.float32), c)


@pytest.mark.gpu
def test_single_columns_out_of_rows(toma):  # noqa: F811
    g = generator(41)
    for m in (1, 5, 40):
        a, w, c = rand(g, 1, m).t(), rand(g, 1, 1), torch.empty(1, m, device="cuda").t()
        toma.toma_linear_act(a, w, c, act="gelu")
        torch.cuda.synchronize()
        assert_linear(c, a, w, None, "gelu")


# ---- the norm where its sum of squares leaves fp32 ----

@pytest.mark.gpu
@pytest.mark.parametrize("dim", [8, 64, 640, 1280, 5120, 16384])
def test_norm_next_to_the_overflow_of_its_sum(toma, dim):  # noqa: F811
    """A row just below sqrt(3.4e38 / dim) is right, one just above is zeros (3 %: bf16 has steps of 0.8 %, the sum errors of 0.1 %)."""
    bound = math.sqrt(torch.finfo(torch.float32).max / dim)
    sign = torch.where(rand(generator(dim), dim) < 0, -1.0, 1.0).double()
    for dtype in (BF16, torch.float32):
        x = torch.stack([sign * bound * f for f in (0.97, 1.03, 0.5, 1e-3)]).to(dtype)
        y = torch.empty_like(x)
        toma.toma_rms_norm(x, None, y)
        torch.cuda.synchronize()
        want = norm(x, None, 1e-6)
        tol = want.abs() * ((2.0 ** -8 if dtype == BF16 else 2.0 ** -24) + 64 * 2.0 ** -24)
        for r in (0, 2, 3):
            assert bool(((y[r].double() - want[r]).abs() <= tol[r]).all()), r
        assert bool((y[1] == 0).all())
    q, scale = torch.empty(4, (dim + 15) // 16 * 16, dtype=F8, device="cuda")[:, :dim], torch.empty(4, device="cuda")
    x = x.to(BF16)
    toma.toma_rms_norm_q8(x, None, q, scale)
    torch.cuda.synchronize()
    p = x.double()
    top = p.abs().amax(1)
    assert torch.equal(q.double(), to_e4m3(p * 448 / top[:, None]))
    want = top / 448 / torch.sqrt(p.square().mean(1) + 1e-6)
    assert float(scale[1]) == 0
    for r in (0, 2, 3):
        assert abs(float(scale[r]) - float(want[r])) <= float(want[r]) * 64 * 2.0 ** -24


# ---- scales far apart, and operands that are no numbers ----

FORMS = [(2, 0), (12, 0), (40, 0), (300, 0), (300, 2), (300, 3), (300, 4), (300, 5), (300, 6), (300, 7), (300, 9), (300, 10)]  # rows, tile form asked for


@pytest.mark.gpu
@pytest.mark.parametrize("m,tile", FORMS)
def test_q8_scales_whose_product_leaves_fp32(toma, tuning, m, tile):  # noqa: F811
    """(sum a_scale) w_scale is a number where a_scale w_scale is none (1e45: above fp32; 1e-43: below the normal numbers, 70 units of the
    least).  The sums are of positive numbers, some 10^7, so that the first product and the result are normal numbers."""
    tuning(linear_tile=tile)
    n, k = 328, 640
    g = generator(m, tile)
    a, _ = eight_bits(rand(g, m, k).abs() + 1)
    w, _ = eight_bits(rand(g, n, k).abs() + 1)
    a[1] = 0
    c = torch.empty(m, n, dtype=BF16, device="cuda")
    for sa, sw in ((1e25, 1e20), (1e-23, 1e-20), (1e-31, 1e-12)):
        a_scale, w_scale = torch.full((m,), sa, device="cuda"), torch.full((n,), sw, device="cuda")
        if sa > 1:  # only the rows of zeros are numbers there
            a_scale[0], a_scale[2:] = 1e-30, 1e-30
        toma.toma_linear_q8(a, a_scale, w, w_scale, c)
        torch.cuda.synchronize()
        assert not torch.isnan(c).any() and bool((c[1] == 0).all())
        assert_linear(c, a.float(), w.float().t(), a_scale=a_scale, w_scale=w_scale)


@pytest.mark.gpu
@pytest.mark.parametrize("m,tile", FORMS)
def test_q8_none_numbers_keep_to_themselves(toma, tuning, m, tile):  # noqa: F811
    """A none-number in a row of a, in a column of w, in a scale of either, and an infinite scale: the other rows and columns as without."""
    tuning(linear_tile=tile)
    n, k = 328, 648
    g = generator(m, tile, 1)
    a, a_scale = eight_bits(rand(g, m, k))
    w, w_scale = eight_bits(rand(g, n, k))
    clean, c = (torch.empty(m, n, dtype=BF16, device="cuda") for _ in range(2))
    nan, inf = float("nan"), float("inf")
    for act in ("none", "gelu", "gelu_tanh", "silu"):
        toma.toma_linear_q8(a, a_scale, w, w_scale, clean, act=act)
        for where in ("a", "w", "a_scale", "w_scale"):
            t = {"a": a.clone(), "w": w.clone(), "a_scale": a_scale.clone(), "w_scale": w_scale.clone()}
            for name in "aw":  # (rows of whole packets again)
                padded = torch.zeros(t[name].shape[0], 656, device="cuda").to(F8)[:, :k]
                padded.copy_(t[name])
                t[name] = padded
            at = 1 if where[0] == "a" else n - 3
            t[where][at if "scale" in where else (at, k - 1)] = nan
            c.fill_(0)
            toma.toma_linear_q8(t["a"], t["a_scale"], t["w"], t["w_scale"], c, act=act)
            torch.cuda.synchronize()
            bad = torch.zeros_like(c, dtype=torch.bool)
            if where[0] == "a":
                bad[at] = True
            else:
                bad[:, at] = True
            assert torch.isnan(c[bad]).all() and torch.equal(c[~bad], clean[~bad]), (act, where)
        a_inf = a_scale.clone()
        a_inf[0] = inf
        toma.toma_linear_q8(a, a_inf, w, w_scale, c, act=act)
        torch.cuda.synchronize()
        assert not torch.isfinite(c[0][clean[0].abs() > 1]).any() and torch.equal(c[1:], clean[1:])


@pytest.mark.gpu
@pytest.mark.parametrize("m", [2, 10, 200])
def test_activations_of_infinities(toma, m):  # noqa: F811
    """+infinity stays, and -infinity, where the formulas have infinity times zero, is the limit 0 for GELU in bf16 and NaN elsewhere."""
    inf = float("inf")
    for dtype in (BF16, torch.float32):
        a, w = torch.zeros(m, 16, dtype=dtype, device="cuda"), torch.zeros(16, 32, dtype=dtype, device="cuda")
        bias, c = torch.zeros(32, dtype=dtype, device="cuda"), torch.empty(m, 32, dtype=dtype, device="cuda")
        bias[3], bias[20] = inf, -inf
        for act in ("none", "gelu", "gelu_tanh", "silu"):
            outs = []
            toma.toma_linear_act(a, w, c, bias=bias, act=act)
            outs.append(c.clone())
            if dtype == BF16:
                toma.toma_linear_q8(a.to(F8), torch.ones(m, device="cuda"), w.t().contiguous().to(F8), torch.ones(32, device="cuda"), c, bias=bias, act=act)
                outs.append(c.clone())
            torch.cuda.synchronize()
            for out in outs:
                assert bool((out[:, 3] == inf).all()) and bool((out[:, [0, 19, 21, 31]] == 0).all())
                low = out[:, 20]
                if act == "none":
                    assert bool((low == -inf).all())
                elif act == "gelu" and dtype == BF16:
                    assert bool((low == 0).all())
                else:
                    assert torch.isnan(low).all()


# ---- every form, where it is the one that runs ----

TILES = {2: "128x192", 3: "256x256", 4: "128x128", 5: "256x320", 6: "split2", 7: "split4", 8: "split8", 9: "pairs2", 10: "pairs3"}


@pytest.mark.gpu
@pytest.mark.parametrize("tile", list(TILES), ids=list(TILES.values()))
@pytest.mark.parametrize("m,n,k", [(129, 328, 1160), (300, 72, 2056), (257, 1288, 1032), (1000, 648, 1096)])
def test_the_form_asked_for_runs_over_long_ragged_contractions(toma, tuning, tile, m, n, k):  # noqa: F811
    """A split by eight has a step for each CTA from 8 on: 1032 elements are 9 steps of e4m3 and 17 of bf16, the last of 8 elements."""
    tuning(linear_tile=tile)
    for f8 in (False, True):
        assert toma.toma_test_linear_plus_form(m, n, k, f8, "gelu") == tile
    run_linear(toma, m, n, k, BF16, True, "gelu", True, pad=8)
    run_linear(toma, m, n, k, BF16, False, "none", False, seed=1)
    run_linear_q8(toma, m, n, k, True, "silu", True, pad=16)
    run_linear_q8(toma, m, n, k, False, "none", False, seed=1)


@pytest.mark.gpu
def test_forms_by_themselves(toma, tuning):  # noqa: F811
    """At most 16 rows have their own form, and a form that a shape does not allow is not taken."""
    form = toma.toma_test_linear_plus_form
    assert all(form(m, 640, 640, f8) == 1 for m in (1, 16) for f8 in (False, True))
    assert all(form(m, 640, 640, f8) in TILES for m in (17, 154, 4096) for f8 in (False, True))
    tuning(linear_tile=8)
    assert form(300, 640, 448) != 8 and form(300, 640, 456) == 8 and form(300, 640, 896, True) != 8 and form(300, 640, 904, True) == 8
    tuning(linear_tile=3)
    assert form(128, 640, 640) != 3 and form(129, 640, 640) == 3


def test_forms_of_bad_shapes(toma):  # noqa: F811
    form = toma.lib.toma_test_linear_plus_form
    assert form(0, 8, 8, 0, 0) == 0 and form(8, 12, 8, 0, 0) == 0 and form(8, 8, 8, 0, 4) == 0
    assert form(2 ** 31 - 1, 8, 8, 0, 0) == 0 and form(8, 2 ** 31 - 8, 8, 0, 0) == 0 and form(8, 8, 2 ** 31 - 8, 1, 0) == 0


# ---- fp32 on the tensor cores: none of the six products missing, chains as short as they are ----

F32_FORMS = ["chosen", "128", "64", "128split2", "128split4", "64split2", "64split4"]


@pytest.mark.gpu
@pytest.mark.parametrize("form", range(7), ids=F32_FORMS)
def test_linear_f32_error_does_not_grow_with_the_contraction(toma, tuning, form):  # noqa: F811
    """The root of the mean square error against 64 bits in units of 2^-24 of the results' root mean square, at most 6 at any length.

    A chain of 128 elements is eight instructions that each add to the sum so far and cut off: 0.5 units of its last place in the mean,
    a unit being 0.72 2^-23 of it in the mean, the sums on the way 0.66 of the last in the mean: 8 x 0.5 x 0.72 x 0.66 = 1.9 of 2^-23,
    3.8 of 2^-24 of a chain's sum, towards zero.  Chains' sums have signs of their own, so the errors add up as the sums do: 3.8 of the result
    at any length.  Adding up k / 128 chains rounds each time, 0.42 of 2^-24 of the sum so far in the root mean square, 0.7 of the
    last: 0.29 sqrt(k / 128), 2.6 at 10240.  Together 4.6.  One of the six products missing is 40 and more (products of a plane
    of 2^-16, root mean square), chains that do not end at 128 grow with k.
    """
    tuning(linear_tile=form)
    for m, n, k in ((512, 256, 640), (512, 256, 4096), (130, 200, 1000), (300, 136, 10240)):
        g = generator(m, n, k, 5)
        a, w, c = rand(g, m, k), rand(g, k, n), torch.empty(m, n, device="cuda")
        toma.toma_linear_act(a, w, c)
        want = a.double() @ w.double()
        off = float(((c.double() - want).square().mean() / want.square().mean()).sqrt()) * 2 ** 24
        print(f"f32 {F32_FORMS[form]} {m} x {n} x {k}: {off:.2f} units of 2^-24")
        assert off <= 6


# ---- the layer: the same every time ----

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, torch.float32], ids=["bf16", "f32"])
def test_layer_repeats_itself(toma, dtype):  # noqa: F811
    """Whatever its scratch and its result hold before, eager and out of a graph."""
    for rows, dim, hidden in ((1, 640, 2560), (154, 1280, 5120), (1024, 1280, 5120), (3000, 640, 2560)):
        g = generator(rows, 3)
        x, delta, nw = rand(g, rows, dim, dtype=dtype), rand(g, rows, dim, dtype=dtype), rand(g, dim, dtype=dtype)
        w1, b1 = rand(g, dim, hidden, dtype=dtype) / math.sqrt(dim), rand(g, hidden, dtype=dtype)
        w2, b2 = rand(g, hidden, dim, dtype=dtype) / math.sqrt(hidden), rand(g, dim, dtype=dtype)
        ws = torch.empty(toma.toma_mlp_layer_workspace_bytes(rows, dim, hidden, "bf16" if dtype == BF16 else "f32"), dtype=torch.uint8, device="cuda")
        first, out = torch.empty_like(x), torch.empty_like(x)
        toma.toma_mlp_layer(x, nw, w1, b1, w2, b2, first, ws, delta=delta)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            toma.toma_mlp_layer(x, nw, w1, b1, w2, b2, out, ws, delta=delta)
        for i in range(6):
            out.fill_(float("nan")), ws.fill_(255 if i % 2 else 0)
            if i < 3:
                toma.toma_mlp_layer(x, nw, w1, b1, w2, b2, out, ws, delta=delta)
            else:
                graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, first)
