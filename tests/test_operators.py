"""The operators between the blocks (norm with the residual's addition, 8-bit rows, projections with their epilogue, the MLP layer)
against their definitions in 64 bits, and what they refuse.

Tolerances.  A result in bf16 is one rounding (2^-8 relative at most) of a value computed in fp32.  A sum of k products in fp32,
in any order and with truncation instead of rounding at worst, is within k 2^-23 of the sum of the products' magnitudes.  An
activation has a slope of at most 1.13 and is computed to 2^-19 of its argument's magnitude at least.  Where a tensor between two
kernels is rounded, the next one is compared on the rounded tensor itself."""
import ctypes
import itertools
import math

import pytest
import torch

import __graft_entry__ as entry

BF16, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
OK, NULL, SHAPE, DTYPE, WS, UNSUP, ARG = 0, 1, 2, 3, 6, 7, 11


@pytest.fixture(scope="module")
def toma():
    entry.build()
    import paper_2509_10918_b200 as t
    return t


@pytest.fixture
def tuning(toma):
    yield toma.toma_test_set_tuning
    toma.toma_test_set_tuning()


# ---- definitions ----

def e4m3_values(device):
    code = torch.arange(127, device=device)
    e, f = code // 8, (code % 8).double()
    return torch.where(e == 0, f * 2.0 ** -9, (1 + f / 8) * torch.exp2(e.double() - 7))


def to_e4m3(v):
    """The nearest e4m3 value, half way between two the one with the even code; beyond 448 it saturates.

    Callers give 448 p / top as (448 p) / top: with p of at most 16 bits the product is exact in 64 bits, and a quotient that is half
    way between two values (5 bits) is exact after its one rounding.  (p / top) 448 is rounded twice and misses such a quotient
    where top has a factor 7: 145 / 280 comes out above 232 / 448.)"""
    values = e4m3_values(v.device)
    middles = (values[1:] + values[:-1]) / 2
    size = v.abs().contiguous()
    low, high = torch.searchsorted(middles, size), torch.searchsorted(middles, size, right=True)
    return torch.sign(v) * values[torch.where(low % 2 == 0, low, high)]


def activation(v, act):
    if act == "gelu":
        return v * torch.special.ndtr(v)
    if act == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
    return v * torch.sigmoid(v) if act == "silu" else v


def norm(h, weight, eps):
    h = h.double()
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    return y if weight is None else y * weight.double()


def linear(a, w, bias, act, residual, a_scale=None, w_scale=None):
    """(result, magnitude of what was summed up), both in 64 bits."""
    a, w = a.double(), w.double()
    v, size = a @ w, a.abs() @ w.abs()
    if a_scale is not None:
        s = torch.outer(a_scale.double(), w_scale.double())
        v, size = v * s, size * s
    if bias is not None:
        v, size = v + bias.double(), size + bias.double().abs()
    y = activation(v, act)
    if residual is not None:
        y, size = y + residual.double(), size + residual.double().abs()
    return y, size


def assert_linear(c, a, w, bias=None, act="none", residual=None, a_scale=None, w_scale=None):
    want, size = linear(a, w, bias, act, residual, a_scale, w_scale)
    k = a.shape[1]
    half = 2.0 ** -8 if c.dtype == BF16 else 2.0 ** -24
    slope = 1.0 if act == "none" else 1.13
    # (8: the epilogue's own roundings; 2^-19 of the magnitude: the activation)
    tol = half * want.abs() + size * (slope * (k + 8) * 2.0 ** -23 + (2.0 ** -19 if act != "none" else 0.0))
    assert not torch.isnan(c).any()
    off = (c.double() - want).abs() - tol * (1 + 1e-6)
    assert float(off.max()) <= 0, f"{float(off.max())} over the bound"


def rand(gen, *shape, dtype=F32):
    return torch.randn(*shape, generator=gen, device="cuda").to(dtype)


def generator(*seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(hash(seed) & 0x7FFFFFFF)
    return g


def canvas(rows, cols, dtype, pad, fill=7.0):
    """A [rows, cols] view with `pad` elements between its rows and rows above (four, so that it begins on a 16-byte boundary for any
    row length in fp32) and below it, and the check that all of those have stayed as they were."""
    whole = torch.full((rows + 5, cols + pad), fill, device="cuda").to(dtype)
    view = whole[4:rows + 4, :cols]

    def untouched():
        around = whole.float().clone()
        around[4:rows + 4, :cols] = fill
        return bool((around == fill).all())

    return view, untouched


# ---- refusals (no GPU needed: nothing is launched) ----

P = ctypes.c_void_p
A, B, C, D, E, G = (P(0x10000000 * i) for i in range(1, 7))  # far apart, never dereferenced


def norm_args(**kw):
    v = dict(rows=4, dim=64, dtype=0, x=A, ldx=64, delta=B, ldd=64, weight=C, eps=1e-6, sum=D, lds=64, y=E, ldy=64, stream=None)
    v.update(kw)
    return list(v.values())


def test_norm_refuses(toma):
    f = toma.lib.toma_rms_norm
    assert f(*norm_args(x=None)) == NULL and f(*norm_args(y=None)) == NULL and f(*norm_args(delta=None)) == NULL
    assert f(*norm_args(dtype=2)) == DTYPE
    for bad in (dict(rows=0), dict(dim=0), dict(dim=63), dict(dim=60), dict(ldx=56), dict(ldx=68), dict(ldd=60), dict(lds=65), dict(ldy=32),
                dict(x=P(A.value + 8)), dict(delta=P(B.value + 2)), dict(weight=P(C.value + 4)), dict(sum=P(D.value + 8)), dict(y=P(E.value + 2))):
        assert f(*norm_args(**bad)) == SHAPE, bad
    assert f(*norm_args(dim=16392, ldx=16392, ldd=16392, lds=16392, ldy=16392)) == UNSUP
    for eps in (0.0, -1e-6, float("nan"), float("inf")):
        assert f(*norm_args(eps=eps)) == ARG
    # overlaps: a partial one, the sum on the result, the result on the weight, in place with another stride
    for bad in (dict(y=P(A.value + 128)), dict(y=D), dict(sum=E), dict(y=C), dict(sum=C), dict(sum=P(B.value + 16)), dict(y=A, ldy=72)):
        assert f(*norm_args(**bad)) == ARG, bad


def q8_args(**kw):
    v = dict(rows=4, dim=64, x=A, ldx=64, delta=B, ldd=64, weight=C, eps=1e-6, sum=D, lds=64, q=E, ldq=64, scale=G, stream=None)
    v.update(kw)
    return list(v.values())


def test_norm_q8_refuses(toma):
    f = toma.lib.toma_rms_norm_q8
    assert f(*q8_args(scale=None)) == NULL and f(*q8_args(q=None)) == NULL and f(*q8_args(x=None)) == NULL
    for bad in (dict(ldq=72), dict(ldq=48), dict(q=P(E.value + 8)), dict(scale=P(G.value + 2)), dict(dim=12)):
        assert f(*q8_args(**bad)) == SHAPE, bad
    for bad in (dict(q=A), dict(q=D), dict(scale=E), dict(scale=P(A.value + 4)), dict(q=B), dict(eps=0.0)):
        assert f(*q8_args(**bad)) == ARG, bad


def linear_args(**kw):
    v = dict(m=4, n=64, k=32, dtype=0, a=A, lda=32, w=B, bias=C, act=1, residual=D, ldr=64, c=E, ldc=64, status=None, stream=None)
    v.update(kw)
    return list(v.values())


def test_linear_refuses(toma):
    f = toma.lib.toma_linear_act
    for name in ("a", "w", "c"):
        assert f(*linear_args(**{name: None})) == NULL
    assert f(*linear_args(dtype=7)) == DTYPE
    for bad in (dict(m=0), dict(n=0), dict(k=-8), dict(n=60), dict(k=20), dict(lda=24), dict(lda=36), dict(ldr=60), dict(ldc=68),
                dict(a=P(A.value + 2)), dict(w=P(B.value + 8)), dict(bias=P(C.value + 2)), dict(residual=P(D.value + 8)), dict(c=P(E.value + 8))):
        assert f(*linear_args(**bad)) == SHAPE, bad
    # (c in place of the residual is allowed, with another stride or shifted it is not)
    for bad in (dict(act=4), dict(act=-1), dict(c=A), dict(c=B), dict(c=C), dict(c=P(D.value + 128)), dict(c=D, ldc=72), dict(c=P(A.value + 16))):
        assert f(*linear_args(**bad)) == ARG, bad


def linear8_args(**kw):
    v = dict(m=4, n=64, k=32, a=A, lda=32, sa=P(A.value + 0x1000), w=B, ldw=32, sw=P(B.value + 0x10000), bias=C, act=1, residual=D, ldr=64, c=E, ldc=64,
             status=None, stream=None)
    v.update(kw)
    return list(v.values())


def test_linear_q8_refuses(toma):
    f = toma.lib.toma_linear_q8
    for name in ("a", "w", "c", "sa", "sw"):
        assert f(*linear8_args(**{name: None})) == NULL
    for bad in (dict(lda=40), dict(ldw=24), dict(ldw=40), dict(k=36), dict(n=4), dict(sw=P(B.value + 0x10004)), dict(sa=P(A.value + 0x1002)), dict(ldc=60)):
        assert f(*linear8_args(**bad)) == SHAPE, bad
    for bad in (dict(c=P(A.value + 0x1000)), dict(c=P(B.value + 0x10000)), dict(c=B), dict(act=9)):
        assert f(*linear8_args(**bad)) == ARG, bad


def test_quantise_weight_refuses(toma):
    f = toma.lib.toma_quantise_weight
    assert f(32, 64, None, B, 32, C, None) == NULL and f(32, 64, A, None, 32, C, None) == NULL and f(32, 64, A, B, 32, None, None) == NULL
    assert f(30, 64, A, B, 32, C, None) == SHAPE and f(32, 60, A, B, 32, C, None) == SHAPE and f(32, 64, A, B, 40, C, None) == SHAPE
    assert f(32, 64, A, A, 32, C, None) == ARG and f(32, 64, A, B, 32, B, None) == ARG


def test_layer_refuses(toma):
    f = toma.lib.toma_mlp_layer
    need = toma.toma_mlp_layer_workspace_bytes(4, 64, 128, "bf16")
    assert need == 512 + 1024 and toma.toma_mlp_layer_workspace_bytes(0, 64, 128, "bf16") == 0

    def args(**kw):
        v = dict(rows=4, dim=64, hidden=128, dtype=0, x=A, delta=B, norm_weight=P(C.value + 0x1000), eps=1e-6, w1=D, b1=P(D.value + 0x100000),
                 act=1, w2=E, b2=P(E.value + 0x100000), out=G, ws=P(G.value + 0x100000), ws_bytes=need, status=None, stream=None)
        v.update(kw)
        return list(v.values())

    for name in ("x", "w1", "w2", "out"):
        assert f(*args(**{name: None})) == NULL
    assert f(*args(dtype=3)) == DTYPE
    for bad in (dict(rows=0), dict(dim=60), dict(hidden=100), dict(hidden=0), dict(x=P(A.value + 2)), dict(b1=P(D.value + 0x100002))):
        assert f(*args(**bad)) == SHAPE, bad
    for bad in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=P(G.value + 0x100008))):
        assert f(*args(**bad)) == WS, bad
    for bad in (dict(eps=0.0), dict(act=5), dict(out=D), dict(out=P(A.value + 16)), dict(ws=A), dict(ws=E), dict(out=P(G.value + 0x100000)),
                dict(out=P(C.value + 0x1000)), dict(out=P(E.value + 0x100000))):
        assert f(*args(**bad)) == ARG, bad


def test_binding_refuses(toma):
    x = torch.zeros(4, 64, dtype=BF16)
    with pytest.raises(ValueError):
        toma.toma_rms_norm(x, None, x)
    with pytest.raises(ValueError):
        toma.toma_linear_act(x, x, x)
    assert toma.toma_status_str(ARG).startswith("bad eps")


# ---- norm ----

ROWS = (1, 3, 154, 5000)  # the last: more rows than a chip's warps
DIMS = (8, 64, 248, 256, 264, 640, 1024, 1280, 2048, 2056, 4096, 5120, 8200, 16384)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("dim", DIMS)
def test_norm_parity(toma, dtype, dim):
    for rows, (add, store, weighted, pad) in zip(ROWS, [(True, True, True, 0), (False, False, True, 24), (True, False, False, 8), (True, True, True, 16)]):
        g = generator(dim, rows)
        x, _ = canvas(rows, dim, dtype, pad)
        x.copy_(rand(g, rows, dim) * torch.exp(rand(g, rows, 1)))
        delta = rand(g, rows, dim, dtype=dtype) if add else None
        weight = rand(g, dim, dtype=dtype) if weighted else None
        total, total_ok = canvas(rows, dim, dtype, pad) if store else (None, lambda: True)
        y, y_ok = canvas(rows, dim, dtype, 2 * pad)
        toma.toma_rms_norm(x, weight, y, 1e-6, delta=delta, sum_out=total)
        torch.cuda.synchronize()
        h = (x.float() + delta.float()).to(dtype) if add else x
        if store:
            assert torch.equal(total, h)
        want = norm(h, weight, 1e-6)
        # squares of at most 40 elements in a chain, a tree over the rest, the root, the quotient, two products
        tol = want.abs() * ((2.0 ** -8 if dtype == BF16 else 2.0 ** -24) + 64 * 2.0 ** -24)
        assert bool(((y.double() - want).abs() <= tol).all())
        assert y_ok() and total_ok()


@pytest.mark.gpu
@pytest.mark.parametrize("dim", DIMS)
def test_norm_q8_parity(toma, dim):
    for rows, (add, weighted, pad) in zip(ROWS, [(True, True, 0), (False, True, 24), (True, False, 8), (True, True, 16)]):
        g = generator(dim, rows, 8)
        x, _ = canvas(rows, dim, BF16, pad)
        x.copy_(rand(g, rows, dim) * torch.exp(rand(g, rows, 1)))
        delta = rand(g, rows, dim, dtype=BF16) if add else None
        weight = rand(g, dim, dtype=BF16) if weighted else None
        total = torch.empty(rows, dim, dtype=BF16, device="cuda") if add else None
        q, q_ok = canvas(rows, dim, F8, (-dim) % 16 + 16)
        scale = torch.full((rows,), float("nan"), device="cuda")
        toma.toma_rms_norm_q8(x, weight, q, scale, 1e-6, delta=delta, sum_out=total)
        torch.cuda.synchronize()
        h = (x.float() + delta.float()).to(BF16) if add else x
        if add:
            assert torch.equal(total, h)
        p = h.double() * (1 if weight is None else weight.double())
        top = p.abs().amax(1)
        assert torch.equal(q.double(), to_e4m3(p * 448 / top[:, None]))
        want = top / 448 / torch.sqrt(h.double().square().mean(1) + 1e-6)
        assert bool(((scale.double() - want).abs() <= want * 64 * 2.0 ** -24).all())
        assert q_ok()


@pytest.mark.gpu
def test_q8_ties_and_borders(toma):
    """Quotients that are exactly half way between two 8-bit values (48 p = m top with small whole numbers), next to such a
    border, and in the subnormal range: the nearest, ties to the even code."""
    tops = [448.0, 3.5, 7.0, 1.0, 0.4375, 447.0, 449.0, 1.5, 113.0, 2.0 ** -60, 2.0 ** 100]
    rows = []
    for top in tops:
        ratio = torch.cat([torch.arange(1, 256).double() / 256, torch.arange(1, 128).double() / 128 / 2 ** 9, torch.arange(17, 32, 2).double() * 3 / 224])
        v = (ratio * top).to(BF16)
        rows.append(torch.cat([v, -v, torch.tensor([top], dtype=BF16), torch.zeros(1, dtype=BF16)]))
    x = torch.stack(rows)
    x = torch.nn.functional.pad(x, (0, (-x.shape[1]) % 16)).cuda()
    q, scale = torch.empty(x.shape, dtype=F8, device="cuda"), torch.empty(x.shape[0], device="cuda")
    weight = torch.ones(x.shape[1], dtype=BF16, device="cuda")
    for w in (None, weight, 1.25 * weight):
        toma.toma_rms_norm_q8(x, w, q, scale)
        torch.cuda.synchronize()
        p = x.double() * (1 if w is None else w.double())
        v = p * 448 / p.abs().amax(1, keepdim=True)
        middle = torch.isin(v.abs() * 2 ** 10, (e4m3_values("cuda")[1:] + e4m3_values("cuda")[:-1]) * 2 ** 9)
        assert int(middle.sum()) > 50  # there are ties among them
        assert torch.equal(q.double(), to_e4m3(v))


@pytest.mark.gpu
def test_norm_of_special_rows(toma):
    dim = 640
    for dtype in (BF16, F32):
        x = rand(generator(1), 6, dim, dtype=dtype)
        x[1] = 0
        x[2, 5] = float("inf")
        x[3, 7] = float("nan")
        x[4] *= 1e-12
        y = torch.empty_like(x)
        toma.toma_rms_norm(x, None, y, 1e-6)
        torch.cuda.synchronize()
        want = norm(x, None, 1e-6)
        assert bool((y[1] == 0).all())
        assert torch.isnan(y[2, 5]) and bool((y[2, :5] == 0).all()) and torch.isnan(y[3]).all()
        for r in (0, 4, 5):
            assert bool(((y[r].double() - want[r]).abs() <= want[r].abs() * 2.0 ** (-7 if dtype == BF16 else -17)).all())
    x = rand(generator(2), 7, dim, dtype=BF16)
    x[1] = 0
    x[2, 5] = float("-inf")
    x[3, 639] = float("nan")
    x[4] *= 2.0 ** -120
    x[5] *= 2.0 ** -90
    q, scale = torch.empty(7, dim, dtype=F8, device="cuda"), torch.empty(7, device="cuda")
    toma.toma_rms_norm_q8(x, None, q, scale, 1e-6)
    torch.cuda.synchronize()
    for r in (1, 4):
        assert bool((q[r].float() == 0).all()) and float(scale[r]) == 0
    for r in (2, 3):
        assert torch.isnan(q[r].float()).all() and torch.isnan(scale[r])
    for r in (0, 5, 6):
        p = x[r].double()
        assert torch.equal(q[r].double(), to_e4m3(p * 448 / p.abs().max())) and math.isfinite(float(scale[r]))


@pytest.mark.gpu
def test_norm_in_place(toma):
    g = generator(3)
    for dtype in (BF16, F32):
        x, delta, w = rand(g, 300, 1280, dtype=dtype), rand(g, 300, 1280, dtype=dtype), rand(g, 1280, dtype=dtype)
        total, y = torch.empty_like(x), torch.empty_like(x)
        toma.toma_rms_norm(x, w, y, delta=delta, sum_out=total)
        for s_on, y_on in (("x", "delta"), ("delta", "x"), ("x", None), (None, "x")):
            t = {"x": x.clone(), "delta": delta.clone(), None: torch.empty_like(x)}
            s_out = t[s_on] if s_on else torch.empty_like(x)
            toma.toma_rms_norm(t["x"], w, t[y_on], delta=t["delta"], sum_out=s_out)
            torch.cuda.synchronize()
            assert torch.equal(s_out, total) and torch.equal(t[y_on], y)


# ---- projections ----

EPILOGUES = [(b, act, r) for b, act, r in itertools.product((False, True), ("none", "gelu", "gelu_tanh", "silu"), (False, True))]


def run_linear(toma, m, n, k, dtype, bias, act, residual, pad=0, seed=0):
    g = generator(m, n, k, seed)
    a, _ = canvas(m, k, dtype, pad)
    a.copy_(rand(g, m, k))
    w = rand(g, k, n, dtype=dtype) / math.sqrt(k)
    b = rand(g, n, dtype=dtype) if bias else None
    r = None
    if residual:
        r, _ = canvas(m, n, dtype, 2 * pad)
        r.copy_(rand(g, m, n))
    c, c_ok = canvas(m, n, dtype, pad)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    toma.toma_linear_act(a, w, c, bias=b, act=act, residual=r, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0 and c_ok()
    assert_linear(c, a, w, b, act, r)


def eight_bits(t, pad=0):
    """(rows of t in e4m3 as a strided view, scales)"""
    scale = t.abs().amax(1).clamp_min(1e-20).float() / 448
    q = torch.zeros(t.shape[0], (t.shape[1] + 15) // 16 * 16 + pad, device="cuda").to(F8)[:, :t.shape[1]]
    q.copy_((t.float() / scale[:, None]).to(F8))
    return q, scale


def run_linear_q8(toma, m, n, k, bias, act, residual, pad=0, seed=0):
    g = generator(m, n, k, seed, 8)
    a, a_scale = eight_bits(rand(g, m, k), pad)
    w, w_scale = eight_bits(rand(g, n, k) / math.sqrt(k), pad)
    b = rand(g, n, dtype=BF16) if bias else None
    r = None
    if residual:
        r, _ = canvas(m, n, BF16, 8)
        r.copy_(rand(g, m, n))
    c, c_ok = canvas(m, n, BF16, pad)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    toma.toma_linear_q8(a, a_scale, w, w_scale, c, bias=b, act=act, residual=r, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0 and c_ok()
    assert_linear(c, a.float(), w.float().t(), b, act, r, a_scale, w_scale)


@pytest.mark.gpu
@pytest.mark.parametrize("bias,act,residual", EPILOGUES)
def test_linear_every_epilogue(toma, bias, act, residual):
    run_linear(toma, 300, 328, 200, BF16, bias, act, residual, pad=16)
    run_linear(toma, 70, 101, 33, F32, bias, act, residual, pad=3)
    run_linear(toma, 3, 328, 200, BF16, bias, act, residual, pad=8)
    run_linear_q8(toma, 300, 328, 200, bias, act, residual, pad=16)
    run_linear_q8(toma, 3, 328, 200, bias, act, residual, pad=16)


SHAPES = [(1, 8, 8), (1, 640, 640), (2, 5120, 1280), (4, 72, 5120), (7, 1288, 648), (8, 640, 2560), (9, 1288, 648), (16, 136, 4096), (31, 640, 5120),
          (33, 2560, 64), (64, 1280, 1280), (65, 320, 2048), (77, 2048, 640), (127, 64, 64), (128, 328, 640), (129, 136, 1032), (154, 1280, 2048),
          (255, 640, 2560), (257, 1288, 1280), (500, 72, 200), (1003, 2560, 640), (1024, 1280, 5120), (4096, 640, 2560), (4097, 1288, 72)]


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_linear_parity(toma, m, n, k):
    run_linear(toma, m, n, k, BF16, True, "gelu", True)
    run_linear(toma, m, n, k, BF16, False, "none", True, seed=1)
    run_linear(toma, m, n, k, BF16, True, "silu", False, pad=8, seed=2)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_linear_q8_parity(toma, m, n, k):
    run_linear_q8(toma, m, n, k, True, "gelu_tanh", True)
    run_linear_q8(toma, m, n, k, False, "none", False, pad=16, seed=1)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 4, 4), (3, 68, 60), (2, 312, 3272), (8, 640, 2560), (9, 132, 5120), (16, 5120, 640), (1, 640, 640), (2, 1280, 320), (5, 7, 1000), (64, 130, 66), (301, 96, 161), (1003, 640, 320)])
def test_linear_f32_parity(toma, m, n, k):
    run_linear(toma, m, n, k, F32, True, "gelu", True)
    run_linear(toma, m, n, k, F32, False, "silu", False, pad=5, seed=1)
    run_linear(toma, m, n, k, F32, True, "none", True, pad=4, seed=2)


F32_SHAPES = [(17, 4, 4), (20, 640, 2560), (128, 64, 64), (130, 200, 132), (300, 72, 1000), (515, 1284, 68), (1003, 2560, 640), (2048, 320, 2560), (64, 64, 20000), (20000, 132, 40)]


@pytest.mark.gpu
@pytest.mark.parametrize("form", range(7), ids=["chosen", "128", "64", "128split2", "128split4", "64split2", "64split4"])
def test_linear_f32_on_the_tensor_cores(toma, tuning, form):
    """Floats as sums of three bf16 numbers: the bound of a sum in fp32, the length of the longest among them."""
    tuning(linear_tile=form)
    for m, n, k in F32_SHAPES:
        run_linear(toma, m, n, k, F32, True, "gelu_tanh", True, pad=8)
        run_linear(toma, m, n, k, F32, False, "none", False, seed=1)


@pytest.mark.gpu
def test_linear_f32_error_is_that_of_fp32_sums(toma):
    """On the tensor cores and not: the root of the mean square error against 64 bits, in units of 2^-24 of the results' root mean
    square.  A sum of k products of random signs has an error of about sqrt(k) / 3 of them at most where it is rounded after each."""
    for m, n, k in ((512, 256, 640), (512, 256, 4096), (512, 257, 640)):
        g = generator(m, n, k)
        a, w, c = rand(g, m, k), rand(g, k, n), torch.empty(m, n, device="cuda")
        toma.toma_linear_act(a, w, c)
        want = a.double() @ w.double()
        off = float(((c.double() - want).square().mean() / want.square().mean()).sqrt()) * 2 ** 24
        print(f"f32 {m} x {n} x {k}: {off:.2f} units of 2^-24")
        assert off <= math.sqrt(k)


@pytest.mark.gpu
def test_linear_f32_with_infinities_and_none_numbers(toma):
    """Rows and columns with infinities have the infinities that the sums have, rows with a none-number have nothing else."""
    g = generator(9)
    a, w = rand(g, 300, 260), rand(g, 260, 136)
    a[3, 7], a[5, 100], a[5, 200], a[290, 259], a[8, 0] = float("inf"), float("-inf"), float("inf"), float("nan"), 3.4e38
    w[11, 50], w[0, 60] = float("inf"), 1e30
    c = torch.empty(300, 136, device="cuda")
    toma.toma_linear_act(a, w, c)
    torch.cuda.synchronize()
    with_inf = a.double() @ w.double()
    want = torch.where(with_inf.abs() > torch.finfo(F32).max, torch.sign(with_inf) * float("inf"), with_inf)
    assert torch.equal(torch.isnan(c), torch.isnan(want)) and torch.isnan(c[290]).all()
    assert torch.equal(torch.isinf(c), torch.isinf(want)) and torch.isinf(c[3]).any() and torch.isinf(c[:, 50]).any()
    assert torch.equal(c[torch.isinf(c)].double(), want[torch.isinf(want)])
    fine = torch.isfinite(want)
    tol = (a.double().abs().nan_to_num(0, 0, 0) @ w.double().abs().nan_to_num(0, 0, 0)) * 268 * 2.0 ** -23 + want.abs().nan_to_num(0, 0, 0) * 2.0 ** -23
    assert bool(((c.double() - want).abs() <= tol)[fine].all())


@pytest.mark.gpu
@pytest.mark.parametrize("tile", [2, 3, 4, 5, 6, 7, 8, 9, 10],
                         ids=["128x192", "256x256", "128x128", "256x320", "split2", "split4", "split8", "pairs2", "pairs3"])
@pytest.mark.parametrize("m,n,k", [(300, 328, 200), (129, 1920, 640), (1024, 72, 136), (9000, 1016, 72), (20000, 64, 200)])
def test_linear_every_tile_form(toma, tuning, tile, m, n, k):
    tuning(linear_tile=tile)
    run_linear(toma, m, n, k, BF16, True, "gelu", True, pad=8)
    run_linear(toma, m, n, k, BF16, True, "none", False, seed=1)
    run_linear_q8(toma, m, n, k, True, "silu", True, pad=16)
    run_linear_q8(toma, m, n, k, False, "none", False, seed=1)


@pytest.mark.gpu
@pytest.mark.parametrize("form", [*range(11, 19), *range(21, 29)], ids=[f"{cols}by{split}" for cols in (64, 32) for split in range(1, 9)])
def test_linear_few_rows_every_split(toma, tuning, form):
    """Blocks that end inside, contractions shorter than a CTA's steps and none for some, clusters that do not divide a block's eights."""
    tuning(linear_tile=form)
    for m, n, k in ((1, 8, 8), (2, 72, 5120), (2, 1288, 648), (1, 5128, 264), (3, 328, 40), (7, 200, 1000), (8, 2568, 136), (16, 1288, 648)):
        run_linear(toma, m, n, k, BF16, True, "gelu", True, pad=8)
        run_linear(toma, m, n, k, BF16, False, "none", False, seed=1)
        run_linear_q8(toma, m, n, k, True, "silu", True, pad=16)
    for m, n, k in ((1, 4, 4), (2, 68, 5120), (2, 1284, 132), (4, 200, 1000), (7, 324, 60), (16, 1292, 644)):
        run_linear(toma, m, n, k, F32, True, "gelu_tanh", True, pad=4)
        run_linear(toma, m, n, k, F32, False, "none", False, seed=1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_linear_few_rows_keep_to_themselves(toma, dtype):
    """One row with a none-number, one column of w with an infinity: the other rows and columns are what they are without."""
    g = generator(31)
    for m in (1, 2, 4, 8, 16):
        for n, k in ((40, 72), (1288, 648), (5128, 320)):
            a, w = rand(g, m, k, dtype=dtype), rand(g, k, n, dtype=dtype) / math.sqrt(k)
            base, c = torch.empty(m, n, dtype=dtype, device="cuda"), torch.empty(m, n, dtype=dtype, device="cuda")
            toma.toma_linear_act(a, w, base)
            a[0, k - 1], w[3, n - 1] = float("nan"), float("inf")
            toma.toma_linear_act(a, w, c)
            torch.cuda.synchronize()
            assert torch.isnan(c[0]).all() and not torch.isfinite(c[:, n - 1]).any()
            assert torch.equal(c[1:, : n - 1], base[1:, : n - 1])


@pytest.mark.gpu
def test_linear_in_place_and_side_by_side(toma):
    g = generator(5)
    for m in (2, 100, 1000):
        a, w, b = rand(g, m, 640, dtype=BF16), rand(g, 640, 320, dtype=BF16) / 25, rand(g, 320, dtype=BF16)
        r = rand(g, m, 320, dtype=BF16)
        c = torch.empty_like(r)
        toma.toma_linear_act(a, w, c, bias=b, act="gelu", residual=r)
        buf = torch.zeros(m, 960, dtype=BF16, device="cuda")
        buf[:, :640], buf[:, 640:] = a, r
        toma.toma_linear_act(buf[:, :640], w, buf[:, 640:], bias=b, act="gelu", residual=buf[:, 640:])
        torch.cuda.synchronize()
        assert torch.equal(buf[:, 640:], c) and torch.equal(buf[:, :640], a)


@pytest.mark.gpu
def test_a_row_that_is_no_number_stays_by_itself(toma):
    g = generator(6)
    for m in (3, 100, 700):
        a, w = rand(g, m, 648, dtype=BF16), rand(g, 648, 328, dtype=BF16)
        clean, c = torch.empty(m, 328, dtype=BF16, device="cuda"), torch.empty(m, 328, dtype=BF16, device="cuda")
        for act in ("none", "gelu", "gelu_tanh", "silu"):
            toma.toma_linear_act(a, w, clean, act=act)
            bad = a.clone()
            bad[1, 640] = float("nan")
            toma.toma_linear_act(bad, w, c, act=act)
            torch.cuda.synchronize()
            assert torch.isnan(c[1]).all()
            keep = [i for i in range(m) if i != 1]
            assert torch.equal(c[keep], clean[keep])


@pytest.mark.gpu
def test_activations_far_out(toma):
    """Arguments whose exponentials leave fp32: v, 0 and no none-number."""
    v = torch.tensor([0.0, 1e-4, -1e-4, 5.0, -5.0, 12.0, -12.0, 60.0, -60.0, 500.0, -500.0, 1e4, -1e4, 1e18, -1e18, 3e38], device="cuda")
    for dtype in (BF16, F32):
        b = v.to(dtype)
        for m in (2, 200):
            a, w = torch.zeros(m, 8, dtype=dtype, device="cuda"), torch.zeros(8, 16, dtype=dtype, device="cuda")
            c = torch.empty(m, 16, dtype=dtype, device="cuda")
            for act in ("gelu", "gelu_tanh", "silu"):
                toma.toma_linear_act(a, w, c, bias=b, act=act)
                torch.cuda.synchronize()
                want = activation(b.double(), act)
                tol = want.abs() * 2.0 ** -8 + 1e-5 * b.double().abs().clamp_max(20) + 1e-30
                assert bool(((c.double() - want).abs() <= tol).all()), (act, c[0], want)


@pytest.mark.gpu
@pytest.mark.parametrize("k,n", [(8, 8), (640, 2560), (200, 328), (1032, 40), (5120, 1280)])
def test_quantise_weight(toma, k, n):
    w = rand(generator(k, n), k, n, dtype=BF16)
    w[:, n // 2] = 0
    q, ok = canvas(n, k, F8, (-k) % 16 + 16)
    scale = torch.empty(n, device="cuda")
    toma.toma_quantise_weight(w, q, scale)
    torch.cuda.synchronize()
    p = w.double().t()
    top = p.abs().amax(1)
    want = to_e4m3(p * 448 / top.clamp_min(1e-300)[:, None])
    assert torch.equal(q.double(), want) and ok()
    assert bool(((scale.double() - top / 448).abs() <= top / 448 * 2.0 ** -22).all())


@pytest.mark.gpu
def test_rows_beyond_32_bits_of_elements(toma):
    """Strided rows whose offsets pass 2^31 elements: the last rows are the ones that a 32-bit offset would miss."""
    rows, ld, dim = 40000, 65536, 64
    g = generator(12)
    buf = torch.zeros(rows, ld, dtype=BF16, device="cuda")
    x, y = buf[:, :dim], buf[:, 1024:1024 + dim]
    x.copy_(rand(g, rows, dim))
    toma.toma_rms_norm(x, None, y)
    a, c = x, buf[:, 2048:2048 + 72]
    w = rand(g, dim, 72, dtype=BF16)
    toma.toma_linear_act(a, w, c, act="silu", residual=buf[:, 4096:4096 + 72])
    torch.cuda.synchronize()
    for part in (slice(0, 300), slice(32700, 33000), slice(rows - 300, rows)):
        want = norm(x[part], None, 1e-6)
        assert bool(((y[part].double() - want).abs() <= want.abs() * 2.0 ** -7).all())
        assert_linear(c[part], a[part], w, None, "silu")
    del buf, x, y, a, c
    f = torch.zeros(rows, ld, device="cuda")
    for n in (72, 73):  # on the tensor cores and not
        w = rand(g, dim, n)
        f[:, :dim].copy_(rand(g, rows, dim))
        toma.toma_linear_act(f[:, :dim], w, f[:, 2048:2048 + n])
        torch.cuda.synchronize()
        for part in (slice(0, 300), slice(rows - 300, rows)):
            assert_linear(f[part, 2048:2048 + n], f[part, :dim], w)


@pytest.mark.gpu
def test_binding_refuses_what_it_can_see(toma):
    x, w, c, b = (torch.zeros(*s, dtype=BF16, device="cuda") for s in ((4, 64), (64, 32), (4, 32), (32,)))
    toma.toma_linear_act(x, w, c, bias=b)
    for bad in (dict(a=x.cpu()), dict(a=x[0]), dict(w=w.t()), dict(w=w[:32]), dict(c=c.float()), dict(c=c[:3]), dict(bias=b[:8]), dict(bias=b[::2].repeat(2)[::2]),
                dict(residual=c.t()), dict(a=x.half()), dict(residual=x), dict(bias=b.float()), dict(a=x.repeat(1, 2)[:, ::2])):
        args = dict(a=x, w=w, c=c, bias=b)
        args.update(bad)
        with pytest.raises(ValueError):
            toma.toma_linear_act(**args)
    for act in ("relu", 4, -1, 2 ** 32 + 1, None):
        with pytest.raises(toma.TomaError):
            toma.toma_linear_act(x, w, c, act=act)
    with pytest.raises(toma.TomaError):
        toma.toma_rms_norm(x, None, x, eps=0.0)
    with pytest.raises(ValueError):
        toma.toma_rms_norm(x, None, c)
    with pytest.raises(ValueError):
        toma.toma_rms_norm_q8(x, None, torch.zeros(4, 64, dtype=torch.uint8, device="cuda"), torch.zeros(4, device="cuda"))
    with pytest.raises(ValueError):
        toma.toma_rms_norm_q8(x, None, x.to(F8), torch.zeros(4, dtype=torch.float64, device="cuda"))


@pytest.mark.gpu
def test_results_are_the_same_every_time(toma):
    g = generator(13)
    for m, n, k in ((2, 640, 5120), (100, 640, 5120), (600, 1280, 2560), (3000, 640, 640)):
        a, w, r = rand(g, m, k, dtype=BF16), rand(g, k, n, dtype=BF16), rand(g, m, n, dtype=BF16)
        for t in ((a, w, r), (a.float(), w.float(), r.float())):
            first = torch.empty_like(t[2])
            toma.toma_linear_act(t[0], t[1], first, act="gelu", residual=t[2])
            for _ in range(5):
                c = torch.full_like(t[2], float("nan"))
                toma.toma_linear_act(t[0], t[1], c, act="gelu", residual=t[2])
                assert torch.equal(c, first)


# ---- the layer, and a run of the operators together ----

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,dim,hidden", [(1, 640, 2560), (6, 64, 72), (77, 1280, 5120), (1003, 320, 1280)])
def test_layer_is_its_operators(toma, dtype, rows, dim, hidden):
    g = generator(rows, dim)
    x, delta, nw = rand(g, rows, dim, dtype=dtype), rand(g, rows, dim, dtype=dtype), rand(g, dim, dtype=dtype)
    w1, b1 = rand(g, dim, hidden, dtype=dtype) / math.sqrt(dim), rand(g, hidden, dtype=dtype)
    w2, b2 = rand(g, hidden, dim, dtype=dtype) / math.sqrt(hidden), rand(g, dim, dtype=dtype)
    ws = torch.empty(toma.toma_mlp_layer_workspace_bytes(rows, dim, hidden, "bf16" if dtype == BF16 else "f32"), dtype=torch.uint8, device="cuda")
    s, y, hid, want = (torch.empty(rows, c, dtype=dtype, device="cuda") for c in (dim, dim, hidden, dim))
    for add, bias in ((True, True), (False, False)):
        d, c1, c2 = (delta, b1, b2) if add else (None, None, None)
        toma.toma_rms_norm(x, nw, y, 1e-5, delta=d, sum_out=s if add else None)
        toma.toma_linear_act(y, w1, hid, bias=c1, act="gelu")
        toma.toma_linear_act(hid, w2, want, bias=c2, residual=s if add else x)
        torch.cuda.synchronize()
        # each step on what the step before it has stored
        assert_linear(hid, y, w1, c1, "gelu")
        assert_linear(want, hid, w2, c2, "none", s if add else x)
        for on in ("out", "x", "delta"):
            t = {"out": torch.empty_like(x), "x": x.clone(), "delta": delta.clone()}
            toma.toma_mlp_layer(t["x"], nw, w1, c1, w2, c2, t[on], ws, act="gelu", eps=1e-5, delta=t["delta"] if add else None)
            torch.cuda.synchronize()
            assert torch.equal(t[on], want), on


def chain(toma, t):
    """What a sampler's step runs between two attention blocks: the block's output joins the stream, the MLP's first projection in
    8 bits, the second added to the stream, the next norm."""
    toma.toma_rms_norm_q8(t["x"], t["nw"], t["q"], t["qs"], delta=t["delta"], sum_out=t["s"])
    toma.toma_linear_q8(t["q"], t["qs"], t["w8"], t["w8s"], t["hid"], bias=t["b1"], act="gelu_tanh", dev_status=t["status"])
    toma.toma_linear_act(t["hid"], t["w2"], t["s"], bias=t["b2"], residual=t["s"], dev_status=t["status"])
    toma.toma_rms_norm(t["s"], t["nw"], t["y"])


def chain_state(toma, rows, seed, dim=640, hidden=2560):
    g = generator(rows, seed, 77)
    t = {"x": rand(g, rows, dim, dtype=BF16), "delta": rand(g, rows, dim, dtype=BF16), "nw": rand(g, dim, dtype=BF16)}
    t["w1"] = rand(g, dim, hidden, dtype=BF16) / math.sqrt(dim)
    t["w2"], t["b1"], t["b2"] = rand(g, hidden, dim, dtype=BF16) / math.sqrt(hidden), rand(g, hidden, dtype=BF16), rand(g, dim, dtype=BF16)
    t["w8"], t["w8s"] = torch.empty(hidden, dim, dtype=F8, device="cuda"), torch.empty(hidden, device="cuda")
    toma.toma_quantise_weight(t["w1"], t["w8"], t["w8s"])
    t["q"], t["qs"] = torch.empty(rows, dim, dtype=F8, device="cuda"), torch.empty(rows, device="cuda")
    t["hid"] = torch.empty(rows, hidden, dtype=BF16, device="cuda")
    t["s"], t["y"] = torch.empty_like(t["x"]), torch.empty_like(t["x"])
    t["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    return t


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 5, 77, 300, 4096])
def test_operators_in_a_row_eager_captured_and_on_another_stream(toma, rows):
    t = chain_state(toma, rows, 0)
    chain(toma, t)
    torch.cuda.synchronize()
    assert int(t["status"]) == 0
    h = (t["x"].float() + t["delta"].float()).to(BF16)
    p = h.double() * t["nw"].double()
    q = to_e4m3(p * 448 / p.abs().amax(1, keepdim=True))
    assert torch.equal(t["q"].double(), q)
    assert_linear(t["hid"], t["q"].float(), t["w8"].float().t(), t["b1"], "gelu_tanh", None, t["qs"], t["w8s"])
    assert_linear(t["s"], t["hid"], t["w2"], t["b2"], "none", h)
    want = {k: t[k].clone() for k in ("s", "y", "hid")}
    # captured into a graph, replayed on new inputs in the same buffers
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        chain(toma, t)
    other = chain_state(toma, rows, 1)
    chain(toma, other)
    for k in ("x", "delta", "nw", "w1", "w2", "b1", "b2", "w8", "w8s"):
        t[k].copy_(other[k])
    graph.replay()
    torch.cuda.synchronize()
    for k in want:
        assert torch.equal(t[k], other[k]), k
    # eagerly on a stream of its own beside another problem on the default one
    first = chain_state(toma, rows, 0)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(5):
            chain(toma, first)
    for _ in range(5):
        chain(toma, other)
    torch.cuda.synchronize()
    for k in want:
        assert torch.equal(first[k], want[k]) and torch.equal(t[k], other[k]), k
