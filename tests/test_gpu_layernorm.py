"""Layer norm forward and backward against the formulas in 64 bits.

Tolerances.  u = 2^-24.  A sum over a row of D elements runs through a thread's
own at most 32 (a long row's D / 1024) and 10 shuffle and block steps, so mean
is off by at most n u mean|x| with n = 42 + D / 1024, the variance and with it
rstd by a relative n + 8 u or so (half of it for the root, twice for the squares
of the centred values), and y by the products' own roundings.  With |mean| of
the inputs at most 8 standard deviations,
  |y - y64| <= u (8 n + (2 n + 16) |xh|) |gamma| + 4 u |y|,
plus half a unit of the output's type.  dx has two more sums of the same kind:
  |dx - dx64| <= rstd u ((4 n + 40) (|w| + (1 + |xh|) mean (|w| (1 + |xh|))) + 8 n max|w|)
  + 4 u |dx|, plus the output's rounding; sums over the rows add their chain's
length times u times the sum of the terms' magnitudes."""
import pytest
import torch

import paper_1701_00485_gb300 as tbn

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF16_HALF = 2.0 ** -8   # 7 stored mantissa bits: a unit is 2^-7 of the binade
F32, BF16 = torch.float32, torch.bfloat16


def _inputs(rows, D, dtype, seed=0, pad=0, offset=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.empty(rows * (D + pad) + offset, device="cuda").normal_(0, 1.5, generator=g)
    x = flat[offset:].view(rows, D + pad) + torch.empty(rows, 1, device="cuda").normal_(0, 2, generator=g)
    store = torch.empty(rows * (D + pad) + offset, dtype=dtype, device="cuda")
    v = store[offset:].view(rows, D + pad)
    v.copy_(x)
    return v[:, :D]


def _reference(x, gamma, beta, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    rstd = ((x - mean).square().mean(1, keepdim=True) + eps).rsqrt()
    xh = (x - mean) * rstd
    g = torch.ones(x.shape[1], dtype=torch.float64, device="cuda") if gamma is None else gamma.double()
    b = 0.0 if beta is None else beta.double()
    return xh * g + b, mean[:, 0], rstd[:, 0], xh, g


def _gradients(x, dy, mean, rstd, gamma, dres):
    """The formulas in 64 bits with the given mean and rstd."""
    x, dy = x.double(), dy.double()
    rstd = rstd.double()[:, None]
    xh = (x - mean.double()[:, None]) * rstd
    w = dy if gamma is None else dy * gamma.double()
    dx = rstd * (w - w.mean(1, keepdim=True) - xh * (w * xh).mean(1, keepdim=True))
    if dres is not None:
        dx = dx + dres.double()
    return dx, (dy * xh).sum(0), dy.sum(0), xh, w


SHAPES = [(1, 1), (3, 1), (5, 7), (2, 64), (33, 65), (7, 128), (19, 200), (300, 256), (4, 511),
          (9, 512), (64, 520), (1, 4096), (37, 4097), (11, 8192), (5, 8200), (3, 16384), (2, 32768),
          (3, 40001)]


@pytest.mark.parametrize("rows,D", SHAPES)
@pytest.mark.parametrize("xdt,ydt", [(BF16, BF16), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("pad,offset", [(0, 0), (8, 8), (3, 1)])
def test_forward_and_backward(rows, D, xdt, ydt, pad, offset):
    x = _inputs(rows, D, xdt, 1, pad, offset)
    gamma = 1 + 0.3 * torch.randn(D, device="cuda")
    beta = torch.randn(D, device="cuda")
    y, mean, rstd = tbn.tbn_layernorm_fwd(x, gamma, beta, eps=1e-5, out_dtype=ydt)
    y64, mean64, rstd64, xh, g = _reference(x, gamma, beta, 1e-5)
    n = 42 + D / 1024
    out = BF16_HALF if ydt == BF16 else U
    assert ((mean - mean64).abs() <= n * U * x.double().abs().mean(1) + U * mean64.abs()).all()
    # rows of one value: the variance is that of the mean's rounding
    floor = (n * U * x.double().abs().mean(1)).square()
    assert ((rstd - rstd64).abs() <= rstd64 * ((n + 8) * U + floor * rstd64.square())).all()
    tol = U * (8 * n + (2 * n + 16) * xh.abs()) * g.abs() * (1 + floor * rstd64.square())[:, None] + \
        (4 * U + out) * y64.abs()
    if D == 1:   # xh is the mean's rounding times rstd
        tol = tol + (x.double().abs() * 4 * U * rstd64[:, None]) * g.abs()
    assert ((y.double() - y64).abs() <= tol).all()

    dy = _inputs(rows, D, ydt, 2, pad, offset)
    dres = _inputs(rows, D, xdt, 3, pad, offset)
    for res in (None, dres):
        dx, dg, db = tbn.tbn_layernorm_bwd(dy, x, mean, rstd, gamma, dres=res)
        dx64, dg64, db64, xh, w = _gradients(x, dy, mean, rstd, gamma, res)
        wa = w.abs()
        tol = rstd.double()[:, None] * U * (
            (4 * n + 40) * (wa + (1 + xh.abs()) * (wa * (1 + xh.abs())).mean(1, keepdim=True)) +
            8 * n * wa.amax(1, keepdim=True)) + (4 * U + (BF16_HALF if xdt == BF16 else U)) * dx64.abs()
        assert dx.dtype == xdt and ((dx.double() - dx64).abs() <= tol).all()
        chain = rows + 64
        assert ((dg - dg64).abs() <= (chain + 8) * U * (dy.double() * xh).abs().sum(0) + 1e-30).all()
        assert ((db - db64).abs() <= chain * U * dy.double().abs().sum(0) + 1e-30).all()
    assert tbn.tbn_device_error() == 0


# many rows: teams with rings, an odd number of rows, strides, short rows four at once
@pytest.mark.parametrize("rows,D", [(1301, 264), (5001, 512), (1301, 520), (2600, 1000), (1219, 2056),
                                    (1300, 4096), (1217, 8192), (1217, 8200), (9001, 64), (5003, 72),
                                    (2447, 136), (2441, 256)])
@pytest.mark.parametrize("xdt,ydt", [(BF16, BF16), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("pad,offset", [(0, 0), (24, 16)])
def test_many_rows(rows, D, xdt, ydt, pad, offset):
    test_forward_and_backward(rows, D, xdt, ydt, pad, offset)


# many rows that are not aligned, of each way to spread a row
@pytest.mark.parametrize("rows,D", [(66001, 64), (38001, 111), (21001, 201), (14002, 300), (8501, 505),
                                    (4871, 1001), (4870, 4095), (4871, 7777)])
@pytest.mark.parametrize("xdt,ydt", [(BF16, BF16), (F32, F32), (F32, BF16)])
def test_many_unaligned_rows(rows, D, xdt, ydt):
    test_forward_and_backward(rows, D, xdt, ydt, 3, 1)


def test_many_rows_in_place_and_equal_bits():
    rows, D = 4001, 1024
    x, dy = _inputs(rows, D, BF16, 21), _inputs(rows, D, BF16, 22)
    gamma = 1 + 0.2 * torch.randn(D, device="cuda")
    y, mean, rstd = tbn.tbn_layernorm_fwd(x, gamma)
    z = x.clone()
    assert torch.equal(tbn.tbn_layernorm_fwd(z, gamma, out=z)[0], y)
    first = tbn.tbn_layernorm_bwd(dy, x, mean, rstd, gamma, dres=x)
    again = tbn.tbn_layernorm_bwd(dy, x, mean, rstd, gamma, dres=x)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    for name in ("dy", "dres"):
        t = {"dy": dy.clone(), "dres": x.clone()}
        got = tbn.tbn_layernorm_bwd(t["dy"], x, mean, rstd, gamma, dres=t["dres"], dx=t[name])
        assert all(torch.equal(a, b) for a, b in zip(first, got))
    assert tbn.tbn_device_error() == 0


@pytest.mark.parametrize("gamma,beta", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("wdt", [F32, BF16])
def test_optional_weights_of_either_type(gamma, beta, wdt):
    x = _inputs(13, 1000, BF16, 5)
    ga = (1 + 0.3 * torch.randn(1000, device="cuda")).to(wdt) if gamma else None
    be = torch.randn(1000, device="cuda").to(wdt) if beta else None
    y, mean, rstd = tbn.tbn_layernorm_fwd(x, ga, be)
    y64, _, _, xh, g = _reference(x, ga, be, 1e-5)
    assert ((y.double() - y64).abs() <= U * (344 + 102 * xh.abs()) * g.abs() +
            (4 * U + BF16_HALF) * y64.abs()).all()
    dy = _inputs(13, 1000, BF16, 6)
    dx, _, _ = tbn.tbn_layernorm_bwd(dy, x, mean, rstd, ga, weight_grads=False)
    dx64 = _gradients(x, dy, mean, rstd, ga, None)[0]
    assert ((dx.double() - dx64).abs() <= BF16_HALF * dx64.abs() + 1e-4 * rstd.double()[:, None]).all()


def test_gradients_match_differences():
    """(L(x + h d) - L(x - h d)) / 2h of L = sum(y dy) in 64 bits, for x, gamma
    and beta in random directions; the cubic term is of the order h^2 = 1e-8."""
    rows, D, h = 17, 384, 1e-4
    x = _inputs(rows, D, F32, 7)
    gamma, beta = 1 + 0.2 * torch.randn(D, device="cuda"), torch.randn(D, device="cuda")
    dy = _inputs(rows, D, F32, 8)
    y, mean, rstd = tbn.tbn_layernorm_fwd(x, gamma, beta)
    dx, dg, db = tbn.tbn_layernorm_bwd(dy, x, mean, rstd, gamma)

    def loss(a, g, b):
        return float((_reference(a, g, b, 1e-5)[0] * dy.double()).sum())

    x, gamma, beta = x.double(), gamma.double(), beta.double()
    for k, (grad, at) in enumerate([(dx, x), (dg, gamma), (db, beta)]):
        d = torch.randn(at.shape, dtype=torch.float64, device="cuda")
        args = [x, gamma, beta]
        up, down = list(args), list(args)
        up[k], down[k] = at + h * d, at - h * d
        want = (loss(*up) - loss(*down)) / (2 * h)
        got = float((grad.double() * d).sum())
        scale = float((grad.double() * d).abs().sum())
        assert abs(got - want) <= 2e-5 * scale


def test_in_place_zero_rows_and_repeatability():
    x = _inputs(700, 776, BF16, 9)
    gamma = torch.randn(776, device="cuda")
    y, mean, rstd = tbn.tbn_layernorm_fwd(x, gamma)
    z = x.clone()
    assert torch.equal(tbn.tbn_layernorm_fwd(z, gamma, out=z)[0], y)
    dy = _inputs(700, 776, BF16, 10)
    first = tbn.tbn_layernorm_bwd(dy, x, mean, rstd, gamma, dres=dy)
    again = tbn.tbn_layernorm_bwd(dy, x, mean, rstd, gamma, dres=dy)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    w = dy.clone()
    assert torch.equal(tbn.tbn_layernorm_bwd(w, x, mean, rstd, gamma, dres=w, dx=w)[0], first[0])
    none = torch.empty(0, 776, dtype=BF16, device="cuda")
    y0, m0, r0 = tbn.tbn_layernorm_fwd(none, gamma)
    dx, dg, db = tbn.tbn_layernorm_bwd(none, none, m0, r0, gamma)
    assert dx.shape == (0, 776) and not dg.any() and not db.any()
    # a NaN stays in its row
    x2 = x.clone()
    x2[5, 7] = float("nan")
    y2, m2, r2 = tbn.tbn_layernorm_fwd(x2, gamma)
    keep = torch.arange(700, device="cuda") != 5
    assert torch.equal(y2[keep], y[keep]) and torch.isnan(y2[5].float()).all()


def test_writes_stay_inside_the_rows():
    """What lies between rows, and a second stream's temporaries, stay as they are."""
    rows, D, wide = 41, 300, 320
    x = _inputs(rows, D, BF16, 11)
    gamma = torch.randn(D, device="cuda")
    out = torch.full((rows + 2, wide), 7.0, dtype=BF16, device="cuda")
    y, mean, rstd = tbn.tbn_layernorm_fwd(x, gamma, out=out[1:-1, :D])
    plain = tbn.tbn_layernorm_fwd(x, gamma)[0]
    assert torch.equal(out[1:-1, :D], plain)
    out[1:-1, :D] = 7.0
    assert (out == 7.0).all()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    want = tbn.tbn_layernorm_bwd(plain, x, mean, rstd, gamma)
    got = tbn.tbn_layernorm_bwd(plain, x, mean, rstd, gamma, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("rows,D", [(1, 64), (41, 300), (1300, 136), (1301, 4096), (5000, 505), (1217, 8200)])
@pytest.mark.parametrize("dt", [BF16, F32])
def test_workspaces_and_results_have_the_stated_sizes(rows, D, dt):
    x, dy = _inputs(rows, D, dt, 31), _inputs(rows, D, dt, 32)
    gamma = torch.randn(D, device="cuda")
    size = tbn.tbn_layernorm_bwd_workspace_bytes(rows, D)
    out = []
    for fill in (0x00, 0xFF):
        stats = [torch.full((rows + 128,), 7.0, device="cuda") for _ in range(2)]
        y, mean, rstd = tbn.tbn_layernorm_fwd(x, gamma, mean=stats[0][64:-64], rstd=stats[1][64:-64])
        ws = torch.full((size + 512,), fill, dtype=torch.uint8, device="cuda")
        sums = [torch.full((D + 128,), 7.0, device="cuda") for _ in range(2)]
        dx, dgamma, dbeta = tbn.tbn_layernorm_bwd(dy, x, mean, rstd, gamma, dgamma=sums[0][64:-64],
                                                  dbeta=sums[1][64:-64], workspace=ws[256:256 + size])
        assert (ws[:256] == fill).all() and (ws[-256:] == fill).all()
        assert all((t[:64] == 7.0).all() and (t[-64:] == 7.0).all() for t in stats + sums)
        out.append((y, dx, dgamma, dbeta))
    assert all(torch.equal(p, q) for p, q in zip(*out))


@pytest.mark.parametrize("dt,ld", [(BF16, 1 << 22), (BF16, (1 << 22) + 1), (F32, 1 << 22)])
def test_many_rows_past_32_bits(dt, ld):
    """1300 rows, the last of which begins beyond element 2^32."""
    rows, D = 1300, 264
    g = torch.Generator(device="cuda").manual_seed(5)
    near = torch.empty((rows, D + (1 if ld % 2 else 0)), dtype=dt, device="cuda")[:, :D]
    near.copy_(torch.empty((rows, D), device="cuda").normal_(generator=g))
    store = torch.empty((rows - 1) * ld + D, dtype=dt, device="cuda")
    far = store.as_strided((rows, D), (ld, 1))
    far.copy_(near)
    gamma = torch.randn(D, device="cuda")
    y, mean, rstd = tbn.tbn_layernorm_fwd(near, gamma)
    assert torch.equal(tbn.tbn_layernorm_fwd(far, gamma)[0], y)
    want = tbn.tbn_layernorm_bwd(y, near, mean, rstd, gamma, dres=near)
    got = tbn.tbn_layernorm_bwd(y, far, mean, rstd, gamma, dres=far, dx=far)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    del store, far
    torch.cuda.empty_cache()


def test_refusals():
    x = torch.zeros(4, 64, device="cuda")
    with pytest.raises(ValueError):
        tbn.tbn_layernorm_fwd(x.cpu())
    with pytest.raises(ValueError):
        tbn.tbn_layernorm_fwd(x.t())            # rows not contiguous
    with pytest.raises(ValueError):
        tbn.tbn_layernorm_fwd(x, torch.zeros(63, device="cuda"))
    with pytest.raises(TypeError):
        tbn.tbn_layernorm_fwd(x.to(torch.float16))
    with pytest.raises(tbn.TBNError) as e:
        tbn.tbn_layernorm_fwd(x.to(BF16), out=torch.zeros(4, 64, device="cuda"))
    assert e.value.status == tbn.TBN_ERR_UNSUPPORTED
    m = torch.zeros(4, device="cuda")
    with pytest.raises(tbn.TBNError):
        tbn.tbn_layernorm_bwd(x, x, m, m, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        tbn.tbn_layernorm_bwd(x, x, m[:3], m)
