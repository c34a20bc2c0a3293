"""Low-rank adapters against the formulas in 64 bits.

Tolerances.  Products of bf16 values are exact in 32 bits; an accumulation step
of the tensor cores (16 products) is taken to cost at most e = 2^-22 of the sum of
the magnitudes so far, and so does a 32-bit addition.  A contraction of length L
in up to 6 bf16 terms then errs by at most c(L) = (6 L / 16 + 40) e times the sum
of its terms' magnitudes (40 steps for partial sums).  v enters expand with 16
bits (2^-16 of itself) for a bf16 result and with 24 (2^-23) for an fp32 one, and
grad with 24; results are rounded once (bf16: 2^-8, fp32: 2^-24).  Errors of v and
du pass on through the magnitudes of what they are multiplied by."""
import pytest
import torch

import paper_1701_00485_gb300 as tbn

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
E = 2.0 ** -22
D64 = torch.float64


def _c(length):
    return (6 * length / 16 + 40) * E


def _rows(T, K, dtype, g, pad=0, offset=0):
    store = torch.empty(T * (K + pad) + offset, dtype=dtype, device="cuda")
    v = store[offset:].view(T, K + pad)
    v.copy_(torch.empty(T, K + pad, device="cuda").normal_(generator=g))
    return v[:, :K]


def _case(T, K_in, K_out, n, r, xdt=BF16, ydt=BF16, pad=0, offset=0, seed=0, plain=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = dict(x=_rows(T, K_in, xdt, g, pad, offset), dy=_rows(T, K_out, ydt, g, pad, offset),
             base=_rows(T, K_out, ydt, g, pad, offset), dbase=_rows(T, K_in, xdt, g, pad, offset))
    for k, K in (("a", K_in), ("b", K_out)):
        w = torch.empty(n * r * K + offset, dtype=BF16, device="cuda")
        w.copy_(torch.empty(n * r * K + offset, device="cuda").normal_(0, 0.1, generator=g))
        c[k] = w[offset:].view(n, r, K)
    if plain:
        c.update(ids=None, scale=None, ranks=None)
        return c
    # adapters in any order, tokens without one, ids out of range
    ids = torch.randint(-1, n, (T,), generator=g, device="cuda", dtype=torch.int32)
    odd = torch.tensor([n, -5, 2 ** 31 - 1, -2 ** 31], device="cuda").to(torch.int32)
    where = torch.randint(0, 12, (T,), generator=g, device="cuda")
    ids = torch.where(where < 4, odd[where.clamp(max=3)], ids) if T > 8 else ids
    c.update(ids=ids, scale=torch.empty(n, device="cuda").uniform_(-2, 2, generator=g),
             ranks=torch.randint(0, r + 1, (n,), generator=g, device="cuda", dtype=torch.int32))
    return c


def _dense(c):
    """a, b with zeros past the ranks and the tokens' rows of them, scale and
    which tokens have an adapter, in 64 bits."""
    n, r, _ = c["a"].shape
    T = c["x"].shape[0]
    ids = torch.zeros(T, dtype=torch.long, device="cuda") if c["ids"] is None else c["ids"].long()
    has = (ids >= 0) & (ids < n)
    ranks = torch.full((n,), r, device="cuda") if c["ranks"] is None else c["ranks"]
    live = torch.arange(r, device="cuda") < ranks[:, None]
    scale = torch.ones(n, device="cuda", dtype=D64) if c["scale"] is None else c["scale"].to(D64)
    a, b = (torch.where(live[:, :, None], c[k].to(D64), 0.0) for k in "ab")
    return ids.clamp(0, n - 1), has, a, b, scale, live


def _forward64(c, base):
    """(y, v, bound on the error before the output's rounding) with 16 and 24 bits of v."""
    ids, has, a, b, scale, _ = _dense(c)
    x = c["x"].to(D64)
    T = x.shape[0]
    v, va = torch.zeros(T, a.shape[1], dtype=D64, device="cuda"), None
    va = torch.zeros_like(v)
    y = torch.zeros(T, b.shape[2], dtype=D64, device="cuda") if base is None else base.to(D64).clone()
    ya, yv = y.abs(), torch.zeros_like(y)
    for i in range(a.shape[0]):
        t = ((ids == i) & has).nonzero()[:, 0]
        if not t.numel():
            continue
        v[t], va[t] = x[t] @ a[i].t(), x[t].abs() @ a[i].abs().t()
        s = scale[i]
        y[t] += s * v[t] @ b[i]
        mag = s.abs() * v[t].abs() @ b[i].abs()
        ya[t] += mag
        yv[t] += _c(x.shape[1]) * s.abs() * va[t] @ b[i].abs()     # what v carries
    bound = lambda out: yv + (_c(a.shape[1]) + (2.0 ** -16 if out == BF16 else 2.0 ** -23)) * ya  # noqa: E731
    return y, v, _c(x.shape[1]) * va, bound


def _round(dt):
    return 2.0 ** -8 if dt == BF16 else 2.0 ** -24


# (T, K_in, K_out, n, r)
SHAPES = [(1, 64, 64, 1, 8), (1, 4096, 4096, 3, 16), (2, 7, 5, 2, 1), (5, 1001, 515, 3, 13),
          (63, 128, 192, 4, 16), (64, 520, 136, 7, 33), (65, 192, 1000, 64, 4), (130, 2048, 72, 2, 64),
          (200, 300, 260, 200, 20), (300, 1024, 1024, 5, 128), (777, 256, 320, 3, 100),
          (1500, 640, 704, 9, 32), (300, 1, 1, 2, 3), (257, 4100, 1028, 1, 16)]


# many bf16 tokens in aligned rows: ranks of each padded size, one adapter and
# many, widths that end inside a tile, tokens that end inside one
MANY = [(513, 4096, 328, 3, 12), (129, 64, 8, 1, 16), (2050, 1032, 2000, 2, 17), (1300, 512, 136, 40, 48),
        (700, 264, 520, 5, 65), (5000, 1024, 768, 3, 32), (9001, 256, 384, 2, 16), (400, 8, 4096, 2, 128)]


@pytest.mark.parametrize("T,K_in,K_out,n,r", MANY)
def test_many_tokens(T, K_in, K_out, n, r):
    test_forward(T, K_in, K_out, n, r, BF16, BF16)
    test_backward(T, K_in, K_out, n, r, BF16, BF16)


@pytest.mark.parametrize("T,K_in,K_out,n,r", SHAPES)
@pytest.mark.parametrize("xdt,ydt", [(BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16)])
def test_forward(T, K_in, K_out, n, r, xdt, ydt):
    for pad, offset, plain in ((0, 0, False), (8, 8, True), (3, 1, False)):
        c = _case(T, K_in, K_out, n, r, xdt, ydt, pad, offset, seed=T + r, plain=plain)
        for base in (None, c["base"]):
            v = torch.full((T, r), 7.0, device="cuda")
            y = tbn.tbn_adapter_fwd(c["x"], c["a"], c["b"], ids=c["ids"], scale=c["scale"],
                                    ranks=c["ranks"], base=base, out_dtype=ydt, v=v)
            y64, v64, v_bound, bound = _forward64(c, base)
            assert y.dtype == ydt
            assert ((y.to(D64) - y64).abs() <= bound(ydt) + _round(ydt) * (y64.abs() + bound(ydt))).all()
            assert ((v.to(D64) - v64).abs() <= v_bound).all()
            _, has, _, _, _, _ = _dense(c)
            rest = torch.zeros_like(y) if base is None else base
            assert torch.equal(y[~has], rest[~has])
    assert tbn.tbn_device_error() == 0


def _backward64(c, v, base):
    ids, has, a, b, scale, live = _dense(c)
    x, dy = c["x"].to(D64), c["dy"].to(D64)
    v = v.to(D64)
    dx = torch.zeros_like(x) if base is None else base.to(D64).clone()
    bx, da, db = dx.abs() * _c(16), torch.zeros_like(a), torch.zeros_like(b)
    ba, bb = torch.zeros_like(a), torch.zeros_like(b)
    for i in range(a.shape[0]):
        t = ((ids == i) & has).nonzero()[:, 0]
        if not t.numel():
            continue
        s, L = scale[i], t.numel()
        du, mag = s * dy[t] @ b[i].t(), s.abs() * dy[t].abs() @ b[i].abs().t()
        err = _c(dy.shape[1]) * mag
        dx[t] += du @ a[i]
        bx[t] += err @ a[i].abs() + (_c(a.shape[1]) + 2.0 ** -16) * (du.abs() @ a[i].abs())
        da[i] = du.t() @ x[t]
        ba[i] = err.t() @ x[t].abs() + (_c(L) + 2.0 ** -21) * (du.abs().t() @ x[t].abs())
        vi = v[t] * live[i]
        db[i] = s * vi.t() @ dy[t]
        bb[i] = (_c(L) + 2.0 ** -21) * s.abs() * (vi.abs().t() @ dy[t].abs())
        # v may have been computed by the library
        bb[i] += s.abs() * (_c(x.shape[1]) * (x[t].abs() @ a[i].abs().t())).t() @ dy[t].abs()
    return dx, da, db, bx, ba, bb


@pytest.mark.parametrize("T,K_in,K_out,n,r", SHAPES)
@pytest.mark.parametrize("xdt,ydt", [(BF16, BF16), (F32, F32), (F32, BF16)])
def test_backward(T, K_in, K_out, n, r, xdt, ydt):
    for pad, offset, plain in ((0, 0, False), (8, 8, True), (3, 1, False)):
        c = _case(T, K_in, K_out, n, r, xdt, ydt, pad, offset, seed=2 * T + r, plain=plain)
        ad = {k: c[k] for k in ("ids", "scale", "ranks")}
        v64 = _forward64(c, None)[1]
        for base, v in ((None, None), (c["dbase"], v64.float())):
            dx, da, db = tbn.tbn_adapter_bwd(c["dy"], c["x"], c["a"], c["b"], v=v, base=base, **ad)
            dx64, da64, db64, bx, ba, bb = _backward64(c, v64, base)
            assert ((dx.to(D64) - dx64).abs() <= bx + _round(xdt) * (dx64.abs() + bx)).all()
            assert ((da.to(D64) - da64).abs() <= ba).all()
            assert ((db.to(D64) - db64).abs() <= bb).all()
            # past the rank and for adapters without tokens: zeros
            _, has, _, _, _, live = _dense(c)
            assert not da[~live].any() and not db[~live].any()
    assert tbn.tbn_device_error() == 0


def test_gradients_match_differences():
    """(L(p + h d) - L(p - h d)) / 2h of L = sum(y dy), in 64 bits, for x, a and b."""
    c = _case(90, 96, 112, 3, 8, F32, F32, seed=4)
    ad = {k: c[k] for k in ("ids", "scale", "ranks")}
    dx, da, db = tbn.tbn_adapter_bwd(c["dy"], c["x"], c["a"], c["b"], **ad)
    at = {k: c[k].to(D64) for k in "xab"}

    def loss(x, a, b):
        return float((_forward64({**c, "x": x, "a": a, "b": b}, None)[0] * c["dy"].to(D64)).sum())

    for k, grad in (("x", dx), ("a", da), ("b", db)):
        d = torch.randn(at[k].shape, dtype=D64, device="cuda")
        h = 1e-3
        want = (loss(**{**at, k: at[k] + h * d}) - loss(**{**at, k: at[k] - h * d})) / (2 * h)
        got = float((grad.to(D64) * d).sum())
        # the loss is linear in each of the three: what is left is rounding
        assert abs(got - want) <= 1e-4 * float((grad.to(D64) * d).abs().sum())


def test_some_gradients_only_and_equal_bits():
    c = _case(700, 512, 384, 4, 24, seed=5)
    ad = {k: c[k] for k in ("ids", "scale", "ranks")}
    args = (c["dy"], c["x"], c["a"], c["b"])
    full = tbn.tbn_adapter_bwd(*args, **ad)
    again = tbn.tbn_adapter_bwd(*args, **ad)
    assert all(torch.equal(p, q) for p, q in zip(full, again))
    for i in range(3):
        need = tuple(j == i for j in range(3))
        got = tbn.tbn_adapter_bwd(*args, need=need, **ad)
        assert torch.equal(got[i], full[i]) and all(g is None for j, g in enumerate(got) if j != i)
    y = tbn.tbn_adapter_fwd(c["x"], c["a"], c["b"], base=c["base"], **ad)
    z = c["base"].clone()
    assert tbn.tbn_adapter_fwd(c["x"], c["a"], c["b"], base=z, out=z, **ad) is z and torch.equal(z, y)
    dx = c["dbase"].clone()
    want = tbn.tbn_adapter_bwd(*args, base=c["dbase"], need=(True, False, False), **ad)[0]
    got = tbn.tbn_adapter_bwd(*args, base=dx, dx=dx, need=(True, False, False), **ad)[0]
    assert torch.equal(got, want)


@pytest.mark.parametrize("T", [9, 700])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_nothing_passes_from_one_request_to_another(T, bad):
    c = _case(T, 256, 264, 3, 12, seed=6)
    c["ids"] = (torch.arange(T, device="cuda") % 4 - 1).to(torch.int32)
    c["ranks"] = torch.tensor([12, 5, 12], device="cuda", dtype=torch.int32)
    ad = {k: c[k] for k in ("ids", "scale", "ranks")}
    run = lambda c: (tbn.tbn_adapter_fwd(c["x"], c["a"], c["b"], base=c["base"], **ad),  # noqa: E731
                     *tbn.tbn_adapter_bwd(c["dy"], c["x"], c["a"], c["b"], base=c["dbase"], **ad))
    y, dx, da, db = run(c)
    other = c["ids"] != 2
    # another adapter's weights
    a2, b2 = c["a"].clone(), c["b"].clone()
    a2[2], b2[2] = bad, bad
    y2, dx2, da2, db2 = run({**c, "a": a2, "b": b2})
    assert torch.equal(y2[other], y[other]) and torch.equal(dx2[other], dx[other])
    assert torch.equal(da2[:2], da[:2]) and torch.equal(db2[:2], db[:2])
    assert not torch.isfinite(y2[~other].float()).any()
    # what lies past a rank
    a2, b2 = c["a"].clone(), c["b"].clone()
    a2[1, 5:], b2[1, 5:] = bad, bad
    assert all(torch.equal(p, q) for p, q in zip(run({**c, "a": a2, "b": b2}), (y, dx, da, db)))
    # one token's activations and gradient
    x2, dy2 = c["x"].clone(), c["dy"].clone()
    x2[5], dy2[5] = bad, bad
    y2, dx2, da2, db2 = run({**c, "x": x2, "dy": dy2})
    i = int(c["ids"][5])
    keep = torch.arange(T, device="cuda") != 5
    assert i == 0 and torch.equal(y2[keep], y[keep]) and torch.equal(dx2[keep], dx[keep])
    assert torch.equal(da2[1:], da[1:]) and torch.equal(db2[1:], db[1:])
    assert not torch.isfinite(y2[5].float()).any() and not torch.isfinite(da2[0]).any()
    # infinite activations of a token without an adapter
    x2 = c["x"].clone()
    x2[4] = bad
    assert torch.equal(run({**c, "x": x2})[0], y)


def test_no_tokens_and_no_adapters():
    c = _case(0, 64, 72, 3, 8, plain=True)
    assert tbn.tbn_adapter_fwd(c["x"], c["a"], c["b"]).shape == (0, 72)
    da, db = torch.ones(3, 8, 64, device="cuda"), torch.ones(3, 8, 72, device="cuda")
    dx, da, db = tbn.tbn_adapter_bwd(c["dy"], c["x"], c["a"], c["b"], da=da, db=db)
    assert dx.shape == (0, 64) and not da.any() and not db.any()
    c = _case(100, 64, 72, 3, 8)
    none = torch.full((100,), -1, dtype=torch.int32, device="cuda")
    assert torch.equal(tbn.tbn_adapter_fwd(c["x"], c["a"], c["b"], ids=none, base=c["base"]), c["base"])
    dx, da, db = tbn.tbn_adapter_bwd(c["dy"], c["x"], c["a"], c["b"], ids=none)
    assert not dx.any() and not da.any() and not db.any()


@pytest.mark.parametrize("T,dt", [(3, BF16), (150, BF16), (3, F32), (150, F32)])
def test_writes_stay_inside_the_rows(T, dt):
    c = _case(T, 200, 300, 2, 16, dt, dt, seed=8)
    ad = {k: c[k] for k in ("ids", "scale", "ranks")}
    out = torch.full((T + 2, 320), 7.0, dtype=dt, device="cuda")
    y = tbn.tbn_adapter_fwd(c["x"], c["a"], c["b"], base=c["base"], out=out[1:-1, :300], **ad)
    assert torch.equal(y, tbn.tbn_adapter_fwd(c["x"], c["a"], c["b"], base=c["base"], **ad))
    out[1:-1, :300] = 7.0
    assert (out == 7.0).all()
    n = tbn.tbn_adapter_workspace_bytes(T, 200, 300, 2, 16, backward=True)
    ws = torch.full((n + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    wide = {k: torch.full((k[1] + 128,), 7.0, device="cuda") for k in (("da", 2 * 16 * 200), ("db", 2 * 16 * 300))}
    da, db = (wide[k][64:-64].view(2, 16, -1) for k in wide)
    got = tbn.tbn_adapter_bwd(c["dy"], c["x"], c["a"], c["b"], dx=out[1:-1, :200], da=da, db=db,
                              workspace=ws[256:256 + n], **ad)
    want = tbn.tbn_adapter_bwd(c["dy"], c["x"], c["a"], c["b"], **ad)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    out[1:-1, :200] = 7.0
    assert (out == 7.0).all() and (ws[:256] == 0x5A).all() and (ws[256 + n:] == 0x5A).all()
    for t in wide.values():
        assert (t[:64] == 7.0).all() and (t[-64:] == 7.0).all()


def test_row_offsets_past_32_bits():
    """Rows 2^30 elements apart: the last one starts beyond element 2^31."""
    T, K, ld = 4, 128, 1 << 30
    g = torch.Generator(device="cuda").manual_seed(9)
    store = torch.empty(3 * ld + K, dtype=BF16, device="cuda")
    far = store.as_strided((T, K), (ld, 1))
    c = _case(T, K, K, 2, 8, seed=9)
    far.copy_(c["x"])
    ids = torch.tensor([0, 1, -1, 1], dtype=torch.int32, device="cuda")
    want = tbn.tbn_adapter_fwd(c["x"], c["a"], c["b"], ids=ids, base=c["base"])
    assert torch.equal(tbn.tbn_adapter_fwd(far, c["a"], c["b"], ids=ids, base=c["base"]), want)
    tbn.tbn_adapter_fwd(far, c["a"], c["b"], ids=ids, base=c["base"], out=far)
    assert torch.equal(far, want)
    far.copy_(c["x"])
    gamma = torch.ones(K, device="cuda")
    y, mean, rstd = tbn.tbn_layernorm_fwd(c["x"], gamma)
    assert torch.equal(tbn.tbn_layernorm_fwd(far, gamma)[0], y)
    dx = tbn.tbn_layernorm_bwd(c["dy"], c["x"], mean, rstd, gamma)[0]
    assert torch.equal(tbn.tbn_layernorm_bwd(c["dy"], far, mean, rstd, gamma, dx=far)[0], dx)
    del store, far
    torch.cuda.empty_cache()
    assert g is not None


@pytest.mark.parametrize("T,K_in,K_out,n,r", [(1, 200, 300, 2, 16), (150, 200, 304, 3, 100), (383, 256, 72, 5, 20),
                                              (700, 512, 384, 4, 32), (900, 136, 1000, 30, 128)])
@pytest.mark.parametrize("dt,pad", [(BF16, 0), (BF16, 3), (F32, 0), (F32, 3)])
def test_workspaces_and_results_have_the_stated_sizes(T, K_in, K_out, n, r, dt, pad):
    """What lies around the workspace, v, da and db stays as it is, and the
    workspace's former contents do not matter."""
    c = _case(T, K_in, K_out, n, r, dt, dt, pad, seed=T)
    ad = {k: c[k] for k in ("ids", "scale", "ranks")}

    def scratch(backward, fill):
        size = tbn.tbn_adapter_workspace_bytes(T, K_in, K_out, n, r, backward=backward)
        ws = torch.full((size + 512,), fill, dtype=torch.uint8, device="cuda")
        return ws, ws[256:256 + size]

    def whole(ws, fill):
        return bool((ws[:256] == fill).all() and (ws[-256:] == fill).all())

    out = []
    for fill in (0x00, 0xFF):
        guard, ws = scratch(False, fill)
        v = torch.full((T * r + 128,), 7.0, device="cuda")
        y = tbn.tbn_adapter_fwd(c["x"], c["a"], c["b"], base=c["base"], v=v[64:-64].view(T, r), workspace=ws, **ad)
        assert whole(guard, fill) and (v[:64] == 7.0).all() and (v[-64:] == 7.0).all()
        wide = [torch.full((n * r * K + 128,), 7.0, device="cuda") for K in (K_in, K_out)]
        guard, ws = scratch(True, fill)
        dx, da, db = tbn.tbn_adapter_bwd(c["dy"], c["x"], c["a"], c["b"], v=v[64:-64].view(T, r), base=c["dbase"],
                                         da=wide[0][64:-64].view(n, r, K_in), db=wide[1][64:-64].view(n, r, K_out),
                                         workspace=ws, **ad)
        assert whole(guard, fill)
        assert all((t[:64] == 7.0).all() and (t[-64:] == 7.0).all() for t in wide)
        out.append((y, v[64:-64], dx, da, db))
    assert all(torch.equal(p, q) for p, q in zip(*out))
    assert tbn.tbn_device_error() == 0


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("T", [300, 1500])
def test_as_many_adapters_as_there_may_be(T, dt):
    test_forward(T, 72, 64, 1023, 4, dt, dt)
    test_backward(T, 72, 64, 1023, 4, dt, dt)


@pytest.mark.parametrize("dt,ld", [(BF16, 1 << 23), (BF16, (1 << 23) + 1), (F32, 1 << 23)])
def test_tiles_of_rows_past_32_bits(dt, ld):
    """520 rows, the last of which begins beyond element 2^32."""
    T, K = 520, 128
    c = _case(T, K, K, 2, 8, dt, dt, seed=19)
    ad = {k: c[k] for k in ("ids", "scale", "ranks")}
    pad = 1 if ld % 2 else 0   # the same kernels for the rows that stand together
    near = {k: _rows(T, K, dt, torch.Generator(device="cuda").manual_seed(1), pad) for k in ("x", "dy", "base")}
    store = torch.empty((T - 1) * ld + K, dtype=dt, device="cuda")
    far = store.as_strided((T, K), (ld, 1))
    for k in near:
        near[k].copy_(c[k])
    want = tbn.tbn_adapter_fwd(near["x"], c["a"], c["b"], base=near["base"], **ad)
    far.copy_(near["x"])
    assert torch.equal(tbn.tbn_adapter_fwd(far, c["a"], c["b"], base=near["base"], **ad), want)
    grads = tbn.tbn_adapter_bwd(near["dy"], near["x"], c["a"], c["b"], base=near["base"], **ad)
    got = tbn.tbn_adapter_bwd(near["dy"], far, c["a"], c["b"], base=near["base"], **ad)
    assert all(torch.equal(p, q) for p, q in zip(got, grads))
    far.copy_(near["base"])   # the base, overwritten by the result
    tbn.tbn_adapter_fwd(near["x"], c["a"], c["b"], base=far, out=far, **ad)
    assert torch.equal(far, want)
    del store, far
    torch.cuda.empty_cache()


def test_on_another_stream():
    c = _case(500, 256, 256, 4, 16, seed=10)
    ad = {k: c[k] for k in ("ids", "scale", "ranks")}
    want = tbn.tbn_adapter_fwd(c["x"], c["a"], c["b"], base=c["base"], **ad)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = tbn.tbn_adapter_fwd(c["x"], c["a"], c["b"], base=c["base"], stream=s, **ad)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)


def test_in_a_graph():
    """Captured once, replayed with other ids and activations."""
    c = _case(40, 512, 512, 6, 16, seed=11)
    ad = {k: c[k] for k in ("ids", "scale", "ranks")}
    ws = torch.empty(tbn.tbn_adapter_workspace_bytes(40, 512, 512, 6, 16), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(c["base"])
    call = lambda: tbn.tbn_adapter_fwd(c["x"], c["a"], c["b"], base=c["base"], out=out, workspace=ws, **ad)  # noqa: E731
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    d = _case(40, 512, 512, 6, 16, seed=12)
    c["x"].copy_(d["x"])
    c["ids"].copy_(d["ids"])
    graph.replay()
    got = out.clone()
    assert torch.equal(got, tbn.tbn_adapter_fwd(c["x"], c["a"], c["b"], base=c["base"], **ad))


def test_refusals():
    c = _case(8, 64, 64, 2, 8)
    x, a, b = c["x"], c["a"], c["b"]
    for bad in (dict(ids=torch.zeros(7, dtype=torch.int32, device="cuda")),
                dict(ids=torch.zeros(8, dtype=torch.int64, device="cuda")),
                dict(scale=torch.ones(3, device="cuda")), dict(base=c["base"].float(), out=c["base"]),
                dict(ranks=torch.ones(2, device="cuda")), dict(v=torch.empty(8, 7, device="cuda"))):
        with pytest.raises(ValueError):
            tbn.tbn_adapter_fwd(x, a, b, **bad)
    with pytest.raises(ValueError):
        tbn.tbn_adapter_fwd(x, a.float(), b)
    with pytest.raises(ValueError):
        tbn.tbn_adapter_fwd(x[:, :32], a, b)
    with pytest.raises(ValueError):
        tbn.tbn_adapter_fwd(x, a, b[:, :4])
    with pytest.raises(TypeError):
        tbn.tbn_adapter_fwd(x.to(torch.float16), a, b)
    with pytest.raises(tbn.TBNError):
        tbn.tbn_adapter_fwd(x, a, b, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        tbn.tbn_adapter_bwd(c["dy"][:, :32], x, a, b)
    with pytest.raises(ValueError):
        tbn.tbn_adapter_bwd(c["dy"], x, a, b, dx=torch.empty(8, 64, device="cuda"))
