"""The AdamW step against the formula in 64 bits.

Tolerances.  With u = 2^-24, a rounding each: grad * grad_scale, the constants
beta and 1 - beta held in 32 bits, each product, the sum.  m's terms carry at most
4 (constant, scaled gradient, product, sum): 4 u (|beta1 m| + |(1 - beta1) g|).
v's second term carries 6 (constant, the scaled gradient twice, two products,
sum): 6 u v.  The step's term m / (sqrt(v) c + eps) adds at most 8 roundings of
its own (root, constants, quotient, products, the sum's) to m's 4 and half of
v's 6: with the magnitudes' sum M for m,
  |p - p64| <= u (3 |p| + lr' / fix1 (16 M) / den).
8-bit moments are checked where the answer is one of two neighbours of the
format, or exact."""
import math

import pytest
import torch

import paper_1701_00485_gb300 as tbn

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
SIZES = [1, 7, 8, 255, 256, 257, 2048, 2049, 70001]


def _rand(n, dtype, g, std=1.0, offset=0):
    t = torch.empty(n + offset, dtype=dtype, device="cuda")
    t.copy_(torch.empty(n + offset, device="cuda").normal_(0, std, generator=g))
    return t[offset:]


def _step64(p, g, m, v, step, lr, b1, b2, eps, wd, gs):
    g = g.double() * gs
    terms = (b1 * m.double()).abs() + ((1 - b1) * g).abs()
    m = b1 * m.double() + (1 - b1) * g
    v = b2 * v.double() + (1 - b2) * g * g
    den = (v / (1 - b2 ** step)).sqrt() + eps
    p = p.double() * (1 - lr * wd) - lr / (1 - b1 ** step) * m / den
    return p, m, v, terms, den


@pytest.mark.parametrize("pdt", [F32, BF16])
@pytest.mark.parametrize("gdt", [F32, BF16])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("step", [1, 1000])
def test_32_bit_moments(pdt, gdt, offset, step):
    gen = torch.Generator(device="cuda").manual_seed(3)
    P, G = ([_rand(n, d, gen, offset=offset) for n in SIZES] for d in (pdt, gdt))
    M = [_rand(n, F32, gen, 0.1, offset) for n in SIZES]
    V = [_rand(n, F32, gen, 0.3, offset).square_() for n in SIZES]
    C = [_rand(n, BF16, gen, offset=offset) for n in SIZES]
    gs = torch.tensor([0.37], device="cuda")
    wd = [0.01 * (i % 3) for i in range(len(SIZES))]
    lrs = [1.0 + i % 2 for i in range(len(SIZES))]
    want = [_step64(p, g, m, v, step, 1e-2 * l, 0.9, 0.999, 1e-8, w, float(gs))
            for p, g, m, v, w, l in zip(P, G, M, V, wd, lrs)]
    old = [p.double().clone() for p in P]
    plan = tbn.AdamWPlan(P, G, M, V, copies=C, weight_decay=wd, lr_scale=lrs)
    tbn.tbn_adamw_step(plan, step=step, lr=1e-2, grad_scale=gs)
    fix1 = 1 - 0.9 ** step
    for p, m, v, c, o, l, (p64, m64, v64, terms, den) in zip(P, M, V, C, old, lrs, want):
        assert ((m - m64).abs() <= 4 * U * terms).all()
        assert ((v - v64).abs() <= 6 * U * v64).all()
        tol = U * (3 * o.abs() + 16 * 1e-2 * l / fix1 * terms / den)
        assert ((p.double() - p64).abs() <= tol + (2.0 ** -8 * p64.abs() if pdt == BF16 else 0)).all()
        assert ((c.double() - p64).abs() <= tol + 2.0 ** -8 * p64.abs()).all()


def _eight(n, gen, offset=0):
    """8-bit moments of a run in progress, and their values."""
    blocks = -(-n // 256)
    m, v = (torch.zeros(n + offset, dtype=torch.uint8, device="cuda")[offset:] for _ in range(2))
    m.copy_(_rand(n, F32, gen, 40.0).to(E4M3).view(torch.uint8))
    v.copy_((_rand(n, F32, gen, 40.0).square() + 1.0).to(E5M2).view(torch.uint8))
    ms, vs = (torch.exp2(torch.randint(-12, -4, (blocks,), device="cuda", generator=gen).float())
              for _ in range(2))
    return m.view(E4M3), v.view(E5M2), ms, vs


def _values(codes, scale):
    return codes.float() * scale.repeat_interleave(256)[:codes.numel()]


def _neighbours(x, scale, low, digits):
    """The format's values on both sides of x (64 bits, with the block's scale)."""
    s = scale.double().repeat_interleave(256)[:x.numel()]
    a = x.abs() / s
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=1e-300))).clamp(min=low) - digits)
    return torch.floor(a / step) * step * s, torch.ceil(a / step) * step * s


@pytest.mark.parametrize("gdt", [F32, BF16])
@pytest.mark.parametrize("offset", [0, 3])
def test_8_bit_moments(gdt, offset):
    gen = torch.Generator(device="cuda").manual_seed(5)
    P, G = [_rand(n, F32, gen, offset=offset) for n in SIZES], [_rand(n, gdt, gen, 0.2, offset) for n in SIZES]
    S = [_eight(n, gen, offset) for n in SIZES]
    want = [_step64(p, g, _values(m, ms), _values(v, vs), 10, 1e-2, 0.9, 0.99, 1e-8, 0.1, 1.0)
            for p, g, (m, v, ms, vs) in zip(P, G, S)]
    old = [p.double().clone() for p in P]
    tbn.tbn_adamw_step(tbn.AdamWPlan(P, G, *map(list, zip(*S)), weight_decay=0.1), step=10, lr=1e-2,
                       betas=(0.9, 0.99), seed=77)
    for p, (m, v, ms, vs), o, (p64, m64, v64, terms, den) in zip(P, S, old, want):
        assert ((p - p64).abs() <= U * (3 * o.abs() + 16 * 1e-2 / (1 - 0.9 ** 10) * terms / den)).all()
        for code, scale, x, top, low, digits in ((m, ms, m64, 448.0, -6, 3), (v, vs, v64, 57344.0, -14, 2)):
            got = _values(code, scale).double()
            # the least power of two that covers the block
            pad = torch.zeros(-(-x.numel() // 256) * 256, dtype=torch.float64, device="cuda")
            pad[:x.numel()] = x.abs()
            most = pad.view(-1, 256).amax(1)
            assert torch.equal(torch.exp2(torch.log2(scale).round()), scale)
            assert (most <= top * scale.double() * (1 + 8 * U)).all()
            assert (most >= 0.5 * top * scale.double() * (1 - 8 * U)).all()
            lo, hi = _neighbours(x, scale, low, digits)
            slack = 8 * U * (x.abs() + (terms if code is m else 0))   # x itself is rounded to 32 bits
            near = (((got.abs() - lo).abs() <= slack) | ((got.abs() - hi).abs() <= slack))
            assert near.all()
            assert ((got * x >= 0) | (x.abs() <= slack)).all()
        assert (v.view(torch.uint8)[v64 > 0] != 0).all()


def test_rounding_is_unbiased_and_keeps_what_the_format_holds():
    n = 1 << 16
    # beta = 1/2 and g equal to m: m stays as it is, in 32 bits and so in 8
    gen = torch.Generator(device="cuda").manual_seed(6)
    m, _, ms, vs = _eight(n, gen)
    v = torch.exp2(torch.randint(-8, 8, (n,), device="cuda", generator=gen).float() * 2).to(E5M2)
    v.view(-1, 256)[:, 0] = torch.tensor(57344.0, device="cuda").to(E5M2)
    m.view(-1, 256)[:, 0] = torch.tensor(448.0, device="cuda").to(E4M3)
    g = _values(m, ms)
    before, scale = m.clone(), ms.clone()
    p = torch.zeros(n, device="cuda")
    for seed in range(3):
        tbn.tbn_adamw_step(tbn.AdamWPlan([p], [g], [m], [v], [ms], [vs]), step=1, lr=0.0,
                           betas=(0.5, 0.0), seed=seed)
        assert torch.equal(m.view(torch.uint8), before.view(torch.uint8)) and torch.equal(ms, scale)
    # a value between two codes goes up as often as it lies near the upper one:
    # a binomial count of n, within 6 standard deviations
    for part in (0.1, 0.5, 0.8):
        x = 1.0 + part / 8
        g = torch.full((n,), 2 * x, device="cuda")
        g[::256] = 2.0 * 1.75          # one value of the block fixes the scale
        m, v, ms, vs = tbn.AdamWPlan.state8(p)
        tbn.tbn_adamw_step(tbn.AdamWPlan([p], [g], [m], [v], [ms], [vs]), step=1, lr=0.0,
                           betas=(0.5, 0.5), seed=11)
        got = _values(m, ms)
        keep = torch.arange(n, device="cuda") % 256 != 0
        assert ((got[keep] == 1.0) | (got[keep] == 1.125)).all()
        count, many = int((got[keep] == 1.125).sum()), int(keep.sum())
        assert abs(count - many * part) <= 6 * math.sqrt(many * part * (1 - part))
        # and not the same elements for another seed
        m2, v2, ms2, vs2 = tbn.AdamWPlan.state8(p)
        tbn.tbn_adamw_step(tbn.AdamWPlan([p], [g], [m2], [v2], [ms2], [vs2]), step=1, lr=0.0,
                           betas=(0.5, 0.5), seed=12)
        assert not torch.equal(m2.view(torch.uint8), m.view(torch.uint8))


def test_v_follows_small_changes():
    """beta2 = 0.999 towards g = 0: after 1000 steps v is 0.37 of itself on the
    average of many elements, where rounding to nearest would leave it."""
    n = 1 << 14
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    m, v, ms, vs = tbn.AdamWPlan.state8(p)
    v.view(torch.uint8).fill_(0x7B)     # 57344, the format's largest
    vs.fill_(1.0)
    plan = tbn.AdamWPlan([p], [g], [m], [v], [ms], [vs])
    for i in range(1000):
        tbn.tbn_adamw_step(plan, step=i + 1, lr=1e-3, seed=i)
    mean = float(_values(v, vs).double().mean()) / 57344.0
    want = 0.999 ** 1000
    # one element's v is a walk of relative variance below 1000 * 0.001 * 0.25;
    # the mean of n of them lies within 6 standard errors
    assert abs(mean - want) <= 6 * want * math.sqrt(0.5 / n) + 16 * 2.0 ** -16


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_what_is_not_finite_stays_with_its_element(bad):
    gen = torch.Generator(device="cuda").manual_seed(8)
    n = 777
    P, G = _rand(n, F32, gen), _rand(n, F32, gen)
    state = _eight(n, gen)
    runs = []
    for value in (None, bad):
        p, g, st = P.clone(), G.clone(), [t.clone() for t in state]
        if value is not None:
            g[300] = value
        tbn.tbn_adamw_step(tbn.AdamWPlan([p], [g], *[[t] for t in st]), step=5, lr=1e-2, seed=3)
        runs.append((p, _values(st[0], st[2]), _values(st[1], st[3])))
    keep = torch.arange(n, device="cuda") != 300
    # the scale of its block may differ only by what that element itself asked for
    top = [t[256:512][keep[256:512]].abs().max() for t in runs[0]]
    for a, b in zip(runs[0], runs[1]):
        far = torch.ones_like(keep)
        far[256:512] = False
        assert torch.equal(a[far], b[far])
    assert torch.equal(runs[0][0][keep], runs[1][0][keep])
    assert torch.isfinite(runs[1][1][keep]).all() and torch.isfinite(runs[1][2][keep]).all()
    assert torch.isnan(runs[1][0][300]) and torch.isnan(runs[1][1][300])
    assert not torch.isfinite(runs[1][2][300])
    assert all(t > 0 for t in top)


def test_many_tensors_of_all_kinds_in_one_call():
    """More tensors than one launch takes, of mixed types, some empty, equal
    bitwise to calls of their own (with 32-bit moments, which draw nothing)."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    sizes = [(37 * i) % 600 for i in range(800)]
    P = [_rand(n, BF16 if i % 3 == 0 else F32, gen) for i, n in enumerate(sizes)]
    G = [_rand(n, BF16 if i % 2 == 0 else F32, gen) for i, n in enumerate(sizes)]
    M, V = [_rand(n, F32, gen) for n in sizes], [_rand(n, F32, gen).square_() for n in sizes]
    copy = lambda ts: [t.clone() for t in ts]  # noqa: E731
    P2, M2, V2 = copy(P), copy(M), copy(V)
    tbn.tbn_adamw_step(tbn.AdamWPlan(P, G, M, V, weight_decay=0.02), step=3, lr=1e-2)
    for i in range(0, 800, 7):
        tbn.tbn_adamw_step(tbn.AdamWPlan(P2[i:i + 1], G[i:i + 1], M2[i:i + 1], V2[i:i + 1],
                                         weight_decay=0.02), step=3, lr=1e-2)
        assert torch.equal(P[i], P2[i]) and torch.equal(M[i], M2[i]) and torch.equal(V[i], V2[i])
    # 8-bit moments: equal arguments, equal bits
    S = [_eight(n, gen) for n in SIZES]
    P = [_rand(n, F32, gen) for n in SIZES]
    G = [_rand(n, F32, gen) for n in SIZES]
    runs = []
    for _ in range(2):
        p, st = copy(P), [[t.clone() for t in s] for s in S]
        tbn.tbn_adamw_step(tbn.AdamWPlan(p, G, *map(list, zip(*st))), step=3, lr=1e-2, seed=4)
        runs.append(p + [t.view(torch.uint8) if t.dtype != F32 else t for s in st for t in s])
    assert all(torch.equal(a, b) for a, b in zip(*runs))
    tbn.tbn_adamw_step(tbn.AdamWPlan([], [], [], []), step=1, lr=1.0)


def test_neighbouring_memory_is_left_alone():
    gen = torch.Generator(device="cuda").manual_seed(10)
    n = 1000
    fills = {"p": 9.0, "c": -5.0}
    wide = {k: torch.full((n + 64,), fills[k], dtype=d, device="cuda") for k, d in
            (("p", F32), ("c", BF16))}
    codes = {k: torch.full((n + 64,), 0x55, dtype=torch.uint8, device="cuda") for k in "mv"}
    scales = {k: torch.full((4 + 8,), 0.25, device="cuda") for k in "mv"}
    mid = slice(32, 32 + n)
    plan = tbn.AdamWPlan([wide["p"][mid]], [_rand(n, F32, gen)], [codes["m"][mid].view(E4M3)],
                         [codes["v"][mid].view(E5M2)], [scales["m"][4:8]], [scales["v"][4:8]],
                         copies=[wide["c"][mid]])
    tbn.tbn_adamw_step(plan, step=1, lr=0.1, seed=1)
    torch.cuda.synchronize()
    for t, fill, k in ([(t, fills[i], 32) for i, t in wide.items()] + [(t, 0x55, 32) for t in codes.values()] +
                       [(t, 0.25, 4) for t in scales.values()]):
        assert (t[:k] == fill).all() and (t[-k:] == fill).all()
        assert (t[k:-k] != fill).any()


def test_refusals():
    t = lambda n=8, d=F32: torch.zeros(n, dtype=d, device="cuda")  # noqa: E731
    ok = tbn.AdamWPlan([t()], [t()], [t()], [t()])
    for kw in (dict(step=0), dict(lr=-1.0), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1.0),
               dict(lr=float("nan"))):
        with pytest.raises(tbn.TBNError):
            tbn.tbn_adamw_step(ok, **{**dict(step=1, lr=0.1), **kw})
    with pytest.raises(ValueError):
        tbn.AdamWPlan([t()], [t(7)], [t()], [t()])
    with pytest.raises(ValueError):
        tbn.AdamWPlan([t()], [t()], [t()], [])
    with pytest.raises(ValueError):
        tbn.AdamWPlan([t()], [t()], [t(d=E4M3)], [t(d=E5M2)])          # no scales
    with pytest.raises(ValueError):
        tbn.AdamWPlan([t()], [t()], [t(d=E4M3)], [t(d=E4M3)], [t(1)], [t(1)])
    with pytest.raises(ValueError):
        tbn.AdamWPlan([torch.zeros(8)], [t()], [t()], [t()])
    with pytest.raises(ValueError):
        tbn.AdamWPlan([t(16)[::2]], [t()], [t()], [t()])
