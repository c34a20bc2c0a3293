"""Performance cases of the training-step and adapter operators.

Three operators that a program with two-bit projections runs beside them:

* low-rank adapters of many requests at once beside a shared projection
  (``tbn_adapter_fwd``, ``tbn_adapter_bwd``);
* layer norm, forward and backward with the reduction of the weights'
  gradients (``tbn_layernorm_fwd``, ``tbn_layernorm_bwd``);
* an AdamW step over many tensors at once, with states in 32 or in 8 bits
  (``AdamWPlan``, ``tbn_adamw_step``).

``listed`` names the fixed cases, ``draw`` gives more of the same ranges.
``run`` makes the library's calls where ``own`` is set and computes the same
in elementary torch operations where it is not; ``exact`` gives the results in
64 bits, from the definitions.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
BLOCK = 256          # elements that share the scale of an 8-bit state
BETA1, BETA2, EPS = 0.9, 0.999, 1e-8
LN_EPS = 1e-5


# ------------------------------------------------------------------ cases
def listed():
    return [
        # one token of one request: what an adapter adds to a step's latency
        _adapter("adapter_fwd_token", "fwd", T=1, requests=1, n=8, r=16, K_in=8192, K_out=8192),
        # a serving step: one token of each of 64 requests, nearly every one
        # with an adapter of its own, every sixteenth with none
        _adapter("adapter_fwd_decode_64", "fwd", T=64, requests=64, n=96, r=16, K_in=4096,
                 K_out=4096),
        # prompts of ragged lengths together, adapters of different ranks
        _adapter("adapter_fwd_prompts_8k", "fwd", T=8209, requests=20, n=12, r=64, K_in=4096,
                 K_out=8192, mixed_ranks=True),
        # a fine-tuning step of two adapters over one projection
        _adapter("adapter_bwd_8k", "bwd", T=8192, requests=8, n=2, r=32, K_in=4096, K_out=4096),
        # odd sizes in 32 bits, where no row is aligned
        _adapter("adapter_bwd_odd_f32", "bwd", T=777, requests=5, n=3, r=13, K_in=1001, K_out=515,
                 f32=True, mixed_ranks=True),
        # the norm before a single token's projections
        _norm("layernorm_fwd_token", "fwd", rows=1, D=4096),
        # a prompt batch
        _norm("layernorm_fwd_16k", "fwd", rows=16384, D=4096),
        # its training step, with the gradient of the residual branch added
        _norm("layernorm_bwd_16k", "bwd", rows=16384, D=4096, dres=True),
        # rows of odd length inside a wider buffer, in 32 bits
        _norm("layernorm_bwd_odd_f32", "bwd", rows=1111, D=1023, pad=9, f32=True),
        # the update of 256 adapter matrices of one model: fp32 master
        # weights, bf16 gradients and working copies, states in 8 bits
        _adamw("adamw_adapters_8bit", "adapters", tensors=256, size=16 * 4096, bits=8, g_bf16=True,
               copy=True),
        # Algorithm 1's real-valued weights of the ResNet-18 shaped network
        _adamw("adamw_resnet18_f32", "resnet18", bits=32),
        # and of the AlexNet shaped one (61 M weights), states in 8 bits
        _adamw("adamw_alexnet_8bit", "alexnet", bits=8),
    ]


def _adapter(name, direction, T, requests, n, r, K_in, K_out, f32=False, mixed_ranks=False):
    return dict(name=name, op="adapter", direction=direction, T=T, requests=requests, n=n, r=r,
                K_in=K_in, K_out=K_out, f32=f32, mixed_ranks=mixed_ranks)


def _norm(name, direction, rows, D, pad=0, f32=False, dres=False):
    return dict(name=name, op="layernorm", direction=direction, rows=rows, D=D, pad=pad, f32=f32,
                dres=dres)


def _adamw(name, model, bits, tensors=0, size=0, g_bf16=False, copy=False):
    return dict(name=name, op="adamw", model=model, tensors=tensors, size=size, bits=bits,
                g_bf16=g_bf16, copy=copy)


def _log(rng, lo, hi):
    n = max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return n - 1 if n == 3072 else n


def _width(rng, hi=8192):
    """A layer's width: a multiple of 64, of 8, or odd."""
    w = _log(rng, 64, hi)
    w = w // 64 * 64 if rng.random() < 0.6 else w // 8 * 8 if rng.random() < 0.6 else w | 1
    return 3008 if w == 3072 else w


def draw(rng):
    op = rng.choice(["adapter_fwd", "adapter_fwd", "adapter_bwd", "layernorm_fwd", "layernorm_bwd",
                     "adamw"])
    f32 = rng.random() < 0.25
    if op == "adapter_fwd" or op == "adapter_bwd":
        bwd = op == "adapter_bwd"
        T = _log(rng, 16 if bwd else 1, 8192)
        # single tokens of as many requests, or prompts
        requests = T if not bwd and T <= 256 and rng.random() < 0.6 else min(T, _log(rng, 1, 24))
        c = _adapter("", "bwd" if bwd else "fwd", T=T, requests=requests,
                     n=rng.randint(1, 4) if bwd else _log(rng, 1, 64), r=rng.choice([4, 8, 13, 16, 32, 64]),
                     K_in=_width(rng, 4096), K_out=_width(rng, 4096 if bwd else 8192), f32=f32,
                     mixed_ranks=rng.random() < 0.4)
    elif op.startswith("layernorm"):
        D = _width(rng)
        c = _norm("", op[-3:], rows=_log(rng, 1, max(1, (16384 * 4096 >> (1 if f32 else 0)) // D)), D=D,
                  pad=rng.choice([0, 0, 8, 9]), f32=f32, dres=op[-3:] == "bwd" and rng.random() < 0.5)
    else:
        tensors = _log(rng, 1, 400)
        c = _adamw("", "adapters", tensors=tensors, size=_log(rng, 100, 30_000_000 // tensors),
                   bits=rng.choice([8, 32]), g_bf16=rng.random() < 0.5, copy=rng.random() < 0.3)
    del c["name"]
    return c


def _sizes(case):
    """Elements of each tensor of an AdamW case."""
    if case["model"] == "adapters":   # a fourth of them a little shorter, as layers differ
        s = case["size"]
        return [s - s // 7 - 1 if i % 4 == 3 else s for i in range(case["tensors"])]
    if case["model"] == "resnet18":
        sizes, cin = [64 * 3 * 49], 64
        for cout in (64, 128, 256, 512):
            sizes += [cout * cin * 9, cout * cout * 9] + ([cout * cin] if cin != cout else [])
            sizes += [cout * cout * 9] * 2
            cin = cout
        return sizes + [1000 * 512]
    return [96 * 363, 256 * 2400, 384 * 2304, 384 * 3456, 256 * 3456, 9216 * 4096, 4096 * 4096,
            4096 * 1000]


def _ranks(case):
    r = case["r"]
    return [max(1, r >> (i % 3)) if case["mixed_ranks"] else r for i in range(case["n"])]


def _used(case):
    """The adapter of each request (-1: none), before the seed permutes the adapters."""
    many = case["requests"] > 15 and case["direction"] == "fwd"
    return [-1 if many and j % 16 == 15 else j % case["n"] for j in range(case["requests"])]


def work(case):
    if case["op"] == "adapter":
        T, kk, e = case["T"], case["K_in"] + case["K_out"], 4 if case["f32"] else 2
        r = sum(_ranks(case)) / case["n"]
        distinct = len(set(_used(case)) - {-1})
        w = distinct * r * kk
        if case["direction"] == "fwd":      # x, base in, y out, the weights in use
            return {"bytes": T * (case["K_in"] + 2 * case["K_out"]) * e + 2 * w + 4 * T,
                    "flops": 2 * T * r * kk}
        # x, dy, v and the base gradient in, dx out, weights in, their fp32 gradients out
        return {"bytes": T * (3 * case["K_in"] + case["K_out"]) * e + 4 * T * case["r"] + 2 * w
                + 4 * case["n"] * case["r"] * kk + 4 * T, "flops": 4 * T * r * kk}
    if case["op"] == "layernorm":
        n, e = case["rows"] * case["D"], 4 if case["f32"] else 2
        if case["direction"] == "fwd":
            return {"bytes": 2 * n * e + 8 * case["D"] + 8 * case["rows"], "flops": 8 * n}
        return {"bytes": (3 + case["dres"]) * n * e + 12 * case["D"] + 8 * case["rows"],
                "flops": 15 * n}
    n = sum(_sizes(case))
    states = 4 + 16 / BLOCK if case["bits"] == 8 else 16
    return {"bytes": n * (8 + states + (2 if case["g_bf16"] else 4) + 2 * case["copy"]),
            "flops": 16 * n}


# ----------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(g, *shape, std=1.0, dtype=torch.float32):
    return torch.empty(shape, device=DEV).normal_(0.0, std, generator=g).to(dtype)


def prepare(case, seed):
    g = _gen(seed)
    return {"adapter": _prepare_adapter, "layernorm": _prepare_norm,
            "adamw": _prepare_adamw}[case["op"]](case, g, seed)


def _prepare_adapter(case, g, seed):
    T, n, r, K_in, K_out = (case[k] for k in ("T", "n", "r", "K_in", "K_out"))
    dt = torch.float32 if case["f32"] else torch.bfloat16
    R = case["requests"]
    # lengths of the requests' tokens: one each, or ragged ones that fill T
    at = torch.randperm(T - 1, generator=g, device=DEV)[:R - 1].sort().values + 1 if R > 1 else \
        torch.empty(0, dtype=torch.int64, device=DEV)
    request = torch.searchsorted(at, torch.arange(T, device=DEV), right=True)
    perm = torch.randperm(n, generator=g, device=DEV)
    used = torch.tensor(_used(case), device=DEV)
    ids = torch.where(used < 0, used, perm[used.clamp(min=0)])[request].to(torch.int32)
    s = {"case": case, "ids": ids, "ranks": torch.tensor(_ranks(case), dtype=torch.int32, device=DEV)}
    s["x"] = _randn(g, T, K_in, dtype=dt)
    s["a"] = _randn(g, n, r, K_in, std=K_in ** -0.5, dtype=torch.bfloat16)
    s["b"] = _randn(g, n, r, K_out, std=r ** -0.5, dtype=torch.bfloat16)
    s["scale"] = torch.empty(n, device=DEV).uniform_(0.5, 2.0, generator=g)
    if case["direction"] == "fwd":
        s["base"] = _randn(g, T, K_out, dtype=dt)
        s["out"] = torch.empty_like(s["base"])
    else:
        s["dy"] = _randn(g, T, K_out, dtype=dt)
        s["base"] = _randn(g, T, K_in, dtype=dt)     # the gradient through the projection
        s["v"] = _low_rank(s["x"].float(), s["a"], ids, s["ranks"])  # kept by the forward pass
        s["dx"] = torch.empty_like(s["x"])
        s["da"] = torch.empty(n, r, K_in, device=DEV)
        s["db"] = torch.empty(n, r, K_out, device=DEV)
    if own:
        import paper_1701_00485_gb300 as tbn
        s["workspace"] = torch.empty(
            tbn.tbn_adapter_workspace_bytes(T, K_in, K_out, n, r, backward=case["direction"] == "bwd"),
            dtype=torch.uint8, device=DEV)
    return s


def _prepare_norm(case, g, seed):
    rows, D, wide = case["rows"], case["D"], case["D"] + case["pad"]
    dt = torch.float32 if case["f32"] else torch.bfloat16
    s = {"case": case}
    s["x"] = (_randn(g, rows, wide) * 2.0 + _randn(g, rows, 1)).to(dt)[:, :D]
    s["gamma"] = 1.0 + _randn(g, D, std=0.2)
    s["beta"] = _randn(g, D, std=0.2)
    if case["direction"] == "fwd":
        s["out"] = torch.empty(rows, D, dtype=dt, device=DEV)
        s["mean"], s["rstd"] = torch.empty(2, rows, device=DEV)
        return s
    s["dy"] = _randn(g, rows, wide, dtype=dt)[:, :D]
    s["dres"] = _randn(g, rows, D, dtype=dt) if case["dres"] else None
    xf = s["x"].float()
    s["mean"] = xf.mean(1)
    s["rstd"] = (xf.var(1, unbiased=False) + LN_EPS).rsqrt()
    s["dx"] = torch.empty(rows, D, dtype=dt, device=DEV)
    s["dgamma"], s["dbeta"] = torch.empty(2, D, device=DEV)
    if own:
        import paper_1701_00485_gb300 as tbn
        s["workspace"] = torch.empty(tbn.tbn_layernorm_bwd_workspace_bytes(rows, D),
                                     dtype=torch.uint8, device=DEV)
    return s


def _prepare_adamw(case, g, seed):
    """All tensors lie in one buffer, each from a multiple of the block size on."""
    sizes = _sizes(case)
    total = sum(-(-n // BLOCK) * BLOCK for n in sizes)
    live = torch.zeros(total, dtype=torch.bool, device=DEV)
    starts, at = [], 0
    for n in sizes:
        live[at:at + n] = True
        starts.append(at)
        at += -(-n // BLOCK) * BLOCK
    s = {"case": case, "step": 100, "lr": 1e-3, "wd": 0.01}
    # gradients of rows differ in size, as filters' do
    size = torch.exp(_randn(g, total // BLOCK, 1)) * 1e-3
    flat = lambda t: (t.view(-1) * live).contiguous()  # noqa: E731
    s["p"] = flat(_randn(g, total, std=0.02))
    grad = flat(_randn(g, total // BLOCK, BLOCK) * size)
    s["g"] = grad.to(torch.bfloat16) if case["g_bf16"] else grad
    m = flat(_randn(g, total // BLOCK, BLOCK) * size * 0.2)
    v = flat((_randn(g, total // BLOCK, BLOCK) * size).square() * 0.5 + (0.3 * size).square())
    s["grad_scale"] = torch.empty(1, device=DEV).uniform_(0.5, 1.0, generator=g)  # clipping's factor
    if case["bits"] == 8:
        for k, t, dt, most in (("m", m, torch.float8_e4m3fn, 256.0), ("v", v, torch.float8_e5m2, 32768.0)):
            top = t.abs().view(-1, BLOCK).amax(1).clamp(min=1e-30)
            scale = torch.exp2(torch.floor(torch.log2(top)) + 1) / most
            s[k] = (t.view(-1, BLOCK) / scale[:, None]).to(dt).view(-1)
            s[k + "_scale"] = scale
    else:
        s["m"], s["v"] = m, v
    s["copy"] = s["p"].to(torch.bfloat16) if case["copy"] else None
    if own:
        import paper_1701_00485_gb300 as tbn
        cut = lambda t: [t[a:a + n] for a, n in zip(starts, sizes)]  # noqa: E731
        scales = lambda t: [t[a // BLOCK:a // BLOCK - (-n // BLOCK)] for a, n in zip(starts, sizes)]  # noqa: E731
        more = {}
        if case["bits"] == 8:
            more.update(m_scale=scales(s["m_scale"]), v_scale=scales(s["v_scale"]))
        if case["copy"]:
            more["copies"] = cut(s["copy"])
        s["plan"] = tbn.AdamWPlan(cut(s["p"]), cut(s["g"]), cut(s["m"]), cut(s["v"]),
                                  weight_decay=s["wd"], **more)
    return s


# -------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if case["op"] == "adapter":
        fwd = case["direction"] == "fwd"
        if own:
            return _own_adapter_fwd(state) if fwd else _own_adapter_bwd(state)
        return _plain_adapter_fwd(state) if fwd else _plain_adapter_bwd(state)
    if case["op"] == "layernorm":
        fwd = case["direction"] == "fwd"
        if own:
            return _own_norm_fwd(state) if fwd else _own_norm_bwd(state)
        return _plain_norm_fwd(state) if fwd else _plain_norm_bwd(state)
    state["step"] += 1
    return _own_adamw(state) if own else _plain_adamw(state)


def _own_adapter_fwd(s):
    import paper_1701_00485_gb300 as tbn
    return tbn.tbn_adapter_fwd(s["x"], s["a"], s["b"], ids=s["ids"], scale=s["scale"],
                               ranks=s["ranks"], base=s["base"], out=s["out"],
                               workspace=s["workspace"])


def _own_adapter_bwd(s):
    import paper_1701_00485_gb300 as tbn
    dx, da, db = tbn.tbn_adapter_bwd(s["dy"], s["x"], s["a"], s["b"], ids=s["ids"],
                                     scale=s["scale"], ranks=s["ranks"], v=s["v"], base=s["base"],
                                     dx=s["dx"], da=s["da"], db=s["db"], workspace=s["workspace"])
    return {"dx": dx, "da": da, "db": db}


def _own_norm_fwd(s):
    import paper_1701_00485_gb300 as tbn
    y, mean, rstd = tbn.tbn_layernorm_fwd(s["x"], s["gamma"], s["beta"], eps=LN_EPS, out=s["out"],
                                          mean=s["mean"], rstd=s["rstd"])
    return {"y": y, "mean": mean, "rstd": rstd}


def _own_norm_bwd(s):
    import paper_1701_00485_gb300 as tbn
    dx, dgamma, dbeta = tbn.tbn_layernorm_bwd(s["dy"], s["x"], s["mean"], s["rstd"], s["gamma"],
                                              dres=s["dres"], dx=s["dx"], dgamma=s["dgamma"],
                                              dbeta=s["dbeta"], workspace=s["workspace"])
    return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}


def _own_adamw(s):
    import paper_1701_00485_gb300 as tbn
    tbn.tbn_adamw_step(s["plan"], step=s["step"], lr=s["lr"], betas=(BETA1, BETA2), eps=EPS,
                       grad_scale=s["grad_scale"], seed=s["step"])
    return _adamw_outputs(s)


def _adamw_outputs(s):
    out = {k: s[k] for k in ("p", "m", "v")}
    if s["case"]["bits"] == 8:
        out.update(m_scale=s["m_scale"], v_scale=s["v_scale"])
    if s["copy"] is not None:
        out["copy"] = s["copy"]
    return out


# ------------------------------------------------------- the plain forms
def _mine(ids, ranks, r):
    """[T, n, r]: whether the rank row is one of the token's adapter."""
    n = ranks.numel()
    there = torch.arange(r, device=ids.device) < ranks[:, None]
    return (ids[:, None] == torch.arange(n, device=ids.device))[:, :, None] & there


def _low_rank(x, a, ids, ranks):
    """v [T, r]: the token's adapter's rows times its activations."""
    n, r, K = a.shape
    v = (x @ a.float().view(n * r, K).t()).view(-1, n, r)
    return torch.where(_mine(ids, ranks, r), v, 0.0).sum(1)


def _spread(v, ids, ranks):
    """v [T, r] in the columns of the token's own adapter: [T, n r]."""
    return torch.where(_mine(ids, ranks, v.shape[1]), v[:, None, :], 0.0).view(v.shape[0], -1)


def _token_scale(s):
    n = s["scale"].numel()
    return torch.where(s["ids"] >= 0, s["scale"][s["ids"].clamp(0, n - 1).long()], 0.0)[:, None]


def _plain_adapter_fwd(s):
    b = s["b"].float()
    v = _low_rank(s["x"].float(), s["a"], s["ids"], s["ranks"]) * _token_scale(s)
    y = s["base"].float() + _spread(v, s["ids"], s["ranks"]) @ b.view(-1, b.shape[2])
    return y.to(s["base"].dtype)


def _plain_adapter_bwd(s):
    x, dy, scale = s["x"].float(), s["dy"].float(), _token_scale(s)
    a, b = s["a"].float(), s["b"].float()
    du = _spread(_low_rank(dy, s["b"], s["ids"], s["ranks"]) * scale, s["ids"], s["ranks"])
    v = _spread(s["v"] * scale, s["ids"], s["ranks"])
    dx = s["base"].float() + du @ a.view(-1, a.shape[2])
    return {"dx": dx.to(s["x"].dtype), "da": (du.t() @ x).view(a.shape), "db": (v.t() @ dy).view(b.shape)}


def _plain_norm_fwd(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = torch.rsqrt((c * c).mean(1, keepdim=True) + LN_EPS)
    y = c * rstd * s["gamma"] + s["beta"]
    return {"y": y.to(s["x"].dtype), "mean": mean.view(-1), "rstd": rstd.view(-1)}


def _plain_norm_bwd(s):
    x, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
    xh = (x - s["mean"][:, None]) * rstd
    w = dy * s["gamma"]
    dx = rstd * (w - w.mean(1, keepdim=True) - xh * (w * xh).mean(1, keepdim=True))
    if s["dres"] is not None:
        dx = dx + s["dres"].float()
    return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}


def _random_bits(seed, n):
    """32 random bits of each element, a mix of (seed, element): inputs of the step."""
    M = 0xFFFFFFFF
    h = (torch.arange(n, device=DEV) + seed * 0x9E3779B9) & M
    h = ((h ^ (h >> 16)) * 0x7FEB352D) & M
    h = ((h ^ (h >> 15)) * 0x846CA68B) & M
    return h ^ (h >> 16)


def _to_8bit(t, rnd, top, bias, drop, least):
    """Codes (7 bits) and scales of t >= 0.  A block's scale is the least power
    of two that brings its largest value to 1.75 * 2^top or below; the bits
    below the format's mantissa go up or down by 16 random ones."""
    bits = t.view(torch.int32).view(-1, BLOCK).amax(1)
    e = ((bits + 0x1FFFFF >> 23) - top).clamp(min=1)
    scale, inv = (e << 23).view(torch.float32), (254 - e << 23).view(torch.float32)
    # the format's exponent field becomes that of the 32-bit number
    u = (t.view(-1, BLOCK) * inv[:, None] * 2.0 ** (bias - 127)).view(-1)
    code = u.view(torch.int32) + (rnd.to(torch.int32) << drop - 16) >> drop
    return torch.where(t > 0, code.clamp(min=least), code), scale


def _plain_adamw(s):
    case = s["case"]
    g = s["g"].float() * s["grad_scale"]
    if case["bits"] == 8:
        m = (s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        v = (s["v"].float().view(-1, BLOCK) * s["v_scale"][:, None]).view(-1)
    else:
        m, v = s["m"], s["v"]
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + (1.0 - BETA2) * g * g
    fix1, fix2 = 1.0 - BETA1 ** s["step"], 1.0 - BETA2 ** s["step"]
    p = s["p"] * (1.0 - s["lr"] * s["wd"]) - s["lr"] / fix1 * (m / (torch.sqrt(v) / math.sqrt(fix2) + EPS))
    s["p"].copy_(p)
    if s["copy"] is not None:
        s["copy"].copy_(p)
    if case["bits"] == 8:
        rnd = _random_bits(s["step"], m.numel())
        mc, ms = _to_8bit(m.abs(), rnd >> 16, 8, 7, 20, 0)
        vc, vs = _to_8bit(v, rnd & 0xFFFF, 15, 15, 21, 1)
        mc = torch.where(m.view(torch.int32) < 0, mc | 0x80, mc)
        s["m"].view(torch.uint8).copy_(mc)
        s["v"].view(torch.uint8).copy_(vc)
        s["m_scale"].copy_(ms)
        s["v_scale"].copy_(vs)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    return _adamw_outputs(s)


# ------------------------------------------------------------ in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"adapter": _exact_adapter, "layernorm": _exact_norm, "adamw": _exact_adamw}[case["op"]](case, s)


def _exact_adapter(case, s):
    D = torch.float64
    fwd = case["direction"] == "fwd"
    ranks = s["ranks"].tolist()
    x, base = s["x"].to(D), s["base"].to(D)
    if not fwd:
        dy, v = s["dy"].to(D), s["v"].to(D)
        da = torch.zeros(s["a"].shape, dtype=D, device=DEV)
        db = torch.zeros(s["b"].shape, dtype=D, device=DEV)
    out = base.clone()
    for i in range(case["n"]):
        rows = (s["ids"] == i).nonzero().view(-1)
        if not rows.numel():
            continue
        k, c = ranks[i], s["scale"][i].to(D)
        a, b = s["a"][i, :k].to(D), s["b"][i, :k].to(D)
        if fwd:
            out[rows] += c * (x[rows] @ a.t()) @ b
        else:
            du = c * dy[rows] @ b.t()
            out[rows] += du @ a
            da[i, :k] = du.t() @ x[rows]
            db[i, :k] = c * v[rows, :k].t() @ dy[rows]
    return out if fwd else {"dx": out, "da": da, "db": db}


def _exact_norm(case, s):
    D = torch.float64
    x, gamma = s["x"].to(D), s["gamma"].to(D)
    if case["direction"] == "fwd":
        var, mean = torch.var_mean(x, 1, unbiased=False)
        rstd = 1.0 / torch.sqrt(var + LN_EPS)
        y = torch.addcmul(s["beta"].to(D), (x - mean[:, None]) * rstd[:, None], gamma)
        return {"y": y, "mean": mean, "rstd": rstd}
    mean, rstd, dy = s["mean"].to(D), s["rstd"].to(D), s["dy"].to(D)
    xh = torch.addcmul(-mean[:, None] * rstd[:, None], x, rstd[:, None])
    n = case["D"]
    s1 = (dy @ gamma) / n
    s2 = torch.einsum("td,td,d->t", dy, xh, gamma) / n
    dx = rstd[:, None] * (dy * gamma - s1[:, None] - xh * s2[:, None])
    if s["dres"] is not None:
        dx += s["dres"].to(D)
    return {"dx": dx, "dgamma": torch.einsum("td,td->d", dy, xh), "dbeta": dy.sum(0)}


def _exact_adamw(case, s):
    D = torch.float64
    t = s["step"] + 1
    g = s["g"].to(D) * s["grad_scale"].to(D)
    m, v = s["m"].to(D), s["v"].to(D)
    if case["bits"] == 8:
        m *= s["m_scale"].to(D).repeat_interleave(BLOCK)
        v *= s["v_scale"].to(D).repeat_interleave(BLOCK)
    m += (1.0 - BETA1) * (g - m)
    v += (1.0 - BETA2) * (g * g - v)
    p = s["p"].to(D)
    p -= s["lr"] * s["wd"] * p
    p -= s["lr"] * (m / (1.0 - BETA1 ** t)) / (torch.sqrt(v / (1.0 - BETA2 ** t)) + EPS)
    out = {"p": p, "m": m, "v": v}
    if case["copy"]:
        out["copy"] = p
    if case["bits"] == 8:
        rnd = _random_bits(t, m.numel())
        for k, u, top, low, digits in (("m", rnd >> 16, 448.0, -6, 3), ("v", rnd & 0xFFFF, 57344.0, -14, 2)):
            x = out[k].abs()
            most = x.view(-1, BLOCK).amax(1)
            e = torch.ceil(torch.log2(most.clamp(min=1e-300) / top)).clamp(min=-126.0)
            scale = torch.exp2(e)
            x = x / scale.repeat_interleave(BLOCK)
            step = torch.exp2(torch.floor(torch.log2(x.clamp(min=1e-300))).clamp(min=low) - digits)
            q = torch.floor(x / step + u.to(D) / 65536.0) * step
            if k == "v":
                q = torch.where(x > 0, q.clamp(min=2.0 ** (low - digits)), q)
            out[k], out[k + "_scale"] = torch.copysign(q, out[k]), scale
    return out
