"""Operators of a model's affine blocks in 8 bits: what is measured of them, their plain forms and their definitions in 64 bits.

A block is: residual addition and RMS norm, quantisation of activations and weights to e4m3 with a scale for each block of 128, the affine layer on
a Pfo x Pfi worker grid with both operands in 8 bits (forward and input gradient), and the AdamW step of the weights.  A case is a dict of plain
values; `kind` names the operator.  All tensors are synthetic, drawn on the device from the seed.  What a layer holds in several workers' blocks is a
list of tensors, as the library takes it; the optimiser's tensors lie in one buffer per kind, each on a 256-byte boundary.

With `own` false, run() computes an operator in elementary torch operations in 32 bits; with `own` true it makes the library's calls.
"""

import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn
BLOCK = 128                     # values under one scale
TINY = 2.0 ** -100              # a block whose largest magnitude is below this is scaled as if it were this
TOP = 448.0                     # largest e4m3 value
EPS = 1e-6                      # of the norm


# ---------------------------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------------------------

def listed():
    return [
        # One token of a decoder: residual addition, norm, 8-bit output for the layer behind it.  Latency.
        {"name": "norm_1x8192_decode", "kind": "norm", "nb": 1, "bf": 8192, "pf": 1, "t": "bf16", "keep": False, "q": True},
        # The forward pass in training: the sum, the norm in 16 bits (for the weight gradient) and in 8 bits (for the layer) on four workers.
        {"name": "norm_8192x8192_train", "kind": "norm", "nb": 8192, "bf": 2048, "pf": 4, "t": "bf16", "keep": True, "q": True},
        # The backward pass in training, gradients in 16 bits.
        {"name": "norm_adj_8192x8192", "kind": "norm_adj", "nb": 8192, "bf": 2048, "pf": 4, "t": "bf16", "tg": "bf16"},
        # The backward pass in 32 bits with rows that are no whole number of vectors.
        {"name": "norm_adj_1021x4x1250", "kind": "norm_adj", "nb": 1021, "bf": 1250, "pf": 4, "t": "f32", "tg": "f32"},
        # The output gradient of a small batch, quantised for the input gradient.  Latency.
        {"name": "quant_rows_256x8192", "kind": "quant_rows", "nb": 256, "bf": 2048, "pf": 4, "t": "bf16"},
        # The weights after an optimiser's step, from their 32-bit copies.
        {"name": "quant_weights_8192x8192", "kind": "quant_weights", "bfi": 2048, "bfo": 2048, "pfo": 4, "pfi": 4, "t": "f32"},
        # One token through the layer: bound by the weights.
        {"name": "affine_fp8_1x8192", "kind": "affine", "nb": 1, "bfi": 2048, "bfo": 2048, "pfo": 4, "pfi": 4, "adj": False, "bias": True, "t": "bf16"},
        # The input gradient of the batch that the 16-bit layer is measured at.
        {"name": "affine_fp8_adj_256x8192", "kind": "affine", "nb": 256, "bfi": 2048, "bfo": 2048, "pfo": 4, "pfi": 4, "adj": True, "bias": False, "t": "bf16"},
        # A ragged batch and blocks that are no whole number of tiles, results in 32 bits.
        {"name": "affine_fp8_777x3x1040", "kind": "affine", "nb": 777, "bfi": 1040, "bfo": 656, "pfo": 2, "pfi": 3, "adj": False, "bias": True, "t": "f32"},
        # The forward pass over many tokens: bound by the tensor cores.
        {"name": "affine_fp8_2048x8192", "kind": "affine", "nb": 2048, "bfi": 2048, "bfo": 2048, "pfo": 4, "pfi": 4, "adj": False, "bias": True, "t": "bf16"},
        # Parameters of a network of many small layers, states in 32 bits: one step over all of them.
        {"name": "adamw_f32_150_tensors", "kind": "adamw", "count": 150, "lo": 5, "hi": 1000003, "state": "f32", "tg": "f32", "copy": False},
        # The weights of one affine layer on 4 x 4 workers, states in 8 bits, 16-bit copies for the layer.
        {"name": "adamw_8bit_16x2048x2048", "kind": "adamw", "count": 16, "lo": 4194304, "hi": 4194304, "state": "8", "tg": "f32", "copy": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_adj", "quant_rows", "quant_weights", "affine", "affine", "adamw"])
    if kind in ("norm", "norm_adj", "quant_rows"):
        pf = rng.choice([1, 2, 3, 4, 8])
        bf = _log_int(rng, 48, 8192 // pf)
        if rng.random() < 0.5:
            bf = -(-bf // 8) * 8
        case = {"kind": kind, "nb": _log_int(rng, 1, 8192), "bf": bf, "pf": pf, "t": rng.choice(["bf16", "bf16", "f32"])}
        if kind == "norm":
            case.update(keep=rng.random() < 0.5, q=True) if rng.random() < 0.7 else case.update(keep=True, q=False)
        if kind == "norm_adj":
            case.update(tg=rng.choice(["bf16", "f32"]))
        return case
    pfo, pfi = rng.choice([1, 2, 3, 4]), rng.choice([1, 2, 3, 4])
    if kind == "quant_weights":
        return {"kind": kind, "bfi": _log_int(rng, 40, 2048), "bfo": _log_int(rng, 40, 2048), "pfo": pfo, "pfi": pfi, "t": rng.choice(["f32", "bf16"])}
    if kind == "affine":
        adj = rng.random() < 0.5
        return {"kind": kind, "nb": _log_int(rng, 1, 2048), "bfi": 16 * _log_int(rng, 4, 128), "bfo": 16 * _log_int(rng, 4, 128), "pfo": pfo, "pfi": pfi,
                "adj": adj, "bias": not adj and rng.random() < 0.5, "t": rng.choice(["bf16", "f32"])}
    hi = _log_int(rng, 1000, 4000000)
    return {"kind": kind, "count": min(_log_int(rng, 1, 200), max(1, 60000000 // hi)), "lo": max(1, _log_int(rng, 1, hi)), "hi": hi,
            "state": rng.choice(["f32", "8"]), "tg": rng.choice(["f32", "bf16"]), "copy": rng.random() < 0.5}


def _sizes(case):
    """Elements of each tensor of an optimiser's case: spread over the logarithm of the range, in no order."""
    n, lo, hi = case["count"], case["lo"], case["hi"]
    return [int(round(lo * (hi / lo) ** ((7 * i + 3) % 16 / 15))) + (i % 5 if hi > lo else 0) for i in range(n)]


def _up(n, m):
    return -(-n // m)


def work(case):
    kind, size = case["kind"], {"f32": 4, "bf16": 2}
    if kind in ("norm", "norm_adj", "quant_rows"):
        nb, pf, bf, e = case["nb"], case["pf"], case["bf"], size[case["t"]]
        n, scales = nb * pf * bf, 4 * nb * pf * _up(bf, BLOCK)
        if kind == "norm":
            return {"bytes": n * (3 * e + (e if case["keep"] else 0) + (1 if case["q"] else 0)) + (scales if case["q"] else 0) + 4 * (pf * bf + nb), "flops": 6 * n}
        if kind == "norm_adj":
            return {"bytes": n * (e + 3 * size[case["tg"]]) + 8 * pf * bf + 4 * nb, "flops": 10 * n}
        return {"bytes": n * (e + 1) + scales, "flops": 3 * n}
    if kind == "adamw":
        n = sum(_sizes(case))
        state = 16 if case["state"] == "f32" else 4 + 16 / BLOCK
        return {"bytes": n * (8 + size[case["tg"]] + state + (2 if case["copy"] else 0)), "flops": 15 * n}
    bfi, bfo, grid = case["bfi"], case["bfo"], case["pfo"] * case["pfi"]
    weights, scales = grid * bfi * bfo, 4 * grid * _up(bfi, BLOCK) * _up(bfo, BLOCK)
    if kind == "quant_weights":
        return {"bytes": weights * (size[case["t"]] + 1) + scales, "flops": 3 * weights}
    nb = case["nb"]
    nin, nout = (bfo * case["pfo"], bfi * case["pfi"]) if case["adj"] else (bfi * case["pfi"], bfo * case["pfo"])
    blocks = case["pfo"] * _up(bfo, BLOCK) if case["adj"] else case["pfi"] * _up(bfi, BLOCK)
    return {"bytes": weights + scales + nb * nin + 4 * nb * blocks + nb * nout * size[case["t"]] + (4 * nout if case["bias"] else 0), "flops": 2 * nb * weights}


# ---------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape, std=1.0):
    return torch.randn(*shape, device=DEV, generator=g) * std


def _activations(g, nb, bf):
    """Normal values; one feature in 64 is ten times as large, as the few large features of a model's residual stream are."""
    a = _normal(g, nb, bf)
    a[:, torch.randint(0, bf, (max(1, bf // 64),), device=DEV, generator=g)] *= 10.0
    return a


def _rows_to_8_bits(x):
    """What a layer in front leaves behind: e4m3 rows and scales [blocks, rows]."""
    nb, bf = x.shape
    a = torch.nn.functional.pad(x, (0, -bf % BLOCK)).view(nb, -1, BLOCK)
    top = a.abs().amax(2).clamp_min(TINY)
    q = (a * (TOP / top)[:, :, None]).clamp(-TOP, TOP).to(E4M3).view(nb, -1)[:, :bf].contiguous()
    return q, (top / TOP).t().contiguous()


def _blocks_to_8_bits(w):
    rows, cols = w.shape
    a = torch.nn.functional.pad(w, (0, -cols % BLOCK, 0, -rows % BLOCK)).view(_up(rows, BLOCK), BLOCK, _up(cols, BLOCK), BLOCK)
    top = a.abs().amax((1, 3)).clamp_min(TINY)
    q = (a * (TOP / top)[:, None, :, None]).clamp(-TOP, TOP).to(E4M3).view(a.shape[0] * BLOCK, -1)[:rows, :cols].contiguous()
    return q, (top / TOP).contiguous()


def _flat(sizes, dtype):
    """One buffer for tensors of these sizes, each on a boundary of 256 elements, and the tensors."""
    at, end = [], 0
    for n in sizes:
        at.append(end)
        end += 256 * _up(n, 256)
    buf = torch.zeros(end, device=DEV, dtype=dtype)
    return buf, [buf[a:a + n] for a, n in zip(at, sizes)]


def prepare(case, seed):
    g, kind = _generator(seed), case["kind"]
    s = {"case": dict(case)}
    empty = lambda *shape, dtype=torch.float32: torch.empty(*shape, device=DEV, dtype=dtype)  # noqa: E731
    if kind in ("norm", "norm_adj", "quant_rows"):
        nb, bf, pf, t = case["nb"], case["bf"], case["pf"], TYPES[case["t"]]
        blocks = _up(bf, BLOCK)
        s["x"] = [_activations(g, nb, bf).to(t) for _ in range(pf)]
        if kind == "quant_rows":
            s.update(q=[empty(nb, bf, dtype=E4M3) for _ in range(pf)], qs=[empty(blocks, nb) for _ in range(pf)])
            return s
        s["gamma"] = [1 + _normal(g, bf, std=0.1) for _ in range(pf)]
        if kind == "norm":
            s["res"] = [_activations(g, nb, bf).to(t) for _ in range(pf)]
            s.update(h=[empty(nb, bf, dtype=t) for _ in range(pf)], rstd=empty(nb))
            s.update(y=[empty(nb, bf, dtype=t) for _ in range(pf)] if case["keep"] else None)
            s.update(q=[empty(nb, bf, dtype=E4M3) for _ in range(pf)] if case["q"] else None, qs=[empty(blocks, nb) for _ in range(pf)] if case["q"] else None)
            return s
        tg = TYPES[case["tg"]]
        s["rstd"] = (sum(x.double().square().sum(1) for x in s["x"]) / (pf * bf) + EPS).rsqrt().float()     # as the forward pass left it
        s["dy"] = [_normal(g, nb, bf, std=0.01).to(tg) for _ in range(pf)]
        s["dres"] = [_normal(g, nb, bf, std=0.01).to(tg) for _ in range(pf)]
        s.update(dh=[empty(nb, bf, dtype=tg) for _ in range(pf)], dgamma=[empty(bf) for _ in range(pf)])
        if own:                                     # scratch that a program keeps for its layers
            import paper_2006_03108_b200 as distdl
            s["ws"] = empty(distdl.rmsnorm_adj_workspace(nb, pf * bf, pf), dtype=torch.uint8)
        return s
    if kind == "adamw":
        sizes = _sizes(case)
        scale_sizes = [_up(n, BLOCK) for n in sizes]
        s["p_flat"], s["p"] = _flat(sizes, torch.float32)
        s["g_flat"], s["g"] = _flat(sizes, TYPES[case["tg"]])
        s["p_flat"].copy_(_normal(g, s["p_flat"].numel(), std=0.02))
        s["g_flat"].copy_(_normal(g, s["g_flat"].numel(), std=1e-3))
        s["w_flat"], s["w"] = _flat(sizes, torch.bfloat16) if case["copy"] else (None, None)
        m = _normal(g, s["p_flat"].numel(), std=3e-4)              # moments in the middle of a training run
        r = 1e-3 * torch.exp(_normal(g, s["p_flat"].numel(), std=0.5))
        if case["state"] == "f32":
            s["m_flat"], s["m"] = _flat(sizes, torch.float32)
            s["v_flat"], s["v"] = _flat(sizes, torch.float32)
            s["m_flat"].copy_(m)
            s["v_flat"].copy_(r.square())
            s.update(ms_flat=None, ms=None, vs_flat=None, vs=None)
        else:
            for name, value in (("m", m), ("v", r)):               # the second moment is held as its root
                s[name + "_flat"], s[name] = _flat(sizes, E4M3)
                s[name + "s_flat"], s[name + "s"] = _flat(scale_sizes, torch.float32)
                at = 0
                for n, q, sc in zip(sizes, s[name], s[name + "s"]):
                    q8, scales = _rows_to_8_bits(value[at:at + n][None])
                    q.copy_(q8[0])
                    sc.copy_(scales[:, 0])
                    at += 256 * _up(n, 256)
        s["step"] = 100
        if own:                                     # the handle that a program keeps
            import paper_2006_03108_b200 as distdl
            s["opt"] = distdl.AdamW(s["p"], s["m"], s["v"], s["ms"], s["vs"], s["w"])
        return s
    bfi, bfo, pfo, pfi = case["bfi"], case["bfo"], case["pfo"], case["pfi"]
    w = [_normal(g, bfo, bfi, std=(bfi * pfi) ** -0.5) for _ in range(pfo * pfi)]
    if kind == "quant_weights":
        s.update(w=[b.to(TYPES[case["t"]]) for b in w], q=[empty(bfo, bfi, dtype=E4M3) for _ in w], qs=[empty(_up(bfo, BLOCK), _up(bfi, BLOCK)) for _ in w])
        return s
    nb, t = case["nb"], TYPES[case["t"]]
    s["w"], s["ws"] = (list(v) for v in zip(*[_blocks_to_8_bits(b) for b in w]))
    if case["adj"]:
        s["x"], s["xs"] = (list(v) for v in zip(*[_rows_to_8_bits(_normal(g, nb, bfo, std=0.01)) for _ in range(pfo)]))
    else:
        s["x"], s["xs"] = (list(v) for v in zip(*[_rows_to_8_bits(_activations(g, nb, bfi)) for _ in range(pfi)]))
    s["bias"] = [_normal(g, bfo, std=0.1) for _ in range(pfo)] if case["bias"] else None
    s["y"] = [empty(nb, bfi if case["adj"] else bfo, dtype=t) for _ in range(pfi if case["adj"] else pfo)]
    return s


# ---------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------

LR, BETA1, BETA2, ADAM_EPS, DECAY, GRAD_SCALE, SEED = 1e-4, 0.9, 0.95, 1e-8, 0.1, 0.5, 1234


def run(s):
    case = s["case"]
    if own:
        return _own(case, s)
    return {"norm": _norm, "norm_adj": _norm_adj, "quant_rows": _quant_rows, "quant_weights": _quant_weights, "affine": _affine,
            "adamw": _adamw}[case["kind"]](case, s, torch.float32)


def _own(case, s):
    import paper_2006_03108_b200 as distdl
    kind = case["kind"]
    if kind == "norm":
        distdl.rmsnorm_fwd(case["nb"], case["pf"] * case["bf"], case["pf"], s["x"], s["res"], s["gamma"], EPS, s["h"], s["y"], s["q"], s["qs"], s["rstd"])
        return {k: s[k] for k in ("h", "y", "q", "qs", "rstd") if s[k] is not None}
    if kind == "norm_adj":
        distdl.rmsnorm_adj(case["nb"], case["pf"] * case["bf"], case["pf"], s["dy"], s["dres"], s["x"], s["gamma"], s["rstd"], s["dh"], s["dgamma"], s["ws"])
        return {"dh": s["dh"], "dgamma": s["dgamma"]}
    if kind == "quant_rows":
        distdl.quantize_rows(case["nb"], case["pf"] * case["bf"], case["pf"], s["x"], s["q"], s["qs"])
        return {"q": s["q"], "qs": s["qs"]}
    grid = (case.get("bfi", 0) * case.get("pfi", 0), case.get("bfo", 0) * case.get("pfo", 0), case.get("pfo"), case.get("pfi"))
    if kind == "quant_weights":
        distdl.quantize_weights(*grid, s["w"], s["q"], s["qs"])
        return {"q": s["q"], "qs": s["qs"]}
    if kind == "affine":
        if case["adj"]:
            distdl.affine_fp8_adj(case["nb"], *grid, s["x"], s["xs"], s["w"], s["ws"], s["y"])
        else:
            distdl.affine_fp8_fwd(case["nb"], *grid, s["x"], s["xs"], s["w"], s["ws"], s["bias"], s["y"])
        return {"y": s["y"]}
    s["step"] += 1
    s["opt"].step(s["g"], LR, s["step"], (BETA1, BETA2), ADAM_EPS, DECAY, seed=SEED, grad_scale=GRAD_SCALE)
    return _adamw_outputs(s)


def _adamw_outputs(s):
    return {k: s[k + "_flat"] for k in ("p", "m", "v", "ms", "vs", "w") if s[k + "_flat"] is not None}


# The plain forms.  `f` is the type they compute in.

def _split(a, pf):
    return [b.contiguous() for b in a.chunk(pf, 1)]


def _divided(a, b):
    """a / b with both on the device (a quotient by a number of the host is a product by its reciprocal)."""
    return torch.div(torch.full_like(b, a) if not isinstance(a, torch.Tensor) else a, b if isinstance(b, torch.Tensor) else torch.full_like(a, b))


def _quantised_rows(x):
    nb, bf = x.shape
    a = torch.nn.functional.pad(x, (0, -bf % BLOCK)).view(nb, -1, BLOCK)
    top = a.abs().amax(2).clamp_min(TINY)
    q = (a * _divided(TOP, top)[:, :, None]).clamp(-TOP, TOP).to(E4M3)
    return q.view(nb, -1)[:, :bf].contiguous(), _divided(top, TOP).t().contiguous()


def _norm(case, s, f):
    t = TYPES[case["t"]]
    h = [(x.to(f) + r.to(f)).to(t) for x, r in zip(s["x"], s["res"])]
    a = torch.cat([v.to(f) for v in h], 1)
    rstd = (a.square().mean(1) + EPS).rsqrt()
    y = a * rstd[:, None] * torch.cat(s["gamma"]).to(f)
    out = {"h": h, "rstd": rstd}
    if case["keep"]:
        out["y"] = [b.to(t) for b in _split(y, case["pf"])]
    if case["q"]:
        out["q"], out["qs"] = (list(v) for v in zip(*[_quantised_rows(b) for b in _split(y, case["pf"])]))
    return out


def _norm_adj(case, s, f):
    tg = TYPES[case["tg"]]
    rstd = s["rstd"].to(f)[:, None]
    hhat = torch.cat([v.to(f) for v in s["x"]], 1) * rstd
    dy = torch.cat([v.to(f) for v in s["dy"]], 1)
    gdy = dy * torch.cat(s["gamma"]).to(f)
    dh = torch.cat([v.to(f) for v in s["dres"]], 1) + rstd * (gdy - hhat * (gdy * hhat).mean(1, keepdim=True))
    return {"dh": [b.to(tg) for b in _split(dh, case["pf"])], "dgamma": list((dy * hhat).sum(0).chunk(case["pf"]))}


def _quant_rows(case, s, f):
    out = [_quantised_rows(x.to(f)) for x in s["x"]]
    return {"q": [q for q, _ in out], "qs": [v for _, v in out]}


def _quant_weights(case, s, f):
    rows, cols = case["bfo"], case["bfi"]
    padded = [torch.nn.functional.pad(w.to(f), (0, -cols % BLOCK, 0, -rows % BLOCK)).view(_up(rows, BLOCK), BLOCK, _up(cols, BLOCK), BLOCK) for w in s["w"]]
    top = [a.abs().amax((1, 3)).clamp_min(TINY) for a in padded]
    q = [(a * _divided(TOP, m)[:, None, :, None]).clamp(-TOP, TOP).to(E4M3) for a, m in zip(padded, top)]
    return {"q": [v.view(-1, _up(cols, BLOCK) * BLOCK)[:rows, :cols].contiguous() for v in q], "qs": [_divided(m, TOP) for m in top]}


def _values(q, scale, f):
    """Rows in 8 bits with scales [blocks, rows]."""
    return q.to(f) * scale.to(f).t().repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _block_values(q, scale, f):
    return q.to(f) * scale.to(f).repeat_interleave(BLOCK, 0)[:q.shape[0]].repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _affine(case, s, f):
    pfo, pfi, t = case["pfo"], case["pfi"], TYPES[case["t"]]
    x = torch.cat([_values(q, v, f) for q, v in zip(s["x"], s["xs"])], 1)
    w = [_block_values(q, v, f) for q, v in zip(s["w"], s["ws"])]
    w = torch.cat([torch.cat(w[i * pfi:(i + 1) * pfi], 1) for i in range(pfo)], 0)
    y = x @ (w if case["adj"] else w.t())
    if case["bias"]:
        y = y + torch.cat(s["bias"]).to(f)
    return {"y": [b.to(t) for b in _split(y, pfi if case["adj"] else pfo)]}


MASK = 0xFFFFFFFF


def _mixed(x):
    """32 well mixed bits of 32 bits (held in 64): multiplications by odd constants and shifted copies."""
    x = x ^ (x >> 16)
    x = (x * 0xB504F333) & MASK
    x = x ^ (x >> 15)
    x = (x * 0x93CD3A2D) & MASK
    return x ^ (x >> 16)


def _random_bits(n, seed, step, tensor):
    """The 32 random bits of each element of a tensor at a step."""
    key = (_mixed((((seed ^ (seed >> 32)) & MASK) + step * 0x9E3779B9) & MASK) + tensor * 0xA54FF53B) & MASK
    e = torch.arange(n, device=DEV, dtype=torch.int64)
    return _mixed(((e & MASK) * 0x9E3779B9 + (e >> 32) * 0xA54FF53B + key) & MASK)


def _rounded(a, u, never_zero):
    """Magnitudes up to 448 to e4m3 values: up where the rest of the division by a step is above 1 - u, down else."""
    grid = (torch.frexp(a)[1] - 1).clamp_min(-6)
    k = torch.floor(torch.ldexp(a, 3 - grid) + u)
    if never_zero:
        k = torch.where((k == 0) & (a > 0), 1.0, k)
    return torch.ldexp(k, grid - 3)


def _to_8_bits(a, u, never_zero):
    n = a.numel()
    blocks = torch.nn.functional.pad(a, (0, -n % BLOCK)).view(-1, BLOCK)
    top = blocks.abs().amax(1).clamp_min(TINY)
    scaled = (blocks * _divided(TOP, top)[:, None]).clamp(-TOP, TOP).view(-1)[:n]
    return torch.copysign(_rounded(scaled.abs(), u, never_zero), scaled), _divided(top, TOP)


def _adamw_tensor(case, s, i, step, f):
    """One tensor's new (p, m, v, ms, vs): moments as they are held."""
    eight, p, n = case["state"] == "8", s["p"][i].to(f), s["p"][i].numel()
    g = s["g"][i].to(f) * GRAD_SCALE
    m, v = s["m"][i].to(f), s["v"][i].to(f)
    if eight:
        m = m * s["ms"][i].to(f).repeat_interleave(BLOCK)[:n]
        v = (v * s["vs"][i].to(f).repeat_interleave(BLOCK)[:n]).square()
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g.square()
    p = p * (1 - LR * DECAY) - LR / (1 - BETA1 ** step) * m / (v.sqrt() / math.sqrt(1 - BETA2 ** step) + ADAM_EPS)
    if not eight:
        return p, m, v, None, None
    bits = _random_bits(n, SEED, step, i)
    m, ms = _to_8_bits(m, (bits & 0xFFFF).to(f) / 65536, False)
    v, vs = _to_8_bits(v.sqrt(), (bits >> 16).to(f) / 65536, True)
    return p, m, v, ms, vs


def _adamw(case, s, f):
    s["step"] += 1
    for i in range(case["count"]):
        new = _adamw_tensor(case, s, i, s["step"], f)
        for name, value in zip(("p", "m", "v", "ms", "vs"), new):
            if value is not None:
                s[name][i].copy_(value)
        if case["copy"]:
            s["w"][i].copy_(new[0])
    return _adamw_outputs(s)


# ---------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------

def exact(case, seed):
    s, kind, d = prepare({**case}, seed), case["kind"], torch.float64
    if kind == "affine" and work(case)["flops"] > 3e11:
        return None
    if kind == "adamw":
        return _exact_adamw(case, s)
    if kind == "affine":
        return {"y": _exact_affine(case, s)}
    if kind == "quant_weights":
        out = [_exact_blocks(w.to(d)) for w in s["w"]]
        return {"q": [q for q, _ in out], "qs": [v for _, v in out]}
    if kind == "quant_rows":
        out = [_exact_rows(x.to(d)) for x in s["x"]]
        return {"q": [q for q, _ in out], "qs": [v for _, v in out]}
    pf, nf = case["pf"], case["pf"] * case["bf"]
    if kind == "norm":
        h = [torch.add(x.to(d), r.to(d)).to(TYPES[case["t"]]) for x, r in zip(s["x"], s["res"])]     # the sum is held, and normed, in its type
        r = 1 / torch.sqrt(sum(torch.einsum("bf,bf->b", v.to(d), v.to(d)) for v in h) / nf + EPS)
        y = [torch.einsum("bf,b,f->bf", v.to(d), r, c.to(d)) for v, c in zip(h, s["gamma"])]
        out = {"h": [v.to(d) for v in h], "rstd": r}
        if case["keep"]:
            out["y"] = y
        if case["q"]:
            out["q"], out["qs"] = (list(v) for v in zip(*[_exact_rows(b) for b in y]))
        return out
    r = s["rstd"].to(d)
    dot = sum(torch.einsum("bf,bf,f->b", a.to(d), b.to(d), c.to(d)) for a, b, c in zip(s["dy"], s["x"], s["gamma"]))
    dh = [e.to(d) + torch.einsum("bf,f,b->bf", a.to(d), c.to(d), r) - torch.einsum("bf,b->bf", b.to(d), r ** 3 * dot / nf)
          for a, b, c, e in zip(s["dy"], s["x"], s["gamma"], s["dres"])]
    return {"dh": dh, "dgamma": [torch.einsum("bf,bf,b->f", a.to(d), b.to(d), r) for a, b in zip(s["dy"], s["x"])]}


def _exact_rows(x):
    q, scales = torch.empty_like(x), []
    for b in range(0, x.shape[1], BLOCK):
        part = x[:, b:b + BLOCK]
        top = torch.maximum(part.abs().max(1).values, torch.tensor(TINY, dtype=x.dtype, device=DEV))
        q[:, b:b + BLOCK] = (part * TOP / top[:, None]).to(E4M3).to(x.dtype)
        scales.append(top / TOP)
    return q, torch.stack(scales)


def _exact_blocks(w):
    out = [_exact_band(w[r:r + BLOCK]) for r in range(0, w.shape[0], BLOCK)]
    return torch.cat([q for q, _ in out]), torch.stack([v for _, v in out])


def _exact_band(band):
    """Up to 128 rows: values and a scale for every 128 columns."""
    q, scales = torch.empty_like(band), []
    for c in range(0, band.shape[1], BLOCK):
        part = band[:, c:c + BLOCK]
        top = part.abs().max().clamp_min(TINY)
        q[:, c:c + BLOCK] = (part * TOP / top).to(E4M3).to(band.dtype)
        scales.append(top / TOP)
    return q, torch.stack(scales)


def _exact_affine(case, s):
    """Block after block: 128 of the contraction of one worker, its product, its scales."""
    d, pfo, pfi, out = torch.float64, case["pfo"], case["pfi"], []
    for o in range(pfi if case["adj"] else pfo):
        y = torch.zeros(s["y"][o].shape, dtype=d, device=DEV)
        for k in range(pfo if case["adj"] else pfi):
            q, v = s["x"][k].to(d), s["xs"][k].to(d)
            w, ws = (s[n][k * pfi + o if case["adj"] else o * pfi + k].to(d) for n in ("w", "ws"))
            w, ws = (w, ws) if case["adj"] else (w.t(), ws.t())             # [contraction, outputs]
            column = torch.arange(w.shape[1], device=DEV) // BLOCK
            for b in range(v.shape[0]):
                span = slice(b * BLOCK, (b + 1) * BLOCK)
                y += (q[:, span] @ w[span]) * v[b][:, None] * ws[b][column]
        out.append(y + s["bias"][o].to(d) if case["bias"] else y)
    return out


def _exact_adamw(case, s):
    d, step, out = torch.float64, s["step"] + 1, {}
    names = ["p", "m", "v"] + (["ms", "vs"] if case["state"] == "8" else []) + (["w"] if case["copy"] else [])
    for name in names:
        out[name] = s[name + "_flat"].to(d)                         # what lies between the tensors stays
    for i, n in enumerate(_sizes(case)):
        where = {k: (s[k][i].storage_offset(), s[k][i].numel()) for k in names}
        g, m, v = s["g"][i].to(d) * GRAD_SCALE, s["m"][i].to(d), s["v"][i].to(d)
        if case["state"] == "8":
            block = torch.arange(n, device=DEV) // BLOCK
            m, v = m * s["ms"][i].to(d)[block], (v * s["vs"][i].to(d)[block]) ** 2
        m, v = m + (1 - BETA1) * (g - m), v + (1 - BETA2) * (g * g - v)
        p = s["p"][i].to(d)
        p = p - LR * DECAY * p - LR * (m / (1 - BETA1 ** step)) / (torch.sqrt(v / (1 - BETA2 ** step)) + ADAM_EPS)
        new = {"p": p, "w": p, "m": m, "v": v}
        if case["state"] == "8":
            bits = _random_bits(n, SEED, step, i)
            for name, value, shift in (("m", m, 0), ("v", torch.sqrt(v), 16)):
                top = torch.zeros(int(block[-1]) + 1, dtype=d, device=DEV).scatter_reduce(0, block, value.abs(), "amax").clamp_min(TINY)
                a = value.abs() * TOP / top[block]
                u = ((bits >> shift) & 0xFFFF).to(d) / 65536
                width = torch.exp2(torch.floor(torch.log2(a.clamp_min(2.0 ** -6))) - 3)      # distance of e4m3 values here
                k = torch.floor(a / width + u)
                if name == "v":
                    k = torch.where((k < 1) & (a > 0), torch.ones_like(k), k)
                new[name], new[name + "s"] = torch.sign(value) * torch.clamp_max(k * width, TOP), top / TOP
        for k in names:
            at, count = where[k]
            out[k][at:at + count] = new[k]
    return out
