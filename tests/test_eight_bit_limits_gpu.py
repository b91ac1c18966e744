"""GPU tests of the operators of 8-bit affine blocks at the ends of their ranges, against the oracle (fp64); tolerances as in test_eight_bit_gpu.py."""

import numpy as np
import pytest

import paper_2006_03108_b200 as distdl
from oracle import eight_bit as o
from paper_2006_03108_b200 import inputs
from test_eight_bit_gpu import DEV, E4, FP8, U, Out, dev, eps_of, f64, rounded, sum_error

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# a chunk of a thread, two, four; sums over the features by a kernel of their own; rows of odd lengths
NEAR_ZERO = [(24, 136, 2), (24, 40, 1), (12, 2048, 2), (12, 2500, 4), (12, 5003, 4)]


@pytest.mark.parametrize("tg", [torch.float32, torch.bfloat16], ids=["gf32", "gbf16"])
@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("nb,bf,pf", NEAR_ZERO, ids=str)
def test_rmsnorm_adj_of_samples_near_zero(t, tg, nb, bf, pf):
    """Samples of zeros and next to zero, whose rstd has no square in fp32: dh is the number that the formula gives, and no NaN."""
    nf = bf * pf
    size = np.array([0.0, 1e-30, 1e-24, 1e-21, 1e-15, 1.0] * (nb // 6))[:, None]
    eps = np.array([1e-44, 1e-42, 1e-44, 1e-40, 2.0 ** -120, 1e-6] * (nb // 6))
    h = [rounded((inputs.normal((nb, bf), 500 + j) * size).astype(np.float32), t) for j in range(pf)]
    dy = [rounded(inputs.normal((nb, bf), 520 + j, 300.0), tg) for j in range(pf)]
    dres = [rounded(inputs.normal((nb, bf), 540 + j, 0.1), tg) for j in range(pf)]
    g = [1 + inputs.normal((bf,), 560 + j, 0.2) for j in range(pf)]
    h64, g64, d64 = ([a.astype(np.float64) for a in v] for v in (h, g, dy))
    rstd = (1 / np.sqrt(sum((a ** 2).sum(1) for a in h64) / nf + eps)).astype(np.float32)
    assert (rstd.max() > 2.0 ** 64) and np.isfinite(rstd).all()
    out = Out()
    dh, dg = [out(nb, bf, dtype=tg) for _ in range(pf)], [out(bf) for _ in range(pf)]
    ws = out(distdl.rmsnorm_adj_workspace(nb, nf, pf), dtype=torch.uint8)
    distdl.rmsnorm_adj(nb, nf, pf, [dev(a, tg) for a in dy], [dev(a, tg) for a in dres], [dev(a, t) for a in h], [dev(a) for a in g], dev(rstd), dh, dg, ws)
    dhw, dgw = o.rmsnorm_adj(d64, [a.astype(np.float64) for a in dres], h64, g64, rstd)
    r = rstd.astype(np.float64)[:, None]
    terms = sum((np.abs(a * b * c)).sum(1, keepdims=True) for a, b, c in zip(d64, h64, g64)) / nf
    for j in range(pf):
        back = np.abs(h64[j]) * r ** 3 * terms
        e = (sum_error(nf, pf) + 8 * U) * back + 4 * U * (np.abs(r * g64[j] * d64[j]) + np.abs(dres[j]) + back)
        assert (np.abs(f64(dh[j]) - dhw[j]) <= e + eps_of(tg) * (np.abs(dhw[j]) + e)).all()
        assert (np.abs(f64(dg[j]) - dgw[j]) <= (28 + 4) * U * np.abs(d64[j] * h64[j] * r).sum(0)).all()
    out.check()


def test_rmsnorm_forward_and_back_with_the_smallest_eps():
    """The forward pass's own rstd at the smallest eps: samples of zeros, next to it and ordinary ones."""
    nb, bf, pf, eps = 9, 200, 2, 2.0 ** -120
    size = np.array([0.0, 2.0 ** -62, 1.0] * 3)[:, None].astype(np.float32)
    h, dy, g = [[inputs.normal(s, 600 + 10 * k + j) for j in range(pf)] for k, s in enumerate(((nb, bf), (nb, bf), (bf,)))]
    h = [a * size for a in h]
    hd, gd, rstd = [dev(a) for a in h], [dev(a) for a in g], torch.empty(nb, device=DEV)
    y, dh, dg = [[torch.empty(*s, device=DEV) for _ in range(pf)] for s in ((nb, bf), (nb, bf), (bf,))]
    distdl.rmsnorm_fwd(nb, bf * pf, pf, hd, None, gd, eps, None, y, None, None, rstd)
    distdl.rmsnorm_adj(nb, bf * pf, pf, [dev(a) for a in dy], None, hd, gd, rstd, dh, dg,
                       torch.empty(distdl.rmsnorm_adj_workspace(nb, bf * pf, pf), dtype=torch.uint8, device=DEV))
    h64, g64, d64 = ([a.astype(np.float64) for a in v] for v in (h, g, dy))
    yw, rw = o.rmsnorm_fwd(h64, g64, eps)
    re = sum_error(bf * pf, pf) / 2 + 4 * U + 2.0 ** -30                       # the last: squares below 2^-126, each to 2^-150
    assert (np.abs(f64(rstd) - rw) <= re * rw).all()
    dhw, _ = o.rmsnorm_adj(d64, None, h64, g64, f64(rstd))
    terms = sum((np.abs(a * b * c)).sum(1, keepdims=True) for a, b, c in zip(d64, h64, g64)) / (bf * pf)
    r = f64(rstd)[:, None]
    for j in range(pf):
        assert (np.abs(f64(y[j]) - yw[j]) <= (re + 3 * U) * np.abs(yw[j]) * (1 + U)).all()
        back = np.abs(h64[j]) * r ** 3 * terms
        e = (sum_error(bf * pf, pf) + 8 * U) * back + 4 * U * (np.abs(r * g64[j] * d64[j]) + back)
        assert (np.abs(f64(dh[j]) - dhw[j]) <= e + U * (np.abs(dhw[j]) + e)).all()


@pytest.mark.parametrize("eight", [False, True], ids=["f32", "8bit"])
def test_adamw_writes_nothing_once_a_tensor_has_moved(eight):
    """A parameter that got other memory: the step is refused, and neither the old memory nor the new one changes."""
    n = 1000
    p = [torch.nn.Parameter(torch.ones(n, device=DEV)) for _ in range(2)]
    state = [[torch.zeros(n, device=DEV, dtype=E4 if eight else torch.float32) for _ in range(2)] for _ in range(2)]
    scales = [[torch.zeros(8, device=DEV) for _ in range(2)] for _ in range(2)] if eight else []
    opt, g = distdl.AdamW(p, *state, *scales), [torch.ones(n, device=DEV) for _ in range(2)]
    opt.step(g, 1e-3, 1)
    before = [a.detach().clone() for a in p]
    old = p[1].data
    p[1].data = p[1].data.clone()
    with pytest.raises(distdl.DistdlError, match="no longer") as e:
        opt.step(g, 1e-3, 2)
    assert e.value.status == 1
    torch.cuda.synchronize()
    assert torch.equal(p[0], before[0]) and torch.equal(p[1], before[1]) and torch.equal(old, before[1])
    distdl.AdamW(p, *state, *scales).step(g, 1e-3, 2)
    torch.cuda.synchronize()
    assert not torch.equal(p[1], before[1]) and torch.equal(old, before[1])


# Batches that the other tests' sizes leave to none: nb, contraction, columns of a result, workers of either, (columns of a tile, runs of its contraction).
# 256 columns in four runs -- whole, ragged, more than one worker -- and in two, in one turn and in three
RUNS = [(200, 16384, 2816, 1, 1, (256, 4)), (250, 16384, 2800, 1, 1, (256, 4)), (129, 8192, 1408, 2, 2, (256, 4)), (256, 16400, 2576, 1, 1, (256, 4)),
        (1200, 4992, 1040, 2, 1, (256, 2)), (900, 13472, 4800, 1, 1, (256, 2))]


def runs_case(case, adj):
    """nb, features of a worker's input and output block, grid (outputs, inputs)."""
    nb, red, out, workers_red, workers_out, _ = case
    return (nb, out, red, workers_red, workers_out) if adj else (nb, red, out, workers_out, workers_red)


@pytest.mark.parametrize("exact", [True, False], ids=["whole", "normal"])
@pytest.mark.parametrize("adj", [False, True], ids=["fwd", "adj"])
@pytest.mark.parametrize("case", RUNS, ids=str)
def test_affine_fp8_in_runs_of_the_contraction(case, adj, exact):
    """Against products in 64 bits on the device: whole numbers, whose sums are exact in fp32 (at most 2^15 of 64), to the bit; normal ones as in
    test_eight_bit_gpu.py."""
    nb, bfi, bfo, pfo, pfi = runs_case(case, adj)
    shape = distdl.selftest_affine_fp8_shape(nb, bfi * pfi, bfo * pfo, pfo, pfi, adj)
    assert shape[:2] == case[5], shape
    g = torch.Generator(device=DEV)
    g.manual_seed(sum(case[:5]) + adj)
    ki, ko = -(-bfi // 128), -(-bfo // 128)
    (red, kr, nred), (blk, nout) = ((bfo, ko, pfo), (bfi, pfi)) if adj else ((bfi, ki, pfi), (bfo, pfo))
    whole = lambda lo, hi, *s: torch.randint(lo, hi, s, device=DEV, generator=g)  # noqa: E731
    normal = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
    e = lambda *s, dtype=torch.float32: torch.empty(*s, device=DEV, dtype=dtype)  # noqa: E731
    if exact:
        a, asc = [whole(-2, 3, nb, red).float().to(E4) for _ in range(nred)], [torch.exp2(whole(0, 3, kr, nb).float()) for _ in range(nred)]
        w, wsc = [whole(-2, 3, bfo, bfi).float().to(E4) for _ in range(pfo * pfi)], [torch.exp2(whole(0, 3, ko, ki).float()) for _ in range(pfo * pfi)]
        bias = [whole(-9, 10, blk).float() for _ in range(nout)]
    else:
        a, asc, w, wsc = [e(nb, red, dtype=E4) for _ in range(nred)], [e(kr, nb) for _ in range(nred)], [e(bfo, bfi, dtype=E4) for _ in range(pfo * pfi)], [e(ko, ki) for _ in range(pfo * pfi)]
        distdl.quantize_rows(nb, red * nred, nred, [normal(nb, red) for _ in range(nred)], a, asc)
        distdl.quantize_weights(bfi * pfi, bfo * pfo, pfo, pfi, [normal(bfo, bfi) * 0.05 for _ in range(pfo * pfi)], w, wsc)
        bias = [normal(blk) for _ in range(nout)]
    av = [q.double() * s.double().t().repeat_interleave(128, 1)[:, :red] for q, s in zip(a, asc)]
    wv = [q.double() * s.double().repeat_interleave(128, 0)[:bfo].repeat_interleave(128, 1)[:, :bfi] for q, s in zip(w, wsc)]
    for t in (torch.float32, torch.bfloat16):
        out = Out()
        y = [out(nb, blk, dtype=t) for _ in range(nout)]
        if adj:
            distdl.affine_fp8_adj(nb, bfi * pfi, bfo * pfo, pfo, pfi, a, asc, w, wsc, y)
        else:
            distdl.affine_fp8_fwd(nb, bfi * pfi, bfo * pfo, pfo, pfi, a, asc, w, wsc, bias, y)
        distdl.device_status()
        for j in range(nout):
            pairs = [(av[i], wv[i * pfi + j] if adj else wv[j * pfi + i].t()) for i in range(nred)]
            want, size = sum(x @ v for x, v in pairs), sum(x.abs() @ v.abs() for x, v in pairs)
            if not adj:
                want, size = want + bias[j].double(), size + bias[j].double().abs()
            if exact:
                assert torch.equal(y[j].double(), want.float().to(t).double())
            else:
                err = (2 * 128 + 2 + kr * nred + 8) * U * size
                assert ((y[j].double() - want).abs() <= err + eps_of(t) * (want.abs() + err)).all()
        out.check()


def test_affine_fp8_cases_reach_every_shape_of_this_device():
    """As in the CPU test of the same rule, with the clusters that this device holds."""
    for adj in (False, True):
        cases = [c for c in FP8 if c[0] > 128] + [runs_case(c, adj) for c in RUNS]
        seen = {distdl.selftest_affine_fp8_shape(c[0], c[1] * c[4], c[2] * c[3], c[3], c[4], adj)[:2] for c in cases}
        assert seen == {(n, r) for n in (256, 128) for r in (1, 2, 4)}, seen


def test_adamw_codes_in_8_bits_decay_under_a_scale_that_stays():
    """One element of each block has a gradient that keeps both its moments, and so the block's scale, where they are; the others have none, and their
    codes have to fall by beta (its root) a step, 0.5 % and 0.05 %, where the codes are 6 to 12 % apart.  Rounded to nearest none would ever move.

    A value x on a code, w = x / 8 at most above the next one, moves down by it with probability (1 - beta) x / w: it keeps the mean, with a variance of
    (1 - beta) x w <= (1 - beta) x^2 / 8.  After n steps that is (1 + (1 - beta) / 8 / beta^2)^n - 1 of the squared mean or less; six deviations of the mean of
    all elements, and the kept moments' own roundings (2 U a step)."""
    n, steps, b1, b2 = 4096, 400, 0.995, 0.999
    p, g = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    m, v = [torch.full((n,), 288.0, device=DEV).to(E4) for _ in range(2)]
    ms, vs = [torch.ones(n // 128, device=DEV) for _ in range(2)]
    m[::128], v[::128], g[::128] = 448.0, 448.0, 448.0
    opt = distdl.AdamW([p], [m], [v], [ms], [vs])
    for t in range(steps):
        opt.step([g], 1e-3, 10 + t, betas=(b1, b2), seed=17)
    rest = np.arange(n) % 128 != 0
    for code, scale, beta in ((m, ms, b1), (v, vs, b2 ** 0.5)):
        c, s = f64(code), f64(scale)
        assert (c[~rest] == 448).all() and (np.abs(s - 1) <= 4 * steps * U).all()
        spread = np.sqrt(((1 + (1 - beta) / 8 / beta ** 2) ** steps - 1) / rest.sum())
        bound = 6 * spread + 4 * steps * U
        mean = (c * np.repeat(s, 128))[rest].mean() / 288
        assert abs(mean / beta ** steps - 1) <= bound, (mean, beta ** steps, bound)
        nearest = np.full(4, 288.0)
        for _ in range(steps):
            nearest = o.e4m3_round(nearest * beta)
        assert (nearest == 288).all() and abs(nearest.mean() / 288 / beta ** steps - 1) > bound
