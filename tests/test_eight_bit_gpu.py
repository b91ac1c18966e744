"""GPU tests of the operators of 8-bit affine blocks against the oracle (fp64), at the sizes and values where they can go wrong.

Tolerances count the roundings: half a step of the type for a value that is rounded to it (bfloat16 2^-8, fp32 2^-24 relative), n 2^-24
of the sum of magnitudes for an fp32 sum with n additions on a path.
"""

import numpy as np
import pytest

import paper_2006_03108_b200 as distdl
from oracle import eight_bit as o
from paper_2006_03108_b200 import inputs

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E4 = torch.float8_e4m3fn
U = 2.0 ** -24
GUARD = 64                                      # elements on either side of an output that have to stay


def dev(a, dtype=torch.float32):
    return torch.from_numpy(np.array(a)).to(DEV).to(dtype)


def f64(t):
    return t.double().cpu().numpy()


class Out:
    """Outputs in buffers of garbage; `check` looks at what lies around them."""

    def __init__(self):
        self.held = []

    def __call__(self, *shape, dtype=torch.float32):
        n = int(np.prod(shape))
        buf = torch.full(((n + 2 * GUARD) * dtype.itemsize,), 0x5b, dtype=torch.uint8, device=DEV).view(dtype)
        self.held.append((buf, n))
        return buf[GUARD:GUARD + n].view(*shape)

    def check(self):
        for buf, n in self.held:
            b = buf.view(torch.uint8)
            size = buf.dtype.itemsize
            assert (b[:GUARD * size] == 0x5b).all() and (b[(GUARD + n) * size:] == 0x5b).all()


def rounded(a, t):
    """fp32 numbers as a tensor of a type holds them."""
    return a.astype(np.float32) if t is torch.float32 else inputs.bf16_bits_to_f32(inputs.f32_to_bf16_bits(a))


def eps_of(t):
    return 2.0 ** -8 if t is torch.bfloat16 else 2.0 ** -24


def same_quant(q, s, want):
    assert np.array_equal(f64(q), want[0], equal_nan=True) and np.array_equal(s.cpu().numpy(), want[1], equal_nan=True)


BF = [1, 7, 8, 16, 100, 127, 128, 129, 130, 250, 1250, 2048, 2052]


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("bf", BF)
@pytest.mark.parametrize("nb,pf", [(1, 1), (3, 2), (17, 3), (40, 8)])
def test_quantize_rows_to_the_bit(t, bf, nb, pf):
    x = [rounded(inputs.normal((nb, bf), 10 + j) * np.float32(10.0) ** inputs.integers((nb, 1), 90 + j, -6, 7), t) for j in range(pf)]
    out = Out()
    q, s = [out(nb, bf, dtype=E4) for _ in range(pf)], [out(-(-bf // 128), nb) for _ in range(pf)]
    distdl.quantize_rows(nb, bf * pf, pf, [dev(a, t) for a in x], q, s)
    for a, b, c in zip(x, q, s):
        same_quant(b, c, o.quantize_rows(a))
    out.check()


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("bfo,bfi,pfo,pfi", [(1, 1, 1, 1), (128, 128, 1, 1), (129, 127, 2, 1), (250, 130, 1, 3), (64, 516, 2, 2), (300, 1000, 1, 2), (7, 2050, 4, 4)])
def test_quantize_weights_to_the_bit(t, bfo, bfi, pfo, pfi):
    w = [rounded(inputs.normal((bfo, bfi), 20 + i, 0.02 * (i + 1)), t) for i in range(pfo * pfi)]
    out = Out()
    q, s = [out(bfo, bfi, dtype=E4) for _ in w], [out(-(-bfo // 128), -(-bfi // 128)) for _ in w]
    distdl.quantize_weights(bfi * pfi, bfo * pfo, pfo, pfi, [dev(a, t) for a in w], q, s)
    for a, b, c in zip(w, q, s):
        same_quant(b, c, o.quantize_weights(a))
    out.check()


@pytest.mark.parametrize("weights", [False, True], ids=["rows", "weights"])
def test_quantize_special_values(weights):
    """Zeros, the smallest and largest numbers, infinities and NaN: a block's fate is its own."""
    x = inputs.normal((8, 640), 5)
    x[0, :128] = 0.0
    x[1] = 0.0
    x[2, 128:256] = 1e-45                       # below every normal number
    x[3, 256:384] *= np.float32(3e38 / 5)
    x[4, 130] = np.inf
    x[5, 300] = np.nan
    x[6, 5] = -np.inf
    x[7, 639] = -0.0
    a = np.ascontiguousarray(x.repeat(128, 0)) if weights else x
    q, s = torch.empty(*a.shape, dtype=E4, device=DEV), torch.empty((8, 5) if weights else (5, 8), device=DEV)
    if weights:
        distdl.quantize_weights(640, 1024, 1, 1, [dev(a)], [q], [s])
    else:
        distdl.quantize_rows(8, 640, 1, [dev(a)], [q], [s])
    with np.errstate(invalid="ignore", over="ignore"):
        value = f64(q) * np.repeat(np.repeat(f64(s), 128, 0), 128, 1) if weights else o.row_values(f64(q), s.cpu().numpy())
        value = value[::128] if weights else value
    bad = np.zeros((8, 5), bool)
    bad[4, 1] = bad[5, 2] = bad[6, 0] = True
    bad = np.repeat(bad, 128, 1)
    assert np.isnan(value[bad]).all() and np.isfinite(value[~bad]).all()
    want = o.quantize_rows(np.where(bad, 0, x))
    ok = np.repeat(want[1].T, 128, 1)
    assert np.array_equal(value[~bad], (want[0] * ok)[~bad]) and (value[1] == 0).all() and (value[2, 128:256] == 0).all()


NORM = [(1, 1, 1), (3, 1, 2), (2, 8192, 1), (5, 100, 8), (300, 128, 1), (297, 40, 3), (400, 1250, 4), (9, 5000, 2), (310, 2048, 4), (2, 16384, 2), (3, 5003, 8), (700, 8, 1),
        (301, 16500, 2)]


def norm_inputs(nb, bf, pf, t, seed=40):
    x = [rounded(inputs.normal((nb, bf), seed + j, 2.0), t) for j in range(pf)]
    r = [rounded(inputs.normal((nb, bf), seed + 20 + j), t) for j in range(pf)]
    g = [1 + inputs.normal((bf,), seed + 40 + j, 0.2) for j in range(pf)]
    return x, r, g


def sum_error(n_features, pf):
    """Additions on a path of the kernel's sum over a sample's features: at most eight for each chunk of a thread, ten through its
    group; the chunks (padded to blocks of 128 per worker) are spread over a thread for every four or more, up to 1024 of them."""
    chunks = pf * -(-(n_features // pf) // 128) * 16
    return (8 * max(4, -(-chunks // 512)) + 12) * U


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("nb,bf,pf", NORM)
def test_rmsnorm_fwd(t, nb, bf, pf):
    eps, nf = 1e-5, bf * pf
    x, r, g = norm_inputs(nb, bf, pf, t)
    out = Out()
    h, y = [out(nb, bf, dtype=t) for _ in range(pf)], [out(nb, bf, dtype=t) for _ in range(pf)]
    q, qs = [out(nb, bf, dtype=E4) for _ in range(pf)], [out(-(-bf // 128), nb) for _ in range(pf)]
    rstd = out(nb)
    distdl.rmsnorm_fwd(nb, nf, pf, [dev(a, t) for a in x], [dev(a, t) for a in r], [dev(a) for a in g], eps, h, y, q, qs, rstd)
    hw = [rounded(a + b, t).astype(np.float64) for a, b in zip(x, r)]          # fp32 sum, rounded to the type
    for a, b in zip(h, hw):
        assert np.array_equal(f64(a), b)
    yw, rw = o.rmsnorm_fwd(hw, [a.astype(np.float64) for a in g], float(np.float32(eps)))
    re = sum_error(nf, pf) / 2 + 4 * U                                          # half of the sum's; mean, + eps, root, quotient
    assert (np.abs(f64(rstd) - rw) <= re * rw).all()
    for j in range(pf):
        ye = (re + 3 * U) * np.abs(yw[j])
        assert (np.abs(f64(y[j]) - yw[j]) <= ye + eps_of(t) * (np.abs(yw[j]) + ye)).all()
        v, scale = o.row_values(f64(q[j]), qs[j].cpu().numpy()), np.repeat(f64(qs[j]).T, 128, 1)[:, :bf]
        assert (np.abs(v - yw[j]) <= np.maximum(2.0 ** -4 * np.abs(yw[j]), 2.0 ** -10 * scale) * (1 + 4 * U) + 2 * ye).all()
        if t is torch.float32:                                                  # y is the value that is quantised
            same_quant(q[j], qs[j], o.quantize_rows(y[j].cpu().numpy()))
    out.check()
    # without a residual, one output at a time, and the sum in place of the residual: the same values
    hx = [dev(a, t) for a in hw]
    for keep in ("y", "q", "rstd"):
        y2, q2, s2, r2 = [torch.zeros_like(a) for a in y], [torch.zeros_like(a) for a in q], [torch.zeros_like(a) for a in qs], torch.zeros_like(rstd)
        distdl.rmsnorm_fwd(nb, nf, pf, hx, None, [dev(a) for a in g], eps, None, y2 if keep == "y" else None, q2 if keep == "q" else None,
                           s2 if keep == "q" else None, r2 if keep == "rstd" else None)
        for a, b in {"y": zip(y, y2), "q": list(zip(q, q2)) + list(zip(qs, s2)), "rstd": [(rstd, r2)]}[keep]:
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    rd = [dev(a, t) for a in r]
    distdl.rmsnorm_fwd(nb, nf, pf, [dev(a, t) for a in x], rd, [dev(a) for a in g], eps, rd)
    for a, b in zip(rd, h):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("tg", [torch.float32, torch.bfloat16], ids=["gf32", "gbf16"])
@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("nb,bf,pf", NORM)
@pytest.mark.parametrize("res", [True, False], ids=["res", "nores"])
def test_rmsnorm_adj(t, tg, nb, bf, pf, res):
    nf = bf * pf
    h, _, g = norm_inputs(nb, bf, pf, t, 140)
    dy = [rounded(inputs.normal((nb, bf), 200 + j, 0.1), tg) for j in range(pf)]
    dres = [rounded(inputs.normal((nb, bf), 220 + j, 0.1), tg) for j in range(pf)] if res else None
    rstd = (1 / np.sqrt(sum((a.astype(np.float64) ** 2).sum(1) for a in h) / nf + 1e-5)).astype(np.float32)
    out = Out()
    dh, dg = [out(nb, bf, dtype=tg) for _ in range(pf)], [out(bf) for _ in range(pf)]
    ws = out(distdl.rmsnorm_adj_workspace(nb, nf, pf), dtype=torch.uint8)
    args = [dev(a, t) for a in h], [dev(a) for a in g], dev(rstd)
    dy_d, dres_d = [dev(a, tg) for a in dy], [dev(a, tg) for a in dres] if res else None
    distdl.rmsnorm_adj(nb, nf, pf, dy_d, dres_d, *args, dh, dg, ws)
    h64, g64, d64 = ([a.astype(np.float64) for a in v] for v in (h, g, dy))
    dhw, dgw = o.rmsnorm_adj(d64, [a.astype(np.float64) for a in dres] if res else None, h64, g64, rstd)
    r = rstd.astype(np.float64)[:, None]
    terms = sum((np.abs(a * b * c)).sum(1, keepdims=True) for a, b, c in zip(d64, h64, g64)) / nf
    total = nb if nb < 20 else 20 + nb / 8                # additions on a path of dgamma: samples of a block, groups, blocks
    for j in range(pf):
        back = np.abs(h64[j]) * r ** 3 * terms
        e = (sum_error(nf, pf) + 8 * U) * back + 4 * U * (np.abs(r * g64[j] * d64[j]) + (np.abs(dres[j]) if res else 0) + back)
        assert (np.abs(f64(dh[j]) - dhw[j]) <= e + eps_of(tg) * (np.abs(dhw[j]) + e)).all()
        assert (np.abs(f64(dg[j]) - dgw[j]) <= (total + 4) * U * np.abs(d64[j] * h64[j] * r).sum(0)).all()
    out.check()
    # the same bits again; without dgamma; in place of dy and of dres
    again = [torch.empty_like(a) for a in dg]
    distdl.rmsnorm_adj(nb, nf, pf, dy_d, dres_d, *args, dy_d, again, ws)
    assert all(torch.equal(a, b) for a, b in zip(again, dg)) and all(torch.equal(a, b) for a, b in zip(dy_d, dh))
    if res:
        distdl.rmsnorm_adj(nb, nf, pf, [dev(a, tg) for a in dy], dres_d, *args, dres_d, None, ws)
        assert all(torch.equal(a, b) for a, b in zip(dres_d, dh))


def test_rmsnorm_gradient_against_differences():
    """<dh, way> and <dgamma, way> against central differences of the fp64 definition."""
    nb, bf, pf, eps = 5, 333, 3, 1e-5
    h, way, g = norm_inputs(nb, bf, pf, torch.float32, 300)
    h64, w64, g64 = ([a.astype(np.float64) for a in v] for v in (h, way, g))
    dy = [inputs.normal((nb, bf), 360 + j) for j in range(pf)]
    rstd = torch.empty(nb, device=DEV)
    hd, gd = [dev(a) for a in h], [dev(a) for a in g]
    distdl.rmsnorm_fwd(nb, bf * pf, pf, hd, None, gd, eps, rstd=rstd)
    dh, dg = [torch.empty_like(a) for a in hd], [torch.empty_like(a) for a in gd]
    distdl.rmsnorm_adj(nb, bf * pf, pf, [dev(a) for a in dy], None, hd, gd, rstd, dh, dg,
                       torch.empty(distdl.rmsnorm_adj_workspace(nb, bf * pf, pf), dtype=torch.uint8, device=DEV))
    loss = lambda a, b: sum((u * v).sum() for u, v in zip(o.rmsnorm_fwd([x + a * w for x, w in zip(h64, w64)], [x + b * w[0] for x, w in zip(g64, w64)], eps)[0], dy))  # noqa: E731
    step = 1e-5
    for got, want, scale in ((sum((f64(a) * b).sum() for a, b in zip(dh, w64)), (loss(step, 0) - loss(-step, 0)) / (2 * step), sum(np.abs(f64(a) * b).sum() for a, b in zip(dh, w64))),
                             (sum((f64(a) * b[0]).sum() for a, b in zip(dg, w64)), (loss(0, step) - loss(0, -step)) / (2 * step), sum(np.abs(f64(a) * b[0]).sum() for a, b in zip(dg, w64)))):
        assert abs(got - want) <= 1e-6 * scale


def test_rmsnorm_of_a_bad_sample_is_its_own():
    """Infinity or NaN in a sample stays in that sample (dgamma sums over all of them)."""
    nb, bf, pf = 40, 136, 2
    x, _, g = norm_inputs(nb, bf, pf, torch.float32, 400)
    clean = [a.copy() for a in x]
    x[0][7, 3], x[1][20, 135], x[0][39, 0] = np.inf, np.nan, -np.inf
    for a in clean:
        a[[7, 20, 39]] = 0.0
    bad = np.isin(np.arange(nb), [7, 20, 39])
    res = []
    for v in (x, clean):
        xd, gd = [dev(a) for a in v], [dev(a) for a in g]
        y, q, s = [torch.empty_like(a) for a in xd], [torch.empty(nb, bf, dtype=E4, device=DEV) for _ in xd], [torch.empty(2, nb, device=DEV) for _ in xd]
        rstd, dh = torch.empty(nb, device=DEV), [torch.empty_like(a) for a in xd]
        distdl.rmsnorm_fwd(nb, bf * pf, pf, xd, None, gd, 1e-6, None, y, q, s, rstd)
        ws = torch.empty(distdl.rmsnorm_adj_workspace(nb, bf * pf, pf), dtype=torch.uint8, device=DEV)
        distdl.rmsnorm_adj(nb, bf * pf, pf, y, None, xd, gd, rstd, dh, None, ws)
        res.append([f64(a)[~bad] for a in y + q + dh] + [f64(a)[:, ~bad] for a in s] + [f64(rstd)[~bad]])
        if v is x:
            assert np.isnan(f64(y[0])[20]).all() and np.isnan(f64(y[0])[7, 3])
    assert all(np.array_equal(a, b) and np.isfinite(a).all() for a, b in zip(*res))
    # a sample of zeros is normed to zeros
    assert (f64(rstd)[7] == np.float32(1) / np.sqrt(np.float32(1e-6))).all() and (f64(y[0])[7] == 0).all() and (f64(q[1])[7] == 0).all()


def test_rmsnorm_of_no_samples():
    dg = [torch.full((130,), 5.0, device=DEV) for _ in range(2)]
    e = [torch.empty(0, 130, device=DEV) for _ in range(2)]
    distdl.rmsnorm_fwd(0, 260, 2, e, e, dg, 1e-6, e, e)
    assert all((a == 5).all() for a in dg)
    distdl.rmsnorm_adj(0, 260, 2, e, None, e, dg, e[0].view(0), e, dg, torch.empty(16, dtype=torch.uint8, device=DEV))
    assert all((a == 0).all() for a in dg)
    distdl.quantize_rows(0, 260, 2, e, [a.to(E4) for a in e], [torch.empty(2, 0, device=DEV)] * 2)
    torch.cuda.synchronize()


def test_host_memory_is_refused():
    t = torch.zeros(4, 128)
    with pytest.raises(distdl.DistdlError) as e:
        distdl.quantize_rows(4, 128, 1, [t], [t.to(E4)], [torch.zeros(1, 4)])
    assert e.value.status == 1


# ---------------------------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------------------------

SIZES = [1, 3, 0, 127, 128, 129, 1000, 8192, 8193, 70001, 16384, 2, 257]
HYPER = dict(lr=2e-3, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1, grad_scale=0.5)


def adam_state(sizes, seed, eight):
    p = [inputs.normal((n,), seed + 5 * i, 0.1) for i, n in enumerate(sizes)]
    g = [inputs.normal((n,), seed + 5 * i + 1, 1e-2) for i, n in enumerate(sizes)]
    m = [inputs.normal((n,), seed + 5 * i + 2, 1e-3) for i, n in enumerate(sizes)]
    r = [np.abs(inputs.normal((n,), seed + 5 * i + 3, 4e-3)) for i, n in enumerate(sizes)]
    if not eight:
        return p, g, m, [a * a for a in r], None, None
    m, ms = zip(*[o.moment_to_8_bits(a, 0.5, False) for a in m])
    r, vs = zip(*[o.moment_to_8_bits(a, 0.5, True) for a in r])
    return p, g, list(m), list(r), list(ms), list(vs)


def adam_check(i, n, got, before, g, step, seed, eight, h=HYPER):
    """One tensor after a step against fp64; got, before: (p, m, v, ms, vs)."""
    p, m, v, ms, vs = before
    m64, v64 = np.asarray(m, np.float64), np.asarray(v, np.float64)
    if eight:
        rep = lambda s: np.repeat(np.asarray(s, np.float64), 128)[:n]  # noqa: E731
        m64, v64 = m64 * rep(ms), (v64 * rep(vs)) ** 2
    b1, b2 = h["betas"]
    c = h["grad_scale"]
    pw, mw, vw = o.adamw(p, g, m64, v64, h["lr"], step, h["betas"], h["eps"], h["weight_decay"], c)
    # m, v: the constants, the products and the sum are rounded; v's square doubles what it gets; p: its own rounding, and the change's
    me = 5 * U * (b1 * np.abs(m64) + (1 - b1) * np.abs(c * g))
    ve = 8 * U * vw
    change = np.abs(h["lr"] * h["weight_decay"] * p) + np.abs(h["lr"] / (1 - b1 ** step) / (np.sqrt(vw / (1 - b2 ** step)) + h["eps"])) * (np.abs(mw) + me / (16 * U))
    assert (np.abs(f64(got[0]) - pw) <= 1.01 * U * np.abs(pw) + 16 * U * change).all(), i
    if not eight:
        assert (np.abs(f64(got[1]) - mw) <= me).all() and (np.abs(f64(got[2]) - vw) <= ve).all(), i
        return
    bits = o.random_bits(0, n, seed, step, i)
    for k, value, u, positive in ((1, mw, bits & 0xFFFF, False), (2, np.sqrt(vw), bits >> 16, True)):
        code, scale = f64(got[k]), f64(got[k + 2])
        pad = np.zeros(len(scale) * 128)
        pad[:n] = value
        top = np.maximum(np.abs(pad.reshape(-1, 128)).max(1), 2.0 ** -100)
        assert (np.abs(scale - top / 448) <= 12 * U * top / 448).all(), i
        a = np.minimum(np.abs(value) * 448 / np.repeat(top, 128)[:n], 448)
        want = np.copysign(o.stochastic_e4m3(a, u / 65536.0, positive), value)
        width = 2.0 ** (np.maximum(np.frexp(a)[1] - 1, -6) - 3.0)
        # a code differs only where the value, known to 20 U, ends next to a random number: twice 20 U * 16 / 2^-16 of them or so
        assert (np.abs(code - want) <= width * 1.0001).all() and (code != want).mean() <= 1e-3 + 2 / n, i
        assert not positive or (code[vw > 0] > 0).all()


@pytest.mark.parametrize("eight", [False, True], ids=["f32", "8bit"])
@pytest.mark.parametrize("tg", [torch.float32, torch.bfloat16], ids=["gf32", "gbf16"])
def test_adamw_against_the_definition(tg, eight):
    p, g, m, v, ms, vs = adam_state(SIZES, 1000, eight)
    g = [rounded(a, tg) for a in g]
    out, held = Out(), E4 if eight else torch.float32

    def put(a, dtype=torch.float32):
        t = out(len(a), dtype=dtype)
        t.copy_(dev(a))
        return t

    pd, md, vd = [put(a) for a in p], [put(a, held) for a in m], [put(a, held) for a in v]
    msd, vsd = ([put(a) for a in ms], [put(a) for a in vs]) if eight else (None, None)
    copies = [out(n, dtype=torch.bfloat16) if i % 3 else None for i, n in enumerate(SIZES)]
    opt = distdl.AdamW(pd, md, vd, msd, vsd, copies)
    gd = [dev(a, tg) for a in g]
    for step in (7, 8):
        before = [[f64(a[i]) if a is not None else None for a in (pd, md, vd, msd, vsd)] for i in range(len(SIZES))]
        opt.step(gd, step=step, seed=99, **HYPER)
        for i, n in enumerate(SIZES):
            if n:
                adam_check(i, n, [a[i] if a is not None else None for a in (pd, md, vd, msd, vsd)], before[i], g[i].astype(np.float64), step, 99, eight)
            if copies[i] is not None:
                assert torch.equal(copies[i], pd[i].bfloat16())
    assert all(torch.equal(a, dev(b, tg)) for a, b in zip(gd, g))
    out.check()


@pytest.mark.parametrize("eight", [False, True], ids=["f32", "8bit"])
def test_adamw_of_many_tensors_is_that_of_each(eight):
    """More tensors than a launch takes: the same bits as one at a time (in 8 bits: up to the random numbers, which go by the tensor)."""
    sizes = [(17 * i) % 300 for i in range(701)]
    p, g, m, v, ms, vs = adam_state(sizes, 7000, eight)
    held = E4 if eight else torch.float32
    state = lambda: [[dev(a) for a in p], [dev(a, held) for a in m], [dev(a, held) for a in v]] + ([[dev(a) for a in ms], [dev(a) for a in vs]] if eight else [])  # noqa: E731
    a, b, gd = state(), state(), [dev(x) for x in g]
    distdl.AdamW(*a).step(gd, step=3, **HYPER)
    for i in range(len(sizes)):
        distdl.AdamW(*[x[i:i + 1] for x in b]).step(gd[i:i + 1], step=3, **HYPER)
    for k in (0, 3, 4) if eight else (0, 1, 2):
        assert all(torch.equal(x, y) for x, y in zip(a[k], b[k])), k
    if eight:
        i = 653                                                      # in the third launch
        adam_check(i, sizes[i], [x[i] for x in a], [p[i], m[i], v[i], ms[i], vs[i]], g[i].astype(np.float64), 3, 0, True)


def test_adamw_first_step_moves_every_weight_by_the_rate():
    """From a state of zeros: |change| = lr for every gradient that is not zero, whatever its size; nothing else moves."""
    n = 1000
    g = inputs.normal((n,), 3) * np.float32(10.0) ** inputs.integers((n,), 4, -6, 7)
    g[::7] = 0.0
    for eight in (False, True):
        p = torch.zeros(n, device=DEV)
        m, v = [torch.zeros(n, device=DEV, dtype=E4 if eight else torch.float32) for _ in range(2)]
        scales = [[torch.zeros(8, device=DEV)] for _ in range(2)] if eight else [None, None]
        distdl.AdamW([p], [m], [v], *scales).step([dev(g)], 1e-2, 1, eps=1e-30, weight_decay=0.0)
        assert (np.abs(np.abs(f64(p)) - 1e-2 * (g != 0)) <= 1e-2 * 16 * U).all() and (np.sign(f64(p)) == -np.sign(g)).all()


def test_adamw_states_in_8_bits_follow_small_decays():
    """A second moment that shrinks by 0.1 % a step does shrink: the codes' mean over 4096 elements after 400 steps without gradients
    (e4m3 steps are 6 to 12 %: rounded to nearest nothing would move), and a first moment at 0.5 % a step."""
    n, steps = 4096, 400
    p, g = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    m, v = [torch.full((n,), 300.0, device=DEV).to(E4) for _ in range(2)]
    ms, vs = [torch.ones(n // 128, device=DEV) for _ in range(2)]
    m[::128] = v[::128] = 448.0                                       # holds the scale of its block, which decays with it
    opt = distdl.AdamW([p], [m], [v], [ms], [vs])
    start = [(a.double() * s.double().repeat_interleave(128)).mean().item() for a, s in ((m, ms), (v, vs))]
    for t in range(steps):
        opt.step([g], 1e-3, 10 + t, betas=(0.995, 0.999))
    end = [(a.double() * s.double().repeat_interleave(128)).mean().item() for a, s in ((m, ms), (v, vs))]
    # each rounding keeps the mean and moves a code by less than 1/8 of itself: after 400 of them the deviation of an element is at most
    # 1/16 sqrt(400) of itself, of the mean of 4096 elements 1.25 / 64 -- the scales are exact but for their roundings
    assert abs(end[0] / start[0] / 0.995 ** steps - 1) < 0.1 and abs(end[1] / start[1] / 0.999 ** (steps / 2) - 1) < 0.1


@pytest.mark.parametrize("eight", [False, True], ids=["f32", "8bit"])
def test_adamw_live_arguments_and_replayed_steps(eight):
    p, g, m, v, ms, vs = adam_state([5000, 300], 500, eight)
    held = E4 if eight else torch.float32
    state = lambda: [[dev(a) for a in p], [dev(a, held) for a in m], [dev(a, held) for a in v]] + ([[dev(a) for a in ms], [dev(a) for a in vs]] if eight else [])  # noqa: E731
    gd = [dev(a) for a in g]
    h = {k: x for k, x in HYPER.items() if k not in ("lr", "grad_scale")}
    live = torch.zeros(3, device=DEV)
    eager, other, replayed = state(), state(), state()
    opts = [distdl.AdamW(*s) for s in (eager, other, replayed)]
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        live.copy_(torch.tensor([0.0, 1.0, 0.0]))
        distdl.AdamW(*state()).step(gd, 0.0, 0, live=live, seed=3, **h)       # loads the kernel
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        opts[2].step(gd, 0.0, 0, live=live, seed=3, **h)
    torch.cuda.synchronize()
    for t in (1, 2, 3, 1000):
        live.copy_(torch.tensor([1e-3 * t, float(t), 0.25]))
        opts[0].step(gd, 0.0, 0, live=live, seed=3, **h)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        opts[1].step(gd, 1e-3 * t, t, seed=3, grad_scale=0.25, **h)
    for a, b in zip(eager, replayed):
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))
    for a, b in zip(eager[0], other[0]):                                # 1 - beta^t in fp32 and fp64
        assert (a - b).abs().max() <= 64 * U * (0.2 + 4 * 1.1)


def test_adamw_bad_gradients_stay_where_they_are():
    n = 1024
    for eight in (False, True):
        p, g, m, v, ms, vs = adam_state([n], 800, eight)
        g[0][5], g[0][600] = np.inf, np.nan
        held = E4 if eight else torch.float32
        s = [[dev(a) for a in p], [dev(a, held) for a in m], [dev(a, held) for a in v]] + ([[dev(a) for a in ms], [dev(a) for a in vs]] if eight else [])
        distdl.AdamW(*s).step([dev(g[0])], step=4, **HYPER)
        touched = np.isin(np.arange(n) // (128 if eight else 1), [0, 4] if eight else [5, 600])
        value = [f64(s[0][0])]
        assert np.isnan(value[0][600]) and np.isfinite(value[0][~np.isin(np.arange(n), [5, 600])]).all()
        for k in (1, 2):
            x = f64(s[k][0]) * (np.repeat(f64(s[k + 2][0]), 128) if eight else 1.0)
            assert np.isfinite(x[~touched]).all() and not np.isfinite(x[touched]).any()


def test_adamw_beyond_32_bits_of_elements():
    n, tail = 2 ** 32 + 333, 1000
    if torch.cuda.get_device_properties(0).total_memory < 80 << 30:
        pytest.skip("needs 40 GB")
    p, g = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV, dtype=torch.bfloat16)
    m, v = [torch.zeros(n, device=DEV, dtype=torch.uint8).view(E4) for _ in range(2)]
    ms, vs = [torch.zeros(-(-n // 128), device=DEV) for _ in range(2)]
    at = (n - tail) // 128 * 128
    pw, gw = inputs.normal((n - at,), 1), rounded(inputs.normal((n - at,), 2), torch.bfloat16)
    p[at:].copy_(dev(pw))
    g[at:].copy_(dev(gw))
    distdl.AdamW([p], [m], [v], [ms], [vs]).step([g], step=2, seed=5, **HYPER)
    zero = np.zeros(n - at)
    _, mw, vw = o.adamw(pw, gw, zero, zero, HYPER["lr"], 2, HYPER["betas"], HYPER["eps"], HYPER["weight_decay"], HYPER["grad_scale"])
    bits = o.random_bits(at, n - at, 5, 2, 0)
    for code, scale, value, u, positive in ((m, ms, mw, bits & 0xFFFF, False), (v, vs, np.sqrt(vw), bits >> 16, True)):
        want, sw = o.moment_to_8_bits(value, u / 65536.0, positive)
        assert (f64(code[at:]) != want).mean() <= 3e-3 and np.allclose(f64(scale[at // 128:]), sw, rtol=12 * U)
    assert not p[:at].any() and not m.view(torch.uint8)[:at].any() and p[at:].ne(dev(pw)).any()


# ---------------------------------------------------------------------------------------------
# The affine layer in 8 bits
# ---------------------------------------------------------------------------------------------

# nb, features of a worker's input and output block, grid
FP8 = [(1, 16, 16, 1, 1), (1, 128, 128, 1, 1), (2, 144, 272, 2, 3), (16, 2048, 2048, 2, 2), (17, 400, 112, 1, 2), (33, 1040, 656, 2, 2), (64, 256, 128, 4, 1),
       (65, 48, 1040, 1, 4), (100, 128, 2048, 1, 1), (128, 1296, 32, 3, 2), (129, 128, 128, 1, 1), (129, 16, 16, 2, 2), (200, 272, 656, 2, 3), (256, 2048, 256, 1, 2),
       (256, 512, 1024, 2, 4), (300, 144, 144, 1, 1), (513, 1040, 80, 3, 1), (777, 208, 400, 2, 2), (1500, 640, 1280, 1, 1), (3000, 256, 2048, 1, 1), (1000, 4096, 96, 1, 4),
       # contractions of more k-blocks than a block's ring has stages, either way
       (3, 16384, 144, 1, 1), (3, 144, 16384, 1, 1), (20, 8192, 512, 1, 2), (20, 512, 8192, 2, 1), (60, 16384, 128, 1, 1), (60, 128, 16384, 1, 1), (90, 8192, 256, 1, 2),
       (90, 256, 8192, 2, 1), (200, 8192, 272, 1, 2), (200, 272, 8192, 2, 1), (2000, 4096, 512, 1, 1), (2000, 512, 4096, 1, 1), (1200, 5000 // 16 * 16, 1040, 1, 2)]


def fp8_inputs(nb, bfi, bfo, pfo, pfi, adj, exact, seed=600):
    """Activations, weights as (values, scales) pairs.  exact: whole numbers, scales that are powers of two, sums below 2^24 steps."""
    blk, n = (bfo, pfo) if adj else (bfi, pfi)
    if exact:
        pow2 = lambda shape, s: np.float32(2.0) ** inputs.integers(shape, s, 0, 3)  # noqa: E731
        a = [(inputs.integers((nb, blk), seed + j, -2, 3).astype(np.float64), pow2((-(-blk // 128), nb), seed + 50 + j)) for j in range(n)]
        w = [(inputs.integers((bfo, bfi), seed + 100 + i, -2, 3).astype(np.float64), pow2((-(-bfo // 128), -(-bfi // 128)), seed + 150 + i)) for i in range(pfo * pfi)]
    else:
        a = [o.quantize_rows(inputs.normal((nb, blk), seed + j) * np.float32(3.0) ** inputs.integers((nb, 1), seed + 50 + j, -3, 4)) for j in range(n)]
        w = [o.quantize_weights(inputs.normal((bfo, bfi), seed + 100 + i, 0.05)) for i in range(pfo * pfi)]
    return a, w


def fp8_call(nb, bfi, bfo, pfo, pfi, adj, a, w, bias, t, out):
    ad, asd = [dev(v, E4) for v, _ in a], [dev(s) for _, s in a]
    wd, wsd = [dev(v, E4) for v, _ in w], [dev(s) for _, s in w]
    y = [out(nb, bfi if adj else bfo, dtype=t) for _ in range(pfi if adj else pfo)]
    if adj:
        distdl.affine_fp8_adj(nb, bfi * pfi, bfo * pfo, pfo, pfi, ad, asd, wd, wsd, y)
    else:
        distdl.affine_fp8_fwd(nb, bfi * pfi, bfo * pfo, pfo, pfi, ad, asd, wd, wsd, None if bias is None else [dev(b) for b in bias], y)
    distdl.device_status()
    return y


@pytest.mark.parametrize("adj", [False, True], ids=["fwd", "adj"])
@pytest.mark.parametrize("case", FP8, ids=str)
def test_affine_fp8_on_whole_numbers(case, adj):
    """Every product and sum is exact in fp32 (at most 2^16 of them, each at most 64 steps): equal to the oracle in any order."""
    nb, bfi, bfo, pfo, pfi = case
    a, w = fp8_inputs(*case, adj, True)
    bias = None if adj else [inputs.integers((bfo,), 700 + i) for i in range(pfo)]
    want = o.affine_fp8_adj(a, w, pfo, pfi) if adj else o.affine_fp8_fwd(a, w, pfo, pfi, bias)
    for t in (torch.float32, torch.bfloat16):
        out = Out()
        for got, ref in zip(fp8_call(*case, adj, a, w, bias, t, out), want):
            assert np.array_equal(f64(got), rounded(ref.astype(np.float32), t).astype(np.float64))
        out.check()


@pytest.mark.parametrize("adj", [False, True], ids=["fwd", "adj"])
@pytest.mark.parametrize("case", FP8, ids=str)
def test_affine_fp8_on_normal_numbers(case, adj):
    nb, bfi, bfo, pfo, pfi = case
    a, w = fp8_inputs(*case, adj, False)
    bias = None if adj else [inputs.normal((bfo,), 700 + i) for i in range(pfo)]
    fn = o.affine_fp8_adj if adj else o.affine_fp8_fwd
    want = fn(a, w, pfo, pfi) if adj else fn(a, w, pfo, pfi, bias)
    size = fn([(np.abs(v), s) for v, s in a], [(np.abs(v), s) for v, s in w], pfo, pfi)
    # 128 additions of a product in the tensor cores, where a sum may be cut off instead of rounded (2 U each), the scales' product, a rounding per block
    blocks = -(-(bfo if adj else bfi) // 128) * (pfo if adj else pfi)
    for t in (torch.float32, torch.bfloat16):
        out = Out()
        for j, (got, ref, s) in enumerate(zip(fp8_call(*case, adj, a, w, bias, t, out), want, size)):
            e = (2 * 128 + 2 + blocks + 8) * U * (s + (0 if bias is None else np.abs(bias[j])))
            assert (np.abs(f64(got) - ref) <= e + eps_of(t) * (np.abs(ref) + e)).all()
            if t is torch.float32:
                assert np.linalg.norm(f64(got) - ref) <= 1e-6 * np.linalg.norm(s)
        out.check()


# ---------------------------------------------------------------------------------------------
# The operators together, as a block of a network runs them
# ---------------------------------------------------------------------------------------------

class Block:
    """Residual addition, norm and 8-bit affine layer on a worker grid: a training step.  All buffers are its own."""

    def __init__(self, nb, bfi, bfo, pfo, pfi, seed, eight=True):
        self.shape = nb, bfi * pfi, bfo * pfo, pfo, pfi
        e = lambda *s, dtype=torch.float32: torch.empty(*s, device=DEV, dtype=dtype)  # noqa: E731
        bf16, n = torch.bfloat16, pfo * pfi
        ki, ko = -(-bfi // 128), -(-bfo // 128)
        self.base = [dev(inputs.normal((nb, bfi), seed + j), bf16) for j in range(2 * pfi)]
        self.dbase = [dev(inputs.normal((nb, bfo), seed + 20 + i, 0.1), bf16) for i in range(pfo)]
        self.gamma = [dev(1 + inputs.normal((bfi,), seed + 30 + j, 0.1)) for j in range(pfi)]
        self.w = [dev(inputs.normal((bfo, bfi), seed + 40 + i, 0.05)) for i in range(n)]
        self.bias = [dev(inputs.normal((bfo,), seed + 60 + i)) for i in range(pfo)]
        self.x = [torch.empty_like(a) for a in self.base]                # x, then the residual
        self.dy = [torch.empty_like(a) for a in self.dbase]
        self.h, self.y = [[e(nb, bfi, dtype=bf16) for _ in range(pfi)] for _ in range(2)]
        self.q, self.qs, self.rstd = [e(nb, bfi, dtype=E4) for _ in range(pfi)], [e(ki, nb) for _ in range(pfi)], e(nb)
        self.w8, self.ws = [e(bfo, bfi, dtype=E4) for _ in range(n)], [e(ko, ki) for _ in range(n)]
        self.out = [e(nb, bfo, dtype=bf16) for _ in range(pfo)]
        self.dq, self.dqs = [e(nb, bfo, dtype=E4) for _ in range(pfo)], [e(ko, nb) for _ in range(pfo)]
        self.dx, self.dh = [[e(nb, bfi, dtype=bf16) for _ in range(pfi)] for _ in range(2)]
        self.dgamma, self.dw, self.db = [e(bfi) for _ in range(pfi)], [e(bfo, bfi) for _ in range(n)], [e(bfo) for _ in range(pfo)]
        self.ws_adj = e(distdl.rmsnorm_adj_workspace(nb, bfi * pfi, pfi), dtype=torch.uint8)
        params = self.w + self.gamma + self.bias
        zeros = lambda: [torch.zeros(a.numel(), device=DEV, dtype=torch.uint8).view(E4) for a in params]  # noqa: E731
        scales = lambda: [torch.zeros(-(-a.numel() // 128), device=DEV) for a in params]  # noqa: E731
        self.copies = [e(bfo, bfi, dtype=bf16) for _ in range(n)] + [None] * (pfi + pfo)
        self.state = [zeros(), zeros(), scales(), scales()]
        self.opt = distdl.AdamW(params, *self.state, self.copies)
        self.factor = torch.ones((), device=DEV)
        self.live = torch.tensor([1e-3, 1.0, 1.0], device=DEV)

    def step(self, wait=lambda: None):
        nb, nfi, nfo, pfo, pfi = self.shape
        for a, b in zip(self.x + self.dy, self.base + self.dbase):       # the inputs, by kernels of another library
            torch.mul(b, self.factor, out=a)
        wait()
        distdl.quantize_weights(nfi, nfo, pfo, pfi, self.w, self.w8, self.ws)
        wait()
        distdl.rmsnorm_fwd(nb, nfi, pfi, self.x[:pfi], self.x[pfi:], self.gamma, 1e-6, self.h, self.y, self.q, self.qs, self.rstd)
        wait()
        distdl.affine_fp8_fwd(nb, nfi, nfo, pfo, pfi, self.q, self.qs, self.w8, self.ws, self.bias, self.out)
        wait()
        distdl.quantize_rows(nb, nfo, pfo, self.dy, self.dq, self.dqs)
        wait()
        distdl.affine_fp8_adj(nb, nfi, nfo, pfo, pfi, self.dq, self.dqs, self.w8, self.ws, self.dx)
        wait()
        distdl.rmsnorm_adj(nb, nfi, pfi, self.dx, self.dy if nfi == nfo and pfi == pfo else None, self.h, self.gamma, self.rstd, self.dh, self.dgamma, self.ws_adj)
        wait()
        distdl.affine_adj_params(nb, nfi, nfo, pfo, pfi, self.dy, self.y, self.dw, self.db)
        wait()
        self.opt.step(self.dw + self.dgamma + self.db, 0.0, 0, betas=(0.9, 0.95), seed=11, live=self.live)
        wait()
        return [a.clone() for a in self.out + self.dh + self.w + self.gamma + self.bias + self.copies[:len(self.w)]]


GRID = [(70, 256, 384, 2, 2), (300, 144, 272, 1, 3), (1, 640, 128, 2, 1)]


@pytest.mark.parametrize("case", GRID, ids=str)
def test_block_of_all_operators_against_fp64(case):
    """Each operator's result from what the one before it left, in fp64; rounding to bfloat16 half a step, sums as in the tests above."""
    nb, bfi, bfo, pfo, pfi = case
    b = Block(*case, 900)
    w0, g0, c0 = [f64(a) for a in b.w], [f64(a) for a in b.gamma], [f64(a) for a in b.bias]
    b.step()
    distdl.device_status()
    h = [f64(a) for a in b.h]
    for j in range(pfi):
        assert np.array_equal(h[j], rounded((f64(b.x[j]) + f64(b.x[pfi + j])).astype(np.float32), torch.bfloat16))
    y, _ = o.rmsnorm_fwd(h, g0, 1e-6)
    for a, want in zip(b.y, y):
        assert (np.abs(f64(a) - want) <= 1.01 * 2.0 ** -8 * np.abs(want)).all()
    for i in range(pfo * pfi):
        same_quant(b.w8[i], b.ws[i], o.quantize_weights(w0[i]))
    pairs = lambda q, s: [(f64(u), v.cpu().numpy()) for u, v in zip(q, s)]  # noqa: E731
    act, w8, dq = pairs(b.q, b.qs), pairs(b.w8, b.ws), pairs(b.dq, b.dqs)
    mag = lambda p: [(np.abs(u), v) for u, v in p]  # noqa: E731
    for got, want, size in list(zip(b.out, o.affine_fp8_fwd(act, w8, pfo, pfi, c0), o.affine_fp8_fwd(mag(act), mag(w8), pfo, pfi, [np.abs(v) for v in c0]))) + \
            list(zip(b.dx, o.affine_fp8_adj(dq, w8, pfo, pfi), o.affine_fp8_adj(mag(dq), mag(w8), pfo, pfi))):
        e = 300 * U * size
        assert (np.abs(f64(got) - want) <= e + 2.0 ** -8 * (np.abs(want) + e)).all()
    for a, d in zip(b.dq, b.dy):
        assert np.array_equal(f64(a), o.quantize_rows(f64(d).astype(np.float32))[0])
    dh, dgamma = o.rmsnorm_adj([f64(a) for a in b.dx], None, h, g0, f64(b.rstd))
    for a, want in zip(b.dh, dh):
        assert (np.abs(f64(a) - want) <= 2.0 ** -8 * np.abs(want) + 1e-5 * np.abs(want).max()).all()
    for a, want in zip(b.dgamma, dgamma):
        assert np.abs(f64(a) - want).max() <= 1e-5 * np.abs(want).max()
    for i in range(pfo):
        for j in range(pfi):
            want = f64(b.dy[i]).T @ f64(b.y[j])
            assert np.abs(f64(b.dw[i * pfi + j]) - want).max() <= 1e-5 * np.abs(want).max()
    zero = np.zeros(1)
    for p, before, g in zip(b.w + b.gamma + b.bias, w0 + g0 + c0, b.dw + b.dgamma + b.db):
        want, _, _ = o.adamw(before, f64(g), zero, zero, float(np.float32(1e-3)), 1, (0.9, 0.95), 1e-8, 0.01)
        assert (np.abs(f64(p) - want) <= 1.01 * U * np.abs(want) + 32 * U * 1e-3 * (1 + np.abs(before))).all()
    for c, p in zip(b.copies, b.w):
        assert torch.equal(c, p.bfloat16())


@pytest.mark.parametrize("case", GRID, ids=str)
def test_block_captured_and_replayed_and_two_at_once(case):
    """Steps one after another with a wait behind every operator; without; replayed from a graph; two blocks on two streams at once: the
    same bits."""
    def drive(b, go, results):
        for t in range(1, 5):
            b.factor.fill_(0.5 * t)
            b.live.copy_(torch.tensor([1e-3 * t, float(t), 1.0], device=DEV))
            results.append(go())

    blocks = [Block(*case, 900 + 100 * (k % 2)) for k in range(6)]
    torch.cuda.synchronize()
    want = [[], []]
    for k in range(2):
        drive(blocks[k], lambda: blocks[k].step(torch.cuda.synchronize), want[k])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[] for _ in range(4)]
    for k in range(2):                                                   # both streams are busy at once
        with torch.cuda.stream(streams[k]):
            drive(blocks[2 + k], blocks[2 + k].step, got[k])
    torch.cuda.synchronize()
    graphs, held = [], []
    for k in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=streams[k]):
            held.append(blocks[4 + k].step())
        graphs.append(g)
    torch.cuda.synchronize()
    for k in range(2):
        def replay(k=k):
            graphs[k].replay()
            return [a.clone() for a in held[k]]
        with torch.cuda.stream(streams[k]):
            drive(blocks[4 + k], replay, got[2 + k])
    distdl.device_status(streams[0])
    torch.cuda.synchronize()
    for k in range(4):
        for a, b in zip(got[k], want[k % 2]):
            assert all(torch.equal(u.view(torch.uint8), v.view(torch.uint8)) for u, v in zip(a, b)), k


def test_blocks_in_host_memory_are_refused():
    """Wherever they stand in their lists: nothing is launched on them."""
    x, host = [torch.ones(4, 128, device=DEV) for _ in range(2)], torch.ones(4, 128)
    q, s = [torch.zeros(4, 128, device=DEV).to(E4) for _ in range(2)], [torch.zeros(1, 4, device=DEV) for _ in range(2)]
    for bad in (dict(x=[x[0], host]), dict(x=[host, x[1]]), dict(q=[q[0], host.to(E4)]), dict(s=[s[0], torch.zeros(1, 4)])):
        a = dict(dict(x=x, q=q, s=s), **bad)
        with pytest.raises(distdl.DistdlError, match="host memory"):
            distdl.quantize_rows(4, 256, 2, a["x"], a["q"], a["s"])
    p, m, v = [torch.ones(130) for _ in range(3)]
    with pytest.raises(distdl.DistdlError, match="host memory"):
        distdl.AdamW([p], [m], [v]).step([p.clone()], 1e-3, 1)
    p, m, v = [torch.ones(130, device=DEV) for _ in range(3)]
    opt = distdl.AdamW([p], [m], [v])
    with pytest.raises(distdl.DistdlError, match="host memory"):
        opt.step([p.clone()], 1e-3, 1, live=torch.ones(3))
    with pytest.raises(distdl.DistdlError, match="host memory"):
        opt.step([torch.ones(130)], 1e-3, 1)
    torch.cuda.synchronize()
    assert all((a.float() == 0).all() for a in q + s) and (p == 1).all()


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("case", [(20, 256, 272, 1, 2), (300, 256, 272, 1, 2), (2000, 128, 1040, 2, 1), (1200, 4096, 528, 1, 1), (300, 128, 288, 2, 1), (2300, 256, 1056, 1, 2)], ids=str)
def test_affine_fp8_into_blocks_on_16_byte_boundaries(case, t):
    """Results that begin on a boundary of 16 bytes and not of 32: the same bits."""
    nb, bfi, bfo, pfo, pfi = case
    a, w = fp8_inputs(*case, False, False)
    bias = [inputs.normal((bfo,), 700 + i) for i in range(pfo)]
    off = 16 // t.itemsize
    held = []

    def odd(*shape, dtype):
        buf = torch.full((shape[0] * shape[1] + 2 * off,), 7.0, device=DEV, dtype=dtype)
        held.append(buf)
        return buf[off:-off].view(*shape)

    want, got = fp8_call(*case, False, a, w, bias, t, Out()), fp8_call(*case, False, a, w, bias, t, odd)
    assert all(g.data_ptr() % 32 == 16 and torch.equal(g, x) for g, x in zip(got, want))
    assert all((b[:off] == 7).all() and (b[-off:] == 7).all() for b in held)


def test_affine_fp8_of_bad_numbers():
    """A sample of infinities or NaN is NaN, a block of weights with one makes its columns NaN; everything else is what it is without."""
    nb, bfi, bfo = 140, 272, 272
    for rows in (nb, 20):
        x, w = inputs.normal((rows, bfi), 1), inputs.normal((bfo, bfi), 2, 0.05)
        outs = []
        for bad in (False, True):
            xb, wb = x.copy(), w.copy()
            if bad:
                xb[3, 200], xb[rows - 1, 0], wb[140, 10] = np.nan, np.inf, -np.inf
            q, s, w8, ws = torch.empty(rows, bfi, device=DEV, dtype=E4), torch.empty(3, rows, device=DEV), torch.empty(bfo, bfi, device=DEV, dtype=E4), torch.empty(3, 3, device=DEV)
            y = torch.empty(rows, bfo, device=DEV)
            distdl.quantize_rows(rows, bfi, 1, [dev(xb)], [q], [s])
            distdl.quantize_weights(bfi, bfo, 1, 1, [dev(wb)], [w8], [ws])
            distdl.affine_fp8_fwd(rows, bfi, bfo, 1, 1, [q], [s], [w8], [ws], None, [y])
            distdl.device_status()
            outs.append(f64(y))
        touched = np.zeros((rows, bfo), bool)
        touched[[3, rows - 1]] = True
        touched[:, 128:256] = True
        assert np.isnan(outs[1][touched]).all() and np.array_equal(outs[1][~touched], outs[0][~touched]) and np.isfinite(outs[0]).all()


def test_operators_on_more_than_2_31_elements():
    """Offsets beyond 32 bits: the first and last samples of the largest batch of the layer, rows in front of and behind 2^31 elements of the others."""
    if torch.cuda.get_device_properties(0).total_memory < 120 << 30:
        pytest.skip("needs 60 GB")
    nb, bfi, bfo = 1 << 20, 128, 2064
    at = [slice(0, 300), slice(nb // 2, nb // 2 + 50), slice(nb - 300, nb)]
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    x = torch.randn(nb, bfi, device=DEV, generator=g, dtype=torch.bfloat16)
    w = [dev(inputs.normal((bfo, bfi), 3, 0.1))]
    q, s = torch.empty(nb, bfi, device=DEV, dtype=E4), torch.empty(1, nb, device=DEV)
    w8, ws = torch.empty(bfo, bfi, device=DEV, dtype=E4), torch.empty(17, 1, device=DEV)
    y = torch.empty(nb, bfo, device=DEV, dtype=torch.bfloat16)
    distdl.quantize_rows(nb, bfi, 1, [x], [q], [s])
    distdl.quantize_weights(bfi, bfo, 1, 1, w, [w8], [ws])
    distdl.affine_fp8_fwd(nb, bfi, bfo, 1, 1, [q], [s], [w8], [ws], None, [y])
    distdl.device_status()
    wv = (f64(w8), ws.cpu().numpy())
    for r in at:
        want = o.affine_fp8_fwd([(f64(q[r]), s[:, r].cpu().numpy())], [wv], 1, 1)[0]
        assert (np.abs(f64(y[r]) - want) <= 1.01 * 2.0 ** -8 * np.abs(want) + 300 * U * np.abs(want).max()).all()
    # the wide result: normed with itself as the residual, quantised, and back
    gamma = [dev(1 + inputs.normal((bfo,), 4, 0.1))]
    rstd, q2, s2 = torch.empty(nb, device=DEV), torch.empty(nb, bfo, device=DEV, dtype=E4), torch.empty(17, nb, device=DEV)
    h = torch.empty_like(y)
    distdl.rmsnorm_fwd(nb, bfo, 1, [y], [y], gamma, 1e-6, [h], None, [q2], [s2], rstd)
    dx = torch.empty(nb, bfi, device=DEV)
    distdl.affine_fp8_adj(nb, bfi, bfo, 1, 1, [q2], [s2], [w8], [ws], [dx])
    distdl.device_status()
    ws_adj = torch.empty(distdl.rmsnorm_adj_workspace(nb, bfo, 1), dtype=torch.uint8, device=DEV)
    dh, dgamma = torch.empty_like(y), torch.empty(bfo, device=DEV)
    distdl.rmsnorm_adj(nb, bfo, 1, [y], None, [h], gamma, rstd, [dh], [dgamma], ws_adj)
    q3, s3 = torch.empty(nb, bfo, device=DEV, dtype=E4), torch.empty(17, nb, device=DEV)
    distdl.quantize_rows(nb, bfo, 1, [dh], [q3], [s3])
    torch.cuda.synchronize()
    for r in at:
        hv = f64(y[r]) * 2
        assert np.array_equal(f64(h[r]), hv)
        yw, rw = o.rmsnorm_fwd([hv], [f64(gamma[0])], 1e-6)
        assert np.allclose(f64(rstd[r]), rw, rtol=1e-5)
        v, scale = o.row_values(f64(q2[r]), s2[:, r].cpu().numpy()), np.repeat(f64(s2[:, r]).T, 128, 1)[:, :bfo]
        assert (np.abs(v - yw[0]) <= np.maximum(2.0 ** -4 * np.abs(yw[0]), 2.0 ** -10 * scale) * 1.001 + 1e-5 * np.abs(yw[0])).all()
        act = [(f64(q2[r]), s2[:, r].cpu().numpy())]
        want, size = o.affine_fp8_adj(act, [wv], 1, 1)[0], o.affine_fp8_adj([(np.abs(act[0][0]), act[0][1])], [(np.abs(wv[0]), wv[1])], 1, 1)[0]
        assert (np.abs(f64(dx[r]) - want) <= 300 * U * size).all()
        dhw, _ = o.rmsnorm_adj([f64(y[r])], None, [hv], [f64(gamma[0])], f64(rstd[r]))
        assert (np.abs(f64(dh[r]) - dhw[0]) <= 2.0 ** -8 * np.abs(dhw[0]) + 1e-5 * (np.abs(dhw[0]).max(1, keepdims=True) + np.abs(f64(y[r]) * f64(rstd[r])[:, None]))).all()
        same_quant(q3[r], s3[:, r], o.quantize_rows(f64(dh[r]).astype(np.float32)))
