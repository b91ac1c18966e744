"""CPU tests of the operators of 8-bit affine blocks: the oracle pinned against torch and brute force, and what the calls refuse."""

import ctypes

import numpy as np
import pytest

import paper_2006_03108_b200 as distdl
from oracle import eight_bit as o

torch = pytest.importorskip("torch")
RNG = np.random.Generator(np.random.Philox(7))


# ---------------------------------------------------------------------------------------------
# The oracle
# ---------------------------------------------------------------------------------------------

def test_oracle_e4m3_values_and_rounding_agree_with_torch():
    codes = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(o.e4m3_value(codes.numpy()), codes.view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)
    grid = np.unique(np.abs(o.e4m3_value(np.arange(127))))
    x = np.concatenate([grid, (grid[1:] + grid[:-1]) / 2, RNG.uniform(0, 448, 20000), RNG.uniform(0, 0.02, 20000)]).astype(np.float32)
    x = np.concatenate([x, np.nextafter(x, np.float32(0)), np.minimum(np.nextafter(x, np.float32(500)), np.float32(448))])
    x = np.concatenate([x, -x])
    assert np.array_equal(o.e4m3_round(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())


def test_oracle_blocks_hold_their_values_to_half_a_step():
    x = (RNG.standard_normal((5, 300)) * 10.0 ** RNG.integers(-20, 20, (5, 1))).astype(np.float32)
    q, s = o.quantize_rows(x)
    assert q.shape == x.shape and s.shape == (3, 5)
    scale = np.repeat(s.T, 128, axis=1)[:, :300].astype(np.float64)
    assert (np.abs(o.row_values(q, s) - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * scale) * (1 + 1e-6)).all()
    for b in range(3):                                      # the largest value of a block is the largest code
        assert (np.abs(q[:, 128 * b:128 * b + 128]).max(1) == 448).all()
    w, ws = o.quantize_weights(x.T)
    assert w.shape == (300, 5) and ws.shape == (3, 1)
    assert (np.abs(o.weight_values(w, ws) - x.T) <= np.maximum(2.0 ** -4 * np.abs(x.T), 2.0 ** -10 * np.repeat(ws, 128, axis=0)[:300]) * (1 + 1e-6)).all()


def test_oracle_norm_adjoint_against_differences_and_autograd():
    nb, bf, pf, eps = 3, 5, 2, 1e-3
    x = [torch.randn(nb, bf, dtype=torch.float64, requires_grad=True) for _ in range(pf)]
    gamma = [torch.randn(bf, dtype=torch.float64, requires_grad=True) for _ in range(pf)]
    dy = [RNG.standard_normal((nb, bf)) for _ in range(pf)]
    h = torch.cat(x, 1)
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + eps) * torch.cat(gamma)
    (y * torch.from_numpy(np.concatenate(dy, 1))).sum().backward()
    hn, gn = [a.detach().numpy() for a in x], [a.detach().numpy() for a in gamma]
    got, rstd = o.rmsnorm_fwd(hn, gn, eps)
    assert np.allclose(np.concatenate(got, 1), y.detach().numpy(), rtol=1e-13)
    dh, dgamma = o.rmsnorm_adj(dy, None, hn, gn, rstd)
    for a, b, c, d in zip(dh, x, dgamma, gamma):
        assert np.allclose(a, b.grad.numpy(), atol=1e-12) and np.allclose(c, d.grad.numpy(), atol=1e-12)
    dh2, _ = o.rmsnorm_adj(dy, dy, hn, gn, rstd)
    assert np.allclose(dh2[1], dh[1] + dy[1])
    step, way = 1e-6, [RNG.standard_normal((nb, bf)) for _ in range(pf)]
    loss = lambda t: sum((a * b).sum() for a, b in zip(o.rmsnorm_fwd([p + t * q for p, q in zip(hn, way)], gn, eps)[0], dy))  # noqa: E731
    assert np.isclose((loss(step) - loss(-step)) / (2 * step), sum((a * b).sum() for a, b in zip(dh, way)), rtol=1e-7)


def test_oracle_affine_is_the_product_of_the_values():
    pfo, pfi, nb, bfi, bfo = 2, 3, 4, 144, 160
    x = [o.quantize_rows(RNG.standard_normal((nb, bfi))) for _ in range(pfi)]
    w = [o.quantize_weights(RNG.standard_normal((bfo, bfi))) for _ in range(pfo * pfi)]
    xg = np.concatenate([o.row_values(*a) for a in x], 1)
    wg = np.concatenate([np.concatenate([o.weight_values(*w[i * pfi + j]) for j in range(pfi)], 1) for i in range(pfo)], 0)
    assert np.allclose(np.concatenate(o.affine_fp8_fwd(x, w, pfo, pfi), 1), xg @ wg.T)
    dy = [o.quantize_rows(RNG.standard_normal((nb, bfo))) for _ in range(pfo)]
    dg = np.concatenate([o.row_values(*a) for a in dy], 1)
    assert np.allclose(np.concatenate(o.affine_fp8_adj(dy, w, pfo, pfi), 1), dg @ wg)


def test_oracle_adamw_agrees_with_torch():
    p0, lr, betas, eps, decay = RNG.standard_normal(50), 1e-2, (0.8, 0.9), 1e-6, 0.3
    p = torch.nn.Parameter(torch.from_numpy(p0.copy()))
    opt = torch.optim.AdamW([p], lr=lr, betas=betas, eps=eps, weight_decay=decay)
    q, m, v = p0, np.zeros(50), np.zeros(50)
    for step in range(1, 6):
        g = RNG.standard_normal(50)
        p.grad = torch.from_numpy(g.copy())
        opt.step()
        q, m, v = o.adamw(q, 2 * g, m, v, lr, step, betas, eps, decay, grad_scale=0.5)
        assert np.allclose(q, p.detach().numpy(), rtol=1e-12, atol=1e-14)


def test_oracle_stochastic_rounding_keeps_the_mean_and_the_grid():
    a = np.concatenate([RNG.uniform(0, 448, 300), RNG.uniform(0, 0.02, 300), o.e4m3_value(np.arange(127))])
    bits = o.random_bits(0, 2000, seed=5, step=1, tensor=0)
    up = (o.random_bits(2 ** 32 - 3, 6, 5, 1, 0), o.random_bits(2 ** 32, 1, 5, 1, 0))
    assert up[0][3] == up[1][0] and len(set(up[0])) == 6
    u = (bits & 0xFFFF) / 65536.0
    r = np.stack([o.stochastic_e4m3(a, x, False) for x in u])
    assert np.isin(r, o.e4m3_value(np.arange(127))).all()
    width = 2.0 ** (np.maximum(np.frexp(a)[1] - 1, -6) - 3.0)
    assert (np.abs(r - a) < width).all()
    # the mean of 2000 draws with a deviation of half a width at most: five standard errors
    assert (np.abs(r.mean(0) - a) <= 5 * width / 2 / np.sqrt(2000)).all()
    assert (o.stochastic_e4m3(np.array([1e-30, 2.0 ** -9]), 0.0, True) == 2.0 ** -9).all() and o.stochastic_e4m3(np.zeros(1), 0.99, True)[0] == 0


# ---------------------------------------------------------------------------------------------
# Refusals: nothing is launched
# ---------------------------------------------------------------------------------------------

vp = ctypes.c_void_p


def _array(n, step=0x10000, first=0x10000):
    return (vp * n)(*[first + step * i for i in range(n)])


def test_quantize_and_norm_refusals():
    lib, a, odd = distdl.lib(), _array(16), _array(16, first=0x10004)
    F32, BF16 = distdl.F32, distdl.BF16
    rows = lambda nb=4, nf=256, pf=2, x=a, t=F32, q=a, s=a: lib.distdl_quantize_rows(nb, nf, pf, x, t, q, s, None)  # noqa: E731
    assert rows(nb=-1) == 1 and rows(nf=0) == 1 and rows(pf=0) == 1 and rows(pf=9, nf=9) == 4 and rows(nf=255) == 2
    assert rows(t=distdl.F64) == 1 and rows(t=distdl.E4M3) == 1 and rows(x=None) == 1 and rows(q=None) == 1 and rows(s=None) == 1
    assert rows(x=odd) == 3 and rows(q=odd) == 3 and rows(s=odd) == 3 and rows(x=(vp * 2)(0x10000, None)) == 1
    assert rows(nb=1 << 36) == 4 and rows(nf=1 << 26) == 4 and rows(nb=0) == 0
    w = lambda nfi=256, nfo=128, pfo=1, pfi=2, w=a, t=F32, q=a, s=a: lib.distdl_quantize_weights(nfi, nfo, pfo, pfi, w, t, q, s, None)  # noqa: E731
    assert w(nfi=255) == 2 and w(nfo=129, pfo=2) == 2 and w(pfo=9) == 4 and w(pfo=4, pfi=8) == 4 and w(t=7) == 1 and w(w=odd) == 3 and w(s=None) == 1
    assert w(nfo=1 << 23) == 4 and w(nfi=0) == 1

    one, zero = ctypes.c_double(1e-6), ctypes.c_double(0)
    fwd = lambda nb=4, nf=256, pf=2, x=a, r=a, g=a, e=ctypes.byref(one), t=BF16, h=a, y=a, q=a, qs=a, rstd=vp(0x50000): \
        lib.distdl_rmsnorm_fwd(nb, nf, pf, x, r, g, e, t, h, y, q, qs, rstd, None)  # noqa: E731
    assert fwd(nb=-1) == 1 and fwd(nf=0) == 1 and fwd(pf=9, nf=18) == 4 and fwd(nf=255) == 2 and fwd(nf=1 << 21) == 4 and fwd(nb=1 << 31) == 4
    assert fwd(e=None) == 1 and fwd(e=ctypes.byref(zero)) == 1 and fwd(e=ctypes.byref(ctypes.c_double(float("nan")))) == 1
    assert fwd(e=ctypes.byref(ctypes.c_double(1e-60))) == 1 and fwd(e=ctypes.byref(ctypes.c_double(float("inf")))) == 1
    assert fwd(t=distdl.F64) == 1 and fwd(x=None) == 1 and fwd(g=None) == 1 and fwd(q=None) == 1 and fwd(qs=None) == 1
    assert fwd(h=None, y=None, q=None, qs=None, rstd=None) == 1
    for name in ("x", "r", "g", "h", "y", "q", "qs"):
        assert fwd(**{name: odd}) == 3, name
    assert fwd(rstd=vp(0x50008)) == 3 and fwd(nb=0) == 0
    n = ctypes.c_int64(0)
    assert lib.distdl_rmsnorm_adj_workspace(4, 255, 2, ctypes.byref(n)) == 2 and lib.distdl_rmsnorm_adj_workspace(4, 256, 2, None) == 1
    adj = lambda nb=4, nf=256, pf=2, dy=a, dr=a, h=a, g=a, rstd=vp(0x50000), t=BF16, tg=F32, dh=a, dg=a, ws=vp(0x60000), b=1 << 30: \
        lib.distdl_rmsnorm_adj(nb, nf, pf, dy, dr, h, g, rstd, t, tg, dh, dg, ws, b, None)  # noqa: E731
    assert adj(nb=-1) == 1 and adj(nf=255) == 2 and adj(pf=9, nf=18) == 4 and adj(t=2) == 1 and adj(tg=3) == 1
    for name in ("dy", "h", "g", "rstd", "dh", "ws"):
        assert adj(**{name: None}) == 1, name
    for name in ("dy", "dr", "h", "g", "dh", "dg"):
        assert adj(**{name: odd}) == 3, name
    assert adj(ws=vp(0x60004)) == 3 and adj(nb=0, dg=None) == 0


def test_python_calls_refuse_lists_types_sizes_and_layouts():
    t = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype)  # noqa: E731
    e4 = torch.float8_e4m3fn
    x, q, s = [t(4, 128), t(4, 128)], [t(4, 128, dtype=e4), t(4, 128, dtype=e4)], [t(1, 4), t(1, 4)]

    def refused(status, fn, *args):
        with pytest.raises(distdl.DistdlError) as e:
            fn(*args, stream=0)
        assert e.value.status == status

    refused(1, distdl.quantize_rows, 4, 256, 2, x[:1], q, s)
    refused(1, distdl.quantize_rows, 4, 256, 2, [], q, s)
    refused(1, distdl.quantize_rows, 4, 256, 2, x, q, s[:1])
    refused(2, distdl.quantize_rows, 4, 255, 2, x, q, s)
    refused(2, distdl.quantize_rows, 5, 256, 2, x, q, s)
    refused(2, distdl.quantize_rows, 4, 256, 2, x, x, s)
    refused(2, distdl.quantize_rows, 4, 256, 2, [t(128, 4).t(), x[1]], q, s)
    refused(2, distdl.quantize_rows, 4, 256, 2, [t(4, 256)[:, :128], x[1]], q, s)
    refused(2, distdl.quantize_weights, 256, 4, 1, 2, x, q, [t(1, 2), t(1, 1)])
    with pytest.raises(TypeError):
        distdl.quantize_rows(4, 256, 2, [t(4, 128, dtype=torch.float16)] * 2, q, s)
    gamma = [t(128), t(128)]
    refused(2, distdl.rmsnorm_fwd, 4, 256, 2, x, [t(4, 128, dtype=torch.bfloat16)] * 2, gamma, 1e-6, x)
    refused(2, distdl.rmsnorm_fwd, 4, 256, 2, x, None, [t(127), t(128)], 1e-6, x)
    refused(2, distdl.rmsnorm_fwd, 4, 256, 2, x, None, gamma, 1e-6, None, None, None, None, t(3))
    refused(1, distdl.rmsnorm_fwd, 4, 256, 2, x, None, gamma, 1e-6, None, None, q, None)
    refused(1, distdl.rmsnorm_fwd, 4, 256, 2, x, None, gamma, -1.0, x)
    refused(2, distdl.rmsnorm_adj, 4, 256, 2, x, None, x, gamma, t(4), q, None, t(1 << 20))
    refused(1, distdl.quantize_rows, 4, 256, 2, x, q, s)              # sizes and types fit, but this is host memory


def test_adamw_refusals():
    lib, a, odd = distdl.lib(), _array(5000), _array(4, first=0x10004)
    n4 = (ctypes.c_int64 * 4)(8, 0, 130, 8)
    good = (1e-3, 0.9, 0.999, 1e-8, 0.1, 1.0)

    def step(count=4, elems=n4, p=a, g=a, tg=distdl.F32, m=a, v=a, ms=a, vs=a, state=distdl.E4M3, copies=a, hyper=good, t=1, live=None):
        h = None if hyper is None else (ctypes.c_double * 6)(*hyper)
        return lib.distdl_adamw_step(count, elems, p, g, tg, m, v, ms, vs, state, copies, h, t, 0, live, None)

    assert step(count=-1) == 1 and step(hyper=None) == 1 and step(elems=None) == 1 and step(count=5000, elems=(ctypes.c_int64 * 5000)()) == 4
    assert step(tg=distdl.F64) == 1 and step(tg=distdl.E4M3) == 1 and step(state=distdl.BF16) == 1
    for k, bad in ((0, -1.0), (0, float("nan")), (0, float("inf")), (1, 1.0), (1, -0.1), (2, 1.0), (2, float("nan")), (3, 0.0), (3, 1e-60), (4, -0.1), (5, float("inf"))):
        assert step(hyper=good[:k] + (bad,) + good[k + 1:]) == 1, (k, bad)
    assert step(t=0) == 1 and step(t=-3) == 1 and step(elems=(ctypes.c_int64 * 4)(8, -1, 8, 8)) == 1 and step(elems=(ctypes.c_int64 * 4)(8, 1 << 41, 8, 8)) == 4
    hole = (vp * 4)(0x10000, None, 0x30000, None)
    for name in ("p", "g", "m", "v", "ms", "vs"):
        assert step(**{name: None}) == 1 and step(**{name: hole}) == 1 and step(**{name: odd}) == 3, name
    assert step(copies=odd) == 3 and step(live=vp(0x10004)) == 3
    assert step(count=0) == 0 and step(elems=(ctypes.c_int64 * 4)()) == 0             # nothing to do


def test_adamw_handle_refuses_tensors_that_do_not_belong_together():
    t = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype)  # noqa: E731
    e4 = torch.float8_e4m3fn
    p = [t(300), t(5)]
    m8 = lambda: [t(300, dtype=e4), t(5, dtype=e4)]  # noqa: E731
    sc = lambda: [t(3), t(1)]  # noqa: E731
    f = lambda: [t(300), t(5)]  # noqa: E731

    def refused(status, *args):
        with pytest.raises(distdl.DistdlError) as e:
            distdl.AdamW(*args)
        assert e.value.status == status

    refused(1, p, f()[:1], f())
    refused(2, p, [t(300), t(6)], f())
    refused(2, p, f(), m8())
    refused(1, p, m8(), m8())
    refused(1, p, m8(), m8(), sc(), None)
    refused(2, p, m8(), m8(), [t(2), t(1)], sc())
    refused(2, p, f(), f(), None, None, [t(300), None])
    refused(2, [t(600)[::2], t(5)], f(), f())
    refused(1, p, [p[0], t(5)], f())                                                   # one buffer in two places
    both = t(600)
    refused(1, p, [both[:300], t(5)], [both[299:599], t(5)])
    opt = distdl.AdamW(p, f(), f(), None, None, [None, t(5, dtype=torch.bfloat16)])
    for g in ([t(300)], [t(300), t(6)], [t(300), t(5, dtype=torch.bfloat16)], [t(2, 300)[:, ::2], t(5)]):
        with pytest.raises(distdl.DistdlError):
            opt.step(g, 1e-3, 1, stream=0)
    with pytest.raises(distdl.DistdlError) as e:
        opt.step(f(), 1e-3, 0, stream=0)
    assert e.value.status == 1
    distdl.AdamW([], [], []).step([], 1e-3, 1)
    lists = [t(64)], [t(64)], [t(64)]
    held = distdl.AdamW(*lists)
    for x in lists:
        x.clear()                                                                      # the handle holds the tensors themselves
    assert [len(k) for k in held._keep if k is not None] == [1, 1, 1]


def test_affine_fp8_refusals():
    lib, a, odd = distdl.lib(), _array(16), _array(16, first=0x10008)

    def fwd(nb=16, nfi=256, nfo=256, pfo=1, pfi=1, x=a, xs=a, w=a, ws=a, bias=a, t=distdl.F32, y=a):
        return lib.distdl_affine_fp8_fwd(nb, nfi, nfo, pfo, pfi, x, xs, w, ws, bias, t, y, None)

    def adj(nb=16, nfi=256, nfo=256, pfo=1, pfi=1, x=a, xs=a, w=a, ws=a, t=distdl.BF16, y=a):
        return lib.distdl_affine_fp8_adj(nb, nfi, nfo, pfo, pfi, x, xs, w, ws, t, y, None)

    for call in (fwd, adj):
        assert call(nb=0) == 1 and call(nfi=0) == 1 and call(pfo=0) == 1 and call(nfi=256, pfi=3) == 2 and call(nfo=100, pfo=3) == 2
        assert call(nfi=264) == 4 and call(nfo=8) == 4 and call(pfo=16) == 4 and call(pfo=4, pfi=8) == 4 and call(nb=(1 << 20) + 1) == 4
        assert call(t=distdl.F64) == 1 and call(t=distdl.E4M3) == 1
        for name in ("x", "xs", "w", "ws", "y"):
            assert call(**{name: None}) == 1 and call(**{name: odd}) == 3 and call(**{name: (vp * 1)(None)}) == 1, name
    assert fwd(bias=odd) == 3
    e4, t = torch.float8_e4m3fn, lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype)
    x, xs, w, ws, y = [t(4, 128, dtype=e4)] * 2, [t(1, 4)] * 2, [t(144, 128, dtype=e4)] * 2, [t(2, 1)] * 2, [t(4, 144)]

    def refused(status, *args):
        with pytest.raises(distdl.DistdlError) as e:
            distdl.affine_fp8_fwd(4, 256, 144, 1, 2, *args, stream=0)
        assert e.value.status == status

    refused(1, x[:1], xs, w, ws, None, y)
    refused(1, x, xs[:1], w, ws, None, y)
    refused(1, x, xs, w[:1], ws, None, y)
    refused(1, x, xs, w, ws, [], y)
    refused(2, x, xs, w, [t(1, 1)] * 2, None, y)
    refused(2, x, xs, [t(128, 144, dtype=e4).t()] * 2, ws, None, y)
    refused(2, x, [t(4)[:0]] * 2, w, ws, None, y)
    refused(2, x, xs, w, ws, [t(143)], y)


class Block:
    """What the checks ask a tensor for, on a device of its own."""

    dtype = torch.float32

    def __init__(self, device, n=8):
        self.device, self.n = device, n

    def get_device(self):
        return self.device

    def numel(self):
        return self.n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1000 + self.device


@pytest.mark.parametrize("devices, words", [([0, -1], "host memory"), ([0, 0, -1], "host memory"), ([-1, 0], "host memory"), ([1, 1, 0], "device 0, others on 1"),
                                            ([0, 1, 2], "device 1, others on 0"), ([1, 1, 1], None)], ids=str)
def test_every_block_is_checked_for_its_device(devices, words):
    """Any block of any list, not the first alone; what is wrong with the sizes is said first."""
    distdl._load()
    for cut in range(len(devices) + 1):
        a, b = [Block(d) for d in devices[:cut]], [Block(d) for d in devices[cut:]]
        lists = (a, cut, 8, torch.float32, "a", None, 3, 8, torch.float32, "none", b, len(b), 8, torch.float32, "b")
        got = distdl._calls.check(*lists)
        if words is None:
            assert [None if v is None else np.frombuffer(v, np.int64).tolist() for v in got] == [[d + 1000 for d in devices[:cut]], None, [d + 1000 for d in devices[cut:]]]
        else:
            assert got[0] == 1 and words in got[1], (cut, got)
        got = distdl._calls.check(*lists, [Block(devices[0], 7)], 1, 8, torch.float32, "c")
        assert got[0] == 2 and got[1].startswith("c[0]")


def test_the_checks_agree_on_tensors_and_subclasses():
    """Plain tensors go through DLPack's table where PyTorch has it, others are asked for their attributes: the same answers."""
    class Other(torch.Tensor):
        pass

    f32, bf16, e4m3, u8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn, torch.uint8
    distdl._float_code("x", [torch.zeros(1)])
    base = torch.zeros(48)
    blocks = [base.view(6, 8), base.view(6, 8).T, base.view(6, 8)[:, :5], base[::2], base.view(48, 1).T, base.view(6, 8)[2:3, :], base[:0].view(0, 4), torch.tensor(1.0),
              base.to(bf16), base.to(e4m3), base.to(u8), base.half(), base.to(torch.float8_e5m2), base.bool(), base.clone().requires_grad_()]
    for b in blocks:
        for t in (f32, bf16, e4m3, u8, torch.float64):
            for n in (b.numel(), b.numel() + 1):
                got, want = [distdl._calls.check([a], 1, n, t, "a") for a in (b, b.as_subclass(Other))]
                assert got == want and got[0] == (1 if b.dtype is t and n == b.numel() and b.is_contiguous() else 2), (b.dtype, b.shape, b.stride(), t, got, want)
    sizes = np.array([48, 24, 1], np.int64).tobytes()
    assert distdl._calls.check([base, base[:24], base[:1]], 3, sizes, f32, "a")[1] == "a: a block is in host memory"
    assert distdl._calls.check([base, base[:23], base[:1]], 3, sizes, f32, "a")[1].startswith("a[1]: contiguous blocks of 24")
    assert distdl._calls.check([base, base[:24], base[:1], base], 3, sizes, f32, "a")[0] == 1
