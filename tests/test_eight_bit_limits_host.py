"""CPU tests of the limits of the operators of 8-bit affine blocks: what they refuse at the ends of their ranges."""

import ctypes

import numpy as np
import pytest

import paper_2006_03108_b200 as distdl

torch = pytest.importorskip("torch")
vp = ctypes.c_void_p


def test_norm_refuses_eps_whose_squares_are_subnormal():
    """What weighs against an eps of 2^-120 has squares whose error is 2^-30 of it; below, they lose the digits that the sums count on."""
    lib, a = distdl.lib(), (vp * 1)(0x10000)

    def status(eps, nb=0):
        return lib.distdl_rmsnorm_fwd(nb, 128, 1, a, None, a, ctypes.byref(ctypes.c_double(eps)), distdl.F32, a, None, None, None, None, None)

    assert status(2.0 ** -120) == 0 and status(1e-6) == 0 and status(3e38) == 0             # no samples: nothing to do
    for eps in (2.0 ** -120 * (1 - 2.0 ** -50), 2.0 ** -121, 2.0 ** -130, 1e-45, 0.0, -1.0, float("nan"), float("inf"), 1e39):
        assert status(eps) == 1 and status(eps, 4) == 1, eps
        assert b"eps" in lib.distdl_last_error()


def test_adamw_refuses_tensors_that_have_moved():
    """Weights and their copies are where they were or the step says so; the memory of all tensors is held, so that no step writes to what is another's."""
    e4 = torch.float8_e4m3fn
    names = "p", "m", "v", "ms", "vs", "copies"
    for k, name in enumerate(names):
        for parameter in (False, True):
            sizes = 300, 0, 5
            lists = [[torch.zeros(n, dtype=t) for n in sizes] for t in (torch.float32, e4, e4)] + [[torch.zeros(-(-n // 128)) for n in sizes] for _ in range(2)]
            lists.append([torch.zeros(300, dtype=torch.bfloat16), None, torch.zeros(5, dtype=torch.bfloat16)])
            if parameter:
                lists[0] = [torch.nn.Parameter(a) for a in lists[0]]
            opt = distdl.AdamW(*lists)
            g = [torch.zeros(n) for n in sizes]

            def step(words):
                with pytest.raises(distdl.DistdlError, match=words) as e:
                    opt.step(g, 1e-3, 1, stream=0)
                assert e.value.status == 1

            step("host memory")                                       # where they were: on to the next check
            with torch.no_grad():
                lists[0][0].add_(1)
                lists[3][2].copy_(torch.ones(1))
            step("host memory")
            t = lists[k][2]
            old = t.data_ptr()
            t.data = t.data.clone()
            assert t.data_ptr() != old and any(m.data_ptr() == old for m in opt._memory)
            step(name + r"\[2\] is no longer where it was" if name in ("p", "copies") else "host memory")
            step("no longer" if name in ("p", "copies") else "host memory")
    with pytest.raises(TypeError):
        distdl._calls.moved((torch.zeros(1),), b"", "p")
    with pytest.raises(TypeError):
        distdl._calls.moved((torch.zeros(1),), b"\0" * 8)


@pytest.mark.parametrize("kind", [np.int64, np.int32, np.int16, np.int8, np.uint8])
def test_whole_numbers_of_any_type(kind):
    """NumPy's numbers are taken as Python's are: all checks pass up to the one that finds host memory, and their products do not wrap around."""
    t = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype)  # noqa: E731
    e4 = torch.float8_e4m3fn
    nb, bf, pf, e = 100, 32, 2, t(100, 32)
    i = [kind(v) for v in (nb, bf * pf, pf)]
    rows, q, s, gamma = [e, e], [t(nb, bf, dtype=e4)] * 2, [t(1, nb)] * 2, [t(bf)] * 2
    w, w8, ws = [t(bf, bf)] * 4, [t(bf, bf, dtype=e4)] * 4, [t(1, 1)] * 4
    grid = i[1], i[1], i[2], i[2]
    calls = (lambda: distdl.quantize_rows(*i, rows, q, s, stream=0), lambda: distdl.quantize_weights(*grid, w, w8, ws, stream=0),
             lambda: distdl.rmsnorm_fwd(*i, rows, rows, gamma, 1e-6, rows, None, q, s, t(nb), stream=0),
             lambda: distdl.rmsnorm_adj(*i, rows, None, rows, gamma, t(nb), rows, None, t(1 << 20), stream=0),
             lambda: distdl.affine_fp8_fwd(i[0], *grid, q, s, w8, ws, gamma, rows, stream=0), lambda: distdl.affine_fp8_adj(i[0], *grid, q, s, w8, ws, rows, stream=0))
    for call in calls:
        with pytest.raises(distdl.DistdlError, match="host memory") as err:
            call()
        assert err.value.status == 1
    with pytest.raises(TypeError):
        distdl.quantize_rows(4.0, 64, 2, rows, q, s, stream=0)
    with pytest.raises(TypeError):
        distdl.affine_fp8_fwd(nb, 64, 64, 2, "2", q, s, w8, ws, None, rows, stream=0)


def test_packed_addresses_and_sizes_are_whole_ones():
    """Bytes that end inside an address or a size are refused, in the calls that took lists alone before too."""
    part = distdl.Partition((8, 8), (2, 2), (1, 1), (1, 1))
    packed = np.array([256] * 4, np.int64).tobytes()
    for cut in (1, 7, 8 * 4 - 1):
        with pytest.raises(ValueError, match="addresses"):
            distdl.halo_fwd(part, packed + b"\0" * cut, stream=0)
        with pytest.raises(ValueError, match="addresses"):
            distdl._calls.quantize_rows(4, 128, 1, packed[:8] + b"\0" * cut, 0, packed, packed, 0, 1, 1, 1)
    with pytest.raises(distdl.DistdlError) as e:
        distdl.halo_fwd(part, packed[:24], stream=0)
    assert e.value.status == 1
    a = torch.zeros(4)
    for sizes in (b"", b"\4" + b"\0" * 7):
        got = distdl._calls.check([a][:len(sizes) // 8], len(sizes) // 8, sizes, torch.float32, "a")
        assert got == (b"",) if not sizes else got[0] == 1 and "host memory" in got[1]
    with pytest.raises(ValueError, match="sizes"):
        distdl._calls.check([a], 1, b"\4" + b"\0" * 8, torch.float32, "a")


@pytest.mark.parametrize("clusters", [(74, 37, 18, 74, 37, 18), (74, 35, 16, 74, 35, 16), (74, 33, 15, 74, 33, 15), (70, 31, 12, 70, 31, 12)], ids=str)
def test_affine_fp8_cases_reach_every_shape(clusters):
    """The sizes that the GPU tests run take the 8-bit layer through all six of its shapes, forward and back: a measured time that is set anew cannot leave
    one untested without a word.  clusters: how many of each shape a device of 148 multiprocessors may hold."""
    from test_eight_bit_gpu import FP8
    from test_eight_bit_limits_gpu import RUNS, runs_case
    for adj in (False, True):
        seen = {}
        for c in [c for c in FP8 if c[0] > 128] + [runs_case(c, adj) for c in RUNS]:
            got = distdl.selftest_affine_fp8_shape(c[0], c[1] * c[4], c[2] * c[3], c[3], c[4], adj, clusters)
            seen.setdefault(got[:2], []).append(got[2] > got[3])
        assert set(seen) == {(n, r) for n in (256, 128) for r in (1, 2, 4)}, seen
        assert all(any(seen[k]) for k in ((256, 1), (256, 2))) and not all(seen[256, 2])           # in one turn and in several
        for c in RUNS:
            n = runs_case(c, adj)
            assert distdl.selftest_affine_fp8_shape(n[0], n[1] * n[4], n[2] * n[3], n[3], n[4], adj, clusters)[:2] == c[5], c
    # what a tile costs decides; a shape that the device cannot hold is never taken
    assert distdl.selftest_affine_fp8_shape(200, 16384, 2816, 1, 1, False, (74, 37, 0, 74, 37, 0))[1] != 4
    with pytest.raises(distdl.DistdlError):
        distdl.selftest_affine_fp8_shape(200, 16384, 2816, 1, 1, False, (0,) * 6)
    for bad in ((128, 128, 128, 1, 1), (200, 128, 130, 4, 1), (200, 0, 128, 1, 1)):
        with pytest.raises(distdl.DistdlError) as e:
            distdl.selftest_affine_fp8_shape(*bad, False, clusters)
        assert e.value.status == 1
