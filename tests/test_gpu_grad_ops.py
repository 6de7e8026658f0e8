"""The gradient's norm, its clipping and Adam over a list (HIP, through the C ABI) against the oracle in 64 bits.

Tolerances, from the roundings made. Sums are fp64 (2000 terms a lane at most here: 1e-12 relative), so norm, factor and the
norms of single tensors are off by one rounding to fp32, 2^-24, where they are normal numbers (half a step, 2^-150, below). A
clipped value is fl_T(fl32(scale * g)) with a scale that is itself rounded: 2^-24 + 2^-24 relative, then half a step of the type
(2^-11 for fp16, 2^-8 for bf16) - and half of the smallest subnormal of each type it is rounded to (2^-150, 2^-25, 2^-134).
Adam over a list is what clipping and pbdr_adam_selective leave, bit for bit; that call has its own test against the oracle.
"""
import numpy as np
import pytest
import torch

import oracle
from paper_2512_20017_amd import binding as B
from paper_2512_20017_amd import synth

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
STEP = {F32: 0.0, F16: 2.0 ** -11, BF16: 2.0 ** -8}
TINY = {F32: 2.0 ** -150, F16: 2.0 ** -25, BF16: 2.0 ** -134}
EPS = 2.0 ** -24


def rows(t):
    """[..., n] on the device -> [n, ...] in fp64"""
    a = t.double().cpu().numpy()
    return np.moveaxis(a, -1, 0) if a.ndim > 1 else a


def make(spec, seed, size=1e-3):
    """spec: (shape, type, share of used points or None for no mask). Unused entries hold NaN, infinities and large numbers."""
    rng = np.random.default_rng(seed)
    ts, ms = [], []
    for shape, dtype, share in spec:
        x = torch.from_numpy(np.asarray(rng.normal(size=shape) * size, dtype=np.float32)).to(dtype)
        mask = None
        if share is not None:
            mask = torch.from_numpy((rng.uniform(size=shape[-1]) < share).astype(np.uint8) * rng.integers(1, 256, size=shape[-1]).astype(np.uint8))
            poison = torch.tensor([float("nan"), float("inf"), float("-inf"), 6e4]).to(dtype)[torch.from_numpy(rng.integers(0, 4, size=shape))]
            x = torch.where(mask != 0, x, poison)
        ts.append(x.cuda())
        ms.append(None if mask is None else mask.cuda())
    return ts, ms


def reference(ts, ms, max_norm):
    return oracle.grad_norm([rows(t) for t in ts], [None if m is None else m.cpu().numpy() for m in ms], max_norm)


def check_result(result, ref, max_norm):
    norm, factor, each = ref
    got = result.double().cpu().numpy()
    want = np.array([norm, factor] + each)
    assert got.shape == want.shape
    for g, w in zip(got, want):      # a norm beyond the range of fp32 is infinite there, its factor is not affected
        assert g == float("inf") if w >= 2.0 ** 128 * (1 - EPS) else abs(g - w) <= (EPS + 1e-12) * w + 2.0 ** -150, (got, want)


def check_clipped(out, before, t, mask, factor):
    want = oracle.grad_clip(rows(t), None if mask is None else mask.cpu().numpy(), factor, rows(before))
    got = rows(out)
    used = np.ones(got.shape[0] if got.ndim else (), bool) if mask is None else mask.cpu().numpy() != 0
    if got.ndim == 0:
        got, want = got[None], want[None]
    g, w = got[used], want[used]
    exact = factor in (0.0, 1.0)
    tol = 0.0 if exact else np.abs(w) * ((2 * EPS + 1e-12) + STEP[t.dtype] * (1 + 1e-6)) + TINY[t.dtype] + TINY[F32]
    assert (np.abs(g - w) <= tol).all()
    if mask is not None:      # unused entries: the very bits that were there
        view = torch.int32 if t.dtype == F32 else torch.int16
        keep = (mask == 0).expand(t.shape)
        assert torch.equal(out.view(view)[keep], before.view(view)[keep])


def run_clip(ts, ms, max_norm, in_place=False):
    ws = B.alloc_grad_workspace(len(ts))
    result = torch.full((2 + len(ts),), 9.0, device="cuda")
    raw = [t.clone() for t in ts]
    out = None if in_place else [torch.full_like(t, 7.0) for t in ts]
    before = raw if in_place else [o.clone() for o in out]
    B.pbdr_grad_clip(B.GradList(ts, visible=ms, out=out), max_norm, result, ws)
    alone = torch.full_like(result, 9.0)
    B.pbdr_grad_norm(B.GradList(raw, visible=ms), max_norm, alone, ws)
    torch.cuda.synchronize()
    assert torch.equal(result.view(torch.int32), alone.view(torch.int32))
    # the boundary takes max_norm as fp32 (1e-3 is 4.7e-8 from its fp32 number, a rounding of the factor allows 6.0e-8): the oracle
    # gets the same number
    ref = reference(raw, ms, float(np.float32(max_norm)))
    check_result(result, ref, max_norm)
    for o, b, t, m in zip(ts if in_place else out, before, raw, ms):
        check_clipped(o, b, t, m, ref[1])
    if not in_place:
        for t, r in zip(ts, raw):
            bits = torch.int32 if t.dtype == F32 else torch.int16
            assert torch.equal(t.view(bits), r.view(bits))
    return result


GAUSS = [((3, 5000), F32, 0.5), ((3, 5000), F32, 0.5), ((4, 5000), F32, 0.5), ((5000,), F32, 0.5), ((16, 3, 5000), F32, 0.5)]
SPECS = {
    "one value": [((1,), F32, None)],
    "one value, a scalar": [((), F32, None)],
    "one point": [((48, 1), F32, 1.0), ((3, 1), F16, 1.0)],
    "short rows": [((7, 2), F32, 0.6), ((9, 3), F32, 0.6), ((5, 5), BF16, 0.6), ((3, 7), F16, 0.8), ((11, 9), BF16, 1.0)],
    "odd rows": [((48, 1003), F32, 0.3), ((17, 2049), F16, 0.3), ((8, 2051), BF16, 0.9), ((1, 4099), F32, 0.02)],
    "a scene": GAUSS,
    "a scene and a network": GAUSS + [((64, 65), BF16, None), ((63,), F16, None), ((4097,), F32, None), ((16385,), BF16, None)],
    "no mask": [((5, 1001), F32, None), ((100003,), F32, None), ((33333,), F16, None), ((70001,), BF16, None)],
    "nothing used": [((3, 777), F32, 0.0), ((2, 100), F16, 0.0)],
    "one of many used": [((3, 1500), F32, 0.0), ((3, 1500), F32, 0.001), ((1,), F32, None)],
    "empty tensors": [((0,), F32, None), ((3, 0), F32, None), ((10,), F32, None), ((0, 4), F16, None), ((3, 0), BF16, 0.5)],
    "many points": [((11, 4_000_005), F32, 0.0003), ((9, 4_000_001), BF16, 0.4), ((3, 4_000_000), F32, 0.3)],
    "more than a workgroup each": [((3, 1_000_001), F32, 0.4), ((9_000_001,), F32, None), ((2, 3_000_000), BF16, 0.4)],
}


@pytest.mark.parametrize("name", SPECS)
@pytest.mark.parametrize("share", [0.25, 0.999, 1.5])      # of the norm that is allowed
def test_norm_and_clipping(name, share):
    ts, ms = make(SPECS[name], sum(name.encode()))
    norm = reference(ts, ms, np.inf)[0]
    run_clip(ts, ms, float(np.float32(norm * share)), in_place=share == 0.999)


@pytest.mark.parametrize("units", [1, 127, 128, 129, 1023, 1024, 1025, 2047, 2048, 2049, 4100])
@pytest.mark.parametrize("masked", [False, True])
def test_lengths_at_which_the_sum_ends_another_way(units, masked):
    """Units are 2,048 values without a mask, 4 planes of 1,024 points with one; a small tensor goes with the large one."""
    spec = [((4, units * 1024 - 3), F32, 0.5)] if masked else [((units * 2048 - 3,), F32, None)]
    ts, ms = make(spec + [((5,), F16, None)], units)
    norm = reference(ts, ms, np.inf)[0]
    run_clip(ts, ms, float(np.float32(norm * 0.5)), in_place=bool(units & 1))


@pytest.mark.parametrize("count", [7, 8, 9, 64, 87, 88, 89, 177, 1024])
def test_many_tensors(count):
    rng = np.random.default_rng(count)
    spec = [((int(rng.integers(0, 300)),), (F32, F16, BF16)[k % 3], None) if k % 5 else ((3, int(rng.integers(1, 2000))), F32, 0.5) for k in range(count)]
    ts, ms = make(spec, count)
    run_clip(ts, ms, 1e-3)


def test_no_tensor_at_all():
    ws = B.alloc_grad_workspace(0)
    for tensors in ([], [torch.empty(0, device="cuda")]):
        result = torch.full((2 + len(tensors),), 9.0, device="cuda")
        B.pbdr_grad_clip(B.GradList(tensors), 0.0, result, ws)
        torch.cuda.synchronize()
        assert result.tolist() == [0.0, 1.0, 0.0][:result.numel()]
    B.pbdr_adam_selective_list(B.AdamList([], [], [], [], []), 0.9, 0.999, 1e-8, 1)


@pytest.mark.parametrize("size", [1e-44, 1e-37, 1e-22, 1e18, 3e38])
def test_squares_that_fp32_cannot_hold(size):
    x = torch.tensor([3.0, -4.0, 0.0, 0.5] * 300, dtype=torch.float64).mul(size / 4).float().cuda()
    run_clip([x], [None], float(np.float32(size)))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_a_gradient_that_is_not_finite_counts_as_zero(bad, dtype):
    ts, ms = make([((3, 1001), F32, 0.5), ((2, 999), dtype, None)], 5)
    ts[1][1, 700] = bad
    result = torch.empty(4, device="cuda")
    B.pbdr_grad_clip(B.GradList(ts, visible=ms), float("inf"), result, B.alloc_grad_workspace(2))
    torch.cuda.synchronize()
    r = result.tolist()
    assert r[1] == 0.0 and (np.isnan(r[0]) and np.isnan(r[3]) if np.isnan(bad) else r[0] == r[3] == float("inf")) and np.isfinite(r[2])
    assert not ts[1].any() and not ts[0][:, ms[0] != 0].any() and torch.isnan(ts[0][:, ms[0] == 0]).any()


def test_zero_gradients_and_a_limit_of_zero():
    z = torch.zeros(3, 100, device="cuda")
    ws, result = B.alloc_grad_workspace(1), torch.empty(3, device="cuda")
    B.pbdr_grad_clip(B.GradList([z]), 0.0, result, ws)
    torch.cuda.synchronize()
    assert result.tolist() == [0.0, 1.0, 0.0]
    z.fill_(2.0)
    B.pbdr_grad_clip(B.GradList([z]), 0.0, result, ws)
    torch.cuda.synchronize()
    assert result[1] == 0.0 and not z.any()


def test_bits_do_not_change_from_run_to_run_or_with_the_stream():
    ts, ms = make(SPECS["more than a workgroup each"], 8)
    gl = B.GradList(ts, visible=ms)
    side = torch.cuda.Stream()
    got = []
    for k in range(4):
        result, ws = torch.empty(5, device="cuda"), B.alloc_grad_workspace(3)
        torch.cuda.synchronize()
        B.pbdr_grad_norm(gl, 0.5, result, ws, stream=side if k % 2 else None)
        torch.cuda.synchronize()
        got.append(result.clone())
    assert all(torch.equal(got[0], g) for g in got)


def test_rows_beyond_32_bits():
    """2^32 + 4100 values of 16 bits in one tensor, and three rows of 2^30 + 3 points; what is far back counts and is scaled."""
    n = (1 << 32) + 4100
    x = torch.zeros(n, dtype=BF16, device="cuda")
    x[-1], x[5], x[1 << 31] = 3.0, 4.0, 12.0
    result, ws = torch.empty(3, device="cuda"), B.alloc_grad_workspace(1)
    B.pbdr_grad_clip(B.GradList([x]), 6.5, result, ws)
    torch.cuda.synchronize()
    assert result.tolist() == [13.0, 0.5, 13.0]
    assert (float(x[-1]), float(x[5]), float(x[1 << 31])) == (1.5, 2.0, 6.0)
    del x
    n = (1 << 30) + 3
    y = torch.full((5, n), float("nan"), dtype=F16, device="cuda")
    mask = torch.zeros(n, dtype=torch.uint8, device="cuda")
    mask[-1] = mask[0] = 1
    y[:, 0], y[:, -1] = 0.0, 2.0
    B.pbdr_grad_clip(B.GradList([y], visible=mask), 1.0, result, ws)
    torch.cuda.synchronize()
    assert float(result[0]) == pytest.approx(20.0 ** 0.5, rel=1e-7)
    want = float(np.float16(np.float32(2.0) * np.float32(1 / 20.0 ** 0.5)))
    assert y[:, -1].tolist() == [want] * 5 and not y[:, 0].any() and torch.isnan(y[4, n - 2]) and torch.isnan(y[4, 1])


# ---------------------------------------------------------------------------------------------------------- Adam over a list
ADAM_SPECS = {
    "one value": [((1,), F32, None)],
    "one point": [((48, 1), F32, 1.0)],
    "short and odd rows": [((7, 2), F32, 0.6), ((9, 3), F32, 0.6), ((5, 5), F32, 0.6), ((17, 2049), F32, 0.3), ((48, 1003), F32, 0.7)],
    "a scene": GAUSS,
    "no mask": [((5, 1001), F32, None), ((100003,), F32, None)],
    "mixed": [((3, 777), F32, 0.0), ((0,), F32, None), ((3, 4100), F32, 0.9), ((4097,), F32, None), ((3, 0), F32, 0.5)],
    "eight": [((9,), F32, None)] * 8,
    "nine": [((3, 501), F32, 0.5)] * 9,
    "forty-nine": [((2, 77), F32, 0.5)] * 49,
    "many points": [((11, 4_000_005), F32, 0.0003), ((4_000_005,), F32, 0.5), ((6, 400_000), F32, 0.0005), ((5, 399_999), F32, 0.2)],
    "large": [((48, 100_001), F32, 0.4), ((5_000_003,), F32, None)],
}


@pytest.mark.parametrize("name", ADAM_SPECS)
@pytest.mark.parametrize("share,zero", [(0.3, False), (None, True), (2.0, True), (0.0, False)])
def test_adam_list_is_clipping_and_adam_bit_for_bit(name, share, zero):
    spec = ADAM_SPECS[name]
    ts, ms = make(spec, 31 + len(name))
    rng = np.random.default_rng(77)
    up = lambda a: torch.from_numpy(np.asarray(a, dtype=np.float32)).cuda()      # noqa: E731
    p = [up(rng.normal(size=t.shape)) for t in ts]
    m = [up(rng.normal(size=t.shape) * 1e-3) for t in ts]
    v = [up(rng.uniform(size=t.shape) * 1e-6) for t in ts]
    lrs = [1e-3 * (k + 1) for k in range(len(ts))]
    one = [[x.clone() for x in xs] for xs in (p, ts, m, v)]
    two = [[x.clone() for x in xs] for xs in (p, ts, m, v)]
    result = None
    if share is not None:
        result, ws = torch.empty(2 + len(ts), device="cuda"), B.alloc_grad_workspace(len(ts))
        norm = reference(ts, ms, np.inf)[0]
        B.pbdr_grad_norm(B.GradList(one[1], visible=ms), float(np.float32(norm * share)), result, ws)
        clipped = [x.clone() for x in ts]
        B.pbdr_grad_clip(B.GradList(clipped, visible=ms), float(np.float32(norm * share)), torch.empty_like(result), ws)
        two[1] = clipped
    B.pbdr_adam_selective_list(B.AdamList(*one, lrs, visible=ms), 0.9, 0.999, 1e-15, 7, clip=result, zero_grad=zero)
    for pp, g, mm, vv, mask, lr in zip(*two, ms, lrs):
        if pp.numel():
            every = torch.ones(pp.shape[-1], dtype=torch.uint8, device="cuda") if mask is None else mask
            B.pbdr_adam_selective(pp, g, mm, vv, every, lr, 0.9, 0.999, 1e-15, 7, zero_grad=zero)
    torch.cuda.synchronize()
    for k in (0, 2, 3):
        for a, b in zip(one[k], two[k]):
            assert torch.equal(a, b), name
    for a, raw, mask in zip(one[1], ts, ms):      # the gradient stays as it was, or its used entries are cleared
        want = raw if not zero else torch.zeros_like(raw) if mask is None else torch.where(mask != 0, 0.0, raw)
        assert torch.equal(a.view(torch.int32), want.contiguous().view(torch.int32))


def test_adam_list_against_the_oracle():
    spec = [((3, 301), F32, 0.5), ((301,), F32, 0.5), ((4, 3, 301), F32, 0.5), ((77,), F32, None)]
    ts, ms = make(spec, 4)
    rng = np.random.default_rng(9)
    up = lambda a: torch.from_numpy(np.asarray(a, dtype=np.float32)).cuda()      # noqa: E731
    p = [up(rng.normal(size=t.shape)) for t in ts]
    m = [torch.zeros_like(t) for t in ts]
    v = [torch.zeros_like(t) for t in ts]
    lr, b1, b2, eps = (float(np.float32(x)) for x in (1.6e-3, 0.9, 0.999, 1e-8))
    result, ws = torch.empty(6, device="cuda"), B.alloc_grad_workspace(4)
    al = B.AdamList(p, ts, m, v, [lr] * 4, visible=ms)
    for step in (1, 2, 3):
        p0, m0, v0 = ([rows(x) for x in xs] for xs in (p, m, v))
        norm, factor, _ = reference(ts, ms, 0.01)
        assert factor < 1
        B.pbdr_grad_norm(B.GradList(ts, visible=ms), 0.01, result, ws)
        B.pbdr_adam_selective_list(al, b1, b2, eps, step, clip=result)
        torch.cuda.synchronize()
        for k, t in enumerate(ts):
            used = np.ones(t.shape[-1]) if ms[k] is None else ms[k].cpu().numpy()
            g = np.where((used != 0).reshape(-1, *[1] * (t.dim() - 1)), rows(t), 0.0) * factor
            rp, rm, rv = oracle.adam_selective(p0[k], g, m0[k], v0[k], used, lr, b1, b2, eps, step)
            # as in the test of pbdr_adam_selective, plus two roundings of the clipped gradient (2^-23) in m, twice that in v
            assert (np.abs(rows(m[k]) - rm) <= 3e-7 * (b1 * np.abs(m0[k]) + (1 - b1) * np.abs(g)) + (1 - b1) * np.abs(g) * 2.0 ** -23 + 1e-30).all()
            np.testing.assert_allclose(rows(v[k]), rv, rtol=4e-7 + 2.0 ** -22, atol=1e-20)
            # m / sqrt(v) moves by the sum of what m and v are off, relative to their own terms
            room = 2e-6 * lr + lr * 2.0 ** -21 * np.maximum(1.0, (b1 * np.abs(m0[k]) + (1 - b1) * np.abs(g)) / np.maximum(np.sqrt(rv), 1e-30))
            assert (np.abs(rows(p[k]) - rp) <= room + 1.2e-7 * np.abs(rp)).all()
        for t, mask in zip(ts, ms):
            new = torch.from_numpy((rng.normal(size=t.shape) * 1e-3).astype(np.float32)).cuda()
            t.copy_(new if mask is None else torch.where(mask != 0, new, t))


def test_refusals_on_the_gpu():
    t = torch.ones(3, 64, device="cuda")
    result, ws = torch.empty(3, device="cuda"), B.alloc_grad_workspace(1)
    for bad in (lambda: B.pbdr_grad_clip(B.GradList([t, t]), 1.0, torch.empty(4, device="cuda"), ws), lambda: B.pbdr_grad_norm(B.GradList([t]), -1.0, result, ws),
                lambda: B.pbdr_grad_norm(B.GradList([t.view(-1)[1:]]), 1.0, result, ws), lambda: B.pbdr_grad_norm(B.GradList([t]), 1.0, result, ws[:256]),
                lambda: B.pbdr_adam_selective_list(B.AdamList([t], [t], [t.clone()], [t.clone()], [1.0]), 0.9, 0.999, 1e-8, 1)):
        with pytest.raises(B.PbdrError):
            bad()
    for bad in (lambda: B.pbdr_grad_norm(B.GradList([t]), 1.0, result[:2], ws), lambda: B.pbdr_grad_norm(B.GradList([t]), 1.0, result.double(), ws),
                lambda: B.pbdr_grad_norm(B.GradList([t]), 1.0, result.cpu(), ws), lambda: B.pbdr_grad_norm(B.GradList([t]), 1.0, result, ws.cpu()),
                lambda: B.GradList([t, t.cpu()])):
        with pytest.raises(ValueError):
            bad()
    torch.cuda.synchronize()
    assert (t == 1).all()


@pytest.mark.parametrize("n", [1, 3, 31, 33, 1023, 1025, 2050, 40_003, 450_001, 4_100_001])
@pytest.mark.parametrize("masked", [True, False])
def test_rows_and_buffers_that_begin_anywhere_on_a_line(n, masked):
    """Parameter, gradient, moments and output each at another multiple of 16 bytes, rows at any multiple of a value: what lies
    before, between and behind keeps its bits, unused entries too (NaN with a payload, infinities)."""
    rng = np.random.default_rng(n)
    planes = 5
    mask = torch.from_numpy((rng.uniform(size=n) < 0.8).astype(np.uint8)).cuda() if masked else None
    used = torch.ones(n, dtype=torch.bool, device="cuda") if mask is None else mask != 0
    guard = 0x7FA12345      # a NaN

    def buffer(shift, values):
        flat = torch.full((planes * n + 64,), guard, dtype=torch.int32, device="cuda").view(F32)
        view = flat[shift:shift + planes * n].view(planes, n)
        bits = torch.from_numpy(values.astype(np.float32)).cuda().view(torch.int32)
        view.view(torch.int32).copy_(torch.where(used, bits, torch.full_like(bits, guard)))
        return flat, view

    values = [rng.normal(size=(planes, n)), rng.normal(size=(planes, n)) * 1e-3, rng.normal(size=(planes, n)) * 1e-3, rng.uniform(size=(planes, n)) * 1e-6]
    flats, (p, g, m, v) = zip(*[buffer(shift, x) for shift, x in zip((4, 8, 28, 16), values)])
    out_flat, out = buffer(12, values[1])
    before = [f.view(torch.int32).clone() for f in (*flats, out_flat)]
    result, ws = torch.empty(3, device="cuda"), B.alloc_grad_workspace(1)
    limit = float(np.float32(reference([g], [mask], np.inf)[0] * 0.5))
    B.pbdr_grad_clip(B.GradList([g], visible=mask, out=[out]), limit, result, ws)
    B.pbdr_adam_selective_list(B.AdamList([p], [g], [m], [v], [1e-2], visible=mask), 0.9, 0.999, 1e-15, 3, clip=result, zero_grad=True)
    # the same on buffers of their own, by pbdr_adam_selective
    q, h, a, b = (torch.from_numpy(x.astype(np.float32)).cuda() for x in values)
    h.mul_(result[1])
    B.pbdr_adam_selective(q, h, a, b, torch.ones(n, dtype=torch.uint8, device="cuda") if mask is None else mask, 1e-2, 0.9, 0.999, 1e-15, 3)
    torch.cuda.synchronize()
    for got, want, name in ((p, q, "p"), (m, a, "m"), (v, b, "v"), (out, h, "out"), (g, torch.zeros_like(h), "g")):
        assert torch.equal(got[:, used], want[:, used]), name
    for flat, old, view in zip((*flats, out_flat), before, (p, g, m, v, out)):
        changed = flat.view(torch.int32) != old
        start = (view.data_ptr() - flat.data_ptr()) // 4
        inside = torch.zeros_like(changed)
        inside[start:start + planes * n] = used.repeat(planes)
        assert not (changed & ~inside).any()


def test_two_graphs_share_a_workspace_and_streams_change():
    """Every form of the sum's end (in the launch, in the scaling, in a launch of its own, over two tables), recorded twice with
    one workspace, replayed in turn with eager calls between, against the eager results; and the eager calls on another stream."""
    specs = [[((3, 900), F32, 0.5), ((64,), BF16, None)], [((14, 30_000), F32, None)], [((48, 30_001), F32, 0.6), ((3, 30_001), F32, 0.6)],
             [((int(k % 7) * 100 + 1,), (F32, F16)[k % 2], None) for k in range(120)]]
    ws = B.alloc_grad_workspace(120)
    for k, spec in enumerate(specs):
        ts, ms = make(spec, k)
        limit = float(np.float32(reference(ts, ms, np.inf)[0] * 0.5))
        adam = [i for i, t in enumerate(ts) if t.dtype == F32]
        def state():
            g = [t.clone() for t in ts]
            p, m, v = ([torch.zeros_like(ts[i]) for i in adam] for _ in range(3))
            s = dict(g=g, out=[torch.zeros_like(t) for t in ts], p=p, m=m, v=v, result=torch.zeros(2 + len(ts), device="cuda"), clip=torch.zeros(2 + len(ts), device="cuda"))
            s["norm"], s["to"] = B.GradList(g, visible=ms), B.GradList(g, visible=ms, out=s["out"])
            s["adam"] = B.AdamList(p, [g[i] for i in adam], m, v, [1e-3] * len(adam), visible=[ms[i] for i in adam])
            return s

        def run(s, stream=None):
            B.pbdr_grad_norm(s["norm"], limit, s["result"], ws, stream=stream)
            B.pbdr_grad_clip(s["to"], limit, s["clip"], ws, stream=stream)
            B.pbdr_adam_selective_list(s["adam"], 0.9, 0.999, 1e-15, 2, clip=s["result"], stream=stream)

        def flat(s):
            return [x.view(torch.int32 if x.dtype == F32 else torch.int16) for x in (s["result"], s["clip"], *s["out"], *s["p"], *s["m"], *s["v"])]

        states, graphs = [state(), state()], []
        ref = state()
        run(state())
        torch.cuda.synchronize()
        for s in states:
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1]):
                run(s)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        for rep in range(3):
            for graph in graphs:
                graph.replay()
            torch.cuda.synchronize()
            run(ref, stream=side if rep == 1 else None)
            torch.cuda.synchronize()
            assert 0 < float(ref["result"][1]) < 1
            for s in states:
                assert all(torch.equal(a, b) for a, b in zip(flat(s), flat(ref))), (k, rep)


def test_calls_in_flight_on_two_streams():
    """Lists of both kinds of ending, each stream with a workspace and result of its own, nothing waiting between."""
    pairs = []
    for spec in (SPECS["odd rows"], SPECS["more than a workgroup each"]):
        ts, ms = make(spec, len(spec))
        pairs.append((B.GradList(ts, visible=ms), B.GradList(ts, visible=ms, out=[torch.zeros_like(t) for t in ts]), len(ts)))
    want = []
    for norm, _, count in pairs:
        result = torch.empty(2 + count, device="cuda")
        B.pbdr_grad_norm(norm, 0.5, result, B.alloc_grad_workspace(count))
        want.append(result)
    streams = [torch.cuda.Stream() for _ in pairs]
    spaces = [B.alloc_grad_workspace(count) for *_, count in pairs]
    results = [[torch.empty(2 + count, device="cuda") for _ in range(20)] for *_, count in pairs]
    torch.cuda.synchronize()
    for rep in range(20):
        for (norm, clip, _), stream, ws, result in zip(pairs, streams, spaces, results):
            (B.pbdr_grad_clip if rep % 3 == 2 else B.pbdr_grad_norm)(clip if rep % 3 == 2 else norm, 0.5, result[rep], ws, stream=stream)
    torch.cuda.synchronize()
    for result, w in zip(results, want):
        assert all(torch.equal(r, w) for r in result)


def test_lists_follow_tensors_that_get_other_memory():
    t, mask = torch.ones(3, 50, device="cuda"), torch.ones(50, dtype=torch.bool, device="cuda")
    mask[10:] = False
    gl = B.GradList([t], visible=mask)
    result, ws = torch.empty(3, device="cuda"), B.alloc_grad_workspace(1)
    B.pbdr_grad_norm(gl, 1e9, result, ws)
    assert float(result[0]) == pytest.approx(30 ** 0.5, rel=1e-6)
    t.data = torch.full((7, 50), 2.0, device="cuda")
    B.pbdr_grad_clip(gl, 1.0, result, ws)
    assert float(result[0]) == pytest.approx((7 * 10 * 4) ** 0.5, rel=1e-6)
    assert float(t[:, :10].norm()) == pytest.approx(1.0, rel=1e-6) and (t[:, 10:] == 2).all()


# ------------------------------------------------------------------------------------------------------- a training iteration
def test_a_training_iteration_eager_and_replayed():
    """Render, loss, backward, norm over the scene and a small network's 16-bit gradients, Adam with the factor: recorded
    once and replayed, with other work between the replays, against the same calls issued one by one, clipping by hand."""
    n, W, H, cap = 12000, 320, 200, 600_000
    sc = synth.random_small_scene(3, n, 1, spread=1.0, ls_mu=-3.2)
    cam = synth.pinhole(W, H, 55.0, *synth.look_at((0.3, -0.2, -3.0), (0, 0, 0), (0, 1, 0)))
    rng = np.random.default_rng(1)
    target = torch.from_numpy(rng.uniform(size=(3, H, W)).astype(np.float32)).cuda()
    net = torch.from_numpy((rng.normal(size=(64, 33)) * 1e-4).astype(np.float32)).to(BF16).cuda()
    names, lrs = ("mean", "log_scale", "quat", "logit", "sh"), (1.6e-4, 5e-3, 1e-3, 5e-2, 2.5e-3)

    def state():
        s = dict(scene=B.Scene.from_numpy(sc), splats=B.Splats.empty(n), ws=B.alloc_workspace(n, W, H, cap), gws=B.alloc_grad_workspace(6))
        s["grads"], s["m"], s["v"] = (s["scene"].zeros_like() for _ in range(3))
        s["visible"] = torch.zeros(n, dtype=torch.uint8, device="cuda")
        s["image"], s["dL"] = (torch.empty((3, H, W), device="cuda") for _ in range(2))
        s["T"], s["last"] = torch.empty((H, W), device="cuda"), torch.empty((H, W), dtype=torch.int32, device="cuda")
        s["loss"], s["result"] = torch.zeros(1, device="cuda"), torch.empty(8, device="cuda")
        g = [getattr(s["grads"], k) for k in names]
        s["list"] = B.GradList(g + [net], visible=[s["visible"]] * 5 + [None])
        s["adam"] = B.AdamList([getattr(s["scene"], k) for k in names], g, *[[getattr(s[x], k) for k in names] for x in "mv"], lrs, visible=s["visible"])
        return s

    def forward_backward(s):
        B.pbdr_preprocess(s["scene"], cam, s["splats"])
        s["visible"].zero_()
        B.pbdr_mark_visible(s["splats"].radius, s["visible"])
        B.pbdr_render_fwd(s["splats"], cam, [0.1, 0.2, 0.3], cap, s["image"], s["T"], s["last"], s["ws"])
        B.pbdr_l1_loss(s["image"], target, s["loss"], s["dL"])
        B.pbdr_render_bwd(s["scene"], s["splats"], cam, [0.1, 0.2, 0.3], cap, s["T"], s["last"], s["dL"], None, s["grads"], s["ws"], first_view=True)
        B.pbdr_grad_norm(s["list"], 1e-3, s["result"], s["gws"])

    def iteration(s):
        forward_backward(s)
        B.pbdr_adam_selective_list(s["adam"], 0.9, 0.999, 1e-15, 5, clip=s["result"])

    got, ref = state(), state()
    warm = state()
    iteration(warm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        iteration(got)
    torch.cuda.synchronize()
    for rep in range(3):
        torch.cuda.synchronize()
        graph.replay()
        (torch.randn(1000, device="cuda") * 2).sum()
        torch.cuda.synchronize()
        forward_backward(ref)
        factor = float(ref["result"][1])
        assert 0 < factor < 1
        for k, lr in zip(names, lrs):
            g = getattr(ref["grads"], k)
            g.mul_(ref["result"][1])
            B.pbdr_adam_selective(getattr(ref["scene"], k), g, getattr(ref["m"], k), getattr(ref["v"], k), ref["visible"], lr, 0.9, 0.999, 1e-15, 5)
        torch.cuda.synchronize()
        assert torch.equal(got["result"], ref["result"])
        for k in names:
            assert torch.equal(getattr(got["scene"], k), getattr(ref["scene"], k)), (rep, k)
            assert torch.equal(getattr(got["m"], k), getattr(ref["m"], k)) and torch.equal(getattr(got["v"], k), getattr(ref["v"], k))
        assert 0 < int(ref["visible"].sum()) < n
    # the list holds the scene's norm and the network's
    r = ref["result"].double()
    assert float(r[0]) == pytest.approx(float(r[2:].norm()), rel=1e-6)
    assert float(r[7]) == pytest.approx(float(net.double().norm()), rel=1e-7)


def test_a_list_that_was_refused_serves_tensors_that_came_back():
    ts = [torch.full((40,), 3.0, device="cuda"), torch.full((30,), 4.0, device="cuda")]
    gl = B.GradList(ts)
    result, ws = torch.empty(4, device="cuda"), B.alloc_grad_workspace(2)
    here = ts[0].data
    ts[0].data = here.cpu()
    with pytest.raises(ValueError):      # one on each side
        B.pbdr_grad_norm(gl, 1.0, result, ws)
    ts[0].data = here
    B.pbdr_grad_norm(gl, 1.0, result, ws)
    torch.cuda.synchronize()
    assert float(result[0]) == pytest.approx(840 ** 0.5, rel=1e-6)


@pytest.mark.parametrize("spec,op,want", [
    ([((3, 900), F32, 0.5)], "norm", dict(k_grad_squares=1)),
    ([((3, 900), F32, 0.5)], "clip", dict(k_grad_squares=1, k_grad_scale=1)),
    ([((14, 90_000), F32, None)], "norm", dict(k_grad_squares=1, k_grad_finish=1)),
    ([((14, 90_000), F32, None)], "clip", dict(k_grad_squares=1, k_grad_scale=1)),
    ([((48, 60_001), F32, None)], "clip", dict(k_grad_squares=1, k_grad_finish=1, k_grad_scale=1)),
    ([((100,), F32, None)] * 89, "norm", dict(k_grad_squares=2)),
    ([((100,), F32, None)] * 89, "clip", dict(k_grad_squares=2, k_grad_scale=2)),
    ([((100,), F32, None)] * 49, "adam", dict(k_adam_list=2)),
    ([((3, 0), F32, None)], "clip", dict(k_grad_squares=1)),
    ([((3, 0), F32, None)], "adam", dict()),
], ids=lambda x: x if isinstance(x, str) else None)
def test_each_launch_is_timed_under_its_kernel(spec, op, want):
    ts, ms = make(spec, 3)
    result, ws = torch.empty(2 + len(ts), device="cuda"), B.alloc_grad_workspace(len(ts))
    gl = B.GradList(ts, visible=ms, out=[torch.empty_like(t) for t in ts])
    al = B.AdamList(*[[t.clone() for t in ts] for _ in range(4)], [1e-3] * len(ts), visible=ms)
    names = B.profile_kernel_names()
    torch.cuda.synchronize()
    B.pbdr_profile_begin((1 << len(names)) - 1, 16)
    try:
        if op == "adam":
            B.pbdr_adam_selective_list(al, 0.9, 0.999, 1e-8, 1)
        else:
            (B.pbdr_grad_norm if op == "norm" else B.pbdr_grad_clip)(gl, 0.5, result, ws)
        torch.cuda.synchronize()
        got = {name: B.pbdr_profile_collect(k) for k, name in enumerate(names)}
    finally:
        B.pbdr_profile_end()
    assert {name: count for name, (ms_, count) in got.items() if count} == want
    assert all(ms_ > 0 for ms_, count in got.values() if count)


# ------------------------------------------------------------------------------------------------------------ sizes and ranges at the ends
@pytest.mark.parametrize("dtype,size", [(F32, 1e-39), (BF16, 1e-38), (F16, 1e-6)])
def test_clipped_values_below_the_normal_numbers(dtype, size):
    """Gradients around the smallest normal number of their type, a quarter of which is left: most of what is written is subnormal."""
    ts, ms = make([((3, 1001), dtype, 0.5), ((5003,), dtype, None)], 21, size)
    norm = reference(ts, ms, np.inf)[0]
    run_clip(ts, ms, float(np.float32(norm * 0.25)))
    x = ts[1].cpu().double() * 0.25
    assert 0 < float(x.abs().median()) < float(torch.finfo(dtype).tiny)


def test_launches_whose_workgroups_take_several_units_each():
    """More units than a launch has workgroups (2^23): rows of one point, 2^24 - 1 of them, three times that for scaling."""
    planes = (1 << 24) - 1
    gen = torch.Generator(device="cuda").manual_seed(4)
    gs = [torch.randn(planes, 1, device="cuda", generator=gen) for _ in range(3)]
    seen = torch.ones(1, dtype=torch.uint8, device="cuda")
    outs = [torch.full_like(g, float("nan")) for g in gs]
    result, ws = torch.empty(5, device="cuda"), B.alloc_grad_workspace(3)
    B.pbdr_grad_clip(B.GradList(gs, visible=seen, out=outs), 100.0, result, ws)
    torch.cuda.synchronize()
    each = [float(g.double().norm()) for g in gs]
    norm = float(np.sqrt(sum(e * e for e in each)))
    # one lane of a workgroup adds all its terms here: 2^23 units / 2048 workgroups * 4 planes * 1.5 = 24,576 terms, 2^-53 each, and
    # the root halves it: 1.4e-12 beside the rounding to fp32
    for got, want in zip(result.tolist(), [norm, 100.0 / norm] + each):
        assert abs(got - want) <= (EPS + 3e-12) * want
    assert 0 < float(result[1]) < 1
    for g, o in zip(gs, outs):
        assert torch.equal(o, g * result[1])
    p, m, v = torch.randn(planes, 1, device="cuda", generator=gen), outs[1], outs[2].square_()
    q, g, a, b = (x.clone().view(1, planes) for x in (p, gs[0], m, v))
    B.pbdr_adam_selective_list(B.AdamList([p], [gs[0]], [m], [v], [1e-2], visible=seen), 0.9, 0.999, 1e-15, 3, zero_grad=True)
    B.pbdr_adam_selective(q, g, a, b, torch.ones(planes, dtype=torch.uint8, device="cuda"), 1e-2, 0.9, 0.999, 1e-15, 3, zero_grad=True)
    torch.cuda.synchronize()
    for got, want in ((p, q), (m, a), (v, b), (gs[0], g)):
        assert torch.equal(got.view(-1), want.view(-1))
    assert not gs[0].any()


def test_adam_beyond_32_bits():
    """Five rows of 2^30 + 3 entries with three used points, then the same memory as one row of all entries."""
    n, planes = (1 << 30) + 3, 5
    spots = [0, 777_777_777, n - 1]
    p, m, v = (torch.zeros(planes, n, device="cuda") for _ in range(3))
    g = torch.full((planes, n), float("nan"), device="cuda")
    seen = torch.zeros(n, dtype=torch.uint8, device="cuda")
    new = torch.arange(1.0, 16.0, device="cuda").view(planes, 3)
    for k, at in enumerate(spots):
        seen[at] = 1
        g[:, at] = new[:, k]

    def check():
        for got, want in zip((p, m, v), small()):
            assert torch.equal(torch.stack([got[:, at] for at in spots], 1), want)
            assert all(int(torch.count_nonzero(row)) == 3 for row in got)

    def small():      # pbdr_adam_selective on the used entries alone
        q, h, a, b = torch.zeros(1, 15, device="cuda"), new.clone().view(1, 15), torch.zeros(1, 15, device="cuda"), torch.zeros(1, 15, device="cuda")
        B.pbdr_adam_selective(q, h, a, b, torch.ones(15, dtype=torch.uint8, device="cuda"), 1e-2, 0.9, 0.999, 1e-8, 2)
        return [x.view(planes, 3) for x in (q, a, b)]

    B.pbdr_adam_selective_list(B.AdamList([p], [g], [m], [v], [1e-2], visible=seen), 0.9, 0.999, 1e-8, 2)
    check()
    for x in (p, m, v, g):
        x.zero_()
    for k, at in enumerate(spots):
        g[:, at] = new[:, k]
    flat = [x.view(-1) for x in (p, g, m, v)]
    assert flat[0].numel() > 1 << 32
    B.pbdr_adam_selective_list(B.AdamList(*[[x] for x in flat], [1e-2]), 0.9, 0.999, 1e-8, 2)
    check()


def test_clipping_and_updates_in_flight_on_several_streams():
    """Each stream clips into buffers and updates parameters of its own, call upon call, nothing waiting between; all that is
    written is compared with what the same calls leave one at a time."""
    def work(name, spec):
        ts, ms = make(spec, len(name))
        adam = [k for k, t in enumerate(ts) if t.dtype == F32]

        def one():
            s = dict(out=[torch.zeros_like(t) for t in ts], result=torch.zeros(2 + len(ts), device="cuda"))
            p, m, v = ([torch.zeros_like(ts[k]) for k in adam] for _ in range(3))
            s["clip"] = B.GradList(ts, visible=ms, out=s["out"])
            s["adam"] = B.AdamList(p, [ts[k] for k in adam], m, v, [1e-3] * len(adam), visible=[ms[k] for k in adam])
            s["all"] = [s["result"], *s["out"], *p, *m, *v]
            return s
        return one

    def run(s, ws, stream=None):
        B.pbdr_grad_clip(s["clip"], 0.1, s["result"], ws, stream=stream)
        B.pbdr_adam_selective_list(s["adam"], 0.9, 0.999, 1e-15, 2, clip=s["result"], stream=stream)

    makers = [work(name, SPECS[name]) for name in ("odd rows", "more than a workgroup each", "a scene")]
    spaces, streams = [B.alloc_grad_workspace(8) for _ in makers], [torch.cuda.Stream() for _ in makers]
    want, states = [one() for one in makers], [[one() for _ in range(6)] for one in makers]
    for s, ws in zip(want, spaces):
        run(s, ws)
        torch.cuda.synchronize()
        assert 0 < float(s["result"][1]) < 1
    for rep in range(6):
        for row, ws, stream in zip(states, spaces, streams):
            run(row[rep], ws, stream)
    torch.cuda.synchronize()
    for s, row in zip(want, states):
        for got in row:
            for a, b in zip(got["all"], s["all"]):
                bits = torch.int32 if a.dtype == F32 else torch.int16
                assert torch.equal(a.view(bits), b.view(bits))


@pytest.mark.parametrize("bad", [None, float("nan"), float("inf")])
def test_a_step_with_other_gradients_in_the_list(bad):
    """Norm over a scene and 16-bit extras, Adam on the scene, the extras times the factor by torch: bit for bit what clipping the
    whole list and pbdr_adam_selective leave, a gradient that is not finite among the extras too."""
    spec = GAUSS + [((64, 33), BF16, None), ((63,), F16, None), ((17,), F32, None)]
    ts, ms = make(spec, 12)
    if bad is not None:
        ts[-2][5] = bad
    rng = np.random.default_rng(2)
    p, m, v = ([torch.from_numpy(f(size=t.shape).astype(np.float32)).cuda() for t in ts[:5]] for f in (rng.normal, rng.normal, rng.uniform))
    one, two = ([[x.clone() for x in xs] for xs in (ts, p, m, v)] for _ in range(2))
    result, ws = torch.empty(2 + len(ts), device="cuda"), B.alloc_grad_workspace(len(ts))
    grads, net_grads = one[0][:5], one[0][5:]
    B.pbdr_grad_norm(B.GradList(grads + net_grads, visible=ms), 0.05, result, ws)
    B.pbdr_adam_selective_list(B.AdamList(one[1], grads, one[2], one[3], [1e-3] * 5, visible=ms[:5]), 0.9, 0.999, 1e-8, 2, clip=result)
    for g in net_grads:
        g.copy_(torch.where(result[1] == 0, 0.0, g.float() * result[1]))
    B.pbdr_grad_clip(B.GradList(two[0], visible=ms), 0.05, torch.empty_like(result), ws)
    for k in range(5):
        B.pbdr_adam_selective(two[1][k], two[0][k], two[2][k], two[3][k], ms[k], 1e-3, 0.9, 0.999, 1e-8, 2)
    torch.cuda.synchronize()
    assert float(result[1]) == 0.0 if bad is not None else 0 < float(result[1]) < 1
    for a, b in zip(one[0][5:], two[0][5:]):
        assert a.dtype == b.dtype and torch.equal(a, b) and bool(a.any()) == (bad is None)
    for a, b in zip(one[1] + one[2] + one[3], two[1] + two[2] + two[3]):
        assert torch.equal(a, b)
