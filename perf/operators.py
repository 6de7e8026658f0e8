"""Workloads of the gradient operators between the backward pass and the update, as a training program calls them.

A case is a dict of plain values:
  op       norm   the global norm of the gradient and the clipping factor, nothing else (monitoring, a loop with its own optimizer)
           clip   the same and the clipped gradient into buffers of its own (the raw one is kept for densification statistics)
           step   norm, then selective Adam on every attribute with the factor applied on the way
  model    gauss (3D Gaussians, five attribute tensors) or surfel (2D Gaussian disks, six)
  n, degree   points and SH degree; an attribute with l components is [l, n]
  visible  share of the points that the batch's views use (in runs: points are stored in Z-order), or 1.0: no mask
  extra    number of further gradient tensors of other learned things (camera corrections, a small appearance network), all used
  kind     their type: f32, f16 or bf16
  ratio    the allowed norm over the norm to expect: below 1 the gradient is clipped, above it is left as it is
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
RUN = 701                                  # points of a run that is seen or not seen as a whole
# components of the attributes, the typical size of their gradients (mean-L1 loss, 1080p) and their learning rates
ATTRS = {
    "gauss": (("mean", 3, 3e-6, 1.6e-4), ("log_scale", 3, 1e-6, 5e-3), ("quat", 4, 4e-7, 1e-3), ("logit", 1, 5e-7, 5e-2), ("sh", 3, 2e-7, 2.5e-3)),
    "surfel": (("mean", 3, 3e-6, 1.6e-4), ("tan_u", 3, 4e-7, 1e-3), ("tan_v", 3, 4e-7, 1e-3), ("log_scale", 2, 1e-6, 5e-3),
               ("logit", 1, 5e-7, 5e-2), ("sh", 3, 2e-7, 2.5e-3)),
}
KINDS = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# hyper-parameters as the boundary takes them: rounded to 32 bits
BETA1, BETA2, EPS = (float(np.float32(x)) for x in (0.9, 0.999, 1e-15))
STEP = 4000


def _case(name, op, model, n, degree, visible=1.0, extra=0, kind="f32", ratio=0.3):
    c = dict(op=op, model=model, n=n, degree=degree, visible=visible, extra=extra, kind=kind, ratio=ratio)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # the smallest configuration of the benchmark: latency counts
        _case("norm_tiny", "norm", "gauss", 4096, 0),
        # the 1M-point scene after a batch of views that see all of it
        _case("norm_mid", "norm", "gauss", 1000000, 3, ratio=4.0),
        # one GPU's share of a city: street-level views use one point in four
        _case("norm_street", "norm", "gauss", 8000000, 3, visible=0.25),
        # an odd number of surfels and the many small tensors of a 16-bit appearance network
        _case("norm_many", "norm", "surfel", 100003, 2, visible=0.6, extra=160, kind="bf16"),
        # a surfel object fit, odd size, everything in view
        _case("clip_tiny", "clip", "surfel", 3001, 2),
        # a ragged scene of the benchmark's tests with a 16-bit network
        _case("clip_mixed", "clip", "gauss", 30011, 2, visible=0.5, extra=40, kind="f16"),
        # the 1M-point scene
        _case("clip_mid", "clip", "gauss", 1000000, 3),
        # two million surfels: twice what the last-level cache holds
        _case("clip_large", "clip", "surfel", 2000000, 3, ratio=0.7),
        # the smallest configuration's update
        _case("step_tiny", "step", "gauss", 4096, 0, visible=0.9),
        # an early iteration of a surfel scene, odd size
        _case("step_loop", "step", "surfel", 200003, 3, visible=0.7),
        # the 1M-point scene
        _case("step_mid", "step", "gauss", 1000000, 3, visible=0.6),
        # one GPU's share of a city
        _case("step_street", "step", "gauss", 8000000, 3, visible=0.25, ratio=4.0),
    ]


def draw(rng):
    def log_uniform(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["norm", "clip", "step"])
    n = log_uniform(500, 8000000)
    visible = 1.0 if n <= 2000000 and rng.random() < 0.35 else round(min(rng.uniform(0.05, 0.95), 2e6 / n), 3)
    extra = 0 if op == "step" or rng.random() < 0.5 else log_uniform(1, 200 if op == "norm" else 40)
    return _case(None, op, rng.choice(["gauss", "gauss", "surfel"]), n, rng.choice([0, 1, 2, 3, 3, 3]), visible, extra,
                 rng.choice(["f32", "f16", "bf16"]), rng.choice([0.1, 0.3, 0.7, 4.0]))


# ----------------------------------------------------------------------------------------------------------------- inputs
def _shapes(case):
    """(shape, typical size of the gradient, learning rate) of each attribute."""
    n, K = case["n"], (case["degree"] + 1) ** 2
    out = []
    for name, l, size, lr in ATTRS[case["model"]]:
        out.append(((K, 3, n) if name == "sh" else (n,) if l == 1 else (l, n), size, float(np.float32(lr))))
    return out


def _extra_lengths(case):
    """Vectors and matrices of a small network, ragged: 1 to 65,664 values."""
    widths = (1, 16, 63, 64, 127, 256)
    out = []
    for k in range(case["extra"]):
        a, b = widths[k % 6], widths[(k // 6 + k) % 6]
        out.append(b if k % 2 else a * b + a // 2)
    return out


def _runs(case):
    """How many runs of points there are and how many of them are seen."""
    runs = -(-case["n"] // RUN)
    return runs, max(1, round(case["visible"] * runs))


def _visible(case, g):
    if case["visible"] >= 1.0:
        return None
    runs, seen = _runs(case)
    order = torch.randperm(runs, generator=g, device=DEV)
    mask = (order < seen).repeat_interleave(RUN)[:case["n"]]
    return (mask & (torch.rand(case["n"], generator=g, device=DEV) < 0.97)).to(torch.uint8)


def _gradient(shape, size, g, visible):
    """Points differ in the size of their gradients by a factor of e or so; points out of view got none."""
    x = torch.randn(shape, generator=g, device=DEV)
    x.mul_(torch.randn(shape[-1], generator=g, device=DEV).exp_().mul_(size))
    return x if visible is None else x.mul_(visible)


def _share(case):
    """Used points over points, near enough."""
    if case["visible"] >= 1.0:
        return 1.0
    runs, seen = _runs(case)
    return 0.97 * seen / runs


def _expected_norm(case):
    square = sum(math.prod(shape) * _share(case) * (size * math.e) ** 2 for shape, size, _ in _shapes(case))
    return math.sqrt(square + sum(_extra_lengths(case)) * 1e-6)


def _carve(lengths, dtype):
    """Tensors of these lengths out of one buffer, 16-byte aligned each, as a bucket of gradients is laid out."""
    pad = [-(-k // 8) * 8 for k in lengths]
    flat = torch.zeros(sum(pad), dtype=dtype, device=DEV)
    return [x[:k] for x, k in zip(torch.split(flat, pad), lengths)]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    visible = _visible(case, g)
    shapes = _shapes(case)
    grads = [_gradient(shape, size, g, visible) for shape, size, _ in shapes]
    masks = [visible] * len(grads)
    lengths = _extra_lengths(case)
    if lengths:
        extra = _carve(lengths, KINDS[case["kind"]])
        for t in extra:
            t.copy_(torch.randn(t.shape, generator=g, device=DEV).mul_(1e-3))
        grads += extra
        masks += [None] * len(extra)
    s = dict(op=case["op"], grads=grads, masks=masks, max_norm=float(np.float32(case["ratio"] * _expected_norm(case))))
    if case["op"] == "clip":
        s["out"] = [torch.zeros_like(t) for t in grads[:len(shapes)]]
        if lengths:
            s["out"] += _carve(lengths, KINDS[case["kind"]])
    if case["op"] == "step":
        s["lrs"] = [lr for _, _, lr in shapes]
        s["params"] = [torch.randn(shape, generator=g, device=DEV) for shape, _, _ in shapes]
        s["m"] = [0.3 * _gradient(shape, size, g, None) for shape, size, _ in shapes]
        s["v"] = [_gradient(shape, size, g, None).square_() + (0.1 * size) ** 2 for shape, size, _ in shapes]
        s["step"] = STEP
    if own:
        from paper_2512_20017_amd import binding as B
        s["list"] = B.GradList(grads, visible=masks, out=s.get("out"))
        s["result"] = torch.empty(2 + len(grads), device=DEV)
        s["ws"] = B.alloc_grad_workspace(len(grads))
        if case["op"] == "step":
            s["adam"] = B.AdamList(s["params"], grads, s["m"], s["v"], s["lrs"], visible=masks)
    return s


# ------------------------------------------------------------------------------------------------------------------- runs
def _plain_norm(s):
    squares = torch.stack([(t.float() if v is None else torch.where(v != 0, t.float(), 0.0)).square().sum() for t, v in zip(s["grads"], s["masks"])])
    norm = squares.sum().sqrt()
    scale = torch.where(torch.isfinite(norm), torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0), 0.0)
    return torch.cat([norm[None], scale[None], squares.sqrt()])


def _plain_scaled(t, scale):
    return torch.where(scale == 0.0, 0.0, t.float() * scale)


def _plain_adam(p, t, m, v, mask, lr, scale, step):
    t = _plain_scaled(t, scale)
    m2 = BETA1 * m + (1.0 - BETA1) * t
    v2 = BETA2 * v + (1.0 - BETA2) * t * t
    p2 = p - lr / (1.0 - BETA1 ** step) * m2 / ((v2 / (1.0 - BETA2 ** step)).sqrt() + EPS)
    for old, new in ((p, p2), (m, m2), (v, v2)):
        old.copy_(new if mask is None else torch.where(mask != 0, new, old))


def run(s):
    if s["op"] == "step":
        s["step"] += 1
    if own:
        from paper_2512_20017_amd import binding as B
        if s["op"] == "clip":
            B.pbdr_grad_clip(s["list"], s["max_norm"], s["result"], s["ws"])
            return [s["result"], s["out"]]
        B.pbdr_grad_norm(s["list"], s["max_norm"], s["result"], s["ws"])
        if s["op"] == "norm":
            return s["result"]
        B.pbdr_adam_selective_list(s["adam"], BETA1, BETA2, EPS, s["step"], clip=s["result"])
        return [s["result"], s["params"], s["m"], s["v"]]
    result = _plain_norm(s)
    if s["op"] == "norm":
        return result
    scale = result[1]
    if s["op"] == "clip":
        for o, t, v in zip(s["out"], s["grads"], s["masks"]):
            new = _plain_scaled(t, scale)
            o.copy_(new if v is None else torch.where(v != 0, new, o.float()))
        return [result, s["out"]]
    for args in zip(s["params"], s["grads"], s["m"], s["v"], s["masks"], s["lrs"]):
        _plain_adam(*args, scale, s["step"])
    return [result, s["params"], s["m"], s["v"]]


def exact(case, seed):
    """From the definitions in 64 bits: a used entry counts, an unused one stays as it is."""
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    one = torch.ones((), dtype=torch.bool, device=DEV)
    used = [one if v is None else v.bool() for v in s["masks"]]
    each = []
    for t, u in zip(s["grads"], used):
        x = t.double()
        x *= u
        each.append(float(torch.linalg.vector_norm(x)) if x.numel() else 0.0)
    norm = math.hypot(*each)
    scale = min(1.0, s["max_norm"] / norm) if norm > 0 else 1.0
    result = torch.tensor([norm, scale] + each, dtype=torch.float64, device=DEV)
    if s["op"] == "norm":
        return result
    if s["op"] == "clip":
        out = []
        for o, t, u in zip(s["out"], s["grads"], used):
            out.append(torch.where(u, t.double() * scale, o.double()))
        return [result, out]
    step, ps, ms, vs = STEP + 1, [], [], []
    for p, t, m, v, u, lr in zip(s["params"], s["grads"], s["m"], s["v"], used, s["lrs"]):
        x = t.double() * scale
        first = m.double().lerp(x, 1.0 - BETA1)
        second = v.double().lerp(x.square(), 1.0 - BETA2)
        del x
        new = p.double().addcdiv_(first / (1.0 - BETA1 ** step), (second / (1.0 - BETA2 ** step)).sqrt_().add_(EPS), value=-lr)
        ps.append(torch.where(u, new, p.double()))
        ms.append(torch.where(u, first, m.double()))
        vs.append(torch.where(u, second, v.double()))
    return [result, ps, ms, vs]


def work(case):
    """Used entries once in and, where they change, once out; the mask once."""
    used = sum(math.prod(shape) for shape, _, _ in _shapes(case)) * _share(case)
    extra = sum(_extra_lengths(case))
    size = 4 if case["kind"] == "f32" else 2
    mask = case["n"] if case["visible"] < 1.0 else 0
    result = 4 * (2 + len(_shapes(case)) + case["extra"])
    gradient = 4 * used + size * extra
    if case["op"] == "norm":
        return {"bytes": gradient + mask + result, "flops": 2 * (used + extra)}
    if case["op"] == "clip":
        return {"bytes": 2 * gradient + mask + result, "flops": 3 * (used + extra)}
    return {"bytes": 28 * used + mask + result, "flops": 16 * used}
