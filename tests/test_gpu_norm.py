"""GPU parity of the norms around a block against their float64 definition and its automatic gradient.

Error bars.  Every output is an fp32 expression rounded once: 2^-8 (bf16) or
2^-24 (fp32) of its value, plus the expression's own error.  That is counted
against `sizes`, the same expression with every term's magnitude (a gradient
through a norm is a difference that can cancel entirely: with one feature, it
is zero).  An fp32 sum over a row, in a tree of at most log2 D + 8 levels, and
the few operations around it leave (log2 D + 16) 2^-24 of the magnitudes; a
value passes at most four of these, 2^-22.  A norm magnifies what its input is
off by, relative to the row's spread: kappa = max |z| / spread of each norm
(1 at least) multiplies the error of everything behind it.  Parameter
gradients add one term per token, each addition 2^-24 of the sum of magnitudes.
"""
import math

import pytest
import torch

import layer_reference as ref
from paper_2306_01926_amd import ga

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
NAMES = ("X", "F", "post_w", "post_b", "gate", "pre_w", "pre_b")
KW = {"post_w": "post_weight", "post_b": "post_bias", "gate": "gate", "pre_w": "pre_weight", "pre_b": "pre_bias"}


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    ga.lib()
    return torch.device("cuda:0")


def make(dtype, B, n, D, kind, post=True, gate=1, pre=True, branch=True, seed=0):
    g = torch.Generator().manual_seed(seed + D)
    new = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    p = dict(X=2 * new(B, n, D) + 0.5, F=1.5 * new(B, n, D) - 0.3 if branch else None,
             post_w=1 + 0.3 * new(D) if post else None, post_b=0.2 * new(D) if post and kind == "layer" else None,
             gate=(None, 0.6 + 0.4 * new(D), 0.6 + 0.4 * new(B, D))[gate],
             pre_w=1 + 0.3 * new(D) if pre else None, pre_b=0.2 * new(D) if pre and kind == "layer" else None)
    p = {k: None if t is None else t.to(DT[dtype]) for k, t in p.items()}
    dY, dH = new(B, n, D).to(DT[dtype]), new(B, n, D).to(DT[dtype]) if pre else None
    return p, dY, dH


def sizes(p, dY, dH, kind, eps, a, b):
    """Magnitudes of the terms of every output (float64), and the product of the norms' kappa for each row."""
    q = {k: None if t is None else t.double() for k, t in p.items()}

    def unit(z, size):
        z = z - z.mean(-1, keepdim=True) if kind == "layer" else z
        r = 1 / (z.square().mean(-1, keepdim=True) + eps).sqrt()
        return (z * r).abs(), r, (size.amax(-1, keepdim=True) * r).clamp(min=1.0)

    def back(d, zn, r):
        return r * (d + zn * (d * zn).mean(-1, keepdim=True) + (d.mean(-1, keepdim=True) if kind == "layer" else 0.0))

    y, size_y, out, kappa = a * q["X"], abs(a) * q["X"].abs(), {}, torch.ones(1, 1, 1, dtype=torch.float64)
    gate = 1.0 if p["gate"] is None else q["gate"] if q["gate"].dim() == 1 else q["gate"][:, None]
    if p["F"] is not None:
        u, su = q["F"], q["F"].abs()
        if p["post_w"] is not None:
            fn, rf, kappa = unit(q["F"], q["F"].abs())
            u = ref.norm(q["F"], kind, eps, q["post_w"], q["post_b"])
            su = fn * q["post_w"].abs() + (0.0 if p["post_b"] is None else q["post_b"].abs())
        y, size_y = y + b * gate * u, size_y + abs(b) * abs(gate) * su
    out["Y"] = size_y
    d = torch.zeros_like(y) if dY is None else dY.double().abs()
    if p["pre_w"] is not None:
        yn, ry, ky = unit(y, size_y)
        kappa = kappa * ky
        out["H"] = q["pre_w"].abs() * (1 + yn) + (0.0 if p["pre_b"] is None else q["pre_b"].abs())
        if dH is not None:
            out["dpre_w"], out["dpre_b"] = dH.double().abs() * (1 + yn), dH.double().abs()
            d = d + back(dH.double().abs() * q["pre_w"].abs(), yn, ry)
    out["dX"] = abs(a) * d
    if p["F"] is not None:
        du = abs(b) * abs(gate) * d
        out["dgate"] = abs(b) * d * su
        if p["post_w"] is not None:
            out["dpost_w"], out["dpost_b"] = du * (1 + fn), du
            du = back(du * q["post_w"].abs(), fn, rf)
        out["dF"] = du
    return out, kappa


def near(got, want, bar, name):
    got = got.detach().cpu().double()
    assert got.shape == want.shape and torch.isfinite(got).all(), name
    over = (got - want).abs() > bar
    assert not over.any(), f"{name}: {over.sum()} of {over.numel()} outside, worst {((got - want).abs() / bar).max()}"


def check(dev, dtype, p, dY, dH, kind, scales=(0.9, 0.7), eps=1e-5):
    gpu = {k: None if t is None else t.to(dev) for k, t in p.items()}
    o = dict(norm=kind, eps=eps, residual_scale=scales[0], branch_scale=scales[1],
             **{KW[k]: gpu[k] for k in KW})
    got = ga.norm_residual(gpu["X"], gpu["F"], **o)
    grads = ga.norm_residual_backward(gpu["X"], gpu["F"], None if dY is None else dY.to(dev),
                                      None if dH is None else dH.to(dev), **o)
    torch.cuda.synchronize()
    # the scales as the fp32 numbers that the call receives
    a, b = (float(torch.tensor(s, dtype=torch.float32)) for s in scales)
    e = float(torch.tensor(eps, dtype=torch.float32))
    leaf = {k: None if t is None else t.double().requires_grad_() for k, t in p.items()}
    Y, H = ref.norm_residual(leaf, kind, e, a, b)
    D = p["X"].shape[-1]
    size, kappa = sizes(p, dY, dH, kind, e, a, b)
    unit = (math.log2(D) + 16) * 2.0 ** -22 * kappa

    def row_bar(name, want):
        return HALF[dtype] * want.abs() + unit * size[name].amax(-1, keepdim=True)

    for name, g, w in zip("YH", got if H is not None else (got,), (Y, H) if H is not None else (Y,)):
        near(g, w.detach(), row_bar(name, w.detach()), name)
    loss = 0.0
    if dY is not None:
        loss = loss + (Y * dY.double()).sum()
    if dH is not None:
        loss = loss + (H * dH.double()).sum()
    used = [k for k in NAMES if leaf[k] is not None and (dH is not None or k not in ("pre_w", "pre_b"))]
    want = dict(zip(("d" + k for k in used), torch.autograd.grad(loss, [leaf[k] for k in used])))
    assert set(grads) == set(want), (set(grads), set(want))
    tokens = p["X"].shape[0] * p["X"].shape[1]
    for k, w in want.items():
        if k in ("dX", "dF"):
            near(grads[k], w, row_bar(k, w), k)
        else:
            assert grads[k].dtype == torch.float32
            each = (unit + tokens * 2.0 ** -24) * size[k]
            near(grads[k], w, each.sum(1) if w.dim() == 2 else each.sum((0, 1)), k)
    return got, grads


WIDTHS = [1, 2, 7, 8, 9, 33, 64, 72, 100, 128, 250, 512, 513, 1000, 1024, 1600, 2048, 4095, 4096, 8191, 8192]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("D", WIDTHS)
def test_widths(dev, dtype, kind, D):
    print(f"\n[case] norm {dtype} {kind} D={D}", flush=True)
    p, dY, dH = make(dtype, 2, 5, D, kind)
    check(dev, dtype, p, dY, dH, kind)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("post,gate,pre", [(False, 0, True), (True, 0, False), (False, 2, False), (True, 2, True),
                                           (False, 1, True), (True, 1, False)])
def test_parts(dev, dtype, kind, post, gate, pre):
    p, dY, dH = make(dtype, 3, 17, 192, kind, post, gate, pre)
    check(dev, dtype, p, dY, dH, kind)


@pytest.mark.parametrize("B,n,D,gate", [(1, 1, 512, 1), (1, 9000, 64, 1), (700, 3, 64, 2), (5, 1000, 136, 2),
                                        (600, 1, 1024, 2), (1100, 2, 40, 1), (3, 2100, 513, 2)])
def test_row_groupings(dev, B, n, D, gate):
    """One row, many, batches split over workgroups and several batches in one."""
    print(f"\n[case] norm B={B} n={n} D={D} gate={gate}", flush=True)
    p, dY, dH = make("f32", B, n, D, "layer", gate=gate)
    check(dev, "f32", p, dY, dH, "layer")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_first_norm_and_single_gradients(dev, dtype, kind):
    p, dY, dH = make(dtype, 2, 33, 320, kind, post=False, gate=0, branch=False)
    check(dev, dtype, p, None, dH, kind)
    X, w = p["X"].to(dev), p["pre_w"].to(dev)
    both = ga.norm_residual(X, None, norm=kind, pre_weight=w)
    assert torch.equal(ga.norm_residual(X, None, norm=kind, pre_weight=w, return_sum=False), both[1])
    assert torch.equal(both[0], X)
    p, dY, dH = make(dtype, 2, 33, 320, kind)
    check(dev, dtype, p, dY, None, kind)
    check(dev, dtype, p, None, dH, kind)


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_rows_of_zeros_and_far_means(dev, kind):
    p, dY, dH = make("f32", 2, 6, 256, kind)
    p["X"][0, 0] = 0.0
    p["F"][0, 0] = 0.0
    p["X"][1, 3] = 0.0
    got, grads = check(dev, "f32", p, dY, dH, kind)
    p, dY, dH = make("f32", 2, 6, 256, kind)
    p["F"][0] += 500.0  # |mean| / spread about 330
    check(dev, "f32", p, dY, dH, kind)


def test_same_bits_captured_and_on_streams(dev):
    p, dY, dH = make("bf16", 4, 600, 512, "layer", gate=2)
    g = {k: t.to(dev) for k, t in p.items()}
    dY, dH = dY.to(dev), dH.to(dev)
    o = {KW[k]: g[k] for k in KW}

    def call():
        return (*ga.norm_residual(g["X"], g["F"], norm="layer", **o),
                *ga.norm_residual_backward(g["X"], g["F"], dY, dH, norm="layer", **o).values())

    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        again = call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(again, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = call()
    for _ in range(3):
        for t in outs:
            t.fill_(3.0)
        call()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_empty_batch(dev):
    X = torch.empty(0, 4, 64, device=dev)
    w = torch.ones(64, device=dev)
    Y, H = ga.norm_residual(X, X, post_weight=w, gate=w, pre_weight=w)
    assert Y.shape == H.shape == X.shape
    grads = ga.norm_residual_backward(X, X, X, X, post_weight=w, gate=w, pre_weight=w)
    assert all((grads[k] == 0).all() for k in ("dpost_w", "dgate", "dpre_w"))
