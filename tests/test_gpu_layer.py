"""The operators together, as a layer uses them: norm, projections, rotary positions, linear attention, output
projection, norms around the residual; for a whole sequence and one token at a time.  2e-2 of the float64 layer's
2-norm: some ten bf16 roundings of 2^-8 on the way, each relative to its stage's values."""
import math

import pytest
import torch

import layer_reference as ref
from paper_2306_01926_amd import ga, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    ga.lib()
    return torch.device("cuda:0")


PAIRS = (24, 8)


def weights(H, seed):
    D = 64 * H
    g = torch.Generator().manual_seed(seed)
    _, Wqkv, Wo = inputs.block_inputs(1, 1, H, seed=seed)
    w = {k: (1 + 0.2 * torch.randn(D, generator=g)).bfloat16() for k in ("first", "post", "pre")}
    gate = (0.5 + 0.2 * torch.randn(D, generator=g)).bfloat16()
    return Wqkv, Wo, w, gate, -math.log(2.0) / (8.0 * 32.0 ** (torch.arange(H) / max(1, H - 1)))


def layer(X, pos, p, H, state=None, step=False):
    Wqkv, Wo, w, gate, g = p
    h = ga.norm_residual(X, None, pre_weight=w["first"], return_sum=False)
    Q, K, V = ga.project_qkv(h, Wqkv, H)
    Q, K = ga.rotary(Q, K, pos, PAIRS)
    if step:
        O, state = ga.linear_step(Q, K, V, g, state)
    else:
        O, state = ga.linear_attend(Q, K, V, g, state=state, return_state=True)
    Y, Hn = ga.norm_residual(X, ga.project_out(O, Wo), post_weight=w["post"], gate=gate, pre_weight=w["pre"])
    return Y, Hn, state


def layer_f64(X, pos, p, H):
    Wqkv, Wo, w, gate, g = (ref.f64(x) if isinstance(x, torch.Tensor) else {k: ref.f64(v) for k, v in x.items()}
                            for x in p)
    X = ref.f64(X)
    B, n, D = X.shape
    h = ref.norm(X, "rms", 1e-6, w["first"], None)
    Q, K, V = (h @ Wqkv.T).view(B, n, 3, H, 64).permute(2, 0, 3, 1, 4)
    Q, K = (ref.rotary(x, pos, PAIRS) for x in (Q, K))
    O, S, _ = ref.linear(Q, K, V, g, 0.125)
    F = O.permute(0, 2, 1, 3).reshape(B, n, D) @ Wo.T
    return (*ref.norm_residual(dict(X=X, F=F, post_w=w["post"], post_b=None, gate=gate, pre_w=w["pre"], pre_b=None),
                               "rms", 1e-6, 1.0, 1.0), S)


def rel(a, b):
    return ((a.detach().cpu().double() - b).norm() / b.norm()).item()


@pytest.mark.parametrize("B,n,H", [(2, 150, 4), (1, 1, 2), (3, 700, 8)])
def test_layer(dev, B, n, H):
    X, _, _ = inputs.block_inputs(B, n, H, seed=4)
    p = weights(H, 5)
    pos = torch.stack((torch.arange(n), torch.arange(n) % 13)).int().view(2, 1, n)
    gpu = [x.to(dev) if isinstance(x, torch.Tensor) else {k: v.to(dev) for k, v in x.items()} for x in p]
    got = layer(X.to(dev), pos.to(dev), gpu, H)
    torch.cuda.synchronize()
    for name, a, b in zip(("Y", "H", "state"), got, layer_f64(X, pos, p, H)):
        assert rel(a, b) <= 2e-2, (name, rel(a, b))


def test_prompt_then_tokens(dev):
    B, n, H, more = 2, 90, 4, 6
    X, _, _ = inputs.block_inputs(B, n + more, H, seed=8)
    p = weights(H, 9)
    pos = torch.stack((torch.arange(n + more), torch.arange(n + more) % 7)).int().view(2, 1, n + more)
    gpu = [x.to(dev) if isinstance(x, torch.Tensor) else {k: v.to(dev) for k, v in x.items()} for x in p]
    Xg, pg = X.to(dev), pos.to(dev)
    want = layer_f64(X, pos, p, H)[0]
    _, _, state = layer(Xg[:, :n].contiguous(), pg[:, :, :n].contiguous(), gpu, H)
    for t in range(n, n + more):
        Y, _, state = layer(Xg[:, t:t + 1].contiguous(), pg[:, :, t:t + 1].contiguous(), gpu, H, state, step=True)
        assert rel(Y[:, 0], want[:, t]) <= 2e-2, t
