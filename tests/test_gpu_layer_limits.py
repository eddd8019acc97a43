"""The layer's operators at their limits: tensors of more than 2^31 values, two calls at once, inputs of one launch
that are outputs of another, infinities where nothing may be read, lists at four-byte alignment."""
import math

import pytest
import torch

import layer_reference as ref
from paper_2306_01926_amd import ga

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    ga.lib()
    yield torch.device("cuda:0")
    torch.cuda.empty_cache()


def say(msg):
    print(f"\n[case] {msg}", flush=True)


def rel(a, b):
    return ((a.detach().cpu().double() - b).norm() / b.norm()).item()


FAR = 4_200_000  # tokens of eight heads of 64, or rows of 512: 2^31 values and more


def test_linear_far(dev):
    """The last head's ends, which decay separates from the rest of the sequence (e^-50 after 1000 tokens)."""
    say("linear far")
    g = torch.Generator(device=dev).manual_seed(3)
    Q, K, V, dO = (torch.randn(1, 8, FAR, 64, device=dev, generator=g, dtype=torch.bfloat16) for _ in range(4))
    log_decay = torch.full((8,), -0.05, device=dev)
    O, S = ga.linear_attend(Q, K, V, log_decay, return_state=True)
    dQ, dK, dV, dS = ga.linear_backward(Q, K, V, dO, log_decay, return_dstate=True)
    tail, head = slice(FAR - 1000, FAR), slice(0, 1000)
    cut = lambda x, s: x[:, 7:, s].cpu()  # noqa: E731
    Or, Sr, _ = ref.linear(cut(Q, tail), cut(K, tail), cut(V, tail), log_decay[7:].cpu(), 0.125)
    assert rel(cut(O, tail)[:, :, -100:], Or[:, :, -100:]) <= 5e-3
    assert rel(S[:, 7:], Sr) <= 1e-5
    at = [ref.linear_grad(*(cut(x, s) for x in (Q, K, V, dO)), log_decay[7:].cpu(), 0.125) for s in (head, tail)]
    assert rel(cut(dQ, tail)[:, :, -100:], at[1]["dQ"][:, :, -100:]) <= 5e-3
    for x, name in ((dK, "dK"), (dV, "dV")):
        assert rel(cut(x, head)[:, :, :100], at[0][name][:, :, :100]) <= 5e-3
        assert rel(cut(x, tail)[:, :, -100:], at[1][name][:, :, -100:]) <= 5e-3
    assert rel(dS[:, 7:], at[0]["dS"]) <= 1e-5


def test_step_far(dev):
    say("step far")
    many, H = 70_000, 8
    pool = torch.zeros(many, H, 64, 64, device=dev)
    g = torch.Generator(device=dev).manual_seed(4)
    Q, K, V = (torch.randn(2, H, 1, 64, device=dev, generator=g) for _ in range(3))
    pool[-1].normal_(generator=g)
    before = pool[-1].cpu()
    log_decay = torch.full((H,), -0.1)
    slots = torch.tensor([many - 1, 5], dtype=torch.int32, device=dev)
    O, _ = ga.linear_step(Q, K, V, log_decay.to(dev), pool, slots=slots)
    state = torch.stack((before, torch.zeros_like(before)))
    Or, Sr, _ = ref.linear(Q.cpu(), K.cpu(), V.cpu(), log_decay, 0.125, None, state)
    assert rel(O, Or) <= 1e-5 and rel(pool[-1], Sr[0]) <= 1e-5 and rel(pool[5], Sr[1]) <= 1e-5


def test_rotary_and_norm_far(dev):
    say("rotary far")
    g = torch.Generator(device=dev).manual_seed(5)
    Q = torch.randn(1, 8, FAR, 64, device=dev, generator=g, dtype=torch.bfloat16)
    pos = torch.arange(FAR, dtype=torch.int32, device=dev).view(1, 1, FAR)
    want = ref.rotary(Q[:, 7:, -50:].cpu(), pos[:, :, -50:].cpu(), (32,))
    ga.rotary(Q, None, pos, (32,), out=(Q, None))
    # fp32 products (2^-21 of the pair) and one rounding to bf16, as a 2-norm: below 2^-8
    assert rel(Q[:, 7:, -50:], want) <= 2.0 ** -8
    say("norm far")
    X = Q.view(1, FAR, 512)
    F = torch.randn(1, FAR, 512, device=dev, generator=g, dtype=torch.bfloat16)
    w = 1 + 0.2 * torch.randn(512, device=dev, generator=g)
    w = w.bfloat16()
    o = dict(norm="layer", post_weight=w, gate=w, pre_weight=w)
    Y, H = ga.norm_residual(X, F, **o)
    p = dict(X=X[:, -60:].cpu().double(), F=F[:, -60:].cpu().double(), post_w=w.cpu().double(), post_b=None,
             gate=w.cpu().double(), pre_w=w.cpu().double(), pre_b=None)
    leaf = {k: p[k].clone().requires_grad_() for k in ("X", "F")}
    Yr, Hr = ref.norm_residual({**p, **leaf}, "layer", 1e-6, 1.0, 1.0)
    assert rel(Y[:, -60:], Yr.detach()) <= 2.0 ** -8 and rel(H[:, -60:], Hr.detach()) <= 2.0 ** -8
    got = ga.norm_residual_backward(X, F, Y, H, **o)
    loss = (Yr * Y[:, -60:].cpu().double()).sum() + (Hr * H[:, -60:].cpu().double()).sum()
    for k, grad in zip(("dX", "dF"), torch.autograd.grad(loss, [leaf["X"], leaf["F"]])):
        assert rel(got[k][:, -60:], grad) <= 2.0 ** -8


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_two_calls_at_once(dev, dtype):
    """Calls with workspaces on two streams, their launches in turn: each gives what it gives alone."""
    say(f"two at once {dtype}")
    g = torch.Generator(device=dev).manual_seed(6)

    def inputs(n, Hk):
        t = [torch.randn(2, h, n, 64, device=dev, generator=g).to(dtype) for h in (4, Hk, Hk, 4)]
        X, F = (torch.randn(2, n, 256, device=dev, generator=g).to(dtype) for _ in range(2))
        return t, X, F

    log_decay = -0.01 * torch.arange(1, 5, device=dev)
    w = torch.ones(256, device=dev, dtype=dtype)

    def call(a):
        (Q, K, V, dO), X, F = a
        d = ga.norm_residual_backward(X, F, F, X, post_weight=w, gate=w, pre_weight=w)
        return [*ga.linear_attend(Q, K, V, log_decay, return_state=True),
                *ga.linear_backward(Q, K, V, dO, log_decay, return_dstate=True), *(d[k] for k in sorted(d))]

    cases = [inputs(3000, 2), inputs(2500, 4)]
    alone = [call(a) for a in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(3):
        got = [[], []]
        for _ in range(2):
            for i, s in enumerate(streams):
                with torch.cuda.stream(s):
                    got[i].append(call(cases[i]))
        torch.cuda.synchronize()
        for i in range(2):
            for outs in got[i]:
                assert all(torch.equal(a, b) for a, b in zip(outs, alone[i]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_infinities_behind_the_end(dev, dtype):
    """Infinities behind a sequence's end, in the buffers that outputs are written to as well, reach nothing."""
    say(f"infinities {dtype}")
    B, H, n = 3, 2, 500
    lengths = torch.tensor([500, 0, 131], dtype=torch.int32)
    g = torch.Generator().manual_seed(7)
    x = [torch.randn(B, H, n, 64, generator=g).to(dtype) for _ in range(4)]
    log_decay = torch.tensor([-0.02, -math.inf])
    live = ref.length_mask(lengths, B, n)[:, None, :, None]
    bad = [torch.where(live, t, float("inf")).to(dev) for t in x]
    out = torch.full_like(bad[0], float("inf"))
    O, S = ga.linear_attend(*bad[:3], log_decay.to(dev), lengths=lengths.to(dev), return_state=True, out=out)
    grads = ga.linear_backward(*bad, log_decay.to(dev), lengths=lengths.to(dev))
    Or, Sr, _ = ref.linear(*x[:3], log_decay, 0.125, lengths)
    want = ref.linear_grad(*x, log_decay, 0.125, lengths)
    bar = 5e-3 if dtype == torch.bfloat16 else 1e-5
    assert rel(O, Or) <= bar and rel(S, Sr) <= 1e-5
    for t, k in zip(grads, ("dQ", "dK", "dV")):
        assert rel(t, want[k]) <= bar, k
        assert (t.cpu()[~live.expand_as(t)] == 0).all()


def test_lists_at_four_bytes(dev):
    """log_decay, lengths, slots and positions at any four-byte address."""
    say("lists at four bytes")
    g = torch.Generator(device=dev).manual_seed(8)
    Q = torch.randn(3, 2, 70, 64, device=dev, generator=g)
    odd = lambda t: torch.cat((t[:1], t)).contiguous()[1:]  # noqa: E731
    decay = torch.tensor([-0.1, -0.2], device=dev)
    lengths = torch.tensor([70, 3, 20], dtype=torch.int32, device=dev)
    assert odd(lengths).data_ptr() % 16 == 4
    assert torch.equal(ga.linear_attend(Q, Q, Q, decay, lengths=lengths),
                       ga.linear_attend(Q, Q, Q, odd(decay), lengths=odd(lengths)))
    pos = torch.arange(70, dtype=torch.int32, device=dev)
    assert torch.equal(ga.rotary(Q, None, pos.view(1, 1, 70), (32,)),
                       ga.rotary(Q, None, odd(pos).view(1, 1, 70), (32,)))
    one, pool = Q[:, :, :1].contiguous(), torch.ones(5, 2, 64, 64, device=dev)
    slots = torch.tensor([4, 0, 2], dtype=torch.int32, device=dev)
    a = ga.linear_step(one, one, one, decay, pool, slots=slots, out_state=torch.empty_like(pool))[0]
    assert torch.equal(a, ga.linear_step(one, one, one, odd(decay), pool, slots=odd(slots),
                                         out_state=torch.empty_like(pool))[0])
