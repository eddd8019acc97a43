"""GPU parity of the linear attention with decays against its float64 definition.

Error bars, with u = 2^-8 (bf16) or 2^-24 (fp32) the largest relative error of
one rounding and A the sum of the magnitudes of all terms of an output:
  * bf16: a term passes one rounding to bf16 on its way (its product q . k, or
    the state it was summed into), and the output one: u A + u |o|, plus fp32
    sums (below).  2-norm over the whole tensor: 5e-3, the header's figure
    (three independent roundings of 2^-8 / sqrt 3 each are 3.9e-3).
  * fp32 and every state: sums of at most n + 64 products, (n + 64) 2^-24 A;
    each decay is 2^(g x) with g x off by two roundings and g x > -32 wherever
    its term is not below 2^-32 A: 32 * 2 * 2^-24 A; a state handed back by a
    bf16 call is formed from decayed keys kept in three bf16 parts: 2^-24 A.
    2-norm: 1e-5.
"""
import math

import pytest
import torch

import layer_reference as ref
from paper_2306_01926_amd import ga

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    ga.lib()
    return torch.device("cuda:0")


def say(msg):
    print(f"\n[case] {msg}", flush=True)


def decays(H, kind="mixed"):
    if kind == "none":
        return torch.zeros(H)
    if kind == "all":  # l = 0: a token sees itself alone
        return torch.full((H,), -math.inf)
    life = 4.0 * 512.0 ** (torch.arange(H) / max(1, H - 1))
    return -math.log(2.0) / life


def case(dev, dtype, B, H, Hk, n, lengths=None, state=False, decay="mixed", seed=0):
    g = torch.Generator().manual_seed(seed + 7919 * n + 31 * H)
    new = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    c = dict(Q=new(B, H, n, 64).to(DT[dtype]), K=new(B, Hk, n, 64).to(DT[dtype]), V=new(B, Hk, n, 64).to(DT[dtype]),
             dO=new(B, H, n, 64).to(DT[dtype]), log_decay=decays(H, decay).float(),
             lengths=None if lengths is None else torch.tensor(lengths, dtype=torch.int32),
             state=new(B, H, 64, 64) * 3 if state else None, dstate=new(B, H, 64, 64) * 0.2 if state else None)
    return c, {k: None if t is None else t.to(dev) for k, t in c.items()}


def close(got, want, A, n, dtype, name, state=False):
    got, want = got.detach().cpu().double(), want
    assert torch.isfinite(got).all(), f"{name}: not finite"
    bar = (n + 64 + 64) * 2.0 ** -24 * A
    if dtype == "bf16":
        bar = bar + (2.0 ** -24 * A if state else 2.0 ** -8 * (A + want.abs()))
    elif not state:
        bar = bar + 2.0 ** -24 * want.abs()
    worst = ((got - want).abs() - bar).max().item()
    assert worst <= 0, f"{name}: {((got - want).abs() > bar).sum()} values outside their bar (by {worst:.3g})"
    norm = want.norm().item()
    rel = (got - want).norm().item() / norm if norm else 0.0
    assert rel <= (5e-3 if dtype == "bf16" and not state else 1e-5), f"{name}: 2-norm error {rel:.3g}"


def check_forward(c, g, dtype, scale=None):
    n = c["Q"].shape[2]
    s = 0.125 if scale is None else scale
    O, S = ga.linear_attend(g["Q"], g["K"], g["V"], g["log_decay"], scale=scale, lengths=g["lengths"], state=g["state"],
                            return_state=True)
    torch.cuda.synchronize()
    Or, Sr, A = ref.linear(c["Q"], c["K"], c["V"], c["log_decay"], s, c["lengths"], c["state"])
    As = ref.linear(c["Q"], c["K"].abs(), c["V"].abs(), c["log_decay"], s, c["lengths"],
                    None if c["state"] is None else c["state"].abs())[1]
    close(O, Or, A, n, dtype, "O")
    close(S, Sr, As, n, dtype, "state", state=True)
    return O, S


def check_backward(c, g, dtype, scale=None):
    n = c["Q"].shape[2]
    got = ga.linear_backward(g["Q"], g["K"], g["V"], g["dO"], g["log_decay"], scale=scale, lengths=g["lengths"],
                             state=g["state"], dstate=g["dstate"], return_dstate=True)
    torch.cuda.synchronize()
    want = ref.linear_grad(c["Q"], c["K"], c["V"], c["dO"], c["log_decay"], 0.125 if scale is None else scale,
                           c["lengths"], c["state"], c["dstate"])
    for x, t in zip(("dQ", "dK", "dV", "dS"), got):
        close(t, want[x], want["a" + x], n, dtype, x, state=x == "dS")
    return got


LENGTHS = [1, 2, 15, 16, 31, 33, 63, 64, 65, 127, 128, 129, 200, 511]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", LENGTHS)
def test_forward_and_backward_over_lengths(dev, dtype, n):
    say(f"linear {dtype} n={n}")
    c, g = case(dev, dtype, 2, 3, 3, n, state=n % 2 == 1)
    check_forward(c, g, dtype)
    check_backward(c, g, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk", [(4, 4), (4, 2), (6, 1), (1, 1)])
def test_shared_heads(dev, dtype, H, Hk):
    say(f"linear {dtype} H={H} Hk={Hk}")
    c, g = case(dev, dtype, 3, H, Hk, 150, state=True)
    check_forward(c, g, dtype)
    check_backward(c, g, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,lengths", [(130, [0, 1, 130, 64]), (200, [65, 0, 199, 63]), (64, [0, 0, 0, 0]),
                                       (300, [-5, 1000, 128, 192])])
def test_padded_batches(dev, dtype, n, lengths):
    """Rows behind a sequence's end hold NaN: they are not read, and outputs there are zero."""
    say(f"linear {dtype} n={n} lengths={lengths}")
    c, g = case(dev, dtype, 4, 2, 1, n, lengths=lengths, state=True)
    live = ref.length_mask(c["lengths"], 4, n)[:, None, :, None].to(dev)
    for x in ("Q", "K", "V", "dO"):
        g[x] = torch.where(live, g[x], float("nan")).contiguous()
    O, _ = check_forward(c, g, dtype)
    grads = check_backward(c, g, dtype)
    for t in (O, *grads[:3]):
        assert (t.float()[~live.expand_as(t)] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("decay", ["none", "all"])
def test_decays_of_one_and_zero(dev, dtype, decay):
    say(f"linear {dtype} decay {decay}")
    c, g = case(dev, dtype, 2, 2, 2, 210, state=True, decay=decay, lengths=[210, 100])
    check_forward(c, g, dtype)
    check_backward(c, g, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,n,lengths", [(1, 2, 3001, None), (1, 1, 5000, [4987]), (40, 8, 130, None),
                                           (3, 5, 1500, [1500, 700, 1])])
def test_long_and_many(dev, dtype, B, H, n, lengths):
    """Sequences split over workgroups, and more slices than compute units."""
    say(f"linear {dtype} B={B} H={H} n={n}")
    c, g = case(dev, dtype, B, H, 1 if H == 8 else H, n, lengths=lengths, state=B < 40)
    check_forward(c, g, dtype)
    check_backward(c, g, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scale_and_missing_pieces(dev, dtype):
    say(f"linear {dtype} scale, no states")
    c, g = case(dev, dtype, 2, 2, 2, 100)
    check_forward(c, g, dtype, scale=-0.75)
    check_backward(c, g, dtype, scale=-0.75)
    only = ga.linear_attend(g["Q"], g["K"], g["V"], g["log_decay"])
    three = ga.linear_backward(g["Q"], g["K"], g["V"], g["dO"], g["log_decay"])
    assert isinstance(only, torch.Tensor) and len(three) == 3
    if dtype == "f32":
        assert torch.equal(only, ga.linear_attend(g["Q"], g["K"], g["V"], g["log_decay"], return_state=True)[0])
        four = ga.linear_backward(g["Q"], g["K"], g["V"], g["dO"], g["log_decay"], return_dstate=True)
        assert all(torch.equal(a, b) for a, b in zip(three, four))
    else:  # a state handed back is formed from three bf16 parts of the keys, and two otherwise: both within the bars
        Or, _, A = ref.linear(c["Q"], c["K"], c["V"], c["log_decay"], 0.125)
        close(only, Or, A, 100, dtype, "O")
        want = ref.linear_grad(c["Q"], c["K"], c["V"], c["dO"], c["log_decay"], 0.125)
        for x, y in zip(("dQ", "dK", "dV"), three):
            close(y, want[x], want["a" + x], 100, dtype, x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,n,ends", [(1, 2, 60000, True), (16, 8, 12000, False)])
def test_long_memory(dev, dtype, B, H, n, ends):
    """Decays so near one that whatever a chunk's factor is off by adds up over all chunks: the header's 1e-5 for every
    state, in sequences of many segments and in ones of a single walk."""
    say(f"linear {dtype} long memory B={B} H={H} n={n}")
    g = torch.Generator(device=dev).manual_seed(n)
    Q, K, V, dO = (torch.randn(B, H, n, 64, device=dev, generator=g).to(DT[dtype]) for _ in range(4))
    log_decay = -(10.0 ** torch.linspace(-7, -4, H, device=dev))
    lengths = torch.full((B,), n - 7 if ends else n, dtype=torch.int32, device=dev)
    _, S = ga.linear_attend(Q, K, V, log_decay, lengths=lengths, return_state=True)
    dS = ga.linear_backward(Q, K, V, dO, log_decay, lengths=lengths, return_dstate=True)[3]
    m = int(lengths[-1])
    t = torch.arange(m, device=dev).double()
    for h in range(H):
        l = log_decay[h].double()
        k, v, q, o = (x[-1, h, :m].cpu().double() for x in (K, V, Q, dO))
        until, since = ((l * x).exp().cpu()[:, None] for x in (m - 1 - t, t + 1))
        for got, want in ((S, (k * until).t() @ v), (dS, 0.125 * (q * since).t() @ o)):
            rel = (got[-1, h].cpu().double() - want).norm() / want.norm()
            assert rel <= 1e-5, (float(l), float(rel))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,n", [(1, 1, 5000), (4, 8, 2000), (2, 2, 333), (32, 8, 70)])
def test_states_in_place(dev, dtype, B, H, n):
    """A state given and handed back in one buffer, split over many segments, a few and none: the same values."""
    say(f"linear {dtype} states in place B={B} H={H} n={n}")
    c, g = case(dev, dtype, B, H, H, n, state=True, lengths=[n] * (B - 1) + [n - 3])
    O, S = ga.linear_attend(g["Q"], g["K"], g["V"], g["log_decay"], lengths=g["lengths"], state=g["state"],
                            return_state=True)
    kept = g["state"].clone()
    O2 = ga.linear_attend(g["Q"], g["K"], g["V"], g["log_decay"], lengths=g["lengths"], state=kept, out_state=kept)
    bar = 5e-3 if dtype == "bf16" else 1e-5
    assert ((kept - S).norm() / S.norm()).item() <= 2e-5
    assert ((O2.double() - O.double()).norm() / O.double().norm()).item() <= 2 * bar
    want = ga.linear_backward(g["Q"], g["K"], g["V"], g["dO"], g["log_decay"], lengths=g["lengths"], state=g["state"],
                              dstate=g["dstate"], return_dstate=True)
    got = [torch.empty_like(g[x]) for x in "QKV"] + [g["dstate"].clone()]
    s = ga.Shape(B, H, n, 64, ga._dtype_code(g["Q"]))
    ws = torch.empty(ga.linear_backward_workspace_bytes(s, H), dtype=torch.uint8, device=dev)
    p = lambda x: x.data_ptr()  # noqa: E731
    ga._check(ga.lib().ga_linear_backward(
        s, H, p(g["Q"]), p(g["K"]), p(g["V"]), p(g["dO"]), p(g["log_decay"]), p(g["lengths"]), p(g["state"]),
        p(got[3]), 0.125, *(p(x) for x in got), p(ws), ws.numel(), torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(got, want)):
        assert ((a.double() - b.double()).norm() / b.double().norm()).item() <= (2e-5 if i == 3 else 2 * bar), i


def test_gradient_against_differences(dev):
    """The outputs are linear in each of Q, K, V and the state: a difference of two forward passes is the gradient's
    product with the step, up to the fp32 sums' rounding (1e-5 of the terms' norms)."""
    c, g = case(dev, "f32", 2, 4, 2, 190, state=True, lengths=[190, 77])
    g["lengths"] = c["lengths"].to(dev)
    gen = torch.Generator().manual_seed(5)

    def loss(**over):
        a = {**g, **over}
        O, S = ga.linear_attend(a["Q"], a["K"], a["V"], a["log_decay"], lengths=a["lengths"], state=a["state"],
                                return_state=True)
        live = ref.length_mask(c["lengths"], 2, 190)[:, None, :, None].to(dev)
        return (O.double() * g["dO"].double() * live).sum() + (S.double() * g["dstate"].double()).sum()

    grads = ga.linear_backward(g["Q"], g["K"], g["V"], g["dO"], g["log_decay"], lengths=g["lengths"], state=g["state"],
                               dstate=g["dstate"], return_dstate=True)
    base = loss()
    for name, grad in zip(("Q", "K", "V", "state"), grads):
        step = torch.randn(g[name].shape, generator=gen).to(dev)
        moved = loss(**{name: (g[name] + step)})
        # the step as it was taken, after the sum's rounding
        want = (grad.double() * ((g[name] + step).double() - g[name].double())).sum()
        room = 1e-5 * (grad.double().norm() * step.double().norm() + base.abs() + moved.abs())
        assert (moved - base - want).abs() <= room, (name, (moved - base).item(), want.item())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_bits_on_every_run_and_stream(dev, dtype):
    c, g = case(dev, dtype, 2, 4, 2, 1300, state=True, lengths=[1300, 900])
    call = lambda: (*ga.linear_attend(g["Q"], g["K"], g["V"], g["log_decay"], lengths=g["lengths"], state=g["state"],  # noqa: E731
                                      return_state=True),
                    *ga.linear_backward(g["Q"], g["K"], g["V"], g["dO"], g["log_decay"], lengths=g["lengths"],
                                        state=g["state"], dstate=g["dstate"], return_dstate=True))
    first = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        second = call()
    third = call()
    torch.cuda.synchronize()
    for a, b, d in zip(first, second, third):
        assert torch.equal(a, b) and torch.equal(a, d)


def test_continued_in_place(dev):
    """A prompt in two parts with the state kept in one buffer."""
    c, g = case(dev, "f32", 2, 2, 2, 333, state=True)
    whole, S = ga.linear_attend(g["Q"], g["K"], g["V"], g["log_decay"], state=g["state"], return_state=True)
    kept, parts = g["state"].clone(), []
    for a, b in ((0, 130), (130, 333)):
        q, k, v = (g[x][:, :, a:b].contiguous() for x in "QKV")
        parts.append(ga.linear_attend(q, k, v, g["log_decay"], state=kept, out_state=kept))
    got = torch.cat(parts, 2)
    assert ((got - whole).norm() / whole.norm()).item() <= 1e-5
    assert ((kept - S).norm() / S.norm()).item() <= 1e-5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hk", [(1, 1, 1), (3, 4, 2), (70, 8, 8)])
def test_steps_follow_the_sequence(dev, dtype, B, H, Hk):
    say(f"linear_step {dtype} B={B} H={H} Hk={Hk}")
    n = 5
    c, g = case(dev, dtype, B, H, Hk, n, state=True)
    S = g["state"].clone()
    outs = []
    for t in range(n):
        q, k, v = (g[x][:, :, t:t + 1].contiguous() for x in "QKV")
        O, S2 = ga.linear_step(q, k, v, g["log_decay"], S)
        assert S2 is S
        outs.append(O)
    Or, Sr, A = ref.linear(c["Q"], c["K"], c["V"], c["log_decay"], 0.125, None, c["state"])
    As = ref.linear(c["Q"], c["K"].abs(), c["V"].abs(), c["log_decay"], 0.125, None, c["state"].abs())[1]
    close(torch.cat(outs, 2), Or, A, n, dtype, "O")
    close(S, Sr, As, n, "f32", "state", state=True)


def test_step_slots(dev):
    """Rows pick their states; padding rows and the later of two rows with one slot leave every state alone."""
    B, H = 6, 2
    c, g = case(dev, "f32", B, H, H, 1)
    pool = torch.randn(9, H, 64, 64, device=dev)
    before = pool.clone()
    slots = torch.tensor([7, -1, 2, 9, 7, 0], dtype=torch.int32, device=dev)
    O, _ = ga.linear_step(g["Q"], g["K"], g["V"], g["log_decay"], pool, slots=slots)
    rows = {0: 7, 2: 2, 5: 0}
    for b in range(B):
        if b not in rows:
            assert (O[b] == 0).all()
            continue
        Or, Sr, A = ref.linear(c["Q"][b:b + 1], c["K"][b:b + 1], c["V"][b:b + 1], c["log_decay"], 0.125, None,
                               before[rows[b]][None].cpu())
        close(O[b:b + 1], Or, A, 1, "f32", "O")
        assert ((pool[rows[b]].cpu().double() - Sr[0]).abs().max() <= 1e-5)
    for s in set(range(9)) - set(rows.values()):
        assert torch.equal(pool[s], before[s])
    away = torch.full_like(pool, 5.0)
    ga.linear_step(g["Q"], g["K"], g["V"], g["log_decay"], before, slots=slots, out_state=away)
    assert torch.equal(away[7], pool[7]) and (away[1] == 5.0).all()


def test_captured_and_replayed(dev):
    """Forward, backward and a step in one graph, replayed with eager work between."""
    c, g = case(dev, "bf16", 2, 4, 2, 700, state=True)
    q1, k1, v1 = (g[x][:, :, :1].contiguous() for x in "QKV")
    kept = g["state"].clone()

    def call():
        O, S = ga.linear_attend(g["Q"], g["K"], g["V"], g["log_decay"], state=g["state"], return_state=True)
        grads = ga.linear_backward(g["Q"], g["K"], g["V"], g["dO"], g["log_decay"], state=g["state"],
                                   dstate=g["dstate"], return_dstate=True)
        return (O, S, *grads, *ga.linear_step(q1, k1, v1, g["log_decay"], kept, out_state=torch.empty_like(kept)))

    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = call()
    for _ in range(3):
        for t in outs:
            t.fill_(1.0)
        call()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
