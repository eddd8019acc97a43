"""GPU parity of the rotary positions against their float64 definition.

Error bar: the sine and cosine of an angle reduced in fp64 carry an absolute
error below 2^-22, and the turn two fp32 products and a sum: 2^-21 (|a| + |b|)
for a pair (a, b); a bf16 result is rounded once more, by 2^-8 of its value.
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


def bar(x, want, interleaved, dtype):
    x = x.double().abs()
    s = x[..., 0::2] + x[..., 1::2] if interleaved else x[..., :32] + x[..., 32:]
    s = s.repeat_interleave(2, -1) if interleaved else torch.cat((s, s), -1)
    return 2.0 ** -21 * s + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * want.abs()


CASES = [  # B, H, Hk, n, pairs, position batches, floats, interleaved, shared
    (2, 4, 4, 100, (32,), 1, False, False, False),
    (2, 4, 2, 65, (20, 12), 2, False, False, True),
    (1, 3, 1, 63, (16, 8, 8), 1, True, True, False),
    (3, 2, 2, 1, (1, 1, 1), 3, True, True, True),
    (2, 8, 8, 257, (5, 3, 2, 7), 2, False, True, False),
    (1, 1, 1, 1, (1,), 1, False, False, False),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("B,H,Hk,n,pairs,PB,floats,interleaved,shared", CASES)
def test_turns(dev, dtype, inverse, B, H, Hk, n, pairs, PB, floats, interleaved, shared):
    print(f"\n[case] rotary {dtype} B={B} H={H} Hk={Hk} n={n} pairs={pairs}", flush=True)
    g = torch.Generator().manual_seed(n)
    Q, K = (torch.randn(B, h, n, 64, generator=g).to(DT[dtype]) for h in (H, Hk))
    if floats:
        pos = torch.rand(len(pairs), PB, n, generator=g) * 2e4 - 1e4
    else:  # far and negative positions among them
        pos = torch.randint(-2 ** 31, 2 ** 31 - 1, (len(pairs), PB, n), generator=g, dtype=torch.int32)
        pos[:, :, ::2] %= 5000
    o = dict(interleaved=interleaved, shared=shared, inverse=inverse)
    got = ga.rotary(Q.to(dev), K.to(dev), pos.to(dev), pairs, **o)
    torch.cuda.synchronize()
    for x, y in zip((Q, K), got):
        want = ref.rotary(x, pos, pairs, **o)
        # fp64 angles of positions up to 2^31 are themselves off by up to 2^31 2^-52 radians
        assert ((y.cpu().double() - want).abs() <= bar(x, want, interleaved, dtype)).all()
        r = sum(pairs)
        for lo, hi in ([(2 * r, 64)] if interleaved else [(r, 32), (32 + r, 64)]):
            assert torch.equal(y.cpu()[..., lo:hi], x[..., lo:hi])


def test_in_place_alone_and_back(dev):
    g = torch.Generator().manual_seed(1)
    Q, K = (torch.randn(2, 3, 90, 64, generator=g).to(dev) for _ in range(2))
    pos = torch.arange(180, dtype=torch.int32, device=dev).view(2, 1, 90)
    Qr, Kr = ga.rotary(Q, K, pos, (20, 10))
    assert torch.equal(ga.rotary(Q, None, pos, (20, 10)), Qr)
    q, k = Q.clone(), K.clone()
    ga.rotary(q, k, pos, (20, 10), out=(q, k))
    assert torch.equal(q, Qr) and torch.equal(k, Kr)
    back, _ = ga.rotary(Qr, Kr, pos, (20, 10), inverse=True)
    assert (back - Q).abs().max() <= 2.0 ** -19 * Q.abs().max()
    zero, _ = ga.rotary(Q, K, torch.zeros_like(pos), (20, 10))
    assert torch.equal(zero, Q)


def test_gradient_against_differences(dev):
    """<dQ', R dQ> = <R^T dQ', dQ>: the turn is linear, so a difference of two turns is the turn of the difference."""
    g = torch.Generator().manual_seed(2)
    Q, D, G = (torch.randn(2, 2, 70, 64, generator=g).to(dev) for _ in range(3))
    pos = torch.randint(0, 9000, (2, 2, 70), generator=g, dtype=torch.int32).to(dev)
    turn = lambda x, **o: ga.rotary(x, None, pos, (24, 8), **o).double()  # noqa: E731
    left = ((turn(Q + D) - turn(Q)) * G.double()).sum()
    right = (turn(G, inverse=True) * ((Q + D).double() - Q.double())).sum()
    assert (left - right).abs() <= 1e-5 * G.double().norm() * (D.double().norm() + Q.double().norm())


def test_many_heads_and_tokens(dev):
    """A launch whose workgroups each take several heads, and one that splits them."""
    for B, H, n in ((8, 8, 20000), (2, 64, 64)):
        Q = torch.randn(B, H, n, 64, device=dev).bfloat16()
        pos = torch.arange(n, dtype=torch.int32, device=dev).view(1, 1, n)
        whole, _ = ga.rotary(Q, Q, pos, (32,))
        part = ga.rotary(Q[:, 1:2, -50:].contiguous(), None, pos[:, :, -50:].contiguous(), (32,))
        assert torch.equal(whole[:, 1:2, -50:], part)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_copied_pairs_bit_for_bit(dev, dtype, interleaved):
    """Pairs behind the last axis' are copied, infinities, NaN and the sign of zeros included."""
    g = torch.Generator().manual_seed(3)
    Q = torch.randn(2, 3, 40, 64, generator=g)
    last = list(range(60, 64)) if interleaved else [30, 31, 62, 63]
    for i, x in enumerate((math.inf, -0.0, -math.inf, math.nan)):
        Q[:, :, ::2, last[i]] = x
    Q = Q.to(DT[dtype]).to(dev)
    pos = torch.arange(40, dtype=torch.int32, device=dev).view(1, 1, 40)
    got = ga.rotary(Q, None, pos, (30,), interleaved=interleaved)
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(got[..., last].contiguous().view(bits), Q[..., last].contiguous().view(bits))
    rest = [i for i in range(64) if i not in last]
    assert torch.isfinite(got[..., rest]).all()


@pytest.mark.parametrize("dtype,n", [("bf16", 200000), ("f32", 100000)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_outputs_larger_than_the_caches(dev, dtype, n, interleaved):
    """Written past the caches (205 MB of outputs), in place as well: the bits of a small call."""
    g = torch.Generator(device=dev).manual_seed(4)
    Q = torch.randn(1, 8, n, 64, device=dev, generator=g).to(DT[dtype])
    pos = torch.arange(n, dtype=torch.int32, device=dev).view(1, 1, n)
    whole = ga.rotary(Q, None, pos, (32,), interleaved=interleaved)
    for h, at in ((0, 0), (3, n // 2), (7, n - 50)):
        part = ga.rotary(Q[:, h:h + 1, at:at + 50].contiguous(), None, pos[:, :, at:at + 50].contiguous(), (32,),
                         interleaved=interleaved)
        assert torch.equal(whole[:, h:h + 1, at:at + 50], part)
    ga.rotary(Q, None, pos, (32,), interleaved=interleaved, out=(Q, None))
    assert torch.equal(Q, whole)
