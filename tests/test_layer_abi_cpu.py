"""Host-side checks of the linear attention's, the rotary positions' and the norms' entry points (no GPU needed): each
error status is forced with fake, never dereferenced device pointers."""
import ctypes

import pytest
import torch

from paper_2306_01926_amd import ga

FAKE = 0x10000000
NAN, INF = float("nan"), float("inf")


def P(x=FAKE):
    return ctypes.c_void_p(x) if x else None


def shape(B=2, H=4, n=100, d=64, dtype=ga.GA_BF16):
    return ga.Shape(B, H, n, d, dtype)


def attend(s=None, Hk=2, Q=FAKE, K=FAKE, V=FAKE, g=FAKE, lengths=0, state=0, scale=0.125, O=FAKE, out=0, ws=FAKE,
           nb=None):
    s = s or shape()
    nb = ga.lib().ga_linear_workspace_bytes(s, Hk) if nb is None else nb
    return ga.lib().ga_linear_attend(s, Hk, P(Q), P(K), P(V), P(g), P(lengths), P(state), scale, P(O), P(out), P(ws),
                                     nb, None)


def backward(s=None, Hk=2, Q=FAKE, K=FAKE, V=FAKE, dO=FAKE, g=FAKE, lengths=0, state=0, dstate=0, scale=0.125,
             dQ=FAKE, dK=FAKE, dV=FAKE, out=0, ws=FAKE, nb=None):
    s = s or shape()
    nb = ga.lib().ga_linear_backward_workspace_bytes(s, Hk) if nb is None else nb
    return ga.lib().ga_linear_backward(s, Hk, P(Q), P(K), P(V), P(dO), P(g), P(lengths), P(state), P(dstate), scale,
                                       P(dQ), P(dK), P(dV), P(out), P(ws), nb, None)


def step(s=None, Hk=2, Q=FAKE, K=FAKE, V=FAKE, g=FAKE, slots=0, states=2, state=FAKE, scale=0.125, O=FAKE, out=FAKE):
    return ga.lib().ga_linear_step(s or shape(n=1), Hk, P(Q), P(K), P(V), P(g), P(slots), states, P(state), scale,
                                   P(O), P(out), None)


def rotary(s=None, Hk=2, Q=FAKE, K=FAKE, pos=FAKE, PB=1, pairs=(20, 12), axes=None, base=10000.0, flags=0, Qo=FAKE,
           Ko=FAKE):
    arr = (ctypes.c_int32 * max(1, len(pairs)))(*pairs) if pairs is not None else None
    return ga.lib().ga_rotary(s or shape(), Hk, P(Q), P(K), P(pos), PB, len(pairs) if axes is None else axes, arr,
                              base, flags, P(Qo), P(Ko), None)


def norm_shape(B=2, n=10, D=128, dtype=ga.GA_BF16, kind=0, gate=1, eps=1e-5, a=1.0, b=1.0):
    return ga.Norm(B, n, D, dtype, kind, gate, eps, a, b)


def norm(s=None, X=FAKE, F=FAKE, pw=FAKE, pb=0, gate=FAKE, qw=FAKE, qb=0, Y=FAKE, H=FAKE):
    return ga.lib().ga_norm_residual(s or norm_shape(), P(X), P(F), P(pw), P(pb), P(gate), P(qw), P(qb), P(Y), P(H),
                                     None)


def norm_back(s=None, X=FAKE, F=FAKE, pw=FAKE, pb=0, gate=FAKE, qw=FAKE, qb=0, dY=FAKE, dH=FAKE, dX=FAKE, dF=FAKE,
              dpw=0, dpb=0, dg=0, dqw=0, dqb=0, ws=FAKE, nb=None):
    s = s or norm_shape()
    nb = ga.lib().ga_norm_backward_workspace_bytes(s) if nb is None else nb
    return ga.lib().ga_norm_residual_backward(s, P(X), P(F), P(pw), P(pb), P(gate), P(qw), P(qb), P(dY), P(dH), P(dX),
                                              P(dF), P(dpw), P(dpb), P(dg), P(dqw), P(dqb), P(ws), nb, None)


HEADS = [(dict(s=shape(dtype=5)), 1), (dict(s=shape(B=-1)), 1), (dict(s=shape(n=0)), 1), (dict(s=shape(d=128)), 2),
         (dict(Hk=3), 1), (dict(Hk=0), 1), (dict(s=shape(B=70000, H=1), Hk=1), 2), (dict(Q=0), 1), (dict(K=FAKE + 8), 1)]
LINEAR = [(dict(scale=NAN), 1), (dict(g=0), 1), (dict(g=FAKE + 2), 1), (dict(lengths=FAKE + 1), 1),
          (dict(state=FAKE + 4), 1), (dict(V=0), 1)]
CASES = (
    [(attend, *c) for c in HEADS + LINEAR] + [(attend, dict(O=0), 1), (attend, dict(out=FAKE + 8), 1)]
    + [(backward, *c) for c in HEADS + LINEAR]
    + [(backward, kw, 1) for kw in (dict(dO=0), dict(dQ=0), dict(dK=0), dict(dV=FAKE + 2), dict(dstate=FAKE + 4),
                                    dict(out=FAKE + 4))]
    + [(backward, kw, 3) for kw in (dict(ws=0), dict(ws=FAKE + 16), dict(nb=100))]
    + [(step, kw, st) for kw, st in ((dict(s=shape(n=2)), 1), (dict(states=1), 1), (dict(states=-1, slots=FAKE), 1),
                                     (dict(state=0), 1), (dict(out=0), 1), (dict(scale=INF), 1), (dict(O=0), 1),
                                     (dict(slots=FAKE + 2), 1), (dict(Hk=3), 1), (dict(s=shape(n=1, d=32)), 2))]
    + [(rotary, *c) for c in HEADS]
    + [(rotary, kw, 1) for kw in (dict(PB=3), dict(PB=0), dict(pairs=(20, 13)), dict(pairs=(0, 4)), dict(pairs=()),
                                  dict(pairs=(1,) * 9), dict(base=0.0), dict(base=INF), dict(base=NAN),
                                  dict(flags=16), dict(pos=0), dict(pos=FAKE + 2), dict(Qo=0), dict(Ko=0))]
    + [(norm, kw, st) for kw, st in (
        (dict(s=norm_shape(dtype=3)), 1), (dict(s=norm_shape(B=-2)), 1), (dict(s=norm_shape(n=0)), 1),
        (dict(s=norm_shape(D=0)), 1), (dict(s=norm_shape(D=8193)), 2), (dict(s=norm_shape(kind=2)), 1),
        (dict(s=norm_shape(gate=3)), 1), (dict(s=norm_shape(eps=0.0)), 1), (dict(s=norm_shape(eps=NAN)), 1),
        (dict(s=norm_shape(a=INF)), 1), (dict(X=0), 1), (dict(F=FAKE + 2), 1), (dict(F=0), 1), (dict(gate=0), 1),
        (dict(s=norm_shape(gate=0)), 1), (dict(pw=0, pb=FAKE), 1), (dict(qw=0, qb=FAKE, H=0), 1), (dict(qw=0), 1),
        (dict(Y=0, H=0), 1), (dict(Y=FAKE + 4), 1))]
    + [(norm_back, kw, st) for kw, st in (
        (dict(dY=0, dH=0), 1), (dict(qw=0), 1), (dict(dpb=FAKE), 1), (dict(dqb=FAKE), 1), (dict(dH=0, dqw=FAKE), 1),
        (dict(gate=0, s=norm_shape(gate=0), dg=FAKE), 1), (dict(F=0, pw=0, gate=0, s=norm_shape(gate=0)), 1),
        (dict(dX=0, dF=0), 1), (dict(dX=FAKE + 2), 1), (dict(ws=0), 3), (dict(ws=FAKE + 64), 3), (dict(nb=16), 3))]
)


@pytest.mark.parametrize("call,kw,status", CASES)
def test_argument_errors(call, kw, status):
    rc = call(**kw)
    message = ga.lib().ga_last_error().decode()
    assert rc == status, (rc, message)
    assert message


@pytest.mark.parametrize("call,s", [(attend, shape(B=0)), (backward, shape(B=0)), (step, shape(B=0, n=1)),
                                    (attend, shape(H=0)), (norm, norm_shape(B=0, gate=0)),
                                    (norm_back, norm_shape(B=0, gate=0))])
def test_empty_batches_enqueue_nothing(call, s):
    assert call(s=s) == 0


def test_workspace_sizes():
    L = ga.lib()
    assert L.ga_linear_workspace_bytes(shape(d=32), 2) == 0
    assert L.ga_linear_backward_workspace_bytes(shape(), 3) == 0
    assert L.ga_norm_backward_workspace_bytes(norm_shape(D=9000)) == 0
    # shared heads keep each query head's share of dK and dV in fp32
    assert L.ga_linear_backward_workspace_bytes(shape(), 2) >= 2 * 4 * 100 * 64 * 4
    for B, n, D, gate in ((1, 1, 8, 0), (40000, 1, 512, 40000), (7, 123457, 8192, 7)):
        assert 0 < L.ga_norm_backward_workspace_bytes(norm_shape(B=B, n=n, D=D, gate=gate)) < 1 << 32


def test_binding_refuses_what_the_library_cannot_see():
    """Wrong shapes, types and places raise before a pointer is taken."""
    q = torch.zeros(1, 2, 4, 64)
    for call in (lambda: ga.linear_attend(q, q, q, torch.zeros(2)),
                 lambda: ga.linear_backward(q, q, q, q, torch.zeros(2)),
                 lambda: ga.linear_step(q, q, q, torch.zeros(2), torch.zeros(1, 2, 64, 64)),
                 lambda: ga.rotary(q, q, torch.zeros(1, 1, 4), (32,)),
                 lambda: ga.norm_residual(q[0]), lambda: ga.norm_residual(q),
                 lambda: ga.norm_residual(q[0], norm="batch"),
                 lambda: ga.norm_residual_backward(q[0], None, q[0])):
        with pytest.raises(ValueError):
            call()
