"""Refusals of the layer norm and the delta rule: C ABI and binding, before
anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2212_14052_amd as h3

OK, EINVAL, EUNSUP, EWS = 0, -1, -2, -3
P = lambda v: ctypes.c_void_p(v)
Q, K, V, G, BE, S, O, W, X, Y = (0x10000000 * i for i in range(1, 11))   # fake, aligned, far apart


def norm(x=X, w=K, b=K + 65536, rows=4, d=64, eps=1e-5, dt=2, y=Y, mean=G, rstd=BE):
    return h3.lib().h3_layernorm(P(x), P(w), P(b), rows, d, eps, dt, P(y), P(mean), P(rstd), None)


def test_layernorm_refusals():
    assert norm(x=0) == EINVAL
    assert norm(y=0) == EINVAL
    assert norm(rows=0) == EINVAL
    assert norm(d=0) == EINVAL
    assert norm(eps=-1.0) == EINVAL
    assert norm(eps=float("nan")) == EINVAL
    assert norm(dt=3) == EUNSUP
    assert norm(x=X + 1) == EINVAL                  # not aligned to its element
    assert norm(dt=0, y=Y + 2) == EINVAL
    assert norm(w=K + 2) == EINVAL
    assert norm(y=X + 64) == EINVAL                 # partly over x
    assert norm(mean=X + 16) == EINVAL              # inside x
    assert norm(rstd=Y) == EINVAL                   # inside y
    assert norm(rstd=G) == EINVAL                   # mean's buffer
    assert norm(w=Y + 128) == EINVAL                # y over the weight


def test_layernorm_widths():
    assert norm(d=(1 << 22) + 1) == EUNSUP
    assert norm_bwd(d=(1 << 22) + 1) == EUNSUP
    assert h3.workspace_size(h3.OP_LAYERNORM_BWD, 4, (1 << 22) + 1, 1, 0, 0, 2) == 0
    with pytest.raises(ValueError):
        h3._rows(torch.empty(1, dtype=torch.float16).expand(2 ** 31, 1))
    assert h3._rows(torch.empty(3, 0)) == 0 and h3._rows(torch.empty(2, 3, 4)) == 6


def norm_bwd(dy=V, x=X, w=K, mean=G, rstd=BE, rows=4, d=64, dt=2, dx=Y, dw=S, db=S + 65536, ws=W, wsb=1 << 20):
    return h3.lib().h3_layernorm_bwd(P(dy), P(x), P(w), P(mean), P(rstd), rows, d, dt, P(dx), P(dw), P(db), P(ws), wsb, None)


def test_layernorm_bwd_refusals():
    for name in ("dy", "x", "mean", "rstd"):
        assert norm_bwd(**{name: 0}) == EINVAL
    assert norm_bwd(rows=0) == EINVAL
    assert norm_bwd(dx=0, dw=0, db=0) == EINVAL     # nothing asked
    assert norm_bwd(dt=9) == EUNSUP
    assert norm_bwd(ws=0) == EWS
    assert norm_bwd(wsb=h3.workspace_size(h3.OP_LAYERNORM_BWD, 4, 64, 1, 0, 0, 2) - 1) == EWS
    assert norm_bwd(ws=W + 8) == EINVAL
    assert norm_bwd(dx=V) == EINVAL                 # in place, but dw and db are still summed from dy
    assert norm_bwd(dw=K) == EINVAL                 # dw over w
    assert norm_bwd(db=S) == EINVAL                 # db over dw
    assert norm_bwd(ws=X) == EINVAL
    assert norm_bwd(dw=S + 1) == EINVAL
    assert h3.workspace_size(h3.OP_LAYERNORM_BWD, 16384, 768, 1, 0, 0, h3.F16) >= 256 * 2 * 768 * 4
    assert h3.workspace_size(h3.OP_LAYERNORM_BWD, 0, 768, 1, 0, 0, h3.F16) == 0


def step(q=Q, k=K, v=V, g=G, beta=BE, scale=0.1, B=2, T=1, H=4, Hk=2, Dk=64, Dv=64, dt=2, S=S, o=O):
    return h3.lib().h3_delta_step(P(q), P(k), P(v), P(g), P(beta), scale, B, T, H, Hk, Dk, Dv, dt, P(S), P(o), None)


def test_delta_step_refusals():
    for name in ("q", "k", "v", "g", "beta", "S", "o"):
        assert step(**{name: 0}) == EINVAL
    for name in ("B", "T", "H", "Hk", "Dk", "Dv"):
        assert step(**{name: 0}) == EINVAL
    assert step(Hk=3) == EINVAL                     # heads not shared evenly
    assert step(Dk=12) == EUNSUP
    assert step(Dk=136) == EUNSUP
    assert step(Dv=20) == EUNSUP
    assert step(Dv=264) == EUNSUP
    assert step(dt=5) == EUNSUP
    assert step(S=S + 8) == EINVAL                  # state not 16-byte aligned
    assert step(q=Q + 1) == EINVAL
    assert step(g=G + 2) == EINVAL
    assert step(o=V) == EINVAL                      # output over v
    assert step(o=S + 256) == EINVAL                # output inside the state
    assert step(S=K) == EINVAL
    assert step(B=1 << 23, H=8, Hk=8, Dk=8, Dv=8, o=O << 8) == EUNSUP      # 2^26 waves


def test_binding_refusals():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        h3.layernorm(x)
    with pytest.raises(TypeError):
        h3.layernorm([1.0])
    with pytest.raises(ValueError):
        h3.layernorm_bwd(x, x, None, x[:, 0], x[:, 0])
    q, v, g = torch.zeros(1, 1, 2, 8), torch.zeros(1, 1, 2, 8), torch.zeros(1, 1, 2)
    with pytest.raises(ValueError):
        h3.delta_step(q, q, v, g, g, torch.zeros(1, 2, 8, 8))


def rule(q=Q, k=K, v=V, g=G, beta=BE, S0=None, lengths=None, scale=0.1, B=2, L=70, H=4, Hk=2, Dk=64, Dv=64, dt=2, o=O, Sf=S,
         saved=None, savedb=0, ws=W, wsb=1 << 26):
    return h3.lib().h3_delta_rule(P(q), P(k), P(v), P(g), P(beta), P(S0), P(lengths), scale, B, L, H, Hk, Dk, Dv, dt, P(o),
                                  P(Sf), P(saved), savedb, P(ws), wsb, None)


def size(op, B=2, L=70, H=4, Dk=64, Dv=64, dt=2):
    return h3.workspace_size(op, B, H, L, Dk, Dv, dt)


def test_delta_rule_refusals():
    for name in ("q", "k", "v", "g", "beta", "o"):
        assert rule(**{name: 0}) == EINVAL
    for name in ("B", "L", "H", "Hk", "Dk", "Dv"):
        assert rule(**{name: 0}) == EINVAL
    assert rule(Hk=3) == EINVAL
    for name, bad in (("Dk", 12), ("Dk", 136), ("Dv", 20), ("Dv", 264), ("dt", 4)):
        assert rule(**{name: bad}) == EUNSUP
    assert rule(B=1 << 20, L=1 << 24, H=2, Hk=2, Dk=8, Dv=8) == EUNSUP     # 2^31 chunks and more
    assert rule(H=65536, Hk=1, Dv=72) == EUNSUP                            # H Dv beyond 2^22
    assert rule(L=2 ** 31 - 1) == EWS
    assert rule(ws=0) == EWS
    assert rule(wsb=size(h3.OP_DELTA) - 1) == EWS
    assert rule(saved=X, savedb=size(h3.OP_DELTA_SAVED) - 1) == EWS
    for name, at in (("q", Q), ("k", K), ("v", V), ("o", O)):
        assert rule(**{name: at + 8}) == EINVAL                            # 16-byte alignment
    assert rule(S0=X + 2) == EINVAL
    assert rule(lengths=X + 2) == EINVAL
    assert rule(o=V) == EINVAL
    assert rule(Sf=O + 256) == EINVAL
    assert rule(S0=X, Sf=X + 4) == EINVAL                                  # partly over the first state
    assert rule(ws=Q - 4096) == EINVAL
    assert rule(saved=W + 4096, savedb=1 << 26) == EINVAL                  # inside the workspace
    assert rule(lengths=W + 64) == EINVAL


def bwd(q=Q, k=K, v=V, g=G, beta=BE, do=X, dS=None, saved=Y, savedb=1 << 27, lengths=None, scale=0.1, B=2, L=70, H=4, Hk=2,
        Dk=64, Dv=64, dt=2, dq=O, dk=O + (1 << 22), dv=O + (1 << 23), dg=S, dbeta=S + (1 << 20), dS0=None, ws=W, wsb=1 << 26):
    return h3.lib().h3_delta_rule_bwd(P(q), P(k), P(v), P(g), P(beta), P(do), P(dS), P(saved), savedb, P(lengths), scale, B,
                                      L, H, Hk, Dk, Dv, dt, P(dq), P(dk), P(dv), P(dg), P(dbeta), P(dS0), P(ws), wsb, None)


def test_delta_rule_bwd_refusals():
    for name in ("q", "k", "v", "g", "beta", "do", "saved", "dq", "dk", "dv", "dg", "dbeta"):
        assert bwd(**{name: 0}) == EINVAL
    for name in ("B", "L", "H", "Hk", "Dk", "Dv"):
        assert bwd(**{name: 0}) == EINVAL
    assert bwd(Hk=3) == EINVAL
    for name, bad in (("Dk", 4), ("Dk", 160), ("Dv", 12), ("Dv", 512), ("dt", -1)):
        assert bwd(**{name: bad}) == (EUNSUP if bad != -1 or name == "dt" else EINVAL)
    assert bwd(savedb=size(h3.OP_DELTA_SAVED) - 1) == EWS
    assert bwd(ws=0) == EWS
    assert bwd(wsb=size(h3.OP_DELTA_BWD) - 1) == EWS
    assert bwd(do=X + 2) == EINVAL
    assert bwd(saved=Y + 4) == EINVAL
    assert bwd(dg=S + 2) == EINVAL
    assert bwd(dq=Q) == EINVAL                                             # over an input
    assert bwd(dk=O) == EINVAL                                             # over dq
    assert bwd(dbeta=G) == EINVAL
    assert bwd(ws=Y + 4096) == EINVAL                                      # inside what was kept
    assert bwd(dS=V + (1 << 24), dS0=V + (1 << 24) + 64) == EINVAL         # partly over dS


def test_delta_sizes():
    assert size(h3.OP_DELTA, H=65536, Dv=72) == 0 and size(h3.OP_DELTA, B=1 << 20, L=1 << 24, H=2) == 0
    assert size(h3.OP_DELTA, Dk=12) == 0 and size(h3.OP_DELTA_SAVED, Dv=0) == 0 and size(h3.OP_DELTA_BWD, L=0) == 0
    # a chunk's state and errors in float32 for every 64 tokens
    assert size(h3.OP_DELTA_SAVED) >= 2 * 4 * 2 * (64 * 64 * 4 + 64 * 64 * 4)
    assert size(h3.OP_DELTA_BWD) >= 2 * 4 * 2 * (64 * 64 * 4 + 64 * 64 * 4)


def test_delta_binding_refusals():
    q, g = torch.zeros(1, 5, 2, 8), torch.zeros(1, 5, 2)
    with pytest.raises(ValueError):
        h3.delta_rule(q, q, q, g, g)
    with pytest.raises(ValueError):
        h3.delta_rule_bwd(q, q, q, g, g, q, torch.zeros(64, dtype=torch.uint8))
    with pytest.raises(TypeError):
        h3.delta_rule(None, q, q, g, g)
