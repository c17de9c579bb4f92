"""The recurrent gated delta rule against the recurrence in 64 bits.

Tolerances: keys of unit length, beta in (0, 1) and decays at most 1 make each
step's map of the state a contraction, so the errors of the steps at most add
up.  One step rounds sums of Dk products (at most Dk 2^-24 of the product of
the column's length and the key's, which is 1), and a few values of that size."""
import pytest
import torch

import paper_2212_14052_amd as h3

pytestmark = pytest.mark.gpu
E32 = 2.0 ** -24
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def inputs(B, T, H, Hk, Dk, Dv, dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)
    q, k = r(B, T, Hk, Dk), r(B, T, Hk, Dk)
    q, k = q / q.norm(dim=-1, keepdim=True), k / k.norm(dim=-1, keepdim=True)
    g = -torch.empty(B, T, H).uniform_(-7, 0, generator=gen).exp()
    ts = [t.to(DTYPES[dtype]).cuda() for t in (q, k, r(B, T, H, Dv))]
    return ts + [g.cuda(), torch.sigmoid(r(B, T, H)).cuda(), r(B, H, Dk, Dv).cuda()]


def reference(q, k, v, g, beta, S, scale):
    q, k, v, g, beta, S = (t.double().cpu() for t in (q, k, v, g, beta, S))
    per, out, size = v.shape[2] // q.shape[2], [], 0.0
    q, k = q.repeat_interleave(per, 2), k.repeat_interleave(per, 2)
    for t in range(v.shape[1]):
        S = S * g[:, t].exp()[..., None, None]
        e = v[:, t] - (S * k[:, t, :, :, None]).sum(2)
        S = S + k[:, t, :, :, None] * (beta[:, t, :, None] * e)[:, :, None, :]
        out.append(scale * (S * q[:, t, :, :, None]).sum(2))
        size = max(size, S.norm(dim=2).max().item() + e.abs().max().item())
    return torch.stack(out, 1), S, size


def run_and_check(q, k, v, g, beta, S, scale=None):
    B, T, H, Dv = v.shape
    Dk = q.shape[-1]
    ro, rS, size = reference(q, k, v, g, beta, S, Dk ** -0.5 if scale is None else scale)
    # lengths of q and k after rounding to 8 bits: at most 1 + 2^-8
    off = 1.02 ** T * T * (Dk + 16) * E32 * size
    o = h3.delta_step(q, k, v, g, beta, S, scale)
    assert o.shape == v.shape and o.dtype == v.dtype
    assert (S.double().cpu() - rS).abs().max() <= off
    tol = ro.abs() * torch.finfo(v.dtype).eps / 2 + abs(Dk ** -0.5 if scale is None else scale) * 2 * off + 2.0 ** -25
    assert ((o.double().cpu() - ro).abs() <= tol).all()
    return o


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,T,H,Hk,Dk,Dv", [
    (1, 1, 1, 1, 8, 8), (2, 1, 6, 6, 128, 128), (3, 5, 4, 2, 64, 96), (1, 9, 3, 1, 96, 40), (5, 2, 6, 3, 16, 256),
    (2, 3, 2, 2, 120, 24), (1, 33, 2, 1, 32, 64), (7, 1, 1, 1, 40, 200)])
def test_step(B, T, H, Hk, Dk, Dv, dtype):
    run_and_check(*inputs(B, T, H, Hk, Dk, Dv, dtype))


def test_tokens_one_by_one_and_together():
    q, k, v, g, beta, S = inputs(3, 6, 4, 2, 64, 64, "bf16", 1)
    S1, S2 = S.clone(), S.clone()
    o = h3.delta_step(q, k, v, g, beta, S1, 0.3)
    for t in range(6):
        at = slice(t, t + 1)
        assert torch.equal(h3.delta_step(q[:, at], k[:, at], v[:, at], g[:, at], beta[:, at], S2, 0.3), o[:, at])
    assert torch.equal(S1, S2)


def test_gates_at_their_ends():
    """beta 0 and g 0 leave a state as it is; g -inf drops it; zero keys write nothing."""
    q, k, v, g, beta, S = inputs(2, 1, 3, 3, 32, 32, "f32", 2)
    S0 = S.clone()
    h3.delta_step(q, k, v, torch.zeros_like(g), torch.zeros_like(beta), S)
    assert torch.equal(S, S0)
    run_and_check(q, k, v, torch.full_like(g, -float("inf")), beta, S)
    S = S0.clone()
    h3.delta_step(q, torch.zeros_like(k), v, torch.zeros_like(g), beta, S)
    assert torch.equal(S, S0)


def test_not_finite_stays_in_its_head():
    q, k, v, g, beta, S = inputs(2, 2, 3, 3, 64, 64, "f16", 3)
    S1, S2 = S.clone(), S.clone()
    o1 = h3.delta_step(q, k, v, g, beta, S1)
    v[0, 0, 1, 5] = float("nan")
    o2 = h3.delta_step(q, k, v, g, beta, S2)
    assert torch.isnan(S2[0, 1, :, 5]).all() and torch.isnan(o2[0, :, 1, 5]).all()
    S2[0, 1, :, 5], o2[0, :, 1, 5] = S1[0, 1, :, 5], o1[0, :, 1, 5]
    assert torch.equal(S1, S2) and torch.equal(o1, o2)


def test_views_and_other_stream():
    q, k, v, g, beta, S = inputs(2, 3, 4, 4, 64, 64, "bf16", 4)
    S1, S2 = S.clone(), S.clone()
    o = h3.delta_step(q, k, v, g, beta, S1)
    qkv = torch.cat([q, k, v], -1)   # slices of one projection
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o2 = h3.delta_step(qkv[..., :64], qkv[..., 64:128], qkv[..., 128:], g, beta, S2)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(o, o2) and torch.equal(S1, S2)
    with pytest.raises(ValueError):
        h3.delta_step(q, k, v, g, beta, S.transpose(-1, -2))   # updated in place: contiguous only
