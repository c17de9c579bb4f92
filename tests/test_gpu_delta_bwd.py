"""Gradients of the gated delta rule against its reverse recurrence in 64 bits,
and against differences.

Tolerances.  Keys of unit length, beta in (0, 1) and decays at most 1: neither the
recurrence nor its reverse stretches an error, so the chunks' errors add up.  Every
gradient is a sum of products of a state S, a state's gradient dS, an error e or
an output's gradient, so what a chunk rounds away is bounded by C times the product of the
largest norms of its two factors: C = 2^-20 in float32 (operands in two fp16 pieces, 2^-22; sums of
up to 128 + 64 terms, 2^-24 each, at a sixteenth by their signs), 2^-15 for 16-bit inputs.  16-bit results are rounded once more: half a step."""
import pytest
import torch

import paper_2212_14052_amd as h3
from tests.test_gpu_delta_rule import DTYPES, MANY, inputs

pytestmark = pytest.mark.gpu
NAMES = ("dq", "dk", "dv", "dg", "dbeta", "dS0")


def reverse(q, k, v, g, beta, S0, do, dS, scale, lengths=None):
    """The gradients, and the largest norms of S, dS, e and scale do."""
    shared = q.shape[2]
    q, k, v, g, beta, do = (t.double() for t in (q, k, v, g, beta, do))
    B, L, H, Dv = v.shape
    per = H // shared
    q, k = q.repeat_interleave(per, 2), k.repeat_interleave(per, 2)
    if lengths is not None:
        gone = torch.arange(L, device=v.device)[None, :, None] >= lengths[:, None, None]
        q, k, v, do = (t.masked_fill(gone[..., None], 0.0) for t in (q, k, v, do))
        g, beta = g.masked_fill(gone, 0.0), beta.masked_fill(gone, 0.0)
    S = torch.zeros(B, H, q.shape[-1], Dv, dtype=torch.float64, device=v.device) if S0 is None else S0.double()
    kept, a = [], g.exp()
    for t in range(L):
        hat = S * a[:, t][..., None, None]
        e = v[:, t] - (hat * k[:, t, :, :, None]).sum(2)
        S = hat + k[:, t, :, :, None] * (beta[:, t, :, None] * e)[:, :, None, :]
        kept.append((hat, e, S))
    dS = torch.zeros_like(S) if dS is None else dS.double()
    dq, dk, dv, dg, dbeta = (torch.zeros_like(t) for t in (q, k, v, g, beta))
    nS = ndS = ne = 0.0
    for t in range(L - 1, -1, -1):
        hat, e, S = kept[t]
        dS = dS + scale * q[:, t, :, :, None] * do[:, t, :, None, :]
        dq[:, t] = scale * (S * do[:, t, :, None, :]).sum(-1)
        u, b = beta[:, t, :, None] * e, beta[:, t, :, None]
        du = (dS * k[:, t, :, :, None]).sum(2)
        dbeta[:, t], dv[:, t] = (e * du).sum(-1), b * du
        dk[:, t] = (dS * u[:, :, None, :]).sum(-1) - (hat * dv[:, t, :, None, :]).sum(-1)
        nS, ndS, ne = max(nS, S.norm(dim=(2, 3)).max().item()), max(ndS, dS.norm(dim=(2, 3)).max().item()), max(ne, e.norm(dim=-1).max().item())
        dS = dS - k[:, t, :, :, None] * dv[:, t, :, None, :]
        dg[:, t] = (dS * hat).sum((-1, -2))
        dS = dS * a[:, t][..., None, None]
    if lengths is not None:
        dg, dbeta = dg.masked_fill(gone, 0.0), dbeta.masked_fill(gone, 0.0)
    to_shared = lambda t: t.view(B, L, shared, per, -1).sum(3)
    return (to_shared(dq), to_shared(dk), dv, dg, dbeta, dS), nS, ndS, ne, scale * do.norm(dim=-1).max().item()


def grads_of(q, k, v, g, beta, S0, do, dS, scale=None, lengths=None):
    saved = h3.delta_rule(q, k, v, g, beta, S0=S0, scale=scale, lengths=lengths, save=True)[2]
    return h3.delta_rule_bwd(q, k, v, g, beta, do, saved, dS=dS, scale=scale, lengths=lengths)


def run_and_check(dtype, q, k, v, g, beta, S0, do, dS, scale=None, lengths=None):
    Dk, per = q.shape[-1], v.shape[2] // q.shape[2]
    refs, nS, ndS, ne, ndo = reverse(q, k, v, g, beta, S0, do, dS, Dk ** -0.5 if scale is None else abs(scale), lengths)
    got = grads_of(q, k, v, g, beta, S0, do, dS, scale, lengths)
    C = (2.0 ** -20 if dtype == "f32" else 2.0 ** -15) * -(-v.shape[1] // 64) * 1.1
    bounds = (per * nS * ndo, per * ndS * (nS + ne), ndS + ndo, nS * ndS, ne * ndS, ndS)
    for name, x, ref, bound in zip(NAMES, got, refs, bounds):
        assert x.shape == ref.shape
        half = torch.finfo(x.dtype).eps / 2 if x.dtype != torch.float32 else 0.0
        far = (x.double() - ref).abs()
        assert (far <= half * ref.abs() + C * bound + (2.0 ** -25 if x.dtype == torch.float16 else 0.0)).all(), (name, far.max().item(), C * bound)
        # In the 2-norm the roundings average out over their signs: a sixteenth of C.  It cannot be under
        # eight float32 roundings of 2^-24 (half of C in float32): with a single token dk = dS u - S dv already rounds exp(g) S,
        # S^T k, e, u, dS's two terms, dv and the difference once each.  dg is a difference of sums: half of C.
        near = max(C / (2 if name == "dg" else 16), 2.0 ** -21 * -(-v.shape[1] // 64))
        assert far.norm() <= (half + near) * ref.norm() + 1e-30, (name, (far.norm() / ref.norm()).item())
    return got


def full_inputs(B, L, H, Hk, Dk, Dv, dtype, seed=0, **more):
    q, k, v, g, beta, S0 = inputs(B, L, H, Hk, Dk, Dv, dtype, seed, **more)
    gen = torch.Generator().manual_seed(seed + 1000)
    return q, k, v, g, beta, S0, torch.randn(v.shape, generator=gen).to(v.dtype).cuda(), 0.3 * torch.randn(S0.shape, generator=gen).cuda()


SIZES = [(1, 1, 1, 1, 8, 8), (2, 63, 2, 2, 16, 16), (1, 64, 3, 1, 128, 128), (2, 65, 2, 1, 64, 64), (3, 150, 4, 2, 96, 40),
         (1, 190, 2, 2, 32, 256), (2, 130, 2, 2, 120, 24), (1, 300, 3, 1, 128, 72)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,L,H,Hk,Dk,Dv", SIZES)
def test_gradients(B, L, H, Hk, Dk, Dv, dtype):
    run_and_check(dtype, *full_inputs(B, L, H, Hk, Dk, Dv, dtype))


@pytest.mark.parametrize("dtype", DTYPES)
def test_without_states_and_with_scale(dtype):
    q, k, v, g, beta, S0, do, dS = full_inputs(2, 100, 2, 2, 64, 64, dtype, 1)
    run_and_check(dtype, q, k, v, g, beta, None, do, None, 1.3)


@pytest.mark.parametrize("dtype", DTYPES)
def test_lengths(dtype):
    q, k, v, g, beta, S0, do, dS = full_inputs(5, 140, 4, 2, 64, 40, dtype, 2)
    lengths = torch.tensor([140, 0, 1, 64, 70], device="cuda", dtype=torch.int32)
    want = run_and_check(dtype, q, k, v, g, beta, S0, do, dS, None, lengths)
    behind = torch.arange(140, device="cuda")[None] >= lengths[:, None]
    for t in (q, k, v, g, beta, do):
        t[behind] = float("nan")
    got = grads_of(q, k, v, g, beta, S0, do, dS, None, lengths)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all((t[behind] == 0).all() for t in got[:5]) and torch.equal(got[5][1], dS[1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,L,H,Hk,Dk,Dv", [(1, 1300, 1, 1, 40, 72), (2, 1100, 2, 1, 64, 64)])
def test_few_heads_long(B, L, H, Hk, Dk, Dv, dtype):
    """Long sequences of few heads, which are worked on in segments."""
    args = full_inputs(B, L, H, Hk, Dk, Dv, dtype, 8)
    run_and_check(dtype, *args)
    for n in (0, 60, L // 2):
        run_and_check(dtype, *args, None, torch.tensor([n, L][:B], device="cuda", dtype=torch.int32))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,L,H,Hk,Dk,Dv", MANY)
def test_many_heads(B, L, H, Hk, Dk, Dv, dtype):
    """Heads that fill the card: workgroups of eight waves for 16-bit inputs, some without columns."""
    run_and_check(dtype, *full_inputs(B, L, H, Hk, Dk, Dv, dtype, 11))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gates_at_their_ends(dtype):
    q, k, v, g, beta, S0, do, dS = full_inputs(2, 100, 2, 2, 32, 32, dtype, 3)
    g[:, 10], g[:, 70], g[:, 71] = -float("inf"), -1e30, 0.0
    beta[:, 20], beta[:, 30] = 0.0, 1.0   # beta's gradient where beta is 0 as well
    run_and_check(dtype, q, k, v, g, beta, S0, do, dS)


def test_against_differences():
    """float32: central differences of the loss <o, do> + <S, dS>."""
    q, k, v, g, beta, S0, do, dS = full_inputs(1, 70, 2, 1, 16, 8, "f32", 4)
    got = grads_of(q, k, v, g, beta, S0, do, dS)

    def loss():
        o, S = h3.delta_rule(q, k, v, g, beta, S0=S0)
        return ((o.double() * do.double()).sum() + (S.double() * dS.double()).sum()).item()

    # step 2^-7: the loss is a sum of about a thousand terms of size one, each off by a few 2^-24 with random signs: under
    # 1e-5, over 2^-6 that is 6e-4; the third derivative's part is h^2 / 6 = 1e-5 times derivatives of the gradient's size
    h, gen = 2.0 ** -7, torch.Generator().manual_seed(5)
    for t, grad in zip((q, k, v, g, beta, S0), got):
        flat = t.view(-1)
        for i in torch.randperm(flat.numel(), generator=gen)[:12].tolist():
            at = flat[i].item()
            flat[i] = at + h
            up = loss()
            flat[i] = at - h
            down = loss()
            flat[i] = at
            assert abs((up - down) / (2 * h) - grad.view(-1)[i].item()) <= 2e-3 * max(1.0, grad.abs().max().item())


def test_repeats_and_in_a_graph_beside_eager_calls():
    args = full_inputs(2, 130, 4, 2, 64, 64, "bf16", 6)
    want = [t.clone() for t in grads_of(*args)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = grads_of(*args)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(torch.equal(a, b) for a, b in zip(grads_of(*args), want))


def test_chunked_training_in_two_parts():
    """The gradient of the first state of one part is that of the last state of the part before."""
    q, k, v, g, beta, S0, do, dS = full_inputs(1, 128, 2, 2, 32, 32, "f32", 7)
    whole = grads_of(q, k, v, g, beta, S0, do, dS)
    part = lambda a, b: [t[:, a:b] for t in (q, k, v, g, beta)]
    o1, S1, saved1 = h3.delta_rule(*part(0, 64), S0=S0, save=True)
    o2, S2, saved2 = h3.delta_rule(*part(64, 128), S0=S1, save=True)
    back = h3.delta_rule_bwd(*part(64, 128), do[:, 64:], saved2, dS=dS)
    front = h3.delta_rule_bwd(*part(0, 64), do[:, :64], saved1, dS=back[5])
    for w, a, b in zip(whole[:5], front, back):
        assert torch.equal(w, torch.cat([a, b], 1))
    assert torch.equal(whole[5], front[5])
