"""The gated delta rule where parts of its inputs differ much in size, against 64 bits.

Tolerances count roundings: a matrix product's operands go in as two fp16 pieces, 2^-22 of
each term at most, and its smallest product of pieces, 2^-22, is left out; a float32 sum of up to 192 terms rounds by
2^-24 of its size a term, with signs that are independent: 14 x 2^-24 in the 2-norm.  Results in 16 bits are
rounded once: half a step."""
import pytest
import torch

import paper_2212_14052_amd as h3
from tests.test_gpu_delta_bwd import NAMES, full_inputs, grads_of, reverse
from tests.test_gpu_delta_rule import DTYPES, inputs, reference

pytestmark = pytest.mark.gpu


def half(dtype):
    return torch.finfo(dtype).eps / 2


@pytest.mark.parametrize("carried", [False, True])
@pytest.mark.parametrize("ratio", [1.0, 30.0, 1000.0])
@pytest.mark.parametrize("dtype", DTYPES)
def test_rewritten_keys(dtype, ratio, carried):
    """32 keys are written twice, the second values smaller, and read: the old values, in the same chunk or in the state,
    cancel.  The chain K S, R, X R, u, P u with Q S cuts seven operands and sums three times: 7 x 2^-22 + 3 x 14 x 2^-24,
    under 2^-17, of the old values."""
    L, first = (96, 32) if carried else (64, 0)
    q, k, v, g, beta, _ = inputs(2, L, 3, 3, 128, 128, dtype, 20)
    k[:, first + 32:first + 64] = k[:, first:first + 32]
    q.copy_(k)
    v[:, first:first + 32] *= ratio
    g.zero_(); beta.fill_(1.0)
    beta[:, :first] = 0.0
    ro, rS, *_ = reference(q, k, v, g, beta, None, 1.0)
    o, S = h3.delta_rule(q, k, v, g, beta, scale=1.0)
    old, new = ro[:, first:first + 32], ro[:, first + 32:]
    off = (o.double() - ro)[:, first + 32:].norm() / new.norm()
    assert off <= (half(v.dtype) if dtype != "f32" else 0.0) + 2.0 ** -17 * (old.norm() / new.norm()), off.item()
    assert (S.double() - rS).norm() <= 2.0 ** -17 * old.norm()


def check_gradients(args, do, dS, lengths=None):
    """All gradients in the 2-norm: a chunk's roundings of 2^-22 (operands) and 2^-24 (sums) are independent, under
    2^-21 together; dg is a difference of sums about four times its size.  Not the 16-bit ones that fp16 holds with
    fewer bits."""
    q, k, v, g, beta, S0 = args
    refs = reverse(q, k, v, g, beta, S0, do, dS, q.shape[-1] ** -0.5, lengths)[0]
    got = grads_of(q, k, v, g, beta, S0, do, dS, None, lengths)
    for name, x, ref in zip(NAMES, got, refs):
        if x.dtype == torch.float16:
            continue
        tol = (half(x.dtype) if x.dtype != torch.float32 else 0.0) + 2.0 ** (-19 if name == "dg" else -21) * -(-v.shape[1] // 64)
        assert (x.double() - ref).norm() <= tol * ref.norm(), (name, ((x.double() - ref).norm() / ref.norm()).item())


GRAD_SIZES = [(2, 192, 2, 2, 128, 128), (1, 150, 4, 2, 64, 40), (2, 130, 2, 2, 32, 72), (1, 2700, 1, 1, 64, 64)]


@pytest.mark.parametrize("size", [2.0 ** -20, 2.0 ** -30])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,L,H,Hk,Dk,Dv", GRAD_SIZES)
def test_only_the_final_state_has_a_small_gradient(B, L, H, Hk, Dk, Dv, dtype, size):
    q, k, v, g, beta, S0, do, dS = full_inputs(B, L, H, Hk, Dk, Dv, dtype, 21)
    check_gradients((q, k, v, g * 0.01, beta, S0), torch.zeros_like(do), dS * size)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,L,H,Hk,Dk,Dv", GRAD_SIZES)
def test_no_gradient_from_a_prompt(B, L, H, Hk, Dk, Dv, dtype):
    """The outputs of the first tokens have no gradient, those of the last ones a small one."""
    q, k, v, g, beta, S0, do, dS = full_inputs(B, L, H, Hk, Dk, Dv, dtype, 22)
    do *= 2.0 ** -14 if dtype == "f16" else 2.0 ** -30
    do[:, :L - 40] = 0.0
    check_gradients((q, k, v, g * 0.01, beta, S0), do, None)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,L,H,Hk,Dk,Dv", GRAD_SIZES)
def test_columns_of_zeros(B, L, H, Hk, Dk, Dv, dtype):
    """Sixteen columns of zeros beside small ones, in the values, the states and the gradients."""
    q, k, v, g, beta, S0, do, dS = full_inputs(B, L, H, Hk, Dk, Dv, dtype, 23)
    for t, size in ((v, 2.0 ** -10), (S0, 2.0 ** -26), (do, 2.0 ** -12), (dS, 2.0 ** -28)):
        t *= size if dtype == "f16" else size * size
        t[..., 16:32] = 0.0
    check_gradients((q, k, v, g, beta, S0), do, dS)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,L,H,Hk,Dk,Dv", [(2, 150, 2, 2, 128, 128), (1, 130, 4, 2, 40, 24), (1, 2700, 1, 1, 64, 72), (16, 65, 16, 16, 128, 128)])
def test_columns_do_not_meet(B, L, H, Hk, Dk, Dv, dtype):
    """A column of the values and states that is much larger, much smaller, or not finite leaves every bit of the
    others as it was, and scales by itself."""
    q, k, v, g, beta, S0, do, dS = full_inputs(B, L, H, Hk, Dk, Dv, dtype, 24)
    rest = torch.arange(Dv, device="cuda") != 3
    o, S = h3.delta_rule(q, k, v, g, beta, S0=S0)
    gr = grads_of(q, k, v, g, beta, S0, do, dS)
    for size in ((2.0 ** 5,) if dtype == "f16" else (2.0 ** 24, 2.0 ** -24, 2.0 ** 60, 2.0 ** -60)):
        f = torch.where(rest, 1.0, size)
        o2, S2 = h3.delta_rule(q, k, v * f.to(v.dtype), g, beta, S0=S0 * f)
        assert torch.equal(o2[..., rest], o[..., rest]) and torch.equal(S2, S * f)
        assert dtype == "f16" or torch.equal(o2, o * f.to(o.dtype))
        gr2 = grads_of(q, k, v, g, beta, S0, do * f.to(do.dtype), dS * f)
        assert torch.equal(gr2[2][..., rest], gr[2][..., rest]) and torch.equal(gr2[5], gr[5] * f)
    for bad in (float("inf"), float("nan")):
        v2, do2 = v.clone(), do.clone()
        v2[:, L // 2, :, 3] = do2[:, L // 2, :, 3] = bad
        o2, S2 = h3.delta_rule(q, k, v2, g, beta, S0=S0)
        assert torch.equal(o2[..., rest], o[..., rest]) and torch.equal(S2[..., rest], S[..., rest])
        assert not S2[..., 3].isfinite().any()
        gr2 = grads_of(q, k, v, g, beta, S0, do2, dS)
        assert torch.equal(gr2[2][..., rest], gr[2][..., rest]) and torch.equal(gr2[5][..., rest], gr[5][..., rest])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,L,H,Hk,Dk,Dv", [(2, 120, 2, 2, 128, 128), (1, 190, 4, 2, 64, 40), (16, 128, 16, 16, 128, 128)])
def test_writes_that_fade(B, L, H, Hk, Dk, Dv, dtype):
    """The last chunk is written to by its first token alone and then decays by up to 2^-45: what is left of that keeps its bits.
    A chunk's roundings of operands and sums, 2^-21, and of its decay: float32 holds the logarithm's sum G by |G| 2^-24, or
    twice that with the change to base 2."""
    q, k, v, g, beta, S0, do, dS = full_inputs(B, L, H, Hk, Dk, Dv, dtype, 25)
    last = (L - 1) // 64 * 64
    g.fill_(-0.5)
    beta[:, last + 1:] = 0.0
    beta[:, :last] = 0.0
    rS = reference(q, k, v, g, beta, None, 1.0)[1]
    S = h3.delta_rule(q, k, v, g, beta)[1]
    assert (S.double() - rS).norm() <= (2.0 ** -21 + 2 * 32 * 2.0 ** -24) * rS.norm()


@pytest.mark.parametrize("late", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,L,H,Hk,Dk,Dv", [(6, 150, 4, 4, 128, 128), (12, 130, 4, 2, 64, 40), (8, 100, 6, 2, 96, 72), (12, 70, 4, 4, 24, 16),
                                            (8, 64, 6, 3, 128, 24)])
def test_gradient_of_strong_decays(B, L, H, Hk, Dk, Dv, dtype, late):
    """Decays of exp(-5) to exp(-60) a token, whose gradients have that factor; all outputs have gradients, or (late) the last
    five only.  Every term of dg is a product of up to five operands of 2^-22 of the largest, at most eight times
    the usual size (5 x 2^-19), times a decay with an error of 87 x 2^-24: under 2^-16 of a token's gradients over all heads."""
    q, k, v, g, beta, S0, do, dS = full_inputs(B, L, H, Hk, Dk, Dv, dtype, 27)
    gen = torch.Generator().manual_seed(28)
    g = -torch.empty(B, L, H).uniform_(5, 60, generator=gen).cuda()
    if late:
        do[:, :L - 5] = 0.0
        dS = None
    ref = reverse(q, k, v, g, beta, S0, do, dS, Dk ** -0.5)[0][3]
    dg = grads_of(q, k, v, g, beta, S0, do, dS)[3]
    far, size = (dg.double() - ref).norm(dim=(0, 2)), ref.norm(dim=(0, 2))
    # Pieces hold 22 bits of what is at least 2^-16 of the largest that shares their scale (2^13 .. 2^14 of fp16, whose
    # second piece ends at 2^-24: 2^-3 is the least value with 22 bits), which the z of a token that only faded gradients reach is
    # not: nothing is promised of tokens whose gradients are smaller than that.
    seen = size >= 2.0 ** -16 * size.max()
    assert (far <= 2.0 ** -16 * size)[seen].all(), (far / size)[seen].max().item()
    assert (dg.double() - ref).norm() <= 2.0 ** -18 * ref.norm()


@pytest.mark.parametrize("dtype", DTYPES)
def test_gradient_of_a_dropped_state(dtype):
    """Nothing passes a decay of -inf: its gradient is 0, and those around it are what they are for -1e30."""
    q, k, v, g, beta, S0, do, dS = full_inputs(2, 150, 4, 2, 64, 64, dtype, 29)
    at = [0, 10, 63, 64, 100, 149]
    g[:, at] = -float("inf")
    got = grads_of(q, k, v, g, beta, S0, do, dS)
    assert (got[3][:, at] == 0).all()
    g[:, at] = -1e30
    assert all(torch.equal(a, b) for a, b in zip(got, grads_of(q, k, v, g, beta, S0, do, dS)))
