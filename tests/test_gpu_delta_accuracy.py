"""The gated delta rule where parts of its inputs differ much in size, against 64 bits.

Tolerances count roundings: a matrix product's operands go in as two fp16 pieces, 2^-22 of
each term at most, and its smallest product of pieces, 2^-22, is left out; a float32 sum of up to 192 terms rounds by
2^-24 of its size a term, with signs that are independent: 14 x 2^-24 in the 2-norm.  Results in 16 bits are
rounded once: half a step."""
import pytest
import torch

import paper_2212_14052_amd as h3
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
