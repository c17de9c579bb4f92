"""The largest calls that the layer norm and the delta rule take, and what is refused beyond (no GPU needed)."""
import pytest
import torch

import paper_2212_14052_amd as h3
from tests.test_abi_mixers import EINVAL, EUNSUP, O, V, bwd, rule, size, step


def test_launches_of_less_than_2_to_32_threads():
    """Scans of four workgroups of 256 threads a head (two of 512), in one launch: 2^22 heads are too many."""
    many = dict(L=1, Dk=8, Dv=256)
    for op in (h3.OP_DELTA, h3.OP_DELTA_SAVED, h3.OP_DELTA_BWD):
        assert size(op, B=1 << 19, H=8, **many) == 0
        assert size(op, B=(1 << 22) - 1, H=1, **many) > 0
        assert size(op, B=1 << 21, L=256, H=1, Dk=128, Dv=8) == 0       # 2^23 chunks, their gradients by 512 threads each
    assert rule(B=1 << 19, H=8, Hk=8, wsb=1 << 62, **many) == EUNSUP
    assert bwd(B=1 << 19, H=8, Hk=8, savedb=1 << 62, wsb=1 << 62, **many) == EUNSUP
    for waves in range((1 << 26) - 3, (1 << 26) + 1):                   # 2^24 workgroups of 256 threads
        assert step(B=waves, H=1, Hk=1, Dk=8, Dv=8, o=O << 8) == EUNSUP
    assert step(B=(1 << 26) - 4, H=1, Hk=1, Dk=8, Dv=8, o=V) == EINVAL  # not too many: refused for its output


def test_workspace_of_the_norm():
    """A partial row of dw and one of db for each of at most 512 workgroups."""
    for rows in (1, 511, 512, 513, 1 << 20):
        assert size(h3.OP_LAYERNORM_BWD, B=rows, H=768) == min(rows, 512) * 2 * 768 * 4


def test_sizes_beyond_an_int():
    """A size of 2^32 + 8 would reach the C entry as 8."""
    one = torch.empty(1, dtype=torch.float16)
    for shape in ((1, 2 ** 32 + 8), (2 ** 31, 1), (1, 2 ** 32 + 64, 1, 8), (1, 1, 2 ** 32 + 1, 8)):
        with pytest.raises(ValueError):
            h3._sizes("x", one.expand(shape))
    for shape in ((), (0,), (0, 2 ** 31 - 1), (2 ** 31 - 1, 2 ** 20)):
        h3._sizes("x", one.reshape(()) if shape == () else one.expand(shape))
