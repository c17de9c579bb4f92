"""The gated delta rule on sequences that are cut into segments, forward and backward, for
every size of the keys' tiles, with workgroups of four and of eight waves.  Tolerances are those of the
uncut form: a segment's map is a product of contractions, off by what its chunks are off by."""
import pytest
import torch

import paper_2212_14052_amd as h3
from tests import test_gpu_delta_bwd as bwd, test_gpu_delta_rule as fwd
from tests.test_gpu_delta_rule import DTYPES

pytestmark = pytest.mark.gpu
CODES = {"f32": h3.F32, "f16": h3.F16, "bf16": h3.BF16}
up = lambda n, to: -(-n // to) * to


def uncut_bytes(B, H, L, Dk, Dv, dtype):
    """Workspaces of the two passes without segments: records (four 6 KB matrices, 800 bytes of gates), keys and
    queries; z, the states' gradients, 16 scales a chunk."""
    chunks, dkp, dvp = B * H * -(-L // 64), up(Dk, 32), up(Dv, 16)
    records, keys = up(chunks * (4 * 6144 + 800), 256), up(chunks * 2 * (2 if dtype == "f32" else 1) * 64 * dkp * 2, 256)
    return records + keys, up(chunks * 64 * dvp * 4, 256) + up(chunks * dkp * dvp * 4, 256) + up(chunks * 16 * 16, 256)


FOUR = [(1, 1500, 1, 1, 8, 8), (2, 1500, 2, 1, 40, 72), (2, 1480, 2, 2, 96, 40), (2, 1500, 2, 1, 128, 128)]
EIGHT = [(2, 2048, 8, 4, 32, 256), (2, 2000, 8, 8, 64, 256), (2, 2048, 8, 8, 96, 256), (2, 2048, 16, 16, 128, 128)]   # of 16-bit inputs


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,L,H,Hk,Dk,Dv", FOUR + EIGHT)
def test_segments(B, L, H, Hk, Dk, Dv, dtype):
    sizes = (B, H, L, Dk, Dv)
    for op, uncut in zip((h3.OP_DELTA, h3.OP_DELTA_BWD), uncut_bytes(*sizes, dtype)):
        assert h3.workspace_size(op, *sizes, CODES[dtype]) > uncut   # there are segments
    q, k, v, g, beta, S0, do, dS = bwd.full_inputs(B, L, H, Hk, Dk, Dv, dtype, 31)
    fwd.run_and_check(dtype, q, k, v, g, beta, S0)
    bwd.run_and_check(dtype, q, k, v, g, beta, S0, do, dS)
    if B == 2:   # ends in the first, a middle and the last segment; whole segments behind them; nothing at all
        for n in (0, 70, L // 2, L - 65):
            lengths = torch.tensor([L, n], device="cuda", dtype=torch.int32)
            fwd.run_and_check(dtype, q, k, v, g, beta, S0, None, lengths)
        lengths = torch.tensor([L - 700, 130], device="cuda", dtype=torch.int32)
        got = bwd.run_and_check(dtype, q, k, v, g, beta, S0, do, dS, None, lengths)
        behind = torch.arange(L, device="cuda")[None] >= lengths[:, None]
        assert all((t[behind] == 0).all() for t in got[:5])


def test_decays_that_empty_segments():
    """The state is dropped at the start of a segment, in the middle of one, and all through another."""
    q, k, v, g, beta, S0, do, dS = bwd.full_inputs(1, 1536, 2, 2, 64, 64, "f32", 32)   # six segments of 256 tokens
    g[:, 256], g[:, 700], g[:, 1024:1280] = -float("inf"), -1e30, -200.0
    fwd.run_and_check("f32", q, k, v, g, beta, S0)
    bwd.run_and_check("f32", q, k, v, g, beta, S0, do, dS)


def test_segments_repeat_in_a_graph_on_another_stream():
    args = bwd.full_inputs(2, 1500, 2, 1, 128, 128, "bf16", 33)
    want = [t.clone() for t in bwd.grads_of(*args)]
    o, S = (t.clone() for t in h3.delta_rule(*args[:5], S0=args[5]))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, fwd2 = bwd.grads_of(*args), h3.delta_rule(*args[:5], S0=args[5])
    side = torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(side):
            graph.replay()
            eager = bwd.grads_of(*args)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(a, b) for a, b in zip(eager, want))
        assert torch.equal(fwd2[0], o) and torch.equal(fwd2[1], S)
