"""The layer norm written over its input, and its gradient over either of its own, as the C entry points allow: the
same bits as elsewhere, for every layout of a row."""
import pytest
import torch

import paper_2212_14052_amd as h3

pytestmark = pytest.mark.gpu
TYPES = {torch.float32: h3.F32, torch.float16: h3.F16, torch.bfloat16: h3.BF16}
p = lambda t: None if t is None else t.data_ptr()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d", [(70, 96), (9, 97), (40, 2560), (700, 5120), (5, 9000), (3, 40000), (600, 33001)])
def test_in_place(rows, d, dtype):
    gen = torch.Generator().manual_seed(d)
    r = lambda *s: torch.randn(*s, generator=gen).cuda()
    x, dy, w, b = r(rows, d).to(dtype), r(rows, d).to(dtype), r(d), r(d)
    y, mean, rstd = h3.layernorm(x, w, b)
    dx = h3.layernorm_bwd(dy, x, w, mean, rstd, want_dw=False, want_db=False)[0]
    st, code = torch.cuda.current_stream().cuda_stream, TYPES[dtype]
    over, mean2, rstd2 = x.clone(), torch.empty_like(mean), torch.empty_like(rstd)
    assert h3.lib().h3_layernorm(p(over), p(w), p(b), rows, d, 1e-5, code, p(over), p(mean2), p(rstd2), st) == 0
    assert torch.equal(over, y) and torch.equal(mean2, mean) and torch.equal(rstd2, rstd)
    ws = torch.empty(h3.workspace_size(h3.OP_LAYERNORM_BWD, rows, d, 1, 0, 0, code), dtype=torch.uint8, device="cuda")
    for name in ("dy", "x"):
        ins = {"dy": dy.clone(), "x": x.clone()}
        assert h3.lib().h3_layernorm_bwd(p(ins["dy"]), p(ins["x"]), p(w), p(mean), p(rstd), rows, d, code, p(ins[name]), None,
                                         None, p(ws), ws.numel(), st) == 0
        assert torch.equal(ins[name], dx)
