"""One token, and one column of the weights, taken out of tensors whose rows lie farther apart than a row stride may be."""
import pytest
import torch

from paper_1705_01626_amd import ffn
from tests import ffn_inputs

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("m,n", [(1, 40), (30, 1), (1, 1)])
@pytest.mark.parametrize("far", [ffn.MAX_COLUMNS + 64, ffn.MAX_COLUMNS * 4 + 3, 75])
def test_single_rows(dtype, m, n, far):
    """Every tensor of one row has that stride; results are those of plain ones, bit for bit."""
    k = 64
    gen = ffn_inputs.generator(m, n, str(dtype))
    base = torch.empty(1 << 16, dtype=dtype, device=DEV)
    used = [0]

    def apart(t):
        if t.shape[0] > 1:
            return t
        out = base.as_strided(t.shape, (far, 1), used[0] * 1024)
        used[0] += 1
        return out.copy_(t)

    make = lambda rows, cols: torch.randn(rows, cols, generator=gen, device=DEV).to(dtype)
    x, wg, wu, dh = make(m, k), make(n, k), make(n, k), make(m, n)
    outs = [torch.empty(m, n, dtype=dtype, device=DEV) for _ in range(3)]
    grads = [torch.empty(m, k, dtype=dtype, device=DEV), *(torch.empty(n, k, dtype=dtype, device=DEV) for _ in range(2))]
    results = []
    for place in (lambda t: t, apart):
        px, pg, pu, ph = (place(t) for t in (x, wg, wu, dh))
        o, g = [place(torch.zeros_like(t)) for t in outs], [place(torch.zeros_like(t)) for t in grads]
        ws = ffn.new_glu_workspace(px, pg, pu, backward=True)
        ffn.zvc_glu_forward(px, pg, pu, o[0], ws, "silu", o[1], o[2], p=0.25, seed=3)
        ffn.zvc_glu_backward(ph, px, pg, pu, *g, ws, "silu", o[1], o[2], p=0.25, seed=3)
        y = place(torch.zeros_like(x))
        ffn.zvc_dropout(px, y, 0.5, 4)
        results.append([t.clone() for t in (*o, *g, y)])
    for a, b in zip(*results):
        assert torch.equal(a, b)
