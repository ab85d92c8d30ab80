"""Gated linear projection at sizes whose products run in 128-wide tiles, forward and
backward, against its plain 64-bit form (bounds in cross_ref.py)."""
import pytest
import torch

import cross_ref as C
import ops_ref as R
from paper_2506_20686_amd import binding as B
from test_gated_linear_gpu import DEV, BF, F4, both, dev, inputs

pytestmark = pytest.mark.gpu

# whole words: [a | b] in 128-wide tiles (272 of them); with dx and dW in one launch, both 128
# wide (102 tiles of dx); dW so and dx in tiles of 64; dx and dW each in a launch of its own; dx
# alone so.  Rows, columns and halves end inside tiles.
WHOLE = [(2050, 136, 1000), (2050, 760, 1000), (2100, 264, 1100), (16500, 200, 200),
         (16500, 200, 136), (2100, 260, 1004)]
# the same of rows that are no whole words
RAGGED = [(2100, 261, 1101), (16500, 201, 203), (16500, 203, 133)]


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("size", WHOLE + RAGGED, ids=str)
def test_forward_and_backward(size, dtype):
    both(*size, (B.ACT_SILU, B.ACT_GELU, B.ACT_SIGMOID)[size[1] % 3], dtype, seed=size[2])


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("size", [(2050, 760, 1000), (16500, 200, 200), (2100, 261, 1101)], ids=str)
def test_results_alone_and_nothing_outside_them(size, dtype):
    m, k, f = size
    x, w, b, dy = inputs(m, k, f, dtype, 1)
    ref, bound = C.gated_bwd(x, w, b, dy, B.ACT_SILU)
    x, w, b, dy = (dev(t) for t in (x, w, b, dy))
    pad, code, L = 64, B.BF16 if dtype == BF else B.F32, B.lib()
    need = B._sized("tri_gated_linear_bwd_workspace_bytes", code, m, k, f)
    ws = torch.full((need + 256,), 9, dtype=torch.uint8, device=DEV)
    s = torch.cuda.current_stream().cuda_stream
    ins = [t.data_ptr() for t in (x, w, b, dy)]
    for which in ((0, 1, 2), (0,), (1,), (2,), (0, 2)):
        big = [torch.full((r.numel() + 2 * pad,), 7.0, dtype=dtype if i == 0 else F4, device=DEV)
               for i, r in enumerate(ref)]
        at = [t.data_ptr() + pad * t.element_size() if i in which else None
              for i, t in enumerate(big)]
        assert L.tri_gated_linear_bwd(code, m, k, f, B.ACT_SILU, *ins, *at, ws.data_ptr(), need,
                                      s) == B.OK
        for i, (t, r, e) in enumerate(zip(big, ref, bound)):
            if i not in which:
                assert bool((t == 7).all())
                continue
            R.check(f"result {i}", t[pad:-pad].view(r.shape), r, e)
            assert bool((t[:pad] == 7).all()) and bool((t[-pad:] == 7).all())
    assert bool((ws[need:] == 9).all())
