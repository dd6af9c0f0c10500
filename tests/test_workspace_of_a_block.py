"""CPU-only: a block's backward passes share one workspace (LayerBuffers.workspace), also where the experts' backward recomputes H and A."""
import pytest

from paper_2112_14397_amd import binding as B


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,d,E,F,P", [(5000, 4096, 1, 64, 1), (4096, 1024, 2, 64, 16), (300, 8192, 64, 64, 300), (18220, 448, 49, 224, 9000)])
def test_one_workspace_for_all_of_them(dtype, T, d, E, F, P):
    s = B.make_shape(T, d, E, F, dtype, "gelu", P)
    norm = min(-(-T // 16), 256) * d * 4                      # a row of dgamma to 16 rows, up to 256 of them
    for n in (B.evomoe_workspace_bytes(s), B.evomoe_workspace_bytes_recompute(s)):
        assert n >= norm
