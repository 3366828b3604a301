"""The operators of a layer of experts where tiles, groups and storage meet awkwardly, against 64 bits.  Bounds are those of
test_gpu_experts.py."""
import pytest
import torch

import paper_1505_04956_b200 as pkg

from .test_gpu_experts import BF, E4, E5, F16, F32, _check_product, _loads, _operand, _values64

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------------------------
# products: pairs of blocks that take several tiles in turn (74 pairs)
# ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("G, R, M, N, out, fa", [
    (48, 48 * 128, 600, 520, F32, E4), (48, 48 * 128, 600, 520, BF, E5), (40, 40 * 128, 344, 1032, F16, E4), (64, 64 * 128, 600, 776, F32, E5)])
def test_inner_groups_without_rows_between_full_ones(G, R, M, N, out, fa):
    # 400 to 770 pair tiles; the last tile row is ragged, so that a warp writes C itself right after copies of a whole tile,
    # and a group of nothing has no K block between the two
    a, sa = _operand(M, R, fa, 1)
    b, sb = _operand(N, R, E4, 2)
    at = _loads(G, R, G + M, 128)
    empty = sum(int(p == q) for p, q in zip(at.tolist(), at.tolist()[1:]))
    assert empty >= G // 4
    a64, b64 = _values64(a, sa), _values64(b, sb)
    offsets, at = at.to(torch.int32).cuda(), at.tolist()
    first = None
    for _ in range(4):
        c = torch.full((G, M, N), 7.0, dtype=out, device="cuda")
        pkg.asgd_product_inner(a, sa, b, sb, offsets, out=c)
        if first is None:
            first = c
            for g in range(G):
                s = slice(at[g], at[g + 1])
                _check_product(c[g], a64[:, s], b64[:, s], at[g + 1] - at[g], out)
        assert torch.equal(c, first)
    pkg.asgd_experts_sync()
