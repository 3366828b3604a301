"""The operators of a layer of experts where tiles, groups and storage meet awkwardly, against 64 bits.  Bounds are those of
test_gpu_experts.py."""
import pytest
import torch

import paper_1505_04956_b200 as pkg
from paper_1505_04956_b200 import binding

from .test_gpu_experts import BF, E4, E5, F16, F32, HALF_STEP, SMALLEST, U, _check_product, _close, _gen, _loads, _operand, _values64

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


# ---------------------------------------------------------------------------------------------------------------
# products: scales and groups that start anywhere
# ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("M, N, K, G", [(37, 136, 512, 3), (203, 264, 512, 4), (1900, 520, 256, 3), (2700, 1100, 1024, 3)])
@pytest.mark.parametrize("first", [0, 1, 2, 3])
def test_scales_and_groups_that_start_anywhere(M, N, K, G, first):
    # the scales lie `first` numbers behind a 16-byte boundary, block after block a whole number of 16 bytes apart, and the
    # groups start at rows of every remainder by 4: a tile's scales are aligned where the array of them is not
    a, sa = _operand(M, K, E4, 1)
    b, sb = _operand(N, K, E4, 2, True, (G,))
    store = torch.zeros(K // 128 * 4096 + 8, device="cuda")
    moved = store[first:first + K // 128 * 4096].view(K // 128, 4096)[:, :M].t()
    moved.copy_(sa)
    assert moved.data_ptr() % 16 == 4 * first
    for start in range(4):
        at = torch.linspace(start, M, G + 1).to(torch.int32)
        at[1:-1] = at[1:-1] // 4 * 4 + (4 - first) % 4
        offsets = at.cuda()
        got = pkg.asgd_product(a, moved, b, sb, offsets=offsets, out=torch.zeros(M, N, device="cuda"))
        want = pkg.asgd_product(a, sa, b, sb, offsets=offsets, out=torch.zeros(M, N, device="cuda"))
        assert torch.equal(got, want)
        a64, b64, rows = _values64(a, sa), _values64(b, sb), at.tolist()
        for g in range(G):
            s = slice(rows[g], rows[g + 1])
            _check_product(got[s], a64[s], b64[g], K, F32)
    pkg.asgd_experts_sync()


# ---------------------------------------------------------------------------------------------------------------
# products: the most rows and columns
# ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("by_groups", [False, True])
def test_products_of_the_most_rows_and_columns(by_groups):
    n = 2 ** 31 - 256                                    # 34 GB of rows of 16 numbers
    long = torch.zeros(n, 16, dtype=torch.uint8, device="cuda")
    scale = torch.ones(n, 1, device="cuda")
    a, sa = _operand(300, 16, E4, 1)
    long[-300:] = a.view(torch.uint8)
    scale[-300:] = sa
    b, sb = _operand(1, 16, E4, 2)
    a64, b64 = _values64(a, sa), _values64(b, sb)
    out = torch.full((n, 1), 5.0, device="cuda")
    if by_groups:
        offsets = torch.tensor([0, 7, 7, n], dtype=torch.int32, device="cuda")
        pkg.asgd_product(long.view(E4), scale, b.view(torch.uint8).expand(3, 1, 16).contiguous().view(E4), sb.expand(3, 1, 1), offsets=offsets, out=out)
    else:
        pkg.asgd_product(long.view(E4), scale, b, sb, out=out)
    pkg.asgd_experts_sync()
    _check_product(out[-300:], a64, b64, 16, F32)
    assert int(out[:-300].count_nonzero()) == 0
    if by_groups:
        return
    out.fill_(5.0)
    pkg.asgd_product(b, sb, long.view(E4), scale, out=out.view(1, n))
    pkg.asgd_experts_sync()
    _check_product(out.view(1, n)[:, -300:], b64, a64, 16, F32)
    assert int(out[:-300].count_nonzero()) == 0


# ---------------------------------------------------------------------------------------------------------------
# reports
# ---------------------------------------------------------------------------------------------------------------

def test_no_report_is_lost_while_another_is_taken():
    # a wait that runs out on one stream, while calls on another stream report offsets that cut a block and are taken one
    # after the other: whichever call takes it, the timeout (the worse status) is seen
    a, sa = _operand(8, 1024, E4, 1)
    b, sb = _operand(512, 1024, E4, 2, True)
    u, su = _operand(16, 400, E4, 3)
    cut = torch.tensor([0, 100, 400], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    pkg.asgd_product(a, sa, b, sb)
    pkg.asgd_product_inner(u, su, u, su, cut[::2].contiguous())
    torch.cuda.synchronize()
    try:
        pkg.asgd_experts_sync()
    except binding.AsgdError:
        pass

    def take(stream=None):
        try:
            pkg.asgd_experts_sync(stream)
            return binding.ASGD_OK
        except binding.AsgdError as err:
            return err.status
    for _ in range(40):
        try:
            pkg.asgd_product_set_wait_drill(2000, True)
            pkg.asgd_product(a, sa, b, sb, stream=side)
        finally:
            pkg.asgd_product_set_wait_drill()
        seen, turns = [], 0
        while not side.query():
            pkg.asgd_product_inner(u, su, u, su, cut)
            seen.append(take())
            turns += 1
            assert turns < 10 ** 6
        seen.append(take(side))
        assert binding.ASGD_ETIMEOUT in seen             # (each of the call's blocks reports: more than one may see it)
        assert all(s == binding.ASGD_EINVAL for s in seen[:-1] if s != binding.ASGD_ETIMEOUT)
    assert take() == binding.ASGD_OK


# ---------------------------------------------------------------------------------------------------------------
# routing
# ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F32, BF, F16])
@pytest.mark.parametrize("E, top_k", [(12, 12), (40, 8), (200, 16), (1000, 32)])
def test_sigmoid_gradient_of_large_logits(E, top_k, dtype):
    # dx = scale * dw * s * (1 - s), relative to itself: both sigmoids (exponential 4 u, sum and reciprocal 1 u each), three
    # products and the factor scale * dw stay below 32 u
    g = _gen(E)
    T = 60
    size = 10 + 20 * torch.rand(T, E, generator=g, device="cuda")
    x = torch.where(torch.rand(T, E, generator=g, device="cuda") < 0.5, size, -size).to(dtype)
    ids = torch.rand(T, E, generator=g, device="cuda").argsort(dim=1)[:, :top_k].to(torch.int32).contiguous()
    dw = torch.randn(T, top_k, generator=g, device="cuda")
    got = pkg.asgd_route_grad(x, ids, dw, score="sigmoid", renormalise=False, scale=1.5)
    z = x.double()
    want = torch.zeros_like(z).scatter(1, ids.long(), 1.5 * dw.double()) / ((1 + torch.exp(-z)) * (1 + torch.exp(z)))
    _close(got, want, (32 * U + HALF_STEP[dtype]) * want.abs() + SMALLEST[dtype])
