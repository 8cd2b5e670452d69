"""NaN and infinities in queries and in the paged cache: they reach the rows that see them, however the work is divided, and no others."""
import numpy as np
import pytest
import torch

import paged_plain as pp
from gpu_util import require_gpu

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def b():
    require_gpu()
    from paper_2312_11462_b200 import binding
    return binding


def attend(b, c, q, masks=None):
    """The operator on a filled case, beside the plain form: what is not finite lies in the same places and is the same, the rest is within the
    bound of finite numbers (the scores' size is taken over the finite entries)."""
    out = torch.full((c.total, q[0].shape[1], c.D), -7.0, dtype=c.dtype, device="cuda")
    tm = None if masks is None else torch.tensor(masks + [0] * (c.total - len(masks)), dtype=torch.int64).cuda()
    b.csd_paged_attention(c.packed(q), c.pool, c.batch(), tree_mask=tm, out=out)
    got = out.double().cpu().numpy()
    tame = lambda x: np.where(np.isfinite(x), x, 0.0)  # noqa: E731
    for s, (r, n) in enumerate(zip(c.rows, c.kv)):
        if not r:
            continue
        mine = None if masks is None else masks[c.start[s]:c.start[s + 1]]
        qs, k, v = q[s].to(c.dtype).double().numpy(), c.held(c.keys[s]), c.held(c.vals[s])
        with np.errstate(invalid="ignore"):
            want, size, _ = pp.attention(qs, k, v, n, c.D ** -0.5, mine)
        top = float(np.abs(tame(qs)).sum(-1).max() * np.abs(tame(k)).max() * c.D ** -0.5)
        far, fine = got[c.start[s]:c.start[s + 1]], np.isfinite(want)
        assert np.array_equal(np.isnan(want), np.isnan(far)), (s, int(np.isnan(want).sum()), int(np.isnan(far).sum()))
        assert np.array_equal(np.where(np.isinf(want), want, 0), np.where(np.isinf(far), far, 0)), s
        bound = pp.attention_bound(tame(want), tame(size), top, n + r, c.D, c.dtype)
        assert (np.abs(np.where(fine, far, 0) - tame(want)) <= bound).all(), s
    assert b.csd_device_status() == 0
    return got


# items with CTAs of their own, and items that lie in parts of a tile each and of several
DIVISIONS = [((40, 40), (30, 100), 2, 1), ((300,), (20,), 4, 2), ((40,), (985,), 1, 1), ((300,), (2005,), 4, 2), ((70, 129), (6075, 4096), 2, 1)]


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rows,kv,heads,kv_heads", DIVISIONS)
def test_a_query_with_a_nan(b, kind, dim, rows, kv, heads, kv_heads):
    """Its head's row is NaN, whole or in parts; all others are what they are without it."""
    c = pp.Case(b, rows, kv, kv_heads, dim, 32, kind, BF16, seed=sum(rows))
    c.fill()
    g = torch.Generator().manual_seed(5)
    q = [torch.randn(r, heads, dim, generator=g) for r in rows]
    for x in q:
        x[len(x) // 3, 0, 7] = float("nan")
        x[-1, -1] = float("nan")
    got = attend(b, c, q)
    for s, x in enumerate(q):
        assert np.isnan(got[c.start[s] + len(x) // 3, 0]).all() and np.isnan(got[c.start[s + 1] - 1, -1]).all()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,kv,heads,kv_heads", [((40,), (985,), 1, 1), ((40,), (89,), 1, 1), ((300,), (1877,), 2, 2), ((33, 65), (3040, 1600), 2, 2), ((1,), (2048,), 1, 1),
                                                    ((7,), (1530,), 2, 1)])
def test_a_nan_that_is_the_only_key_of_a_part(b, kind, dtype, rows, kv, heads, kv_heads):
    """The newest position is the first of a tile of keys and a NaN: its own row, which sees nothing else in that tile, is NaN."""
    c = pp.Case(b, rows, kv, kv_heads, 128, 64, kind, dtype, seed=sum(kv))
    for k in c.keys:
        k[-1, :, 3] = float("nan")
    c.fill()
    g = torch.Generator().manual_seed(6)
    q = [torch.randn(r, heads, 128, generator=g) for r in rows]
    got = attend(b, c, q)
    for s in range(len(rows)):
        assert np.isnan(got[c.start[s + 1] - 1]).all() and not np.isnan(got[c.start[s]:c.start[s + 1] - 1]).any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rows,kv,heads,kv_heads,tree", [((1, 1), (40, 500), 2, 1, False), ((5, 3), (300, 77), 4, 4, False), ((9, 12), (20, 0), 4, 2, True),
                                                         ((60,), (700,), 2, 1, False), ((300,), (2005,), 2, 2, False),
                                                         ((1, 2), (600, 20), 8, 4, False)])
def test_infinite_keys(b, dtype, dim, rows, kv, heads, kv_heads, tree):
    """A score of -inf is no weight, one of +inf makes its row NaN, whatever terms a query enters the products in."""
    c = pp.Case(b, rows, kv, kv_heads, dim, 16, "bf16", dtype, seed=3)
    for k, n in zip(c.keys, c.kv):
        k[2 * len(k) // 3, 0, 1] = float("inf")
        k[len(k) // 4, -1, 2] = -float("inf")
        k[-1, 0, dim - 1] = float("inf")
    c.fill()
    masks = pp.trees(rows, 9) if tree else None
    g = torch.Generator().manual_seed(7)
    q = [torch.randn(r, heads, dim, generator=g) for r in rows]
    for x in q:                                       # (most rows: scores of -inf alone)
        x[..., [1, dim - 1]] = -x[..., [1, dim - 1]].abs()
        x[..., 2].abs_()
        x[len(x) // 2, 0, 1] = 1.7
        x[-1, -1, 2] = -0.3
    got = attend(b, c, q, masks)
    assert np.isnan(got[:c.start[-1]]).any()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,heads", [(1, 1), (3, 2), (20, 1), (50, 2)])
def test_a_nan_of_hardly_any_weight(b, kind, dtype, rows, heads):
    """Values that are NaN reach every row that sees them, also where the weight is below fp32's range."""
    c = pp.Case(b, (rows,), (700,), 1, 128, 32, kind, dtype, seed=rows)
    c.keys[0][5] = -30.0
    c.vals[0][5] = float("nan")
    c.fill()
    got = attend(b, c, [torch.ones(rows, heads, 128)])
    assert np.isnan(got[:rows]).all()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("dim", [64, 128])
def test_blocks_of_two_halves_before_blocks_of_one(b, kind, dim):
    """A CTA's run of many short items: what is not a number in the last tiles of a block of 200 rows reaches its second half's rows, however long
    the three blocks of 36 rows behind it, which have no second half, run ahead."""
    rows, kv = (200, 36, 36, 36) * 100, tuple(n for i in range(100) for n in ((7 * i) % 130, 90, 0, (5 * i) % 220))
    c = pp.Case(b, rows, kv, 1, dim, 16, kind, BF16, seed=dim)
    for s in range(0, 400, 4):
        n = kv[s]
        c.vals[s][n + 150, 0, 5] = float("nan")
        if kind == "bf16":
            c.vals[s][n + 199, 0, dim - 1], c.vals[s][n + 130, 0, 8] = float("inf"), -float("inf")
    c.fill()
    g = torch.Generator().manual_seed(8)
    q = [torch.randn(r, 1, dim, generator=g) for r in rows]
    got = attend(b, c, q)
    for s in range(0, 400, 4):
        mine = got[c.start[s]:c.start[s + 1], 0, 5]
        assert not np.isnan(mine[:150]).any() and np.isnan(mine[150:]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_what_an_8_bit_row_may_hold(b, dtype):
    """Whatever is appended, a row's byte is 27 to 247 and none of its numbers is NaN, or the byte is 255."""
    g = torch.Generator().manual_seed(4)
    x = torch.randn(400, 3, 64, generator=g) * torch.exp2(torch.randint(-149, 128, (400, 3, 1), generator=g).float())
    x[::7, 0, 5], x[::11, 1, 6], x[::13, 2, 7] = float("inf"), -float("inf"), float("nan")
    x[5], x[6], x[7], x[8] = 0.0, torch.finfo(F32).max, 480.0, -torch.finfo(F32).max
    c = pp.Case(b, (400,), (0,), 3, 64, 16, "e4m3", dtype, pad_rows=0)
    c.keys, c.vals = [x.to(dtype)], [(-x).to(dtype)]
    c.fill()
    at = torch.arange(400)
    page, slot = c.table[0, at // 16].long(), at % 16
    for rows, exps, given in ((c.pool.k, c.pool.k_exp, c.keys[0]), (c.pool.v, c.pool.v_exp, c.vals[0])):
        numbers, e = rows.view(torch.uint8).cpu()[page, :, slot].int(), exps.cpu()[page, :, slot].int()
        odd = given.isnan().any(-1)
        assert (e[odd] == 255).all() and ((e[~odd] >= 27) & (e[~odd] <= 247)).all() and ((numbers[~odd] & 0x7F) != 0x7F).all()
    assert b.csd_device_status() == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,kv", [(1, 0), (3, 40), (40, 985), (300, 20)])
def test_rows_whose_every_score_is_no_weight(b, dtype, rows, kv):
    """Scores of -inf alone: 0, like a row that sees nothing, whole or in parts."""
    c = pp.Case(b, (rows,), (kv,), 1, 64, 16, "bf16", dtype, seed=kv)
    c.keys[0][..., 3] = -float("inf")
    c.fill()
    out = b.csd_paged_attention(c.packed([torch.randn(rows, 2, 64).abs()]), c.pool, c.batch())
    assert (out[:rows] == 0).all() and b.csd_device_status() == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rows,kv,heads,tree", [((1, 3), (40, 700), 2, False), ((7, 5), (30, 0), 2, True), ((20,), (300,), 1, False), ((60, 40), (50, 985), 2, False)])
def test_a_nan_behind_a_score_of_no_weight(b, dtype, dim, rows, kv, heads, tree):
    """A position whose key gives -inf and whose value is NaN: every row that sees it is NaN there, in tiles that all rows see and in those that
    some see, whole or in parts; the others are not."""
    c = pp.Case(b, rows, kv, 1, dim, 16, "bf16", dtype, seed=dim)
    for k, v in zip(c.keys, c.vals):
        for at in (len(k) // 5, len(k) - 1 - len(k) // 20):
            k[at, 0, 3], v[at, 0, 9] = -float("inf"), float("nan")
    c.fill()
    g = torch.Generator().manual_seed(2)
    attend(b, c, [torch.randn(r, heads, dim, generator=g).abs() for r in rows], pp.trees(rows, 4) if tree else None)
