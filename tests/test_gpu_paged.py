"""The paged cache and the attention over it against plain 64-bit forms, at the sizes and masks where they can go wrong."""
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


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,kv,heads,dim,page", [((1,), (0,), 1, 64, 16), ((3, 0, 5), (15, 4, 31), 3, 128, 16), ((40, 1), (0, 129), 5, 64, 64),
                                                    ((17, 2, 33, 9), (100, 63, 0, 128), 2, 128, 128), ((2,) * 70, tuple(range(70)), 2, 64, 32)])
def test_append_and_read(b, kind, dtype, rows, kv, heads, dim, page):
    c = pp.Case(b, rows, kv, heads, dim, page, kind, dtype, seed=len(rows) + dim, lead_rows=1)
    new = c.fill()
    whole = [r + n for r, n in zip(rows, kv)]
    start = np.concatenate([[0], np.cumsum(whole)])
    everything = b.PagedBatch(c.table.cuda(), torch.tensor(start, dtype=torch.int32).cuda(), torch.zeros(len(rows), dtype=torch.int32).cuda(),
                              int(start[-1]), max(whole))
    for out_type in (F32, BF16):
        got = b.csd_paged_read(c.pool, everything, out_type)
        for g, parts in zip(got, (c.keys, c.vals)):
            want = np.concatenate([c.held(p) for p in parts])
            assert np.array_equal(g.double().cpu().numpy(), want)          # both are exact in 16 bits
    # only the batch's rows are written, whatever lies around them
    out = tuple(torch.full((c.total, heads, dim), -7.0, dtype=dtype, device="cuda") for _ in range(2))
    b.csd_paged_read(c.pool, new, dtype, out)
    for g, parts in zip(out, (c.keys, c.vals)):
        g = g.double().cpu().numpy()
        assert (g[:c.start[0]] == -7).all() and (g[c.start[-1]:] == -7).all()
        for s, p in enumerate(parts):
            assert np.array_equal(g[c.start[s]:c.start[s + 1]], c.held(p)[kv[s]:])
    # slots that no sequence has are as they were
    used = torch.zeros(c.pool.k.shape[0] * page, dtype=torch.bool)
    for s, n in enumerate(whole):
        t = torch.arange(n)
        used[c.table[s, t // page].long() * page + t % page] = True
    raw = c.pool.k.view(torch.uint8).cpu().view(-1, heads, page, dim * c.pool.k.element_size()).transpose(1, 2).reshape(len(used), -1)
    assert (raw[~used] == 0xFF).all() and b.csd_device_status() == 0


def test_rows_of_every_size(b):
    """Zeros, the largest and smallest numbers, infinities, NaN, ties, each row with its own scale."""
    x = torch.randn(64, 2, 64)
    x[0] = 0
    x[1] *= 1e37
    x[2] *= 1e-38
    x[3, :, 5] = float("inf")
    x[4, :, 6] = -float("inf")
    x[5, :, 7] = float("nan")
    x[6] = float("nan")
    x[7] = 448.0
    x[8] = torch.nextafter(torch.tensor(448.0), torch.tensor(1e9))
    x[9] = torch.finfo(F32).max
    x[10] = 2.0 ** -149
    x[11:40] = (torch.arange(29 * 128).view(29, 2, 64) % 512) * 2.0 ** -6          # ties
    c = pp.Case(b, (64,), (0,), 2, 64, 16, "e4m3", F32)
    c.keys, c.vals = [x], [-x]
    new = c.fill()
    for g, parts in zip(b.csd_paged_read(c.pool, new, F32), (c.keys, c.vals)):
        g, want = g[:64].double().cpu().numpy(), c.held(parts[0])
        assert np.array_equal(np.isnan(g), np.isnan(want)) and np.array_equal(g[~np.isnan(g)], want[~np.isnan(want)])
    _, e = pp.quantise(x.double().numpy())
    at = torch.arange(64)
    e = np.where(np.isnan(x.numpy()).any(-1), 128, e)
    assert np.array_equal(c.pool.k_exp.cpu()[c.table[0, at // 16].long(), :, at % 16].numpy().astype(int) - 127, e)


def attend(b, c, heads, scale=None, masks=None, seed=1, wide=0, ws=None):
    """Runs the operator on a case that has been filled and compares it; returns the output."""
    g = torch.Generator().manual_seed(seed)
    q = [torch.randn(r, heads, c.D, generator=g) * 1.5 for r in c.rows]
    packed = c.packed(q)
    if wide:                                       # rows of a wider buffer
        buf = torch.full((c.total, wide + heads * c.D), float("nan"), dtype=c.dtype, device="cuda")
        buf[:, 8:8 + heads * c.D] = packed.view(c.total, -1)
        packed = buf[:, 8:8 + heads * c.D].unflatten(1, (heads, c.D))
    out = torch.full((c.total, heads, c.D), -7.0, dtype=c.dtype, device="cuda")
    tm = None
    if masks is not None:
        tm = torch.zeros(c.total, dtype=torch.int64)
        tm[c.start[0]:c.start[-1]] = torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], dtype=torch.int64)
        tm = tm.cuda()
    new = c.batch()
    b.csd_paged_attention(packed, c.pool, new, scale, tm, ws, out)
    got = out.double().cpu().numpy()
    assert (got[:c.start[0]] == -7).all() and (got[c.start[-1]:] == -7).all()
    compare(c, got, q, c.D ** -0.5 if scale is None else scale, masks)
    return out


def compare(c, got, q, scale, masks):
    for s, r in enumerate(c.rows):
        if not r:
            continue
        mine = None if masks is None else masks[c.start[s] - c.start[0]:c.start[s + 1] - c.start[0]]
        want, size, top = pp.attention(q[s].to(c.dtype).double().numpy(), c.held(c.keys[s]), c.held(c.vals[s]), c.kv[s], scale, mine)
        far = np.abs(got[c.start[s]:c.start[s + 1]] - want)
        bound = pp.attention_bound(want, size, top, c.kv[s] + r, c.D, c.dtype)
        assert (far <= bound).all(), (s, float((far - bound).max()), float(far.max()))


SHAPES = [((1,), (0,), 1, 1), ((1,), (203,), 12, 12), ((5, 3, 5), (128, 77, 301), 4, 4), ((1, 1, 1, 1), (15, 16, 17, 0), 8, 2), ((17, 0, 1), (63, 9, 64), 7, 1),
          ((16, 31, 33), (0, 1, 1000), 4, 2), ((60,), (5,), 14, 2), ((130, 2), (100, 700), 2, 1), ((1,) * 40, tuple(range(0, 400, 10)), 4, 4)]


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (128, 16), (64, 128)])
@pytest.mark.parametrize("rows,kv,heads,kv_heads", SHAPES)
def test_attention(b, kind, dtype, dim, page, rows, kv, heads, kv_heads):
    c = pp.Case(b, rows, kv, kv_heads, dim, page, kind, dtype, seed=sum(kv) + dim, lead_rows=1)
    c.fill()
    attend(b, c, heads)
    assert b.csd_device_status() == 0


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rows,kv,heads,kv_heads", [((20,), (6000,), 8, 2), ((300,), (2000,), 4, 2), ((40, 0, 1, 70), (900, 5, 0, 3000), 4, 2), ((129,), (4000,), 2, 1),
                                                    ((33,) * 37, (70,) * 36 + (150,), 4, 4), ((33,) * 38, (70,) * 38, 4, 4), ((34, 0, 3) * 12, (5, 9, 300) * 12, 6, 6),
                                                    ((50, 36), (0, 1200), 1, 1), ((1, 400), (2500, 2500), 2, 2)])
def test_chunks_whole_and_in_parts(b, kind, dim, rows, kv, heads, kv_heads):
    """Blocks of many rows whose items have CTAs of their own, and those that lie in up to dozens of parts; twice on one workspace."""
    c = pp.Case(b, rows, kv, kv_heads, dim, 32, kind, BF16, seed=sum(rows) + dim, lead_rows=2)
    c.fill()
    ws = b.csd_paged_attention_workspace(c.pool, c.batch(), heads, BF16)
    ws[4096:] = 0xff                                   # (what is behind the tickets may be anything)
    one = attend(b, c, heads, ws=ws)
    assert torch.equal(one.nan_to_num(), attend(b, c, heads, ws=ws).nan_to_num())
    assert b.csd_device_status() == 0


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,kv,heads,kv_heads", [((12, 5, 1), (77, 0, 300), 4, 4), ((64, 33), (0, 40), 4, 2), ((17,), (16,), 8, 1)])
def test_trees(b, kind, dtype, rows, kv, heads, kv_heads):
    c = pp.Case(b, rows, kv, kv_heads, 128, 32, kind, dtype, seed=sum(rows))
    c.fill()
    attend(b, c, heads, masks=pp.trees(rows, 3))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_that_see_nothing(b, dtype):
    """Empty masks behind an empty cache give zeros, behind a cache what the cache gives."""
    rows, kv = (6, 40, 4), (0, 0, 20)
    c = pp.Case(b, rows, kv, 2, 64, 16, "bf16", dtype)
    c.fill()
    out = attend(b, c, 4, masks=pp.trees(rows, 5, empty=(0, 3, 5, 10, 44, 47)))
    assert (out[[0, 3, 5, 10, 44]] == 0).all()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,kv,heads,kv_heads,dim,tree", [((6, 5), (40, 0), 4, 2, 128, False), ((7,), (9,), 2, 2, 64, True), ((300, 40), (30, 500), 4, 2, 128, False),
                                                             ((150,), (0,), 4, 1, 64, False)])
def test_odd_numbers_stay_with_the_rows_that_see_them(b, kind, dtype, rows, kv, heads, kv_heads, dim, tree):
    """Infinities and NaN in keys and values of new rows: rows that do not see them are what they are without them."""
    c = pp.Case(b, rows, kv, kv_heads, dim, 16, kind, dtype, seed=7)
    masks = pp.trees(rows, 11) if tree else None
    g = torch.Generator().manual_seed(3)
    q = [torch.randn(r, heads, dim, generator=g) for r in rows]
    first = [3 * r // 5 for r in rows]                     # rows before this one see none of them
    for s, (r, n) in enumerate(zip(rows, kv)):
        at = n + first[s]
        c.vals[s][at, 0, 5], c.vals[s][at, 0, 6] = float("nan"), float("inf")
        if kind == "bf16":
            c.vals[s][at + 1, -1, 9], c.vals[s][n + r - 1, 0, dim - 1] = -float("inf"), float("inf")
        c.keys[s][n + r - 1, -1, 0] = float("nan")
    c.fill()
    out = torch.full((c.total, heads, dim), -7.0, dtype=dtype, device="cuda")
    tm = torch.tensor(masks + [0] * (c.total - len(masks)), dtype=torch.int64).cuda() if tree else None
    b.csd_paged_attention(c.packed(q), c.pool, c.batch(), tree_mask=tm, out=out)
    got = out.double().cpu().numpy()
    for s, (r, n) in enumerate(zip(rows, kv)):
        mine = None if masks is None else masks[c.start[s]:c.start[s + 1]]
        with np.errstate(invalid="ignore"):
            want, size, top = pp.attention(q[s].to(dtype).double().numpy(), c.held(c.keys[s]), c.held(c.vals[s]), n, dim ** -0.5, mine)
        far = got[c.start[s]:c.start[s + 1]]
        fine = np.isfinite(want)
        assert np.array_equal(fine, np.isfinite(far)) and np.array_equal(np.isnan(want), np.isnan(far))
        assert np.array_equal(want[~fine & ~np.isnan(want)], far[~fine & ~np.isnan(want)])
        assert fine[:first[s]].all() or tree
        top = 40.0                                        # (scores of finite keys here are far below; the plain form's bound is NaN)
        bound = pp.attention_bound(np.where(fine, want, 0), np.where(fine, size, 0), top, n + r, dim, dtype)
        assert (np.abs(np.where(fine, far, 0) - np.where(fine, want, 0)) <= bound).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale,amplitude", [(0.0, 1.0), (-0.2, 1.0), (3.0, 1.0), (1.0, 12.0)])
def test_scales(b, dtype, scale, amplitude):
    """No weight on the scores, negative ones, and softmaxes that a few keys decide, with maxima that keep growing."""
    c = pp.Case(b, (5, 20), (300, 90), 2, 128, 16, "bf16", dtype, amplitude=amplitude)
    c.keys = [k * torch.linspace(0.2, 1.5, len(k))[:, None, None].to(k.dtype) for k in c.keys]
    c.fill()
    attend(b, c, 4, scale)


def test_strides_and_a_kept_workspace(b):
    """Query rows inside wider rows; one workspace for calls of different shapes."""
    ws = None
    for i, (rows, kv, heads, kv_heads, dim, dtype) in enumerate([((3, 9), (900, 40), 8, 2, 128, BF16), ((1,), (2000,), 4, 4, 64, F32), ((3, 9), (900, 40), 8, 2, 128, BF16),
                                                                ((200,), (50,), 4, 2, 128, BF16), ((1, 1), (3000, 5), 2, 1, 128, BF16)]):
        c = pp.Case(b, rows, kv, kv_heads, dim, 64, "bf16", dtype, seed=i)
        c.fill()
        need = b.csd_paged_attention_workspace(c.pool, c.batch(), heads, dtype)
        ws = need if ws is None else torch.cat([ws, torch.zeros(max(need.numel() - ws.numel(), 0), dtype=torch.uint8, device="cuda")])
        one = attend(b, c, heads, wide=24, ws=ws)
        two = attend(b, c, heads, ws=ws)
        assert torch.equal(one.nan_to_num(), two.nan_to_num())


def test_same_inputs_same_bits(b):
    for rows, kv, heads, kv_heads, dtype in [((5,) * 8, tuple(range(100, 2100, 250)), 8, 8, BF16), ((1,) * 3, (5000, 70, 900), 4, 2, F32), ((150,), (3000,), 4, 2, BF16)]:
        c = pp.Case(b, rows, kv, kv_heads, 128, 16, "bf16", dtype)
        c.fill()
        q = c.packed([torch.randn(r, heads, 128) for r in rows])
        ws = b.csd_paged_attention_workspace(c.pool, c.batch(), heads, dtype)
        outs = [b.csd_paged_attention(q, c.pool, c.batch(), workspace=ws)[:sum(rows)] for _ in range(20)]
        assert all(torch.equal(o, outs[0]) for o in outs)


def test_bad_pages_and_lengths(b):
    """Page ids outside the pool: their positions are written nowhere, read back as zeros and seen by nobody."""
    for dtype in (F32, BF16):
        c = pp.Case(b, (4, 3), (60, 5), 2, 64, 16, "bf16", dtype)
        c.fill()
        assert b.csd_device_status() == 0
        good = c.table.clone()
        c.table[0, 1] = c.pool.k.shape[0]              # positions 16 .. 31 of sequence 0
        before = c.pool.k.clone().view(torch.int16)
        q = [torch.randn(r, 2, 64) for r in c.rows]
        out = torch.full((c.total, 2, 64), -7.0, dtype=dtype, device="cuda")
        b.csd_paged_attention(c.packed(q), c.pool, c.batch(), out=out)
        assert b.csd_device_status() == 9
        want, size, top = pp.attention(q[0].to(dtype).double().numpy(), c.held(c.keys[0]), c.held(c.vals[0]), 60, 64 ** -0.5, hide=range(16, 32))
        assert (np.abs(out[:4].double().cpu().numpy() - want) <= pp.attention_bound(want, size, top, 64, 64, dtype)).all()
        read = b.PagedBatch(c.table.cuda(), torch.tensor([0, 64, 64], dtype=torch.int32).cuda(), torch.zeros(2, dtype=torch.int32).cuda(), 64, 64)
        k, _ = b.csd_paged_read(c.pool, read, F32)
        assert b.csd_device_status() == 9 and (k[16:32] == 0).all() and np.array_equal(k.double().cpu().numpy()[32:], c.held(c.keys[0])[32:])
        b.csd_paged_append(c.pool, read, torch.zeros(64, 2, 64, device="cuda", dtype=dtype), torch.zeros(64, 2, 64, device="cuda", dtype=dtype))
        assert b.csd_device_status() == 9
        changed = (before != c.pool.k.view(torch.int16)).any(-1).any(1)            # [page, slot]
        assert sorted(set(changed.nonzero()[:, 0].tolist())) == sorted(good[0, [0, 2, 3]].tolist())


def test_lengths_outside_their_range(b):
    """Lengths that the caller got wrong are cut, never followed: the status says so, what lies elsewhere stays."""
    c = pp.Case(b, (4, 3), (60, 5), 2, 64, 16, "bf16", F32)
    c.fill()
    q = c.packed([torch.randn(r, 2, 64) for r in c.rows])
    rows = torch.randn(c.total, 2, 64, device="cuda")
    state = c.pool.k.clone().view(torch.int16)
    for kw, code in [(dict(kv=[62, 5]), 3), (dict(kv=[1 << 30, 5]), 3), (dict(kv=[-1, 5]), 1), (dict(max_rows=2), 1), (dict(start=[0, 4, 1000]), 1),
                     (dict(start=[0, -9, 5]), 1), (dict(start=[-3, 4, 7]), 1), (dict(kv=[2 ** 31 - 1, -2 ** 31]), None)]:
        for call in (lambda x: b.csd_paged_attention(q, c.pool, x), lambda x: b.csd_paged_read(c.pool, x, F32)):
            call(c.batch(**kw))
            got = b.csd_device_status()
            assert got == code if code else got in (1, 3), (kw, got)
    assert torch.equal(state, c.pool.k.view(torch.int16))
    b.csd_paged_append(c.pool, c.batch(kv=[62, 5]), rows, rows)                # positions 62 and 63 exist, 64 and 65 do not
    assert b.csd_device_status() == 3
    changed = (state != c.pool.k.view(torch.int16)).any(-1).any(1).nonzero().tolist()
    want = [[int(c.table[0, 3]), 14], [int(c.table[0, 3]), 15]] + [[int(c.table[1, 0]), s] for s in (5, 6, 7)]
    assert sorted(changed) == sorted(want)


@pytest.mark.parametrize("rows,kv,heads,kv_heads,dtype", [((2, 3), (40, 500), 4, 2, F32), ((1, 1), (700, 3), 4, 4, BF16), ((150, 1), (20, 500), 4, 2, BF16)])
def test_captured_calls_replay_with_other_lengths(b, rows, kv, heads, kv_heads, dtype):
    """Append and attention in a graph, on a stream of their own; the lengths on the device change between replays."""
    c = pp.Case(b, rows, kv, kv_heads, 128, 16, "bf16", dtype)
    c.fill()
    new = c.batch()
    k = c.packed([x[n:] for x, n in zip(c.keys, c.kv)])
    v = c.packed([x[n:] for x, n in zip(c.vals, c.kv)])
    parts = [torch.randn(r, heads, 128) for r in rows]
    q = c.packed(parts)
    out = torch.full((c.total, heads, 128), -7.0, dtype=dtype, device="cuda")
    ws = b.csd_paged_attention_workspace(c.pool, new, heads, dtype)
    graphs = []
    for _ in range(2):                                 # two graphs on one workspace, replayed in turn
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            b.csd_paged_append(c.pool, new, k, v)
            b.csd_paged_attention(q, c.pool, new, workspace=ws, out=out)
        graphs.append(g)
    for i, shorter in enumerate([(0, 0), (1, 7), (20, 3), (0, 0)]):
        lens = [max(n - s, 0) for n, s in zip(kv, shorter)]
        new.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        was = c.keys, c.vals, c.kv
        # the new rows now lie at their shorter sequences' ends
        c.keys, c.vals = ([torch.cat([x[:m], x[n:]]) for x, m, n in zip(t, lens, kv)] for t in was[:2])
        c.kv = lens
        compare(c, out.double().cpu().numpy(), parts, 128 ** -0.5, None)
        c.keys, c.vals, c.kv = was
        c.fill()
    assert b.csd_device_status() == 0


def test_far_pages(b):
    """Pages whose offsets pass 32 bits, in bytes and in elements."""
    for kind, heads in (("bf16", 8), ("e4m3", 8)):
        n = (1 << 32) // (heads * 128 * 128) + 40        # elements past 2^32
        pool = b.KvPool.empty(n, 128, heads, 128, BF16 if kind == "bf16" else torch.float8_e4m3fn)
        c = pp.Case(b, (3,), (300,), heads, 128, 128, kind, BF16)
        c.pool, c.table = pool, torch.tensor([[n - 1, 5, n - 20]], dtype=torch.int32)
        c.fill()
        attend(b, c, heads)
        assert b.csd_device_status() == 0


def test_a_long_cache(b):
    """70000 positions: the sums stay exact enough, and every page is read."""
    c = pp.Case(b, (1, 2), (70000, 33), 1, 64, 64, "bf16", F32)
    c.fill()
    attend(b, c, 2)
