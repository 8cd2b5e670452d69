"""The review forward over a paged cache, and a serving step as a run of calls: reviews of several sequences over pages, and the
verification of their drafts, against the contiguous cache, the oracle and a plain 64-bit forward."""
import numpy as np
import pytest
import torch

import paged_plain as pp
import workloads
from gpu_util import LOGIT_MAX_ABS, LOGIT_REL_L2, rel_l2, require_gpu, to_dev_i32

pytestmark = pytest.mark.gpu
TINY = workloads.SHAPES["tiny_target"]
BIG_HEADS = workloads.llama_shape(2, 256, 2, 512, 600, 200)          # d_head 128


@pytest.fixture(scope="module")
def b():
    require_gpu()
    from paper_2312_11462_b200 import binding
    return binding


def pools_of(b, shape, n_pages, page, dtype=torch.bfloat16):
    return [b.KvPool.empty(n_pages, page, shape.n_heads, shape.d_head, dtype) for _ in range(shape.n_layers)]


def batch_of(b, table, rows, kv, pad=0):
    start = np.concatenate([[0], np.cumsum(rows)])
    return b.PagedBatch(table, to_dev_i32(start), to_dev_i32(kv), int(start[-1]) + pad, max(max(rows), 1))


@pytest.mark.parametrize("shape", [TINY, BIG_HEADS], ids=["64", "128"])
def test_as_over_the_contiguous_cache(b, orc, shape):
    """Three sequences of ragged blocks, several steps, with rollbacks: the oracle's logits, and those of handles of their own."""
    blob = workloads.make_weights(shape, seed=3, device="cpu", gain_std=0.1)
    model, om = b.Model(shape, blob.cuda()), [orc.Model(shape, orc.blob_to_u16(blob)) for _ in range(3)]
    own = [b.Model(shape, blob.cuda()) for _ in range(3)]
    pools = pools_of(b, shape, 3 * 13 + 2, 16)
    table = torch.randperm(41, generator=torch.Generator().manual_seed(1))[:39].view(3, 13).int().cuda()
    toks = [workloads.make_prompt(shape.vocab, 150, seed=s) for s in range(3)]
    kv = [0, 0, 0]
    ws = b.csd_paged_attention_workspace(pools[0], batch_of(b, table, [1, 1, 1], kv), shape.n_heads, torch.float32)
    for rows, keep in [((5, 7, 5), (5, 7, 5)), ((0, 17, 0), (0, 16, 0)), ((5, 3, 5), (2, 3, 1)), ((1, 1, 1), (1, 1, 1)), ((6, 0, 11), (6, 0, 11))]:
        blocks = [toks[s][kv[s]:kv[s] + r] for s, r in enumerate(rows)]
        got = model.csd_review_forward_paged(to_dev_i32(np.concatenate(blocks)), pools, batch_of(b, table, rows, kv), workspace=ws)
        assert b.csd_device_status() == 0
        at = 0
        for s, r in enumerate(rows):
            if not r:
                continue
            g, want = got[at:at + r].cpu().numpy(), om[s].review_forward(blocks[s], kv[s])
            other = own[s].csd_review_forward(to_dev_i32(blocks[s]), kv[s]).cpu().numpy()
            assert rel_l2(g, want) <= LOGIT_REL_L2 and np.abs(g - want).max() <= LOGIT_MAX_ABS, (rows, s, rel_l2(g, want))
            assert rel_l2(g, other) <= LOGIT_REL_L2
            at += r
        kv = [n + k for n, k in zip(kv, keep)]


@pytest.mark.parametrize("shape", [TINY, BIG_HEADS], ids=["64", "128"])
def test_trees(b, shape):
    """A tree's rows over pages as over the handle's own cache."""
    blob = workloads.make_weights(shape, seed=5, device="cpu").cuda()
    model, own = b.Model(shape, blob), b.Model(shape, blob)
    pools = pools_of(b, shape, 12, 16)
    table = torch.randperm(12, generator=torch.Generator().manual_seed(2))[None, :8].int().contiguous().cuda()
    toks = workloads.make_prompt(shape.vocab, 60, seed=4)
    for n in range(0, 45, 15):
        model.csd_review_forward_paged(to_dev_i32(toks[n:n + 15]), pools, batch_of(b, table, [15], [n]), append_only=True)
        own.csd_review_forward(to_dev_i32(toks[n:n + 15]), n)
    parent = [-1, 0, 0, 0, 1, 4, 2, 6, 3, 0, 5]
    masks = []
    for r, p in enumerate(parent):
        masks.append((masks[p] if r else 0) | 1 << r)
    block = to_dev_i32(toks[45:45 + len(parent)])
    got = model.csd_review_forward_paged(block, pools, batch_of(b, table, [len(parent)], [45]), torch.tensor(masks, dtype=torch.int64).cuda())
    want = own.csd_review_forward_tree(block, parent, 45)
    assert rel_l2(got.cpu().numpy(), want.cpu().numpy()) <= LOGIT_REL_L2 and b.csd_device_status() == 0


def plain_forward(shape, blob, tokens, keep):
    """Logits of all positions in 64 bits; keep(rows [n, heads, d]): what the cache holds of keys and values."""
    at = {name: (off, shp) for name, off, shp in workloads.blob_layout(shape)[0]}
    part = lambda name: blob[at[name][0]:at[name][0] + int(np.prod(at[name][1]))].view(*at[name][1]).double()  # noqa: E731
    norm = lambda x, g: x / torch.sqrt((x * x).mean(-1, keepdim=True) + shape.norm_eps) * g  # noqa: E731
    n, H, D = len(tokens), shape.n_heads, shape.d_head
    half = D // 2
    angle = torch.arange(n, dtype=torch.float64)[:, None] * shape.rope_theta ** (-torch.arange(half, dtype=torch.float64) / half)
    cos, sin = torch.cos(angle).float().double()[:, None], torch.sin(angle).float().double()[:, None]
    turn = lambda x: torch.cat([x[..., :half] * cos - x[..., half:] * sin, x[..., :half] * sin + x[..., half:] * cos], -1)  # noqa: E731
    x = part("embed")[torch.as_tensor(tokens, dtype=torch.long)]
    hidden = torch.ones(n, n, dtype=torch.bool).triu(1)
    for l in range(shape.n_layers):
        name = [k for k in at if k.startswith(f"l{l}.")]
        w = {k.split(".")[-1]: part(k) for k in name}
        y = norm(x, w["norm1"])
        q, k, v = (turn((y @ w["wq"].T).view(n, H, D)), turn((y @ w["wk"].T).view(n, H, D)), (y @ w["wv"].T).view(n, H, D))
        k, v = keep(k), keep(v)
        s = torch.einsum("ihd,jhd->hij", q, k) / D ** 0.5
        p = torch.softmax(s.masked_fill(hidden, -torch.inf), -1)
        x = x + torch.einsum("hij,jhd->ihd", p, v).reshape(n, H * D) @ w["wo"].T
        y = norm(x, w["norm2"])
        g = y @ w["wgate"].T
        x = x + (g / (1 + torch.exp(-g)) * (y @ w["wup"].T)) @ w["wdown"].T
    return (norm(x, part("final_norm")) @ part("lm_head").T).numpy()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_against_a_plain_forward(b, kind):
    """Both kinds of cache against a 64-bit forward whose keys and values are rounded in the same way."""
    shape = BIG_HEADS
    blob = workloads.make_weights(shape, seed=8, device="cpu", gain_std=0.1)
    toks = workloads.make_prompt(shape.vocab, 51, seed=6)
    keep = (lambda t: t.bfloat16().double()) if kind == "bf16" else (lambda t: torch.from_numpy(pp.quantise(t.float().double().numpy())[0]))
    want = plain_forward(shape, blob, toks, keep)
    model = b.Model(shape, blob.cuda())
    pools = pools_of(b, shape, 5, 16, torch.bfloat16 if kind == "bf16" else torch.float8_e4m3fn)
    table = to_dev_i32([[4, 0, 2, 3]])
    got = torch.cat([model.csd_review_forward_paged(to_dev_i32(toks[n:n + 17]), pools, batch_of(b, table, [17], [n])) for n in (0, 17, 34)]).cpu().numpy()
    # Values of the second layer that round the other way: a difference of d upstream moves a share of about 8 d of the e4m3 numbers by
    # an eighth or less.  The first layer's keys differ by 1e-6: sqrt(8e-6) / 16 = 2e-4 behind it, and so sqrt(1.6e-3) / 16 = 2.5e-3
    # of the second layer's keys and values, which reach the logits through one of their terms: twice that is allowed.
    assert rel_l2(got, want) <= (LOGIT_REL_L2 if kind == "bf16" else 5e-3), rel_l2(got, want)


def test_a_serving_step_captured(b, orc):
    """Reviews of three sequences over pages and the verification of their drafts, in one graph that replays while the sequences grow."""
    shape = TINY
    blob = workloads.make_weights(shape, seed=0, device="cpu", std=0.6)
    model, om = b.Model(shape, blob.cuda()), [orc.Model(shape, orc.blob_to_u16(blob)) for _ in range(3)]
    pools = pools_of(b, shape, 24, 16)
    table = torch.randperm(24, generator=torch.Generator().manual_seed(5)).view(3, 8).int().cuda()
    k, seqs = 4, [list(workloads.make_prompt(shape.vocab, n, seed=n)) for n in (20, 33, 9)]
    for s, text in enumerate(seqs):
        for n in range(0, len(text) - 1, 17):
            part = text[:-1][n:n + 17]
            rows, kv = [0, 0, 0], [0, 0, 0]
            rows[s], kv[s] = len(part), n
            model.csd_review_forward_paged(to_dev_i32(part), pools, batch_of(b, table, rows, kv), append_only=True)
        om[s].review_forward(np.asarray(text[:-1], dtype=np.int32), 0)
    batch = batch_of(b, table, [5, 5, 5], [len(t) - 1 for t in seqs])
    tokens, drafts = torch.zeros(15, dtype=torch.int32, device="cuda"), torch.zeros(3, k, dtype=torch.int32, device="cuda")
    uniforms, count = torch.zeros(3, k + 1, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    logits = torch.zeros(15, shape.vocab, device="cuda")
    out = (torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, k + 1, dtype=torch.int32, device="cuda"))
    ws = b.csd_paged_attention_workspace(pools[0], batch, shape.n_heads, torch.float32)

    def step():
        model.csd_review_forward_paged(tokens, pools, batch, workspace=ws, logits_out=logits)
        b.csd_spec_verify(logits.softmax(-1).view(3, k + 1, -1), None, drafts, uniforms, count, out)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    rng = np.random.default_rng(1)
    for _ in range(4):
        cand = [[int(x) for x in rng.integers(0, shape.vocab, k)] for _ in seqs]
        want = [om[s].review_forward(np.asarray([t[-1]] + c, dtype=np.int32), len(t) - 1) for s, (t, c) in enumerate(zip(seqs, cand))]
        for s in range(3):                            # the first draft is the likeliest token, and accepted for certain
            cand[s][0] = int(want[s][0].argmax())
            want[s] = om[s].review_forward(np.asarray([seqs[s][-1]] + cand[s], dtype=np.int32), len(seqs[s]) - 1)
        n = rng.integers(1, k + 1, 3)
        u = rng.random((3, k + 1)).astype(np.float32)
        u[:, 0] = 0.0
        tokens.copy_(to_dev_i32(np.concatenate([[t[-1]] + c for t, c in zip(seqs, cand)])))
        drafts.copy_(to_dev_i32(cand))
        uniforms.copy_(torch.from_numpy(u))
        count.copy_(to_dev_i32(n))
        batch.kv_len.copy_(to_dev_i32([len(t) - 1 for t in seqs]))
        g.replay()
        torch.cuda.synchronize()
        assert b.csd_device_status() == 0
        for s in range(3):
            mine = logits[5 * s:5 * s + 5].cpu().numpy()
            assert rel_l2(mine, want[s]) <= LOGIT_REL_L2
            p = torch.softmax(logits[5 * s:5 * s + 5], -1).double().cpu().numpy()
            a, row = pp.verify(p, None, cand[s], u[s].astype(np.float64), int(n[s]))
            assert (int(out[0][s]), out[1][s].tolist()) == (a, row) and a >= 1
            seqs[s] += row[:a + 1]
            om[s].review_forward(np.asarray(seqs[s][:-1], dtype=np.int32), 0)


def test_refusals(b):
    blob = workloads.make_weights(TINY, seed=1, device="cpu").cuda()
    model = b.Model(TINY, blob)
    pools = pools_of(b, TINY, 8, 16)
    table = to_dev_i32([[0, 1, 2]])
    tok = to_dev_i32(list(range(18)))
    with pytest.raises(b.CsdError):                      # more rows than a pass takes
        model.csd_review_forward_paged(tok, pools, batch_of(b, table, [18], [0]))
    wrong = [b.KvPool.empty(8, 16, TINY.n_heads + 1, TINY.d_head) for _ in range(TINY.n_layers)]
    with pytest.raises(b.CsdError) as e:
        model.csd_review_forward_paged(tok[:2], wrong, batch_of(b, table, [2], [0]))
    assert e.value.code == 2
    with pytest.raises(b.CsdError) as e:                 # a workspace that is too small
        model.csd_review_forward_paged(tok[:2], pools, batch_of(b, table, [2], [0]), workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))
    assert e.value.code == 3
    # a rotary position that the model has no table for
    long = b.PagedBatch(torch.zeros(1, 200, dtype=torch.int32, device="cuda"), to_dev_i32([0, 2]), to_dev_i32([TINY.max_seq - 1]), 2, 2)
    model.csd_review_forward_paged(tok[:2], pools, long)
    assert b.csd_device_status() == 3
