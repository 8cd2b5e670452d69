"""Tree masks over pages whose bits reach behind the chunk's rows."""
import pytest
import torch

import workloads
from gpu_util import require_gpu, to_dev_i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    require_gpu()
    from paper_2312_11462_b200 import binding
    return binding


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float8_e4m3fn])
def test_bits_without_a_row_are_nobody(b, kind):
    """A row's rotary position counts the rows that its mask names and that exist: the same logits and the same cache, bit for bit."""
    shape = workloads.SHAPES["tiny_target"]
    blob = workloads.make_weights(shape, seed=5, device="cpu").cuda()
    toks = workloads.make_prompt(shape.vocab, 40, seed=4)
    rows, kv = [5, 0, 7], [6, 3, 0]
    trees = [0b1, 0b11, 0b101, 0b1011, 0b10000, 0b1, 0b11, 0b101, 0b1101, 0b10001, 0b110011, 0b1000000]
    beyond = [m | (-1 << (5 if i < 5 else 7)) for i, m in enumerate(trees)]               # every bit behind the sequence's rows
    got = []
    for masks in (trees, beyond):
        model = b.Model(shape, blob)
        pools = [b.KvPool(*(torch.zeros(6, shape.n_heads, 16, shape.d_head, dtype=kind, device="cuda") for _ in range(2)),
                          *(() if kind == torch.bfloat16 else (torch.zeros(6, shape.n_heads, 16, dtype=torch.uint8, device="cuda") for _ in range(2))))
                 for _ in range(shape.n_layers)]
        table = to_dev_i32([[4, 1], [0, 2], [5, 3]])
        batch = lambda r, n: b.PagedBatch(table, to_dev_i32([0, r[0], r[0] + r[1], sum(r)]), to_dev_i32(n), sum(r), max(r))  # noqa: E731
        model.csd_review_forward_paged(to_dev_i32(toks[:9]), pools, batch(kv, [0, 0, 0]), append_only=True)
        logits = model.csd_review_forward_paged(to_dev_i32(toks[9:21]), pools, batch(rows, kv), torch.tensor(masks, dtype=torch.int64).cuda())
        got.append([logits] + [t.view(torch.uint8) for p in pools for t in (p.k, p.v)])
    assert b.csd_device_status() == 0 and torch.isfinite(got[0][0]).all()
    for one, two in zip(*got):
        assert torch.equal(one, two)
