"""Verification of drafts against given probabilities against a plain 64-bit form: integers, equal."""
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


def make(rows, k, V, seed, dtype=F32, point=False, cut=0.0, sharp=2.0, near=0.6):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, k + 1, V, generator=g, device="cuda") * sharp

    def law(t):
        t = t.softmax(-1)
        if cut:
            t = torch.where(t < cut * t.amax(-1, keepdim=True), 0.0, t)
            t = t / t.sum(-1, keepdim=True)
        return t.to(dtype)
    p = law(x)
    q = None if point else law(x[:, :k] + near * torch.randn(rows, k, V, generator=g, device="cuda"))
    if k == 0:
        tok = torch.zeros(rows, 0, dtype=torch.int32, device="cuda")
    elif point:
        tok = torch.where(torch.rand(rows, k, generator=g, device="cuda") < 0.7, x[:, :k].argmax(-1), torch.randint(V, (rows, k), generator=g, device="cuda")).int()
    else:
        tok = torch.multinomial(q.float().view(rows * k, V), 1, generator=g).view(rows, k).int()
    return p, q, tok, torch.rand(rows, k + 1, generator=g, device="cuda")


def compare(b, p, q, tok, u, n=None, status=0, **kw):
    """Equal to the plain form; a draw whose target lies within 1e-12 of an entry's edge would be excused (none is)."""
    rows, k1, V = p.shape
    a, out = b.csd_spec_verify(p, q, tok, u, n, **kw)
    assert b.csd_device_status() == status
    a, out = a.cpu().numpy(), out.cpu().numpy()
    P, Q = p.double().cpu().numpy(), None if q is None else q.double().cpu().numpy()
    U, T = u.double().cpu().numpy(), tok.cpu().numpy()
    for r in range(rows):
        want = pp.verify(P[r], None if Q is None else Q[r], list(T[r]), U[r], k1 - 1 if n is None else min(max(int(n[r]), 0), k1 - 1))
        assert (a[r], list(out[r])) == want, (r, a[r], out[r], want)


@pytest.mark.parametrize("V", [1, 2, 7, 31, 255, 1000, 1024, 4097, 32000, 50257, 128256, 262147])
@pytest.mark.parametrize("rows,k", [(1, 0), (1, 4), (5, 3)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sizes(b, V, rows, k, dtype):
    for point in (False, True):
        p, q, tok, u = make(rows, k, V, V + k, dtype, point)
        compare(b, p, q, tok, u)


@pytest.mark.parametrize("rows,k,V", [(37, 64, 300), (300, 5, 5003), (1000, 1, 64), (150, 2, 32128)])
def test_many_rows(b, rows, k, V):
    p, q, tok, u = make(rows, k, V, rows, cut=0.01)
    n = torch.randint(0, k + 1, (rows,), device="cuda").int()
    compare(b, p, q, tok, u, n)
    compare(b, p, None, tok, u, n)


def test_edges_of_the_uniforms(b):
    p, q, tok, _ = make(64, 3, 1000, 3, cut=0.05)
    for value in (0.0, 1.0 - 2.0 ** -24):
        compare(b, p, q, tok, torch.full((64, 4), value, device="cuda"))
    # dyadic laws: targets that lie exactly on the entries' edges
    law = torch.zeros(8, 2, 16, device="cuda")
    law[..., ::2] = 0.125
    u = torch.arange(16, device="cuda").float().view(8, 2) / 16
    compare(b, law, law[:, :1].contiguous(), torch.full((8, 1), 2, dtype=torch.int32, device="cuda"), u)


def test_laws_without_mass(b):
    V = 600
    p, q, tok, u = make(8, 2, V, 5)
    same = p[:, :2].contiguous()                     # equal laws: accepted, or nothing is left
    off = tok.clone()
    p2, q2 = p.clone(), same.clone()
    q2[:, 0] = 2 * p2[:, 0]                          # nothing left: the target's own law
    compare(b, p2, q2, off, torch.full((8, 3), 0.9, device="cuda"))
    p3 = torch.zeros_like(p)                         # no law at all: token 0
    compare(b, p3, q, tok, u)
    p4 = p.clone()
    p4[:, :, 100:] = float("nan")                    # entries that are not numbers carry nothing
    p4[:, :, 50] = -1.0
    p4[:, :, 51] = float("inf")
    q4 = q.clone()
    q4[:, :, 300:] = float("nan")
    q4[:, :, 7], q4[:, :, 9] = float("inf"), -0.25
    tok4 = torch.randint(0, 50, (8, 2), device="cuda").int()
    compare(b, p4, q4, tok4, u)
    p5 = torch.zeros_like(p)                         # one entry
    p5[..., V - 1] = 1e-30
    compare(b, p5, q, tok, u)


def test_bad_tokens_counts_and_numbers(b):
    p, q, tok, u = make(6, 3, 500, 9)
    u *= 0.01                                        # (nearly everything is accepted)
    bad = tok.clone()
    bad[1, 0], bad[2, 2], bad[3, 1] = -1, 500, 2 ** 31 - 1
    compare(b, p, q, bad, u, status=6)
    compare(b, p, None, bad, u, status=6)
    compare(b, p, q, tok, u, torch.tensor([0, 3, 4, -2, 1, 2 ** 30], dtype=torch.int32, device="cuda"), status=1)
    odd = u.clone()
    odd[0, 3], odd[1, 3], odd[2, 3] = 1.0, float("nan"), -0.5
    a, out = b.csd_spec_verify(p, q, tok, odd)
    assert b.csd_device_status() == 1 and ((out >= -1) & (out < 500)).all()
    # what lies behind a row's drafts is not looked at
    n = torch.tensor([1, 0, 2, 3, 0, 1], dtype=torch.int32, device="cuda")
    junk = tok.clone()
    junk[torch.arange(3, device="cuda")[None] >= n[:, None]] = -77
    compare(b, p, q, junk, u, n)


def test_strided_laws_and_streams(b):
    """Laws inside rows of a padded vocabulary, odd starts; a stream of its own; a captured call."""
    for dtype in (F32, BF16):
        p, q, tok, u = make(7, 3, 1001, 11, dtype)
        wide_p = torch.full((7, 4, 1037), 9.0, dtype=dtype, device="cuda")
        wide_q = torch.full((7, 3, 1040), 9.0, dtype=dtype, device="cuda")
        wide_p[..., 3:1004], wide_q[..., :1001] = p, q
        want = b.csd_spec_verify(p, q, tok, u)
        compare(b, wide_p[..., 3:1004], wide_q[..., :1001], tok, u)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = b.csd_spec_verify(p, q, tok, u)
        side.synchronize()
        out = tuple(torch.zeros_like(t) for t in want)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            b.csd_spec_verify(p, q, tok, u, out=out)
        g.replay()
        torch.cuda.synchronize()
        for x, y, z in zip(want, got, out):
            assert torch.equal(x, y) and torch.equal(x, z)


def test_far_laws(b):
    """Laws whose offsets pass 32 bits."""
    V, rows, k = 128256, 800, 20
    p = torch.zeros(rows, k + 1, V, device="cuda", dtype=BF16)
    p[:, :, 7] = 1.0
    p[-1, -1, 7], p[-1, -1, V - 1] = 0.0, 1.0
    tok = torch.full((rows, k), 7, dtype=torch.int32, device="cuda")
    a, out = b.csd_spec_verify(p, None, tok, torch.full((rows, k + 1), 0.5, device="cuda"))
    assert (a == k).all() and (out[:-1] == 7).all() and (out[-1, :-1] == 7).all() and int(out[-1, -1]) == V - 1
