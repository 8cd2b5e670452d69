"""Verification where sums round: targets beside pieces of the vocabulary that hold nothing."""
import pytest
import torch

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu
V, PIECES = 32000, 64                        # one row of so many entries is summed in 64 pieces
EMPTY = 6

# Masses of the first pieces, and of those behind six empty ones: half of the whole lies between two roundings of the first pieces' sum, so that an
# empty piece seems to hold it (found with the sums' order written out in Python).
LAWS = [(("0x1.1442f8p-15", "0x1.4fa7b6p-21", "0x1.0ec9eep-39", "0x1.a064f4p-9", "0x1.d354b2p-11", "0x1.3698f6p-7", "0x1.758092p-30", "0x1.165604p-32", "0x1.dec1dp-6",
          "0x1.a1b78ep-35", "0x1.66f0d2p-25", "0x1.b6fdb2p-33"), ("0x1.5ea13ep-5", "0x1.5c8894p-29", "0x1.5p-53")),
        (("0x1.5b0872p-33", "0x1.79ac5ap-10", "0x1.26c50cp-29", "0x1.20779ap-15", "0x1.df8596p-14", "0x1.8cfa78p-30", "0x1.517992p-24", "0x1.c0fd5ap-32", "0x1.ca19dap-2",
          "0x1.8b644ap-22", "0x1.95f67cp-32", "0x1.45c6f8p-8"), ("0x1.d0d1bcp-2", "0x1.342a22p-27", "0x1.8p-53")),
        (("0x1.268ddep-30", "0x1.7f6fccp-27", "0x1.566388p-23", "0x1.b7acf4p-5", "0x1.181972p-6", "0x1.53ce5ap-4", "0x1.7ffa34p-10", "0x1.4fc12ap-36", "0x1.60ec28p-26"),
         ("0x1.3dd5a6p-3", "0x1.d3e8ep-29", "0x1.4p-53"))]


@pytest.fixture(scope="module")
def b():
    require_gpu()
    from paper_2312_11462_b200 import binding
    return binding


@pytest.mark.parametrize("first,others", LAWS)
@pytest.mark.parametrize("into", [0, 3, 490])
def test_a_target_beside_pieces_that_hold_nothing(b, first, others, into):
    """The token is one of the two that carry mass beside the target, whichever way the sums round; never one without mass, and always one."""
    law, tokens = torch.zeros(V), []
    for i, mass in [*enumerate(first), *enumerate(others, len(first) + EMPTY)]:
        tokens.append((i * V // PIECES & ~7) + into)
        law[tokens[-1]] = float.fromhex(mass)
    fine = tokens[len(first) - 1:len(first) + 1]
    law, half = law.cuda(), torch.full((1, 2), 0.5, device="cuda")
    none = torch.zeros(1, 0, dtype=torch.int32, device="cuda")
    a, out = b.csd_spec_verify(law.view(1, 1, V), None, none, half[:, :1].contiguous())
    assert int(a) == 0 and int(out[0, 0]) in fine
    # behind a draft that is refused: what is left of the law is all of it
    draft = torch.full((1, 1), V - 1, dtype=torch.int32, device="cuda")
    q = torch.zeros(1, 1, V, device="cuda")
    q[..., V - 1] = 1.0
    for laws in (q, None):
        out = (torch.full((1,), -7, dtype=torch.int32, device="cuda"), torch.full((1, 2), -7, dtype=torch.int32, device="cuda"))
        b.csd_spec_verify(law.expand(1, 2, V).contiguous(), laws, draft, half, out=out)
        assert int(out[0]) == 0 and int(out[1][0, 0]) in fine and int(out[1][0, 1]) == -1
    assert b.csd_device_status() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_drafts_whose_entries_are_negative_or_not_numbers(b, dtype):
    """They count as 0 in the tests of the drafts: accepted iff u * max(q, 0) < max(p, 0), a NaN as 0."""
    nan, inf = float("nan"), float("inf")
    #        p     q    u   accepted
    cases = [(0.0, -0.5, 0.5, 0), (0.25, -0.5, 0.5, 1), (0.0, nan, 0.5, 0), (0.25, nan, 0.5, 1), (-0.25, -0.5, 0.5, 0), (-0.25, 0.5, 0.0, 0), (nan, 0.5, 0.5, 0),
             (nan, nan, 0.5, 0), (nan, -0.5, 0.5, 0), (0.25, 0.5, 0.5, 0), (0.25, 0.375, 0.5, 1), (0.0, 0.0, 0.5, 0), (0.25, inf, 0.5, 0), (inf, 0.5, 0.5, 1), (inf, inf, 0.5, 0)]
    n, x = len(cases), 5
    p, q = torch.zeros(n, 2, 40), torch.zeros(n, 1, 40)
    p[..., 9] = 0.5                                   # (the output token, after a rejection and behind the draft)
    for i, (px, qx, _, _) in enumerate(cases):
        p[i, 0, x], q[i, 0, x] = px, qx
    u = torch.tensor([[c[2], 0.25] for c in cases], device="cuda")
    tok = torch.full((n, 1), x, dtype=torch.int32, device="cuda")
    a, out = b.csd_spec_verify(p.to(dtype).cuda(), q.to(dtype).cuda(), tok, u)
    assert a.tolist() == [c[3] for c in cases] and b.csd_device_status() == 0
    assert out.tolist() == [[x, 9] if c[3] else [9, -1] for c in cases]
    a, out = b.csd_spec_verify(p.to(dtype).cuda(), None, tok, u)                # point masses: q = 1
    want = [int(c[0] > c[2]) for c in cases]
    assert a.tolist() == want and out.tolist() == [[x, 9] if w else [9, -1] for w in want] and b.csd_device_status() == 0
