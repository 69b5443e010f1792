"""Queries that see no key and keys that no query sees, although they count: zero results of their own, and what they hold reaches nobody."""
import pytest
import torch

from test_gpu_attention import BF, F32, check, make

pytestmark = pytest.mark.gpu

ROUTES = [(BF, 64), (BF, 128), (BF, 72), (BF, 20), (BF, 136), (F32, 64), (F32, 128), (F32, 192)]       # tensor cores, then CUDA cores
BAD = [float("nan"), float("inf")]


def dirty(t, rows, bad):
    t = t.clone()
    t[rows] = bad
    return t


@pytest.mark.parametrize("dtype,d", ROUTES)
@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("nq,nk", [(200, 150), (256, 128), (400, 3), (300, 299), (700, 130)])
def test_more_queries_than_keys(dtype, d, window, nq, nk):
    from paper_2609_21594_b200 import functional as F

    q, k, v, do = make(1, nq, nk, 4, 2, d, dtype)
    clean = check(q, k, v, do, window=window)
    blind = (slice(None), slice(0, nq - nk))
    assert not clean[0][blind].any() and not clean[2][blind].any()
    for bad in BAD:
        qq, dd, oo = dirty(q, blind, bad), dirty(do, blind, bad), dirty(clean[0], blind, bad)
        o, lse = F.attention_forward(qq, k, v, True, window)
        assert torch.equal(o, clean[0]) and torch.equal(lse, clean[1])
        for a, b in zip(F.attention_backward(dd, qq, k, v, oo, lse, True, window), clean[2:]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,d", ROUTES)
def test_more_queries_than_keys_in_padded_and_packed_rows(dtype, d):
    from paper_2609_21594_b200 import functional as F

    ql, kl = [300, 260, 130, 7], [170, 300, 1, 0]
    q, k, v, do = make(4, 300, 300, 4, 2, d, dtype)
    i = torch.arange(300, device="cuda")
    lens = {"q_lens": torch.tensor(ql, dtype=torch.int32, device="cuda"), "k_lens": torch.tensor(kl, dtype=torch.int32, device="cuda")}
    unseeing = (i[None] < (lens["q_lens"] - lens["k_lens"])[:, None]) | (i[None] >= lens["q_lens"][:, None])
    clean = check(q, k, v, do, **lens)
    qq, dd, oo = (dirty(t, unseeing, float("nan")) for t in (q, do, clean[0]))
    o, lse = F.attention_forward(qq, k, v, **lens)
    assert torch.equal(o, clean[0]) and torch.equal(lse, clean[1])
    assert all(torch.equal(a, b) for a, b in zip(F.attention_backward(dd, qq, k, v, oo, lse, **lens), clean[2:]))

    qo, ko = ([0] + torch.tensor(x).cumsum(0).tolist() for x in (ql, kl))
    q, k, v, do = (t[0] for t in make(1, qo[-1], max(qo[-1], ko[-1]), 4, 2, d, dtype))
    k, v = k[:ko[-1]], v[:ko[-1]]
    offs = {"q_offsets": torch.tensor(qo, dtype=torch.int32, device="cuda"), "k_offsets": torch.tensor(ko, dtype=torch.int32, device="cuda")}
    unseeing = torch.cat([torch.arange(n, device="cuda") < n - m for n, m in zip(ql, kl)])
    clean = check(q, k, v, do, **offs)
    qq, dd, oo = (dirty(t, unseeing, float("nan")) for t in (q, do, clean[0]))
    o, lse = F.attention_forward(qq, k, v, **offs)
    assert torch.equal(o, clean[0]) and torch.equal(lse, clean[1])
    assert all(torch.equal(a, b) for a, b in zip(F.attention_backward(dd, qq, k, v, oo, lse, **offs), clean[2:]))


@pytest.mark.parametrize("dtype,d", ROUTES)
def test_results_of_the_unseen_are_zero_whatever_the_others_hold(dtype, d):
    """Queries that see nothing beside keys full of NaN, keys outside every window beside queries full of NaN."""
    from paper_2609_21594_b200 import functional as F

    q, k, v, do = make(1, 200, 150, 2, 1, d, dtype)
    k, v = torch.full_like(k, float("nan")), torch.full_like(v, float("nan"))
    o, lse = F.attention_forward(q, k, v)
    assert not o[:, :50].any() and (lse[..., :50] == -float("inf")).all() and o[:, 50:].isnan().all()
    dq, _, _ = F.attention_backward(do, q, k, v, o, lse)
    assert not dq[:, :50].any()
    q, k, v, do = make(1, 30, 150, 2, 1, d, dtype)
    q, do = torch.full_like(q, float("nan")), torch.full_like(do, float("nan"))
    o, lse = F.attention_forward(q, k, v, window=20)
    _, dk, dv = F.attention_backward(do, q, k, v, o, lse, window=20)
    assert not dk[:, :101].any() and not dv[:, :101].any() and dv[:, 101:].isnan().all()
