"""Gradients of short sequences keep the precision that two bf16 terms of P and dS give, whatever they are packed or padded with.

Tolerance: P and dS as two bf16 terms are off by 2^-16 together; with fp32's 2^-14 for the sums 2^-13 of the absolute sums; dS = P (dP - delta)
cancels in fp32 (2^-16 of the sum before it does); the result is rounded to bf16."""
import pytest
import torch

import layer_reference as ref
from test_gpu_attention import BF, close, make

pytestmark = pytest.mark.gpu


def gradients(q, k, v, do, **lens):
    from paper_2609_21594_b200 import functional as F

    o, lse = F.attention_forward(q, k, v, **lens)
    return o, lse, F.attention_backward(do, q, k, v, o, lse, **lens)


def tight(got, r, rows, name):
    tol = 2.0 ** -13 * r[name + "_abs"] + 2.0 ** -8 * 1.01 * r[name].abs() + 1e-30
    if name != "dv":
        tol = tol + 2.0 ** -16 * r[name + "_pre"]
    close(got[rows], r[name][rows], tol[rows], name)


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("lens", [[10] * 70, [2, 3, 128, 1, 129, 128, 127, 300, 512, 64, 1], [700, 4, 5, 6, 900, 20], [40, 1500]])
def test_short_documents_among_others(lens, d):
    n = sum(lens)
    at = [0] + torch.tensor(lens).cumsum(0).tolist()
    offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
    packed = dict(q_offsets=offsets, k_offsets=offsets)
    q, k, v, do = (t[0] for t in make(1, n, n, 4, 2, d, BF, seed=n + d))
    o, lse, got = gradients(q, k, v, do, **packed)
    r = ref.attention(q[None], k[None], v[None], do=do[None], o=o[None], lse=lse[None], **packed)
    short = torch.cat([torch.full((m,), m <= 128, device="cuda") for m in lens])
    for name, g in zip(("dq", "dk", "dv"), got):
        tight(g[None], r, (0, short), name)
    for a, b in zip(at, at[1:]):                       # and alone in a row a document has the same bits
        s, own = slice(a, b), torch.tensor([0, b - a], dtype=torch.int32, device="cuda")
        _, _, alone = gradients(q[s], k[s], v[s], do[s], q_offsets=own, k_offsets=own)
        assert all(torch.equal(x, y[s]) for x, y in zip(alone, got))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 128])
def test_short_rows_of_a_long_batch(d, causal):
    lens = [400, 5, 128, 2, 31, 1]
    kl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    q, k, v, do = make(6, 400, 400, 4, 2, d, BF, seed=d)
    from paper_2609_21594_b200 import functional as F

    o, lse = F.attention_forward(q, k, v, causal, q_lens=kl, k_lens=kl)
    got = F.attention_backward(do, q, k, v, o, lse, causal, q_lens=kl, k_lens=kl)
    r = ref.attention(q, k, v, causal, do=do, o=o, lse=lse, q_lens=kl, k_lens=kl)
    for name, g in zip(("dq", "dk", "dv"), got):
        tight(g, r, slice(1, None), name)
    for i, n in enumerate(lens):
        if n > 128:
            continue
        one = tuple(t[i:i + 1, :n] for t in (q, k, v))
        oi, li = F.attention_forward(*one, causal)
        for a, b in zip(F.attention_backward(do[i:i + 1, :n], *one, oi, li, causal), got):
            assert torch.equal(a[0], b[i, :n])
