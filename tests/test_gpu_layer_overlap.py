"""Results that lie over an input or over another result are refused before anything is launched; exact in-place calls and interleaved views run."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

FREQ = 10000.0 ** (-np.arange(32) / 32)


def refused(call, context):
    from paper_2609_21594_b200 import binding as mb

    before = context.muon_launch_count()
    with pytest.raises(mb.MuonError) as e:
        call()
    assert e.value.code == mb.ERR_INVALID_ARG and context.muon_launch_count() == before


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rotary_out(dtype):
    from paper_2609_21594_b200 import functional as F

    c = F.context()
    store = torch.randn(2 * 50 * 12 * 64 + 4096, device="cuda").to(dtype)
    fused = store[:2 * 50 * 12 * 64].view(2, 50, 12, 64)
    q, k = fused[:, :, :8], fused[:, :, 8:10]
    want = F.rotary_forward([q, k], FREQ)
    refused(lambda: F.rotary_forward([q], FREQ, out=[store[64:64 + q.numel()].view(q.shape)]), c)        # part of it, at other places
    refused(lambda: F.rotary_forward([q[:, 1:]], FREQ, out=[q[:, :-1]]), c)                              # shifted by a token
    refused(lambda: F.rotary_forward([k, k], FREQ, out=[torch.empty_like(k), k]), c)                     # over another input
    two = torch.empty_like(q)
    refused(lambda: F.rotary_forward([q, q], FREQ, out=[two, two]), c)                                   # both results in one place
    refused(lambda: F.rotary_forward([q[:, :, :2], k], FREQ, out=[two[:, :, :2], two[:, :, 1:3]]), c)    # one head in common
    half = torch.empty(2, 50, 8, 64, dtype=dtype, device="cuda").as_strided((2, 50, 8, 64), (50 * 512, 512, 32, 1))
    refused(lambda: F.rotary_forward([q], FREQ, out=[half]), c)                                          # heads of the result half over one another
    got = F.rotary_forward([q, k], FREQ, out=[two, two.new_empty(2, 50, 4, 64)[:, :, ::2]])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    F.rotary_forward([q, k], FREQ, out=[q, k])                                                           # in place, interleaved views of one buffer
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_norm_results():
    from paper_2609_21594_b200 import binding as mb
    from paper_2609_21594_b200 import functional as F

    c = F.context()
    desc = mb.NormDesc(mb.DTYPE_FP32, mb.DTYPE_FP32, 1, 64, 40, 1e-5, 0)
    store = torch.randn(41 * 128, device="cuda")
    p, w = store.data_ptr(), torch.ones(64, device="cuda")
    mean, rstd, y = torch.empty(40, device="cuda"), torch.empty(40, device="cuda"), torch.empty(40, 64, device="cuda")
    m, r = mean.data_ptr(), rstd.data_ptr()

    def forward(x, ldx, y, ldy, weight=w.data_ptr(), mean=m, rstd=r):
        c.muon_layer_norm_forward(desc, x, ldx, weight, None, y, ldy, mean, rstd)

    def backward(dy, lddy, x, ldx, dx, lddx, dw=None):
        c.muon_layer_norm_backward(desc, dy, lddy, x, ldx, w.data_ptr(), m, r, dx, lddx, dw, None, None, 0)

    for call in (lambda: forward(p, 64, p + 256, 64), lambda: forward(p, 128, p + 128, 128), lambda: forward(p, 64, p + 16, 64),
                 lambda: forward(p, 64, y.data_ptr(), 64, weight=y.data_ptr() + 512), lambda: forward(p, 64, y.data_ptr(), 64, mean=r),
                 lambda: forward(p, 64, y.data_ptr(), 64, rstd=p), lambda: backward(p, 64, y.data_ptr(), 64, p + 256, 64),
                 lambda: backward(y.data_ptr(), 64, p, 64, p + 64, 64), lambda: backward(p, 64, p, 64, y.data_ptr(), 64, dw=y.data_ptr())):
        refused(call, c)
    side = store[:40 * 128].view(40, 128)                  # x and y as the two halves of rows of 128
    want = F.layer_norm_forward(side[:, :64].contiguous(), w)[0]
    forward(p, 128, p + 256, 128)
    assert torch.equal(side[:, 64:], want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_results(dtype):
    from paper_2609_21594_b200 import binding as mb
    from paper_2609_21594_b200 import functional as F

    c = F.context()
    n = lambda h: torch.randn(1, 100, h, 64, device="cuda").to(dtype)  # noqa: E731
    q, k, v, do = n(4), n(2), n(2), n(4)
    o, lse = F.attention_forward(q, k, v)
    grads = F.attention_backward(do, q, k, v, o, lse)
    desc = mb.AttentionDesc(int(dtype == torch.float32), 1, 100, 100, 4, 2, 64, 1, 0, 0.125, 0, 0, None, None, None, None)
    h, e = F._heads, q.element_size()
    moved = lambda t, by: mb.Heads(t.data_ptr() + by * e, *t.stride()[:3])  # noqa: E731
    ws = torch.empty(mb.muon_attention_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    room = torch.empty(q.numel() + 4096, dtype=dtype, device="cuda")
    inside = lambda t, by: mb.Heads(room.data_ptr() + by * e, *t.stride()[:3])  # noqa: E731

    def forward(q, o, lse=lse.data_ptr()):
        c.muon_attention_forward(desc, q, h(k), h(v), o, lse)

    def backward(dq, dk, dv, ws=ws.data_ptr()):
        c.muon_attention_backward(desc, h(do), h(q), h(k), h(v), h(o), lse.data_ptr(), dq, dk, dv, ws, mb.muon_attention_workspace_bytes(desc))

    dq, dk, dv = (torch.empty_like(t) for t in (q, k, v))
    for call in (lambda: forward(inside(q, 0), inside(q, 256)), lambda: forward(h(q), moved(k, 64)), lambda: forward(h(q), h(o), o.data_ptr()),
                 lambda: forward(h(q), mb.Heads(o.data_ptr(), 25600, 256, 32)),
                 lambda: backward(moved(q, 256), h(dk), h(dv)), lambda: backward(h(dq), moved(v, 64), h(dv)), lambda: backward(h(dq), h(dk), moved(dk, 64)),
                 lambda: backward(h(dq), h(dk), moved(o, 512)), lambda: backward(h(dq), moved(dq, 128), h(dv)), lambda: backward(moved(ws.view(dtype).view(1, -1, 1, 64).expand(1, -1, 4, 64), 0), h(dk), h(dv))):
        refused(call, c)
    backward(h(dq), h(dk), h(dv))
    assert all(torch.equal(a, b) for a, b in zip((dq, dk, dv), grads))
    # dk and dv as interleaved views of one buffer, dq inside it too
    fused = torch.zeros(1, 100, 8, 64, dtype=dtype, device="cuda")
    parts = fused[:, :, :4], fused[:, :, 4:6], fused[:, :, 6:]
    backward(*(h(t) for t in parts))
    assert all(torch.equal(a, b) for a, b in zip(parts, grads))
