"""Attention, forward and backward, against the definition in 64 bits, on both routes: tensor cores (bf16, aligned) and CUDA cores.

Tolerances, derived element by element from sums of absolute values.  bf16: P, dS and results are each rounded once to bf16 (2^-8 of
their value); scores, statistics and sums are fp32, which adds less than 2^-14 relative for the lengths used here.  So
  o:  2^-8 sum p |v| (rounding of P) + 2^-8 |o|,      dv: the same with do,
  dq: 2^-8 sum |dS| |k| + 2^-16 sum p (|do| |v| + |do| |o|) |k| (dS = P (dP - delta) cancels in fp32) + 2^-8 |dq|,   dk likewise.
fp32: the factor 2^-8 becomes 2^-16 (sums of up to 2^8 products of head and keys at 2^-24) and no rounding of results counts.
lse: 2^-20 (|lse| + max |score|) + 2^-18."""
import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def make(b, nq, nk, hq, hkv, d, dtype, seed=0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: (torch.randn(s, generator=g, device="cuda") * spread).to(dtype)  # noqa: E731
    return n(b, nq, hq, d), n(b, nk, hkv, d), n(b, nk, hkv, d), n(b, nq, hq, d)


def close(got, want, tol, what):
    off = (got.double() - want).abs()
    assert torch.isfinite(got).all(), what
    assert (off <= tol).all(), f"{what}: {(off / tol.clamp_min(1e-300)).max().item():.2f} of the tolerance"


def check(q, k, v, do, causal=True, window=0, scale=None, backward=True, **lens):
    from paper_2609_21594_b200 import functional as F

    packed = lens.get("q_offsets") is not None
    up = (lambda t: t[None]) if packed else (lambda t: t)
    o, lse = F.attention_forward(q, k, v, causal, window, scale, **lens)
    r = ref.attention(up(q), up(k), up(v), causal, window, scale, **lens)
    bf = q.dtype == BF
    w = 2.0 ** -8 + 2.0 ** -14 if bf else 2.0 ** -16
    e = 2.0 ** -8 * 1.01 if bf else 0.0
    tiny = 1e-30
    close(up(o), r["o"], w * r["o_abs"] + e * r["o"].abs() + tiny, "o")
    live = r["lse"] > -float("inf")
    assert torch.equal(up(lse) == -float("inf"), ~live)
    size = float(q.double()[q.isfinite()].abs().max() if q.numel() else 0) ** 2 * q.shape[-1] * (scale or q.shape[-1] ** -0.5)
    close(up(lse)[live], r["lse"][live], 2.0 ** -20 * (r["lse"][live].abs() + size) + 2.0 ** -18, "lse")
    if not backward:
        return o, lse
    dq, dk, dv = F.attention_backward(do, q, k, v, o, lse, causal, window, scale, **lens)
    r = ref.attention(up(q), up(k), up(v), causal, window, scale, do=up(do), o=up(o), lse=up(lse), **lens)
    close(up(dv), r["dv"], w * r["dv_abs"] + e * r["dv"].abs() + tiny, "dv")
    for name, got in (("dq", dq), ("dk", dk)):
        close(up(got), r[name], w * r[name + "_abs"] + 2.0 ** -16 * r[name + "_pre"] + e * r[name].abs() + tiny, name)
    return o, lse, dq, dk, dv


LENGTHS = [(1, 1), (1, 2), (2, 1), (1, 200), (17, 17), (64, 64), (127, 127), (128, 128), (129, 129), (130, 257), (255, 256), (256, 128),
           (300, 300), (301, 77), (513, 513), (1025, 1025)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq,nk", LENGTHS)
def test_lengths(dtype, causal, nq, nk):
    check(*make(2, nq, nk, 2, 1, 64, dtype), causal=causal)


@pytest.mark.parametrize("d", [1, 7, 8, 16, 24, 40, 64, 72, 80, 96, 104, 120, 128, 136, 192, 256])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_head_sizes(dtype, d):
    check(*make(1, 200, 200, 2, 2, d, dtype))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 4), (4, 2), (8, 1), (6, 2), (5, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_shared_heads(hq, hkv, d):
    check(*make(2, 190, 190, hq, hkv, d, BF))


@pytest.mark.parametrize("window", [1, 2, 50, 127, 128, 129, 200, 400, 100000])
@pytest.mark.parametrize("nq,nk", [(400, 400), (150, 400), (400, 150)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_windows(dtype, window, nq, nk):
    check(*make(1, nq, nk, 2, 1, 64, dtype), window=window)


@pytest.mark.parametrize("d", [64, 128])
def test_longer_window_many_blocks(d):
    check(*make(1, 2000, 2000, 1, 1, d, BF), window=300)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("causal", [True, False])
def test_padded_batches_do_not_see_what_padding_holds(dtype, causal):
    q, k, v, do = make(6, 300, 300, 4, 2, 64, dtype)
    lens = torch.tensor([300, 1, 0, 128, 129, 255], dtype=torch.int32, device="cuda")
    dead = torch.arange(300, device="cuda")[None] >= lens[:, None]
    clean = check(q, k, v, do, causal=causal, q_lens=lens, k_lens=lens)
    for bad in (float("nan"), float("inf"), torch.finfo(dtype).min):
        qq, kk, vv, dd = (t.clone() for t in (q, k, v, do))
        for t in (qq, kk, vv, dd):
            t[dead] = bad
        from paper_2609_21594_b200 import functional as F

        o, lse = F.attention_forward(qq, kk, vv, causal, q_lens=lens, k_lens=lens)
        oo = o.clone()
        oo[dead] = bad
        got = F.attention_backward(dd, qq, kk, vv, oo, lse, causal, q_lens=lens, k_lens=lens)
        for a, b in zip((o, lse) + got, clean):
            assert torch.equal(a, b)
    assert not clean[0][dead].any() and all(not t[dead].any() for t in clean[2:])


def test_keys_shorter_than_queries_and_cross_attention():
    q, k, v, do = make(4, 200, 333, 2, 2, 128, BF)
    kl = torch.tensor([333, 0, 5, 130], dtype=torch.int32, device="cuda")
    check(q, k, v, do, causal=False, k_lens=kl)
    check(q, k, v, do, causal=True, k_lens=kl)             # queries before the first key see nothing
    check(q, k, v, do, causal=True, window=40, k_lens=kl, q_lens=torch.tensor([200, 17, 200, 0], dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (BF, 96), (F32, 64)])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 100), (False, 0)])
def test_packed(dtype, d, causal, window):
    lens = [1, 0, 127, 128, 300, 2, 0, 129, 65]
    off = torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int32, device="cuda")
    t = sum(lens) + 70                                       # the last 70 tokens belong to no sequence
    q, k, v, do = (x[0] for x in make(1, t, t, 4, 2, d, dtype))
    clean = check(q, k, v, do, causal=causal, window=window, q_offsets=off, k_offsets=off)
    for x in (clean[0], clean[2], clean[3], clean[4]):
        assert not x[sum(lens):].any()
    from paper_2609_21594_b200 import functional as F

    qq, kk, vv, dd = (x.clone() for x in (q, k, v, do))
    for x in (qq, kk, vv, dd):
        x[sum(lens):] = float("nan")
    a, l = 128 + 128, 128 + 128 + 300                        # and a NaN in one sequence stays there
    kk[a:l], vv[a:l] = float("nan"), float("inf")
    o, lse = F.attention_forward(qq, kk, vv, causal, window, q_offsets=off, k_offsets=off)
    got = F.attention_backward(dd, qq, kk, vv, o, lse, causal, window, q_offsets=off, k_offsets=off)
    keep = torch.ones(t, dtype=torch.bool, device="cuda")
    keep[a:l] = False
    assert torch.equal(o[keep], clean[0][keep]) and torch.equal(lse[:, keep], clean[1][:, keep])
    for x, y in zip(got, clean[2:]):
        assert torch.equal(x[keep], y[keep])


def test_packed_with_other_key_lengths():
    qo = torch.tensor([0, 10, 10, 200, 340], dtype=torch.int32, device="cuda")
    ko = torch.tensor([0, 130, 140, 140, 300], dtype=torch.int32, device="cuda")
    q, k, v, do = (x[0] for x in make(1, 340, 300, 2, 1, 64, BF))
    check(q, k, v, do, causal=True, q_offsets=qo, k_offsets=ko)
    check(q, k, v, do, causal=False, q_offsets=qo, k_offsets=ko)


@pytest.mark.parametrize("n", [40, 100])
def test_many_packed_sequences(n):
    g = torch.Generator().manual_seed(n)
    lens = torch.randint(0, 40, (n,), generator=g)
    off = torch.cat([torch.zeros(1, dtype=torch.int64), lens.cumsum(0)]).to(torch.int32).cuda()
    t = int(lens.sum())
    q, k, v, do = (x[0] for x in make(1, t, t, 2, 1, 64, BF))
    check(q, k, v, do, q_offsets=off, k_offsets=off)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_bad_length_tables_stay_inside_the_tensors(dtype):
    """Lengths and offsets live on the device and are clamped: results of a bad table mean nothing, but no other memory is touched."""
    from paper_2609_21594_b200 import functional as F

    q, k, v, do = make(2, 150, 150, 2, 1, 64, dtype)
    want = F.attention_forward(q, k, v)
    lens = torch.tensor([2 ** 31 - 1, 151], dtype=torch.int32, device="cuda")
    got = F.attention_forward(q, k, v, q_lens=lens, k_lens=lens)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    none = torch.tensor([-5, -2 ** 31], dtype=torch.int32, device="cuda")
    o, lse = F.attention_forward(q, k, v, q_lens=none, k_lens=none)
    assert not o.any() and (lse == -float("inf")).all()
    off = torch.tensor([-7, 900, 3, 2 ** 31 - 1, -1], dtype=torch.int32, device="cuda")
    o, lse = F.attention_forward(q[0], k[0], v[0], q_offsets=off, k_offsets=off)
    F.attention_backward(do[0], q[0], k[0], v[0], o, lse, q_offsets=off, k_offsets=off)
    torch.cuda.synchronize()


@pytest.mark.parametrize("d", [64, 128])
def test_views_and_orders(d):
    g = torch.Generator(device="cuda").manual_seed(9)
    fused = torch.randn((2, 210, 8, d), generator=g, device="cuda").to(BF)
    q, k, v = fused[:, :, :4], fused[:, :, 4:6], fused[:, :, 6:]
    do = torch.randn((2, 4, 210, d), generator=g, device="cuda").to(BF).transpose(1, 2)      # stored head by head
    views = check(q, k, v, do)
    dense = check(*(t.contiguous() for t in (q, k, v, do)))
    assert all(torch.equal(a, b) for a, b in zip(views, dense))
    # one token of padding per row, shared keys over the batch (stride 0), and a base that is not 16-byte aligned
    wide = torch.randn((2, 210, 4, d + 3), generator=g, device="cuda").to(BF)[..., :d]
    check(wide, k, v, do)
    check(q, k[:1].expand(2, -1, -1, -1), v[:1].expand(2, -1, -1, -1), do)
    odd = torch.randn((2 * 210 * 4 * d + 1,), generator=g, device="cuda").to(BF)[1:].view(2, 210, 4, d)
    check(odd, k, v, do)


@pytest.mark.parametrize("spread", [0.02, 1.0, 6.0])
@pytest.mark.parametrize("d", [64, 128])
def test_flat_and_peaked_rows(spread, d):
    check(*make(1, 300, 300, 2, 1, d, BF, spread=spread))


def test_scores_that_rise_along_the_row():
    """Every block of keys raises the running maximum by far more than one block's rounding."""
    q, k, v, do = make(1, 1500, 1500, 1, 1, 64, BF)
    q = q.abs()
    k = (k.abs() * torch.linspace(0.01, 8, 1500, device="cuda")[None, :, None, None]).to(BF)
    check(q, k, v, do, causal=False)
    check(q, k.flip(1), v, do, causal=False)
    check(q, k, v, do)


def test_other_scales():
    q, k, v, do = make(1, 140, 140, 2, 1, 64, BF)
    for scale in (1e-3, 0.5):
        check(q, k, v, do, scale=scale)


def test_special_values_reach_only_rows_that_see_them():
    from paper_2609_21594_b200 import functional as F

    q, k, v, do = make(1, 300, 300, 1, 1, 64, BF)
    o, lse = F.attention_forward(q, k, v)
    kk = k.clone()
    kk[0, 200, 0, 3] = float("nan")
    oo, ll = F.attention_forward(q, kk, v)
    assert torch.equal(oo[:, :200], o[:, :200]) and torch.equal(ll[..., :200], lse[..., :200])
    assert oo[:, 200:].isnan().all()
    qq = q.clone()
    qq[0, 7] = float("nan")
    oo, _ = F.attention_forward(qq, k, v)
    assert oo[0, 7].isnan().all()
    oo = torch.cat([oo[:, :7], oo[:, 8:]], 1)
    assert torch.equal(oo, torch.cat([o[:, :7], o[:, 8:]], 1))


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 64)])
def test_same_bits_every_time_and_on_another_stream(dtype, d):
    q, k, v, do = make(2, 700, 700, 4, 2, d, dtype)
    from paper_2609_21594_b200 import functional as F

    def run():
        o, lse = F.attention_forward(q, k, v)
        return (o, lse) + F.attention_backward(do, q, k, v, o, lse)

    first = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = run()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    assert F.context().muon_last_device_status() == 0


def test_batching_does_not_change_a_sequence():
    from paper_2609_21594_b200 import functional as F

    q, k, v, do = make(3, 260, 260, 4, 2, 64, BF)
    o, lse = F.attention_forward(q, k, v)
    grads = F.attention_backward(do, q, k, v, o, lse)
    for i in range(3):
        s = slice(i, i + 1)
        oi, li = F.attention_forward(q[s], k[s], v[s])
        gi = F.attention_backward(do[s], q[s], k[s], v[s], oi, li)
        assert torch.equal(oi, o[s]) and torch.equal(li, lse[s]) and all(torch.equal(a, b[s]) for a, b in zip(gi, grads))


def test_autograd_against_differences():
    """fp32: <gradient, direction> against the central difference of the 64-bit loss (off by h^2 / 6 of the third derivative, below 1e-6
    here); the gradients' own error is 2^-16 of the absolute sums: 1e-4 covers both."""
    from paper_2609_21594_b200 import functional as F

    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v, c = make(2, 33, 40, 4, 2, 24, F32, seed=4)
    lens = torch.tensor([40, 9], dtype=torch.int32, device="cuda")
    q, k, v = (t.requires_grad_() for t in (q, k, v))
    F.attention(q, k, v, True, 12, k_lens=lens).backward(c)
    loss = lambda a: (ref.attention(*a, True, 12, k_lens=lens)["o"] * c.double()).sum()  # noqa: E731
    base = [t.detach().double() for t in (q, k, v)]
    h = 1e-4
    for i, t in enumerate((q, k, v)):
        d = torch.randn(t.shape, generator=g, device="cuda").double()
        hi, lo = list(base), list(base)
        hi[i], lo[i] = base[i] + h * d, base[i] - h * d
        diff = float(loss(hi) - loss(lo)) / (2 * h)
        assert abs(float((t.grad.double() * d).sum()) - diff) <= 1e-4 * float((t.grad.double() * d).abs().sum())


def test_autograd_takes_broadcast_gradients():
    from paper_2609_21594_b200 import functional as F

    q, k, v, _ = make(1, 70, 70, 2, 1, 64, BF)
    q, k, v = (t.requires_grad_() for t in (q, k, v))
    F.attention(q, k, v).sum().backward()
    one = torch.ones_like(q)
    o, lse = F.attention_forward(q.detach(), k.detach(), v.detach())
    for t, g in zip((q, k, v), F.attention_backward(one, q.detach(), k.detach(), v.detach(), o, lse)):
        assert torch.equal(t.grad, g)


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("cuts", [[2], [3], [20], [128], [0, 2, 4, 20, 21, 149, 470, 512]])
def test_few_keys_keep_the_gradients_precision(cuts, d):
    """Up to 128 keys (512 packed ones) P and dS are two bf16 terms, 2^-16 together: with fp32's 2^-14 for the sums, 2^-13 of the absolute sums
    instead of 2^-8; only the rounding of the result is that of bf16."""
    from paper_2609_21594_b200 import functional as F

    n = cuts[-1]
    q, k, v, do = make(1, n, n, 4, 2, d, BF, seed=n + d)
    lens = {}
    if len(cuts) > 1:
        q, k, v, do = (t[0] for t in (q, k, v, do))
        at = torch.tensor(cuts, dtype=torch.int32, device="cuda")
        lens = dict(q_offsets=at, k_offsets=at)
    up = (lambda t: t[None]) if lens else (lambda t: t)
    o, lse = F.attention_forward(q, k, v, **lens)
    got = F.attention_backward(do, q, k, v, o, lse, **lens)
    r = ref.attention(up(q), up(k), up(v), do=up(do), o=up(o), lse=up(lse), **lens)
    for name, g in zip(("dq", "dk", "dv"), got):
        tol = 2.0 ** -13 * r[name + "_abs"] + 2.0 ** -8 * 1.01 * r[name].abs() + 1e-30
        if name != "dv":
            tol = tol + 2.0 ** -16 * r[name + "_pre"]
        close(up(g), r[name], tol, name)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_empty_calls(dtype):
    from paper_2609_21594_b200 import functional as F

    for b, nq, nk in ((0, 5, 5), (2, 0, 5), (2, 5, 0), (1, 0, 0)):
        q, k, v, do = make(b, nq, nk, 2, 1, 64, dtype)
        o, lse = F.attention_forward(q, k, v)
        dq, dk, dv = F.attention_backward(do, q, k, v, o, lse)
        assert o.shape == dq.shape == q.shape and dk.shape == dv.shape == k.shape
        assert all(not t.any() for t in (o, dq, dk, dv)) and (lse == -float("inf")).all()


def test_refusals():
    from paper_2609_21594_b200 import binding as mb
    from paper_2609_21594_b200 import functional as F

    q, k, v, do = make(2, 20, 20, 4, 2, 64, BF)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for call in (lambda: F.attention_forward(q, k.float(), v), lambda: F.attention_forward(q.half(), k.half(), v.half()),
                 lambda: F.attention_forward(q.cpu(), k.cpu(), v.cpu()), lambda: F.attention_forward(q, k[:, :, :1].expand(2, 20, 3, 64), v),
                 lambda: F.attention_forward(q, k, v[:, :19]), lambda: F.attention_forward(q, k[:1], v[:1]), lambda: F.attention_forward(q[0], k[0], v[0]),
                 lambda: F.attention_forward(q, torch.zeros((2, 20, 3, 64), dtype=BF, device="cuda"), torch.zeros((2, 20, 3, 64), dtype=BF, device="cuda")),
                 lambda: F.attention_forward(q, k, v, q_lens=i32(1, 2, 3)), lambda: F.attention_forward(q, k, v, q_lens=i32(1, 2).long()),
                 lambda: F.attention_forward(q[0], k[0], v[0], q_offsets=i32(0, 20)),
                 lambda: F.attention_forward(q[0], k[0], v[0], q_offsets=i32(0, 20), k_offsets=i32(0, 5, 20)),
                 lambda: F.attention_forward(q[0], k[0], v[0], q_offsets=i32(0), k_offsets=i32(0))):
        with pytest.raises(ValueError):
            call()
    for kw in ({"scale": 0.0}, {"scale": -1.0}, {"scale": float("nan")}, {"scale": float("inf")}, {"window": -1}, {"causal": False, "window": 4}):
        with pytest.raises(mb.MuonError) as e:
            F.attention_forward(q, k, v, **kw)
        assert e.value.code == mb.ERR_INVALID_ARG
    with pytest.raises(mb.MuonError) as e:
        F.attention_forward(*(torch.zeros((1, 4, 1, 264), dtype=BF, device="cuda") for _ in range(3)))
    assert e.value.code == mb.ERR_UNSUPPORTED
    o, lse = F.attention_forward(q, k, v)
    with pytest.raises(ValueError):
        F.attention_backward(do, q, k, v, o, lse[:1])
    with pytest.raises(ValueError):
        F.attention_backward(do[:, :5], q, k, v, o, lse)
    c = F.context()
    desc = mb.AttentionDesc(0, 2, 20, 20, 4, 2, 64, 1, 0, 0.125, 0, 0, None, None, None, None)
    h = F._heads
    before = c.muon_launch_count()
    for args in ((h(q), h(k), h(v), h(q), lse.data_ptr()), (h(q), h(k), h(v), mb.Heads(o.data_ptr(), 0, 256, 64), lse.data_ptr()),
                 (h(q), h(k), h(v), h(o), None), (mb.Heads(None, 1, 1, 1), h(k), h(v), h(o), lse.data_ptr()),
                 (mb.Heads(q.data_ptr() + 1, 1, 1, 1), h(k), h(v), h(o), lse.data_ptr())):
        with pytest.raises(mb.MuonError) as e:
            c.muon_attention_forward(desc, *args)
        assert e.value.code == mb.ERR_INVALID_ARG
    g = [torch.empty_like(t) for t in (q, k, v)]
    with pytest.raises(mb.MuonError) as e:
        c.muon_attention_backward(desc, h(do), h(q), h(k), h(v), h(o), lse.data_ptr(), h(g[0]), h(g[1]), h(g[2]), None, 0)
    assert e.value.code == mb.ERR_WORKSPACE_TOO_SMALL
    n = mb.muon_attention_workspace_bytes(desc)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    with pytest.raises(mb.MuonError) as e:
        c.muon_attention_backward(desc, h(do), h(q), h(k), h(v), h(o), lse.data_ptr(), h(g[0]), h(g[1]), h(g[1]), ws.data_ptr(), n)
    assert e.value.code == mb.ERR_INVALID_ARG              # dk and dv in one place
    assert c.muon_launch_count() == before
