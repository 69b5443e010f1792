"""A bounded wait that expires in one thread's call is seen by the others: backward passes run in threads of autograd's that nobody can ask."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


def in_a_thread(f):
    out = []
    t = threading.Thread(target=lambda: out.append(f()))
    t.start()
    t.join()
    return out[0]


def test_every_thread_sees_an_expired_wait():
    from paper_2609_21594_b200 import binding as mb
    from paper_2609_21594_b200 import functional as F

    F.synchronize_and_check()
    mine = F.context().handle.value

    def fails():
        c = F.context()
        c.muon_self_test_bounded_wait()                      # waits a millisecond for what never comes, records it and ends
        torch.cuda.synchronize()
        return c.handle.value

    assert in_a_thread(fails) != mine
    try:
        assert F.context().muon_last_device_status() == 100 and F.context().muon_synchronize_and_check() == mb.ERR_DEVICE_TIMEOUT
        assert in_a_thread(lambda: F.context().muon_last_device_status()) == 100
        with pytest.raises(mb.MuonError) as e:
            F.synchronize_and_check()
        assert e.value.code == mb.ERR_DEVICE_TIMEOUT
    finally:
        F.context().muon_clear_device_status()
    F.synchronize_and_check(torch.device("cuda"))
    assert in_a_thread(lambda: F.context().muon_last_device_status()) == 0


def test_backward_passes_record_where_the_main_thread_looks():
    from paper_2609_21594_b200 import functional as F

    seen = []

    class Probe(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return x.clone()

        @staticmethod
        def backward(ctx, g):
            seen.append((threading.get_ident(), F.context().handle.value, F.context().muon_device_status_word()))
            return g

    x = torch.randn(4, 64, device="cuda", requires_grad=True)
    F.layer_norm(Probe.apply(x)).sum().backward()
    assert seen[0][0] != threading.get_ident() and seen[0][1] != F.context().handle.value
    assert seen[0][2] == F.context().muon_device_status_word()


def test_contexts_of_a_program_share_a_word_when_told_to():
    from paper_2609_21594_b200 import binding as mb

    a, b = mb.Context(), mb.Context()
    own = b.muon_device_status_word()
    assert own != a.muon_device_status_word()
    b.muon_share_device_status(a.muon_device_status_word())
    b.muon_self_test_bounded_wait()
    torch.cuda.synchronize()
    assert a.muon_last_device_status() == b.muon_last_device_status() == 100
    b.muon_share_device_status(None)
    assert b.muon_device_status_word() == own and b.muon_last_device_status() == 0
    with pytest.raises(mb.MuonError) as e:
        b.muon_share_device_status(own + 2)
    assert e.value.code == mb.ERR_INVALID_ARG
    a.muon_clear_device_status()
    # the whole-iteration launch of small sets counts arrivals in the context's own memory, whatever word it shares
    x = torch.randn(256, 256, device="cuda").bfloat16()
    want, got = torch.empty_like(x), torch.empty_like(x)
    b.muon_share_device_status(a.muon_device_status_word())
    for c, out in ((a, want), (b, got), (a, want), (b, got)):
        c.ensure_workspace([(256, 256)])
        c.muon_orthogonalize_batched([x], [out], [(256, 256)], 5, (3.4445, -4.7750, 2.0315))
    torch.cuda.synchronize()
    assert torch.equal(want, got) and a.muon_last_device_status() == 0
    b.close()
    a.close()
