"""Bounded waits of the matrix products around the feed-forward block, read from the kernels' text: none may cover more than its limit allows for, however
large the call; and where long sums are cut into parts."""
import os
import re

import pytest

from paper_2609_21594_b200 import binding as mb
from test_layer_sources import CSRC, kernel


def number(file, name):
    """A constant as the source defines it: digits, or 1 << digits."""
    text = re.search(name + r" = (1 << )?(\d+)(?:LL)?[;,]", open(os.path.join(CSRC, file)).read())
    return (1 << int(text.group(2))) if text.group(1) else int(text.group(2))


def test_a_tile_is_done_long_before_its_wait_gives_up():
    wait, longest, most = number("tc_common.cuh", "WAIT_CYCLES"), number("product_ops.h", "kLongestSum"), number("product_ops.h", "kMostSum")
    clocks = 800                                             # of a k-block: 560 on CTA pairs, 48 KiB at 64 bytes a clock in the few-token kernel
    assert longest <= most and most // 64 * clocks * 100 < wait
    take = open(os.path.join(CSRC, "product_tc.cu")).read()
    take = take[take.index("bool products_tc_take("):]
    assert "if (!e.sums && int64_t(p.k) * p.segments > kMostSum) return false;" in take[:take.index("\n}\n")]


def test_the_last_products_are_waited_for_when_the_tiles_are_done():
    body = kernel("product_tc.cu", "product_pair_kernel")
    waits = [m.start() for m in re.finditer(r"mbar_wait\(drain_bar", body)]
    assert len(waits) == 1
    before = body[:waits[0]]
    assert before.rindex("give_up(34)") < before.rindex("__syncthreads();") < waits[0] < body.rindex("cluster_sync_all();")


@pytest.mark.parametrize("tokens,more", [(1 << 18, False), ((1 << 18) + 1, True), (1 << 22, True)])
def test_room_for_the_parts_of_long_sums(tokens, more):
    up = lambda n, m=256: -(-n // m) * m  # noqa: E731
    d = mb.FeedForwardDesc(mb.DTYPE_BF16, mb.ACTIVATION_SILU, mb.KEEP_FULL, tokens, 64, 136)
    parts = 2 * up(136 * 64 * 4) + up(64 * 192 * 4)
    assert mb.muon_feed_forward_workspace_bytes(d, True) == 3 * up(tokens * 136 * 2) + (parts if more else 0)
    assert mb.muon_feed_forward_workspace_bytes(d, False) == up(tokens * 136 * 2)
    d.dtype = mb.DTYPE_FP32
    assert mb.muon_feed_forward_workspace_bytes(d, True) == 3 * up(tokens * 136 * 4)
    lin = mb.LinearBlocksDesc(tokens, 64, 136, 0)
    assert mb.muon_linear_blocks_workspace_bytes(lin, True) == (up(tokens * 144) + up(tokens * 16) + up(tokens * 64 * 2) + (up(136 * 64 * 4) if more else 0))
