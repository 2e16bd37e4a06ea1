"""CPU: the workspace of the attention over chosen blocks against the bound that the header states, over the whole range of its arguments."""
import pytest

import paper_2104_05343_amd as opt

GIB = 1 << 30


def bound(matrices, s, d, block, count):
    """For each (sequence, head) 9 bytes an entry of its choice, 40 a query and 1024; and partial results of 1 GiB, or of one (sequence, head)."""
    return matrices * (s * (9 * count + 40) + 1024) + max(GIB, d * (3 * s * count + 8 * (s + block))) + 4096


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", [-1, 0, 1])
def test_no_more_than_the_header_says(d, form):
    opt.debug_set_attention_selected_form(form)
    try:
        for block in (64, 128, 192, 256, 448, 512, 1024, 1088, 2048, 3584, 4096):
            for s in (1, 63, 64, 1000, 4096, 10000, 32768, 65536, 65537, 1 << 17, (1 << 18) + 1, 1 << 19, (1 << 20) - 1, 1 << 20):
                for count in (1, 2, 3, 8, 16, 24, 64):
                    for heads, b in ((1, 1), (8, 1), (3, 5), (16, 16)):
                        sel = opt.make_selection(block, count)
                        got = opt.attention_selected_workspace_bytes(b, s, heads * d, heads, 1, 0, 0, sel)
                        assert (got == 0) == ((s - 1) // block >= 1024)
                        assert got <= bound(b * heads, s, d, block, count), (block, s, count, heads, b, got / GIB)
    finally:
        opt.debug_set_attention_selected_form(-1)


def test_several_matrices_share_a_portion():
    """More (sequence, head)s cost their lists only, once 1 GiB, or one of them, is full of partial results."""
    size = lambda heads, s, block, count: opt.attention_selected_workspace_bytes(1, s, heads * 128, heads, 1, 0, 0, opt.make_selection(block, count))   # noqa: E731
    for s, block, count in ((16384, 64, 4), (65536, 128, 16), (1 << 18, 512, 8), (1 << 18, 4096, 8), (1 << 20, 4096, 1)):
        few, many = size(16, s, block, count), size(64, s, block, count)
        assert many - few <= 48 * (s * (9 * count + 40) + 1024) + GIB
