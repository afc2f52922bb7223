"""Workspaces of tree attention (no GPU): one that is made for the largest step serves every smaller
one, whatever form of the kernel that takes.  Sizes are refused before any HIP call."""
import pytest

from paper_2606_03077_amd import libra

P = 4096  # an aligned address that nothing here reads
WORKSPACE = 3
HEADS = [(32, 8), (28, 4), (8, 1), (16, 1), (4, 4)]


@pytest.mark.parametrize("hq,hkv", HEADS)
def test_the_size_for_the_most_is_enough_for_less(hq, hkv):
    rows = [1, 3, 16, 64, 65, 128, 200, 512, 1024, 1025, 2047, 2048, 8192, 40000]
    batches = [1, 2, 7, 32, 33, 64, 256]
    size = {(r, b): libra.libra_tree_attn_workspace_bytes(r, b, hq, hkv) for r in rows for b in batches}
    for (r, b), most in size.items():
        assert most > 0
        assert all(size[s, c] <= most for s in rows for c in batches if s <= r and c <= b), (r, b)


@pytest.mark.parametrize("rows,batch", [(2048, 32), (1024, 32), (640, 20), (2048, 16), (5, 3)])
def test_a_call_takes_the_workspace_of_a_larger_one(rows, batch):
    """32 / 8 heads, 64 nodes a request or half of that: only below its own size is one refused."""
    most = libra.libra_tree_attn_workspace_bytes(2048, 32, 32, 8)
    layout = libra.libra_kv_layout_create(P, P, 10, 8)
    need = libra.libra_tree_attn_workspace_bytes(rows, batch, 32, 8)
    short = libra.load().libra_tree_attn(layout, P, rows, P, P, None, 0, P, 4, batch, 32, 0.1, P, need - 1, 2 * P,
                                         None, None)
    assert need <= most and short == WORKSPACE
    libra.libra_kv_layout_destroy(layout)
