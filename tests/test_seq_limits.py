"""Ranges of the sequence descriptors that their launches need, by host-only calls."""
from paper_2607_22696_amd import _binding as B
from tests.test_seq_abi import append, forward, paged, paged_desc, seq_desc

import paper_2607_22696_amd as dsa


def test_workgroups():
    """2^31 - 2^22 workgroups: sequences + 1 (and a tile per 128 rows) times heads."""
    most = (1 << 31) - (1 << 22)
    for heads in (127, 128):
        d = seq_desc(batch=(1 << 24) - 1, heads=heads, kv_heads=heads, rel_buckets=0)
        fits = heads << 24 <= most
        assert fits == (heads == 127)
        assert (dsa.dsa3d_seq_backward_workspace_size(d) > 0) == fits
        if not fits:
            assert forward(d) == B.DSA3D_ERR_INVALID_SHAPE
    # the groups' heads share their key head's tiles in the paged form
    wide = dict(batch=(1 << 24) - 1, max_kv=16, rel_buckets=0)
    assert paged(paged_desc(heads=128, kv_heads=128, **wide)) == B.DSA3D_ERR_INVALID_SHAPE
    # a write has a wave per token, whatever the requests and heads: refused for its table alone
    d = paged_desc(heads=128, kv_heads=128, max_kv=0, batch=(1 << 24) - 1)
    assert append(d, k=None) == B.DSA3D_ERR_NULL_POINTER


def test_tokens_of_a_request():
    """2^30 at most for the forward, by max_kv or by the page table."""
    long = dict(page_size=1 << 20, num_pages=8, max_pages=1 << 11, rel_buckets=0)
    assert paged(paged_desc(**long)) == B.DSA3D_ERR_INVALID_SHAPE
    for bound, refused in (((1 << 30) + 1, True), (1 << 30, False)):
        d = paged_desc(max_kv=bound, **long)
        assert (dsa.dsa3d_paged_forward_workspace_size(d) == 0) == refused
