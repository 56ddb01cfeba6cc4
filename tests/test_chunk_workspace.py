"""The workspace of the attention of chunks, on the host: its size from the shape alone."""
import pytest

import paper_2507_01663_amd as ra


def shape(T=7, B=7, most=1, Hq=8, Hkv=2, D=128, pages=40, kv=ra.RA_KV_BF16):
    p = ra.ra_extend()
    p.num_seqs, p.total_tokens, p.max_chunk_len = B, T, most
    p.Hq, p.Hkv, p.D, p.page_size, p.num_pages, p.max_pages_per_seq, p.kv_dtype = Hq, Hkv, D, 16, 900, pages, kv
    return p


@pytest.mark.parametrize("kv", [ra.RA_KV_BF16, ra.RA_KV_FP8_E4M3])
@pytest.mark.parametrize("B,Hq,Hkv,D,pages", [(7, 8, 2, 128, 40), (256, 28, 4, 128, 300), (1, 4, 2, 64, 3), (64, 32, 2, 64, 12)])
def test_the_size_is_the_shape_s(B, Hq, Hkv, D, pages, kv):
    """A descriptor with dimensions, page counts and the pools' type alone is told what the call will want, also for single tokens."""
    p = shape(B, B, 1, Hq, Hkv, D, pages, kv)
    bare = ra.rollout_attn_extend_workspace_size(None, p)
    p.q_stride_token = Hq * D
    assert ra.rollout_attn_extend_workspace_size(None, p) == bare
    p.q_stride_token = Hq * D + 64
    assert ra.rollout_attn_extend_workspace_size(None, p) == bare
    d = ra.ra_problem()
    d.B, d.Hq, d.Hkv, d.D, d.page_size, d.num_pages, d.max_pages_per_seq, d.kv_dtype = B, Hq, Hkv, D, 16, 900, pages, kv
    assert bare >= ra.rollout_attn_workspace_size(None, d)
