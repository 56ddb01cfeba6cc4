"""CPU-side checks of the C ABI for chunks of new tokens: exported symbols, struct layouts, the host-only argument checks."""
import ctypes
import os
import re

import pytest

import paper_2507_01663_amd as ra

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "rollout_attn_chunk.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(rollout_attn_[a-z_]+)\s*\(", text)))
    assert len(names) == 7, names
    lib = ra.load_library()
    for n in names:
        assert getattr(lib, n) is not None and hasattr(ra, n)


def test_struct_layouts():
    assert ctypes.sizeof(ra.ra_rotate) == 16 + 32 + 32 + 16 + 8 + 16 + 16
    assert ctypes.sizeof(ra.ra_append_chunk) == 136 + 16 + 8 + 16 + 16 + 24 + 24 + 8 + 16
    assert ctypes.sizeof(ra.ra_extend) == 24 + 16 + 16 + 16 + 24 + 24 + 8 + 16 + 8 + 16


def rotate():
    r = ra.ra_rotate()
    r.num_tokens, r.Hq, r.Hkv, r.D = 5, 8, 2, 128
    r.q, r.k, r.q_out, r.k_out = 0x10000, 0x20000, 0x30000, 0x40000
    r.q_stride_token, r.k_stride_token, r.q_out_stride_token, r.k_out_stride_token = 12 * 128, 12 * 128, 8 * 128, 2 * 128
    r.q_weight, r.k_weight, r.eps = 0x50000, 0x60000, 1e-6
    r.positions, r.rope, r.rope_len, r.rot_dim = 0x70000, 0x80000, 100, 128
    return r


def cache(p, fp8=False):
    p.num_seqs, p.max_chunk_len = 3, 4
    p.cu_seqlens, p.seq_lens, p.block_table = 0x90000, 0xA0000, 0xB0000
    p.page_size, p.num_pages, p.max_pages_per_seq = 16, 64, 8
    p.k_pool, p.v_pool = 0xC0000, 0xD0000
    p.kv_stride_token, p.kv_stride_head, p.kv_stride_page = 128, 16 * 128, 2 * 16 * 128
    if fp8:
        p.kv_dtype, p.k_scale, p.v_scale = ra.RA_KV_FP8_E4M3, 0xE0000, 0xF0000
    return p


def append(fp8=False):
    p = ra.ra_append_chunk()
    p.rot = rotate()
    p.rot.k_out = None
    p.v, p.v_stride_token = 0x100000, 12 * 128
    return cache(p, fp8)


def extend(fp8=False):
    p = ra.ra_extend()
    p.total_tokens, p.Hq, p.Hkv, p.D = 5, 8, 2, 128
    p.q, p.q_stride_token, p.out, p.lse, p.softmax_scale = 0x10000, 8 * 128, 0x20000, 0x30000, 0.1
    return cache(p, fp8)


BAD, NOT = ra.RA_ERR_INVALID_ARG, ra.RA_ERR_UNSUPPORTED
ROWS = [
    (dict(num_tokens=-1), BAD, "dimension"), (dict(Hq=-1), BAD, "dimension"), (dict(D=0), BAD, "dimension"), (dict(D=96), NOT, "D="),
    (dict(rot_dim=129), BAD, "rot_dim"), (dict(rot_dim=-16), BAD, "rot_dim"), (dict(rot_dim=24), NOT, "rot_dim"),
    (dict(eps=-1.0), BAD, "eps"), (dict(eps=float("nan")), BAD, "eps"), (dict(q_out=None), BAD, "q_out"), (dict(q=0x10008), BAD, "aligned"),
    (dict(q_stride_token=8 * 128 - 8), BAD, "stride"), (dict(k_stride_token=12 * 128 + 4), BAD, "stride"), (dict(q_weight=0x50004), BAD, "aligned"),
    (dict(rope=None), BAD, "rope"), (dict(rope=0x80008), BAD, "aligned"), (dict(rope_len=-1), BAD, "rope_len"), (dict(q_stride_token=2 ** 44), NOT, "large"),
]
CACHE = [
    (dict(num_seqs=-1), BAD, "dimension"), (dict(max_chunk_len=-1), BAD, "dimension"), (dict(page_size=0), BAD, "dimension"),
    (dict(page_size=32), NOT, "page_size"), (dict(kv_dtype=2), BAD, "kv_dtype"), (dict(cu_seqlens=None), BAD, "pointer"), (dict(seq_lens=None), BAD, "pointer"),
    (dict(block_table=None), BAD, "pointer"), (dict(v_pool=None), BAD, "pointer"), (dict(kv_stride_token=64), BAD, "stride"),
    (dict(kv_stride_page=-16), BAD, "stride"), (dict(kv_stride_head=16 * 128 + 4), BAD, "16 bytes"), (dict(k_pool=0xC0008), BAD, "aligned"),
    (dict(kv_stride_token=2 ** 27), NOT, "large"), (dict(num_seqs=2 ** 20, max_pages_per_seq=2 ** 12), NOT, "large"),
]


def refused(check, make, changes, inner=lambda p: p):
    assert check(make()) == (ra.RA_OK, "")
    assert check(None)[0] == BAD
    for change, status, word in changes:
        p = make()
        for k, v in change.items():
            setattr(inner(p), k, v)
        st, msg = check(p)
        assert st == status and word in msg, (change, st, msg)


def test_check_rotate():
    refused(ra.rollout_attn_check_rotate, rotate, ROWS + [(dict(positions=None), BAD, "positions"), (dict(k_out=None), BAD, "k_out")])
    for gone in (("q", "q_out"), ("k", "k_out"), ("rope", "positions", "rot_dim"), ("q_weight", "k_weight")):     # parts that may be absent
        r = rotate()
        for f in gone:
            setattr(r, f, 0 if f == "rot_dim" else None)
        assert ra.rollout_attn_check_rotate(r)[0] == ra.RA_OK
    r = ra.ra_rotate()
    r.D = 64
    assert ra.rollout_attn_check_rotate(r)[0] == ra.RA_OK              # nothing to do needs no pointers


def test_check_append_chunk():
    for fp8 in (False, True):
        refused(ra.rollout_attn_check_append_chunk, lambda: append(fp8), CACHE + [(dict(v=None), BAD, "v"), (dict(v=0x100008), BAD, "aligned"),
                                                                                 (dict(v_stride_token=128), BAD, "stride")])
        refused(ra.rollout_attn_check_append_chunk, lambda: append(fp8), ROWS + [(dict(k=None), BAD, "k"), (dict(k_out=0x40000), BAD, "k_out"),
                                                                                (dict(Hkv=0), BAD, "Hkv")], inner=lambda p: p.rot)
    p = append(True)
    p.v_scale = None
    assert ra.rollout_attn_check_append_chunk(p)[0] == BAD
    p = append()
    p.rot.positions, p.rot.q, p.rot.q_out = None, None, None           # positions from the cache, keys and values alone
    assert ra.rollout_attn_check_append_chunk(p)[0] == ra.RA_OK


def test_check_extend():
    own = [(dict(total_tokens=-1), BAD, "dimension"), (dict(Hkv=0), BAD, "dimension"), (dict(Hq=7), BAD, "multiple"), (dict(softmax_scale=0.0), BAD, "positive"),
           (dict(softmax_scale=float("inf")), BAD, "finite"), (dict(D=96), NOT, "D="), (dict(Hq=258), NOT, "Hq/Hkv"), (dict(q=None), BAD, "pointer"),
           (dict(out=None), BAD, "pointer"), (dict(lse=None), BAD, "pointer"), (dict(q=0x10008), BAD, "aligned"), (dict(lse=0x30002), BAD, "aligned"),
           (dict(q_stride_token=7 * 128), BAD, "stride"), (dict(q_stride_token=8 * 128 + 4), BAD, "stride"),
           (dict(max_chunk_len=2 ** 30), NOT, "large"), (dict(total_tokens=2 ** 24, max_pages_per_seq=2 ** 14), NOT, "large")]
    for fp8 in (False, True):
        refused(ra.rollout_attn_check_extend, lambda: extend(fp8), CACHE + own)
    p = extend(True)
    p.k_scale = None
    assert ra.rollout_attn_check_extend(p)[0] == BAD


def test_extend_workspace_size():
    p = extend()
    assert ra.rollout_attn_extend_workspace_size(None, p) % 256 == 0
    p.max_pages_per_seq = 200                                          # long enough to be shared by workgroups
    n = ra.rollout_attn_extend_workspace_size(None, p)
    assert n > 0 and n % 256 == 0
    p.D = 100
    with pytest.raises(ra.RolloutAttnError) as e:
        ra.rollout_attn_extend_workspace_size(None, p)
    assert e.value.status == NOT
    p.D, p.Hq = 128, 7
    with pytest.raises(ra.RolloutAttnError) as e:
        ra.rollout_attn_extend_workspace_size(None, p)
    assert e.value.status == BAD


def test_calls_without_a_context_are_rejected():
    for call, desc, more in ((ra.rollout_attn_rotate, rotate(), ()), (ra.rollout_attn_append_chunk, append(), ()), (ra.rollout_attn_extend, extend(), (None, 0))):
        with pytest.raises(ra.RolloutAttnError) as e:
            call(None, desc, *more)
        assert e.value.status == BAD
