"""What the entry points around the paged cache refuse, before anything is launched (no GPU), and what they take as nothing to do."""
import ctypes as C

import pytest

from paper_2505_21070_amd import binding as B

L = B._lib
AT = 1 << 20                                                  # an aligned address that no refused call looks at


def packed(struct):
    """The bytes that the binding hands over, None as a null pointer."""
    return bytes(struct)


def cache(**kw):
    d = dict(kv_heads=2, head_dim=128, page_tokens=16, n_pages=8, dtype=B.DP_BF16, format=1, data=AT, scales=AT)
    d.update(kw)
    return packed(B.KvCacheDesc(**d))


def norm(**kw):
    d = dict(q_heads=4, kv_heads=2, head_dim=128, dtype=B.DP_BF16, rope_theta=1e4, eps=1e-6, gq=AT, gk=AT, pos=AT)
    d.update(kw)
    return packed(B.NormRope(**d))


def attn(**kw):
    d = dict(q_heads=4, n_seqs=3, max_q=5, max_kv=60, table_width=4, causal_group=0, scale=0.1)
    d.update(kw)
    return packed(B.AttnConfig(**d))


def rows(heads, d=128, data=AT, ts=None, hs=None):
    return packed(B.KvRows(data, heads * d if ts is None else ts, d if hs is None else hs))


BAD_CACHE = [dict(kv_heads=0), dict(kv_heads=1025), dict(head_dim=96), dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=1 << 17),
             dict(n_pages=0), dict(n_pages=1 << 27), dict(dtype=2), dict(format=2), dict(data=None), dict(scales=None), dict(data=AT + 8)]
BAD_NORM = [dict(q_heads=0), dict(q_heads=2000), dict(kv_heads=-1), dict(head_dim=32), dict(dtype=7), dict(rope_theta=0.5), dict(rope_theta=float("nan")),
            dict(eps=-1.0), dict(eps=float("inf")), dict(gq=None), dict(gk=AT + 4), dict(pos=None), dict(pos=AT + 2)]
BAD_ATTN = [dict(q_heads=3), dict(q_heads=0), dict(n_seqs=-1), dict(n_seqs=65536), dict(max_q=-1), dict(max_q=(1 << 24) + 1), dict(max_kv=-1),
            dict(max_kv=2 ** 31 - 1), dict(table_width=-1), dict(causal_group=-1), dict(scale=0.0), dict(scale=float("nan")), dict(scale=float("inf"))]
BAD_ROWS = [dict(data=None), dict(data=AT + 2), dict(ts=260), dict(hs=132), dict(ts=-512), dict(ts=1 << 50)]


def write(c=None, k=None, v=None, slot=AT, n=3):
    return L.dp_kv_write(c or cache(), k or rows(2), v or rows(2), slot, n, None)


def read(c=None, k=None, v=None, slot=AT, n=3):
    return L.dp_kv_read(c or cache(), slot, n, k or rows(2), v or rows(2), None)


def qk(m=None, q=None, k=None, qo=None, ko=None, n=3):
    return L.dp_qk_norm_rope(m or norm(), q or rows(4), k or rows(2), n, qo or rows(4), ko or rows(2), None)


def qkv(c=None, m=None, q=None, k=None, v=None, slot=AT, n=3, qo=None):
    return L.dp_kv_write_qkv(c or cache(), m or norm(), q or rows(4), k or rows(2), v or rows(2), slot, n, qo or rows(4), None)


def attend(c=None, a=None, q=None, n=7, start=AT, lens=AT, table=AT, out=None, work=AT, nbytes=0):
    return L.dp_attn_paged(c or cache(), a or attn(), q or rows(4), n, start, lens, table, out or rows(4), work, nbytes, None)


def refused(rc, entry):
    assert rc == B.DP_EINVAL and B.last_error().startswith(entry + ": "), (rc, B.last_error())


@pytest.mark.parametrize("bad", BAD_CACHE, ids=str)
def test_bad_caches(bad):
    refused(write(c=cache(**bad)), "dp_kv_write")
    refused(read(c=cache(**bad)), "dp_kv_read")
    refused(qkv(c=cache(**bad)), "dp_kv_write_qkv")
    refused(attend(c=cache(**bad)), "dp_attn_paged")
    assert L.dp_attn_paged_workspace_bytes(cache(**bad), attn(), 7) == 0


@pytest.mark.parametrize("bad", BAD_NORM, ids=str)
def test_bad_norms(bad):
    refused(qk(m=norm(**bad)), "dp_qk_norm_rope")
    refused(qkv(m=norm(**bad)), "dp_kv_write_qkv")


@pytest.mark.parametrize("bad", BAD_ATTN, ids=str)
def test_bad_attention_configs(bad):
    refused(attend(a=attn(**bad)), "dp_attn_paged")
    assert L.dp_attn_paged_workspace_bytes(cache(), attn(**bad), 7) == 0


@pytest.mark.parametrize("bad", BAD_ROWS, ids=str)
def test_bad_rows(bad):
    for r in ("q", "k", "qo", "ko"):
        refused(qk(**{r: rows(4 if r[0] == "q" else 2, **bad)}), "dp_qk_norm_rope")
    for r in ("k", "v"):
        refused(write(**{r: rows(2, **bad)}), "dp_kv_write")
        refused(read(**{r: rows(2, **bad)}), "dp_kv_read")
    for r in ("q", "k", "v", "qo"):
        refused(qkv(**{r: rows(4 if r[0] == "q" else 2, **bad)}), "dp_kv_write_qkv")
    for r in ("q", "out"):
        refused(attend(**{r: rows(4, **bad)}), "dp_attn_paged")


def test_written_rows_do_not_overlap():
    for ts, hs in ((0, 128), (512, 0), (512, 120), (384, 128), (120, 1024), (128, 256)):
        refused(qk(qo=rows(4, ts=ts, hs=hs)), "dp_qk_norm_rope")
        refused(attend(out=rows(4, ts=ts, hs=hs)), "dp_attn_paged")
    refused(read(k=rows(2, ts=128)), "dp_kv_read")


def test_norm_and_cache_agree():
    for other in (dict(kv_heads=4), dict(head_dim=64), dict(dtype=B.DP_F32)):
        refused(qkv(m=norm(**other)), "dp_kv_write_qkv")


def test_null_pointers_and_counts():
    refused(L.dp_kv_write(None, rows(2), rows(2), AT, 3, None), "dp_kv_write")
    refused(L.dp_qk_norm_rope(None, rows(4), rows(2), 3, rows(4), rows(2), None), "dp_qk_norm_rope")
    refused(L.dp_attn_paged(cache(), None, rows(4), 7, AT, AT, AT, rows(4), AT, 0, None), "dp_attn_paged")
    refused(L.dp_attn_paged(cache(), attn(), None, 7, AT, AT, AT, rows(4), AT, 0, None), "dp_attn_paged")
    for n in (-1, (1 << 24) + 1):
        refused(write(n=n), "dp_kv_write")
        refused(read(n=n), "dp_kv_read")
        refused(qk(n=n), "dp_qk_norm_rope")
        refused(qkv(n=n), "dp_kv_write_qkv")
        refused(attend(n=n), "dp_attn_paged")
    for slot in (None, AT + 1):
        refused(write(slot=slot), "dp_kv_write")
        refused(read(slot=slot), "dp_kv_read")
        refused(qkv(slot=slot), "dp_kv_write_qkv")
    for kw in (dict(start=None), dict(lens=None), dict(table=None), dict(start=AT + 2), dict(lens=AT + 1), dict(table=AT + 3)):
        refused(attend(**kw), "dp_attn_paged")


def test_workspaces():
    big = attn(q_heads=4, n_seqs=1, max_q=1, max_kv=4000, table_width=250)
    need = L.dp_attn_paged_workspace_bytes(cache(), big, 1)
    assert need > 0 and L.dp_attn_paged_workspace_bytes(cache(), big, 0) == 0
    for work, nbytes in ((None, need), (AT, need - 1), (AT, 0)):
        assert attend(a=big, n=1, work=work, nbytes=nbytes) == B.DP_ENOMEM and "workspace" in B.last_error()
    refused(attend(a=big, n=1, work=AT + 128, nbytes=need), "dp_attn_paged")
    refused(attend(a=attn(q_heads=512), n=1 << 22, q=rows(512), out=rows(512)), "dp_attn_paged")
    refused(attend(a=attn(q_heads=512), n=(1 << 20) + 1, q=rows(512), out=rows(512)), "dp_attn_paged")
    refused(attend(c=cache(kv_heads=64), a=attn(q_heads=64, n_seqs=(1 << 15) + 1), q=rows(64), out=rows(64)), "dp_attn_paged")


def test_workspaces_stay_bounded():
    """Partial results take at most 16 times as many blocks as the chip holds, whatever the bounds of the launch."""
    for dtype in (B.DP_F32, B.DP_BF16):
        for heads, d in ((1, 64), (40, 128), (1024, 64)):
            for n_seqs in (1, 40, 2000):
                for max_q in (1, 30, 100, 5000, 1 << 24):
                    for max_kv in (1, 5000, 2 ** 31 - 1 - 65536):
                        c = cache(dtype=dtype, kv_heads=heads, head_dim=d, page_tokens=65536)
                        a = attn(q_heads=heads, n_seqs=n_seqs, max_q=max_q, max_kv=max_kv, table_width=1 << 16)
                        assert L.dp_attn_paged_workspace_bytes(c, a, min(1 << 24, (1 << 29) // heads)) <= 16 * 512 * 128 * (d + 2) * 4


def test_nothing_to_do():
    assert write(n=0, slot=None) == read(n=0, slot=None) == qk(n=0) == qkv(n=0, slot=None) == B.DP_OK
    assert L.dp_kv_write(cache(), None, None, None, 0, None) == B.DP_OK
    assert attend(n=0, start=None, lens=None, table=None) == B.DP_OK
    assert attend(a=attn(n_seqs=0)) == attend(a=attn(max_q=0)) == B.DP_OK
    assert C.sizeof(B.KvCacheDesc) == 40 and C.sizeof(B.KvRows) == 24 and C.sizeof(B.NormRope) == 48 and C.sizeof(B.AttnConfig) == 28
