"""What the entry points of the cache in 4 bits refuse, before anything is launched (no GPU)."""
import pytest

import test_paged_refusals as P
from paper_2505_21070_amd import binding as B


def cache4(**kw):
    return P.cache(**dict(dict(format=4), **kw))


@pytest.mark.parametrize("bad", [dict(scales=None), dict(data=None), dict(data=P.AT + 8), dict(head_dim=96), dict(head_dim=32), dict(page_tokens=8), dict(dtype=2),
                                 dict(n_pages=0), dict(kv_heads=0), dict(format=3), dict(format=5), dict(format=-4)], ids=str)
def test_bad_caches(bad):
    P.refused(P.write(c=cache4(**bad)), "dp_kv_write")
    P.refused(P.read(c=cache4(**bad)), "dp_kv_read")
    P.refused(P.qkv(c=cache4(**bad)), "dp_kv_write_qkv")
    P.refused(P.attend(c=cache4(**bad)), "dp_attn_paged")
    assert P.L.dp_attn_paged_workspace_bytes(cache4(**bad), P.attn(), 7) == 0


def test_nothing_to_do():
    assert P.write(c=cache4(), n=0) == P.read(c=cache4(), n=0) == P.qkv(c=cache4(), n=0) == P.attend(c=cache4(), n=0) == B.DP_OK
