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


def gated(x=P.AT, xs=128, y=P.AT, ys=128, n=3, xo=P.AT, xos=128, h=P.AT, hs=128, **kw):
    d = dict(dim=128, dtype=B.DP_BF16, stream_dtype=B.DP_F32, norm=1, n_groups=2, eps=1e-6, res_scale=1.0, gain=P.AT, post_gain=P.AT, gate=P.AT, scale=P.AT, shift=P.AT, group=P.AT)
    return P.L.dp_gated_norm(bytes(B.GatedNorm(**dict(d, **kw))), x, xs, y, ys, n, xo, xos, h, hs, None)


@pytest.mark.parametrize("bad", [dict(dim=0), dict(dim=12), dict(dim=16392), dict(dtype=2), dict(stream_dtype=2), dict(dtype=B.DP_F32, stream_dtype=B.DP_BF16), dict(norm=2), dict(n_groups=0),
                                 dict(eps=-1.0), dict(eps=float("inf")), dict(res_scale=float("inf")), dict(scale=None), dict(shift=None), dict(gain=P.AT + 4), dict(gate=P.AT + 8),
                                 dict(group=P.AT + 1), dict(n=-1), dict(n=(1 << 24) + 1), dict(x=None), dict(y=None), dict(h=None), dict(x=P.AT + 8), dict(y=P.AT + 2), dict(xs=130),
                                 dict(ys=132), dict(hs=-128), dict(xos=0), dict(hs=64), dict(xs=1 << 40), dict(y=None, xo=None, post_gain=None), dict(y=None, xo=None, gate=None),
                                 dict(h=None, gain=None), dict(h=None, xo=None, gain=None, scale=None, shift=None)], ids=str)
def test_bad_gated_norms(bad):
    P.refused(gated(**bad), "dp_gated_norm")


def test_gated_norms_of_nothing():
    assert gated(n=0) == B.DP_OK
    assert P.L.dp_gated_norm(None, P.AT, 0, P.AT, 0, 0, P.AT, 0, P.AT, 0, None) == B.DP_EINVAL


def test_the_binding_packs_what_the_struct_holds():
    assert B._PACK_GATED(1, 2, 3, 4, 5, 6.0, 7.0, 8, 9, 10, 11, 12, 13) == bytes(B.GatedNorm(1, 2, 3, 4, 5, 6.0, 7.0, 8, 9, 10, 11, 12, 13))


def linear(w=True, x=P.AT, xs=64, n=3, act=0, y=P.AT, ys=40, **kw):
    d = dict(out=40, in_=64, dtype=B.DP_BF16, codes=P.AT, scales=P.AT, bias=P.AT)
    return P.L.dp_linear_fp4(bytes(B.Fp4Matrix(**dict(d, **kw))) if w else None, x, xs, n, act, y, ys, None)


def pack(src=P.AT, stride=64, out=40, in_=64, dtype=B.DP_BF16, codes=P.AT, scales=P.AT):
    return P.L.dp_fp4_pack(src, stride, out, in_, dtype, codes, scales, None)


BAD_MATRIX = [dict(out=0), dict(out=(1 << 24) + 1), dict(in_=0), dict(in_=48), dict(in_=(1 << 20) + 32), dict(dtype=2), dict(codes=None), dict(scales=None), dict(codes=P.AT + 8)]


@pytest.mark.parametrize("bad", BAD_MATRIX + [dict(w=False), dict(n=-1), dict(n=(1 << 24) + 1), dict(n=1 << 12, out=1 << 24), dict(act=3), dict(act=-1), dict(x=None), dict(y=None), dict(x=P.AT + 8),
                                              dict(xs=68), dict(xs=-64), dict(xs=1 << 23), dict(y=P.AT + 1), dict(bias=P.AT + 1), dict(ys=39), dict(ys=1 << 39),
                                              dict(dtype=B.DP_F32, y=P.AT + 2)], ids=str)
def test_bad_linears(bad):
    P.refused(linear(**bad), "dp_linear_fp4")


@pytest.mark.parametrize("bad", BAD_MATRIX + [dict(src=None), dict(src=P.AT + 1), dict(stride=-1), dict(out=1 << 24, in_=1 << 13)], ids=str)
def test_bad_packs(bad):
    P.refused(pack(**bad), "dp_fp4_pack")


def test_linears_of_nothing():
    assert linear(n=0) == linear(n=0, x=None, y=None) == B.DP_OK
