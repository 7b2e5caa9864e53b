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


def gated(x=P.AT, xs=128, y=2 * P.AT, ys=128, n=3, xo=P.AT, xos=128, h=2 * P.AT, hs=128, **kw):
    d = dict(dim=128, dtype=B.DP_BF16, stream_dtype=B.DP_F32, norm=1, n_groups=2, eps=1e-6, res_scale=1.0, gain=P.AT, post_gain=P.AT, gate=P.AT, scale=P.AT, shift=P.AT, group=P.AT)
    return P.L.dp_gated_norm(bytes(B.GatedNorm(**dict(d, **kw))), x, xs, y, ys, n, xo, xos, h, hs, None)


@pytest.mark.parametrize("bad", [dict(dim=0), dict(dim=12), dict(dim=16392), dict(dtype=2), dict(stream_dtype=2), dict(dtype=B.DP_F32, stream_dtype=B.DP_BF16), dict(norm=2), dict(n_groups=0),
                                 dict(eps=-1.0), dict(eps=float("inf")), dict(res_scale=float("inf")), dict(scale=None), dict(shift=None), dict(gain=P.AT + 4), dict(gate=P.AT + 8),
                                 dict(group=P.AT + 1), dict(n=-1), dict(n=(1 << 24) + 1), dict(x=None), dict(y=None), dict(h=None), dict(x=P.AT + 8), dict(y=P.AT + 2), dict(xs=130),
                                 dict(ys=132), dict(hs=-128), dict(xos=0), dict(hs=64), dict(xs=1 << 40), dict(y=None, xo=None, post_gain=None), dict(y=None, xo=None, gate=None),
                                 dict(h=None, gain=None), dict(h=None, xo=None, gain=None, scale=None, shift=None), dict(h=P.AT),
                                 dict(n=(1 << 24) - 1, dim=2056, xs=2056, ys=2056, xos=2056, hs=2056)], ids=str)
def test_bad_gated_norms(bad):
    P.refused(gated(**bad), "dp_gated_norm")


def test_gated_norms_of_nothing():
    assert gated(n=0) == B.DP_OK
    assert P.L.dp_gated_norm(None, P.AT, 0, P.AT, 0, 0, P.AT, 0, P.AT, 0, None) == B.DP_EINVAL


def test_the_binding_packs_what_the_struct_holds():
    assert B._PACK_GATED(1, 2, 3, 4, 5, 6.0, 7.0, 8, 9, 10, 11, 12, 13) == bytes(B.GatedNorm(1, 2, 3, 4, 5, 6.0, 7.0, 8, 9, 10, 11, 12, 13))


def linear(w=True, x=P.AT, xs=64, n=3, act=0, y=2 * P.AT, ys=40, work=P.AT, nbytes=1 << 40, **kw):
    d = dict(out=40, in_=64, dtype=B.DP_BF16, laid=P.AT, bias=P.AT)
    return P.L.dp_linear_fp4(bytes(B.Fp4Matrix(**dict(d, **kw))) if w else None, x, xs, n, act, y, ys, work, nbytes, None)


def pack(src=P.AT, stride=64, out=40, in_=64, dtype=B.DP_BF16, codes=P.AT, scales=P.AT):
    return P.L.dp_fp4_pack(src, stride, out, in_, dtype, codes, scales, None)


def lay(codes=P.AT, scales=P.AT, out=40, in_=64, laid=P.AT):
    return P.L.dp_fp4_lay(codes, scales, out, in_, laid, None)


BAD_SIZES = [dict(out=0), dict(out=-1), dict(out=(1 << 24) + 1), dict(in_=0), dict(in_=48), dict(in_=(1 << 20) + 32), dict(out=1 << 24, in_=1 << 13)]
BAD_CODES = [dict(codes=None), dict(scales=None), dict(codes=P.AT + 8)]


@pytest.mark.parametrize("bad", BAD_SIZES + [dict(w=False), dict(dtype=2), dict(n=-1), dict(n=(1 << 24) + 1), dict(n=1 << 12, out=1 << 24), dict(act=3), dict(act=-1), dict(x=None), dict(y=None),
                                             dict(laid=None), dict(laid=P.AT + 32), dict(x=P.AT + 8), dict(xs=68), dict(xs=-64), dict(xs=1 << 22), dict(y=P.AT + 1), dict(bias=P.AT + 1),
                                             dict(ys=39), dict(ys=1 << 39), dict(y=P.AT), dict(dtype=B.DP_F32, y=P.AT + 2), dict(out=512, in_=13824, ys=512, xs=13824, work=P.AT + 128)], ids=str)
def test_bad_linears(bad):
    P.refused(linear(**bad), "dp_linear_fp4")


@pytest.mark.parametrize("bad", BAD_SIZES + BAD_CODES + [dict(dtype=2), dict(src=None), dict(src=P.AT + 1), dict(stride=-1), dict(stride=1 << 39)], ids=str)
def test_bad_packs(bad):
    P.refused(pack(**bad), "dp_fp4_pack")


@pytest.mark.parametrize("bad", BAD_SIZES + BAD_CODES + [dict(laid=None), dict(laid=P.AT + 16)], ids=str)
def test_bad_lays(bad):
    P.refused(lay(**bad), "dp_fp4_lay")
    if bad in BAD_SIZES:
        assert P.L.dp_fp4_laid_bytes(bad.get("out", 40), bad.get("in_", 64)) == 0


def test_sizes_and_linears_of_nothing():
    assert linear(n=0) == linear(n=0, x=None, y=None, laid=None) == B.DP_OK
    assert P.L.dp_fp4_laid_bytes(1, 32) == 1088 and P.L.dp_fp4_laid_bytes(17, 160) == 4 * 1088 and P.L.dp_fp4_laid_bytes(1 << 24, 1 << 12) == (1 << 25) * 1088
    w = bytes(B.Fp4Matrix(512, 13824, B.DP_BF16, P.AT, None))
    need = P.L.dp_linear_fp4_workspace_bytes(w, 2)
    assert need >= 2 * 512 * 4 * 2 and P.L.dp_linear_fp4_workspace_bytes(w, 0) == 0 and P.L.dp_linear_fp4_workspace_bytes(w, -1) == 0
    assert linear(out=512, in_=13824, ys=512, xs=13824, n=2, nbytes=need - 1) == linear(out=512, in_=13824, ys=512, xs=13824, n=2, work=None) == B.DP_ENOMEM


def test_workspaces_are_bounded():
    """Ranges only where the tiles do not fill the chip: at most 8 ranges of 768 blocks' outputs."""
    for out in (1, 100, 5120, 1 << 20, 1 << 24):
        for in_ in (32, 5120, 13824, 1 << 20):
            for n in (1, 17, 64, 100, 1000, 1 << 16):
                if out * in_ <= 1 << 36 and n * out <= 1 << 35:
                    for dtype in (B.DP_BF16, B.DP_F32):
                        assert P.L.dp_linear_fp4_workspace_bytes(bytes(B.Fp4Matrix(out, in_, dtype, P.AT, None)), n) <= 768 * 256 * 256 * 4
