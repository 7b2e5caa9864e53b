"""Gated residual with the norms around it on the GPU, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import fp4 as F
from paged import HALF, TD, U, np64

pytestmark = pytest.mark.gpu
TYPES = [("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32")]            # of the stream, of the rows
SUM = 46                                                            # roundings of a row's sum: 32 values a lane, 6 steps over lanes, 8 wavefronts


def normed(v, dv, kind, eps):
    """N(v), and a bound of what fp32 makes of it from v with an error of up to dv: the mean's sum, the centred values, the squares' sum (SUM roundings and
    the products' own, halved by the root; the root and its product 3), and how far dv moves mean and deviation."""
    n = F.norm(v, kind, eps)
    mean = v.mean(-1, keepdims=True) if kind == "layer" else 0.0
    dev = np.sqrt(((v - mean) ** 2).mean(-1, keepdims=True) + eps)
    shift = (dv.mean(-1, keepdims=True) + SUM * U * np.abs(v).mean(-1, keepdims=True)) if kind == "layer" else 0.0
    dz = dv + shift + U * np.abs(v - mean)
    rel = (SUM / 2 + 5) * U + np.sqrt((dz ** 2).mean(-1, keepdims=True)) / dev
    return n, dz / dev + np.abs(n) * rel


def bounds(x, y, kind, eps, res_scale, gain, post_gain, gate, scale, shift, group):
    """x', h and their bounds before the last rounding."""
    x = np64(x)
    of = (lambda v: np64(v)[group]) if group is not None else (lambda v: np64(v)[0])
    dx = np.zeros_like(x)
    if y is not None:
        t, dt = np64(y), np.zeros_like(x)
        if post_gain is not None:
            t, dt = normed(t, dt, kind, eps)
            g = np64(post_gain)
            dt = dt * np.abs(g) + U * np.abs(t * g)
            t = t * g
        f = res_scale * (np.ones_like(x) if gate is None else of(gate))
        x = x + f * t
        dx = np.abs(f) * dt + 2 * U * np.abs(f * t) + U * np.abs(x)
    h, dh = normed(x, dx, kind, eps)
    if gain is not None:
        g = np64(gain)
        h, dh = h * g, dh * np.abs(g) + U * np.abs(h * g)
    if scale is not None:
        m = 1 + of(scale)
        h, dh = h * m + of(shift), dh * np.abs(m) + 2 * U * np.abs(h * m)
        dh = dh + U * np.abs(h)
    return x, dx, h, dh


def check(got, ref, work, dtype, where):
    err, tol = np.abs(np64(got) - ref), (HALF[dtype] * np.abs(ref) + work) * (1 + 2.0 ** -7) + 1e-37
    bad = ~(err <= tol) & where[:, None]
    assert not bad.any(), (np.argwhere(bad)[:4].tolist(), float((err / tol)[bad].max()))


def inputs(n, d, stream, dtype, groups, seed=0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen)   # noqa: E731
    x, y = (r(n, d) * 2 + 0.5).to(TD[stream]), r(n, d).to(TD[dtype])
    x[:, ::16] *= 5
    gains = [(r(d) * 0.2 + 1).to(TD[dtype]).cuda() for _ in range(2)]
    vectors = [(r(groups, d) * 0.5).cuda() for _ in range(3)]
    return x.cuda(), y.cuda(), gains, vectors


FORMS = {
    "everything": (True, True, True, True), "modulated": (False, True, False, True), "gains": (True, True, True, False), "bare": (False, False, False, False),
}


@pytest.mark.parametrize("stream,dtype", TYPES)
@pytest.mark.parametrize("n,d,groups", [(1, 8, 1), (3, 64, 2), (5, 520, 5), (130, 1536, 3), (2, 2048, 1), (9, 2056, 2), (4, 4104, 4), (6, 5120, 2), (3, 8192, 3), (2, 8200, 1), (2, 16384, 2),
                                        (70, 1000, 64), (5, 1032, 2), (3, 6152, 1), (2, 12296, 2)])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_against_the_definition(kind, n, d, groups, stream, dtype):
    from paper_2505_21070_amd import binding as B
    x, y, (gain, post), (gate, scale, shift) = inputs(n, d, stream, dtype, groups, seed=d)
    group = torch.randint(0, groups, (n,), generator=torch.Generator().manual_seed(1)).to(torch.int32)
    all_ = np.ones(n, bool)
    for with_gain, with_gate, with_post, modulated in FORMS.values():
        kw = dict(gain=gain if with_gain else None, post_gain=post if with_post else None, gate=gate if with_gate else None, scale=scale if modulated else None,
                  shift=shift if modulated else None)
        xo, h = B.gated_norm(x, y, norm=kind, res_scale=-0.75, eps=1e-5, group=group.cuda() if with_gate else None, **kw)
        assert xo.dtype == TD[stream] and h.dtype == TD[dtype]
        rx, dx, rh, dh = bounds(x, y, kind, float(np.float32(1e-5)), -0.75, group=group.numpy() if with_gate else None, **kw)
        check(xo, rx, dx, stream, all_)
        check(h, rh, dh, dtype, all_)
    # before the first branch and behind the last one
    none, first = B.gated_norm(x, gain=gain, norm=kind, dtype=dtype)
    _, _, rh, dh = bounds(x, None, kind, float(np.float32(1e-6)), 1.0, gain, None, None, None, None, None)
    assert none is None
    check(first, rh, dh, dtype, all_)
    last, none = B.gated_norm(x, y, post_gain=post, norm=kind, next_norm=False)
    both, _ = B.gated_norm(x, y, post_gain=post, norm=kind)
    assert none is None and torch.equal(last, both)


@pytest.mark.parametrize("stream,dtype", TYPES)
@pytest.mark.parametrize("d", [256, 5120])
def test_padding_strides_and_in_place(d, stream, dtype):
    from paper_2505_21070_amd import binding as B
    n = 11
    x, y, (gain, post), (gate, scale, shift) = inputs(n, d, stream, dtype, 3)
    group = torch.tensor([0, 2, 1, -1, 0, 3, 2, -2 ** 31, 2 ** 31 - 1, 1, 2], dtype=torch.int32, device="cuda")
    live = ((group >= 0) & (group < 3)).cpu().numpy()
    kw = dict(gain=gain, post_gain=post, gate=gate, scale=scale, shift=shift, group=group, norm="rms")
    xo, h = torch.full_like(x, 7.0), torch.full_like(y, 7.0)
    a, b = B.gated_norm(x, y, x_out=xo, out=h, **kw)
    assert a is xo and b is h and (xo[~live] == 7).all() and (h[~live] == 7).all()
    ref = bounds(x, y, "rms", float(np.float32(1e-6)), 1.0, gain, post, gate, scale, shift, np.where(live, group.cpu().numpy(), 0))
    check(xo, ref[0], ref[1], stream, live)
    check(h, ref[2], ref[3], dtype, live)
    # in place, in wider rows, every second one
    wide = torch.zeros((2 * n, d + 8), dtype=TD[stream], device="cuda")[::2, :d]
    wide_y = torch.zeros((n, 3 * d), dtype=TD[dtype], device="cuda")[:, d: 2 * d]
    wide.copy_(x)
    wide_y.copy_(y)
    a, b = B.gated_norm(wide, wide_y, x_out=wide, out=wide_y, **kw)
    assert a is wide and torch.equal(wide[live], xo[live]) and torch.equal(wide_y[live], h[live]) and torch.equal(wide[~live], x[~live]) and torch.equal(wide_y[~live], y[~live])
    # one row as all rows' stream
    one = x[:1].expand(n, d)
    xo2, h2 = B.gated_norm(one, y, **kw)
    ref = B.gated_norm(one.contiguous(), y, **kw)
    assert torch.equal(xo2[live], ref[0][live]) and torch.equal(h2[live], ref[1][live])


@pytest.mark.parametrize("d", [64, 4096])
def test_values_that_are_not_finite_and_rows_of_zeros(d):
    from paper_2505_21070_amd import binding as B
    x, y = torch.zeros((5, d), device="cuda"), torch.zeros((5, d), device="cuda")
    x[1, 3], x[2, 4], y[3, 5] = float("nan"), float("inf"), float("inf")
    x[4] = 3.0
    xo, h = B.gated_norm(x, y)
    assert (h[0] == 0).all() and torch.isnan(h[1:4]).all() and (h[4] == 0).all() and torch.equal(xo[4], x[4])
    xo, h = B.gated_norm(x, y, norm="rms")
    assert (h[0] == 0).all() and torch.isnan(h[1]).all() and torch.isnan(h[2, 4]) and (h[2, :4] == 0).all() and torch.isinf(xo[3, 5]) and (xo[3, :5] == 0).all()
    # a branch behind its norm: NaN where it was infinite, whole rows where it was NaN, other rows not touched
    post = torch.ones(d, device="cuda")
    xo, h = B.gated_norm(x, y, post_gain=post, norm="layer")
    assert torch.isnan(xo[3]).all() and torch.equal(xo[4], x[4]) and (h[0] == 0).all()


def test_no_rows_and_repeated_bits():
    from paper_2505_21070_amd import binding as B
    x, y, (gain, post), (gate, scale, shift) = inputs(300, 5120, "f32", "bf16", 2)
    kw = dict(gain=gain, post_gain=post, gate=gate, scale=scale, shift=shift, group=(torch.arange(300, device="cuda") % 2).to(torch.int32))
    xo, h = B.gated_norm(x[:0], y[:0], **dict(kw, group=kw["group"][:0]))
    assert xo.shape == h.shape == (0, 5120) and xo.dtype == torch.float32 and h.dtype == torch.bfloat16
    a, b = B.gated_norm(x, y, **kw), B.gated_norm(x, y, **kw)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # a row's bits do not depend on the rows around it
    c = B.gated_norm(x[17:18], y[17:18], **dict(kw, group=kw["group"][17:18]))
    assert torch.equal(c[0][0], a[0][17]) and torch.equal(c[1][0], a[1][17])


def test_captured_and_replayed_beside_eager_calls():
    from paper_2505_21070_amd import binding as B
    x, y, (gain, post), (gate, scale, shift) = inputs(40, 1536, "f32", "bf16", 1)
    kw = dict(gain=gain, post_gain=post, gate=gate, scale=scale, shift=shift)
    xo, h = torch.empty_like(x), torch.empty_like(y)
    B.gated_norm(x, y, x_out=xo, out=h, **kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.gated_norm(x, y, x_out=xo, out=h, **kw)
    for k in range(4):
        x.add_(0.25)
        graph.replay()
        torch.cuda.synchronize()
        ex, eh = B.gated_norm(x, y, **kw)
        assert torch.equal(ex, xo) and torch.equal(eh, h)


def test_on_a_named_stream():
    from paper_2505_21070_amd import binding as B
    x, y, (gain, post), _ = inputs(2000, 5120, "f32", "bf16", 1)
    ref = B.gated_norm(x, y, post_gain=post)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = B.gated_norm(x, y, post_gain=post, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


def test_refused_by_the_binding():
    from paper_2505_21070_amd import binding as B
    x, y, (gain, post), (gate, scale, shift) = inputs(4, 64, "f32", "bf16", 2)
    group = torch.zeros(4, dtype=torch.int32, device="cuda")
    for args, kw in (((x, y[:3]), {}), ((x, y.cpu()), {}), ((x.bfloat16(), y.float()), {}), ((x.double(), y), {}), ((x, y), dict(gain=gain.float())), ((x, y), dict(gate=gate[0])),
                     ((x, y), dict(gate=gate, scale=scale[:1], shift=shift[:1], group=group)), ((x, y), dict(group=group.long())), ((x, y), dict(group=group[:3])),
                     ((x,), dict(next_norm=False)), ((x,), dict(x_out=x)), ((x, y), dict(next_norm=False, out=y)), ((x, y.t().contiguous().t()), {}), ((x, y), dict(out=x))):
        with pytest.raises(AssertionError):
            B.gated_norm(*args, **kw)
    with pytest.raises(KeyError):
        B.gated_norm(x, y, norm="batch")
    for args, kw in (((x, y), dict(scale=scale)), ((x, y), dict(eps=-1.0)), ((x, y), dict(res_scale=float("nan"))), ((x[:, :60], y[:, :60]), {}), ((x,), dict(gate=gate)),
                     ((x, y), dict(x_out=x[:1].expand(4, 64)))):
        with pytest.raises(B.DualParalError) as e:
            B.gated_norm(*args, **kw)
        assert e.value.code == B.DP_EINVAL
