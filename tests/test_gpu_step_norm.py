"""wsr_block_norm against its formula in 64 bits: both kinds and types, every optional part, widths from 8 to
32768, strided and in-place rows, infinities and NaN."""
import pytest
import torch

import step_util as su
from gpu_util import needs_gpu, stream
from paper_2608_12114_amd import wsr

pytestmark = [pytest.mark.gpu, needs_gpu]
FMT = {torch.float16: wsr.WSR_F16, torch.bfloat16: wsr.WSR_BF16}


def _call(y, h, T, d, dt, kind, post, gate=None, res=1.0, vec=None, eps=1e-5, want_h=True, want_x=True, h_out=None, x=None, **over):
    vec = vec or {}
    h_out = torch.full((T, d), float("nan"), device="cuda") if want_h and h_out is None else h_out
    x = torch.full((T, d), float("nan"), dtype=dt, device="cuda") if want_x and x is None else x
    st = lambda t: 0 if t is None or t.dim() < 2 or t.shape[0] == 1 else t.stride(0) * t.element_size()  # noqa: E731
    f = dict(kind=wsr.WSR_NORM_LAYER if kind == "layer" else wsr.WSR_NORM_RMS, fmt=FMT[dt], n_tokens=T, d=d, eps=eps,
             flags=wsr.WSR_BLOCK_POST if post else 0, res_scale=res, y=y, y_tok_stride=st(y), gate=gate, gate_tok_stride=st(gate),
             h=h, h_tok_stride=st(h), h_out=h_out, h_out_tok_stride=st(h_out) if h_out is not None else 0, x=x,
             x_tok_stride=st(x) if x is not None else 0, **vec)
    b = wsr.make_block(**{**f, **over})
    wsr.wsr_block_norm(b, stream())
    torch.cuda.synchronize()
    return h_out, x


def _inputs(T, d, dt, kind, post, gate, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    vec = {"pre_w": (1 + 0.2 * r(d)).to(dt)}
    if post:
        vec["post_w"] = (1 + 0.2 * r(d)).to(dt)
    if kind == "layer":
        vec["pre_b"] = (0.1 * r(d)).to(dt)
        if post:
            vec["post_b"] = (0.1 * r(d)).to(dt)
    gt = None if gate == "none" else (0.5 + 0.3 * r(*((T, d) if gate == "token" else (d,)))).to(dt)
    return r(T, d) * 2 + 0.5, r(T, d) * 3, vec, gt


def _check(h_out, x, y, h, kind, post, gate, res, vec, dt, eps=1e-5):
    eh, ex = su.block64(y, h, kind=kind, post=post, gate=gate, res=res, eps=eps, **vec)
    # a row's statistics carry a few roundings of 32 bits, each product and sum one more: 16 covers them;
    # magnitudes: of the terms of the sums
    size = eh.abs() + (0 if h is None else (res * h.double()).abs()) + (0 if y is None else 1.0)
    row = eh.abs().amax(-1, keepdim=True)
    if h_out is not None:
        err = (h_out.double() - eh).abs()
        assert (err <= 32 * su.U32 * (size + row)).all(), float((err / (size + row)).max())
    if x is not None:
        err = (x.double() - ex).abs()
        slack = 64 * su.U32 * (ex.abs() + ex.abs().amax(-1, keepdim=True) + 1)
        assert (err <= su.U16[dt] * ex.abs() + slack + 2.0 ** -25).all(), float(err.max())


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("T,d", [(1, 8), (3, 120), (2, 512), (5, 520), (1, 2048), (7, 2056), (1, 4096), (16, 8192),
                                 (2, 8200), (3, 16384), (2, 16392), (1, 32768), (513, 1160), (2049, 256)])
def test_matches_formula(T, d, kind, dt):
    gate = ("none", "channel", "token")[(T + d // 8) % 3]
    y, h, vec, gt = _inputs(T, d, dt, kind, True, gate, seed=T + d)
    h_out, x = _call(y, h, T, d, dt, kind, True, gt, 0.9, vec)
    _check(h_out, x, y, h, kind, True, gt, 0.9, vec, dt)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("parts", ["no_y", "no_h", "no_weights", "no_x", "no_h_out"])
def test_optional_parts(parts, post, kind):
    T, d, dt = 5, 1032, torch.bfloat16
    y, h, vec, gt = _inputs(T, d, dt, kind, post, "token", seed=3)
    y, h = (None if parts == "no_y" else y), (None if parts == "no_h" else h)
    vec = {} if parts == "no_weights" else vec
    h_out, x = _call(y, h, T, d, dt, kind, post, gt, 1.25, vec, want_x=parts != "no_x", want_h=parts != "no_h_out")
    _check(h_out, x, y, h, kind, post, gt, 1.25, vec, dt)


def test_in_place_and_strided():
    T, d, dt = 6, 2048, torch.float16
    y, h, vec, gt = _inputs(T, d, dt, "rms", True, "channel", seed=9)
    ya, ha = torch.zeros((T, d + 40), device="cuda"), torch.zeros((T, d + 8), device="cuda")
    xa = torch.full((T, d + 24), 7.0, dtype=dt, device="cuda")
    ya[:, :d], ha[:, :d] = y, h
    _call(ya[:, :d], ha[:, :d], T, d, dt, "rms", True, gt, 0.5, vec, h_out=ha[:, :d], x=xa[:, :d])
    _check(ha[:, :d], xa[:, :d], y, h, "rms", True, gt, 0.5, vec, dt)
    assert (xa[:, d:] == 7).all() and (ha[:, d:] == 0).all()


def test_zero_rows_and_broken_rows_stay_apart():
    """A row of zeros gives zeros (eps), and a row with an infinity or a NaN leaves the others alone."""
    T, d, dt = 4, 4096, torch.bfloat16
    y, h, vec, _ = _inputs(T, d, dt, "rms", True, "none", seed=5)
    y[0], h[0] = 0, 0
    y[1, 7], h[2, 9] = float("nan"), float("inf")
    h_out, x = _call(y, h, T, d, dt, "rms", True, None, 1.0, vec)
    assert (h_out[0] == 0).all() and (x[0] == 0).all()
    assert torch.isnan(h_out[1]).all() and torch.isnan(x[1]).all()
    assert h_out[2, 9] == float("inf") and torch.isfinite(h_out[2]).sum() == d - 1
    _check(h_out[3:], x[3:], y[3:], h[3:], "rms", True, None, 1.0, vec, dt)


def test_same_bits_and_other_stream():
    T, d, dt = 33, 4096, torch.bfloat16
    y, h, vec, gt = _inputs(T, d, dt, "layer", True, "token", seed=6)
    a = _call(y, h, T, d, dt, "layer", True, gt, 0.9, vec)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = _call(y, h, T, d, dt, "layer", True, gt, 0.9, vec)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_nothing_to_do():
    wsr.wsr_block_norm(wsr.make_block(kind=0, fmt=1, n_tokens=0, d=64), stream())
    wsr.wsr_block_norm(wsr.make_block(kind=0, fmt=1, n_tokens=3, d=0), stream())
