"""Layer norm, preference loss and orthogonalised updates on the GPU against their float64 definitions.

Tolerances, with u = 2^-24 (an fp32 rounding) and half(t) = torch.finfo(t).eps / 2 (the one rounding of an output of type t):
* Sums of n terms in fp32, n_seq of them one after the other and the rest in a tree, are off by at most (n_seq + log2 n + 2) u times the
  sum of the terms' magnitudes; the bounds below take n_seq from the kernels' layout, rounded up.
* ex2.approx is off by 2^-22 relative; an exponent of magnitude r by r u (the FMA) and 2^-26 r (the constant).
* Newton-Schulz: a product of split operands is off by d = 3 * 2^-22 + ceil(K / 16) * 2^-24 of its size (two terms of 11 bits each and
  the product left out; an MMA of 16 terms truncates its sum, which grows linearly, by 2^-23 at most); three products per step
  and the polynomial's slope, at most 1.8 in the two or three steps in which singular values are near one (before them error
  and value grow alike), give 5 * 3 * 1.8^3 d < 90 d.
"""
import ctypes
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import dp_oracle
from oracle import operators_oracle as O
from paper_2609_40335_b200 import binding as dp

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
QUINTIC = ((3.4445, -4.7750, 2.0315),) * 5


def half(dtype):
    return torch.finfo(dtype).eps / 2


def f64(t):
    return t.detach().double().cpu().numpy()


def close(got, want, abs_err, dtype=torch.float32):
    """|got - want| within abs_err (of fp32 arithmetic) and the rounding of the result."""
    got, want = f64(got), np.asarray(want)
    off = np.abs(got - want)
    room = abs_err + half(dtype) * (np.abs(want) + abs_err)
    assert got.shape == want.shape and np.isfinite(got).all()
    assert (off <= room).all(), (float((off - room).max()), float(off.max()), np.unravel_index(np.argmax(off - room), off.shape))


def tensor(shape, dtype, seed, std=1.0, mean=0.0, pitch=None, offset=0):
    """Normal values in a tensor of rows `pitch` apart that starts `offset` elements into its buffer; NaN around them."""
    g = torch.Generator().manual_seed(seed)
    p = shape[-1]
    pitch = pitch or p
    rows = math.prod(shape[:-1])
    buf = torch.full((offset + rows * pitch,), float("nan"), dtype=dtype, device="cuda")
    view = buf[offset:].view(*shape[:-1], pitch)[..., :p]
    view.copy_((torch.randn(*shape, generator=g) * std + mean).to(dtype))
    return view


def surroundings_untouched(t, pitch, offset):
    """Nothing was written around a tensor made by tensor()."""
    if pitch and pitch > t.shape[-1]:
        base = t.as_strided(t.shape[:-1] + (pitch,), t.stride(), t.storage_offset())
        assert torch.isnan(base[..., t.shape[-1]:].float()).all()
    if offset:
        assert torch.isnan(t.as_strided((offset,), (1,), 0).float()).all()


# ------------------------------------------------------------------------------------- layer norm
LN_WIDTHS = [1, 2, 7, 8, 31, 64, 100, 257, 520, 768, 1000, 1001, 1024, 1032, 2049, 4096, 8200, 16383, 16384]


@pytest.mark.parametrize("p", LN_WIDTHS)
@pytest.mark.parametrize("dtype,params,pad,offset", [("f32", "f32", 0, 0), ("bf16", "f32", 0, 0), ("bf16", "bf16", 8, 0), ("f32", "bf16", 3, 1),
                                                     ("bf16", "f32", 5, 3)])
def test_layernorm(p, dtype, params, pad, offset):
    rows, dt, pt = 21, DT[dtype], DT[params]
    x = tensor((rows, p), dt, p, mean=0.3, pitch=p + pad, offset=offset)
    gain, shift = tensor((1, p), pt, p + 1, 0.3, 1.0)[0], tensor((1, p), pt, p + 2, 0.2)[0]
    y, hat = (tensor((rows, p), dt, 5, pitch=p + pad, offset=offset) for _ in range(2))
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dp.dp_layernorm(x, gain, shift, 1e-5, Y=y, X_hat=hat, mean=mean, rstd=rstd)
    wy, wh, wm, wr = O.layernorm(f64(x), f64(gain), f64(shift), 1e-5)
    # 32 values of a thread one after the other, 10 joins, a division
    s = 45 * U
    size = np.abs(f64(x)).mean(-1, keepdims=True)
    close(mean, wm, s * size[:, 0])
    # mean enters the variance to second order; half of its relative error, square root and division
    wr_err = wr * (0.5 * s + 4 * U + 0.5 * (s * size[:, 0] * wr) ** 2)
    close(rstd, wr, wr_err)
    h_err = (s * size + 2 * U * (np.abs(f64(x)) + np.abs(wm)[:, None])) * wr[:, None] + np.abs(wh) * (wr_err / wr)[:, None]
    close(hat, wh, h_err, dt)
    close(y, wy, h_err * np.abs(f64(gain)) + 2 * U * (np.abs(wy) + np.abs(f64(shift))), dt)
    for t in (y, hat):
        surroundings_untouched(t, p + pad, offset)


def test_layernorm_optional_outputs_and_in_place():
    x = tensor((3, 5, 96), torch.bfloat16, 1, mean=1.0)
    hat = torch.empty_like(x)
    y = torch.empty_like(x)
    dp.dp_layernorm(x, None, None, 1e-5, Y=y, X_hat=hat)
    assert torch.equal(y, hat)                                       # no gain, no shift
    gain = tensor((1, 96), torch.float32, 2)[0]
    dp.dp_layernorm(x, gain, None, 1e-5, Y=y)
    z = x.clone()
    dp.dp_layernorm(z, gain, None, 1e-5, Y=z)                        # in place
    assert torch.equal(y, z)
    only = torch.empty(15, device="cuda")
    dp.dp_layernorm(x, None, None, 1e-5, mean=only)
    close(only, f64(x).reshape(15, 96).mean(-1), 45 * U * 1.5)


def test_layernorm_rows_of_equal_values_and_values_that_are_not_finite():
    x = torch.full((4, 64), 3.0, device="cuda")
    x[1, 5], x[2, 7] = float("nan"), float("inf")
    y, rstd = torch.empty_like(x), torch.empty(4, device="cuda")
    dp.dp_layernorm(x, None, None, 1e-5, Y=y, rstd=rstd)
    assert not y[0].any() and not y[3].any() and abs(rstd[0].item() * math.sqrt(1e-5) - 1) < 1e-6
    assert torch.isnan(y[1]).all() and torch.isnan(y[2]).all()       # and no other row


BACK = [
    # B, T, p: one token; one example; odd; wide; ragged against the cluster's parts; more parts than rows
    (1, 1, 1), (4, 16, 64), (3, 1, 768), (2, 5, 7), (5, 33, 100), (21, 40, 257), (2, 203, 768), (1, 300, 1001), (7, 9, 1024),
    (2, 17, 1032), (1, 64, 2049), (3, 12, 4096), (1, 20, 8200), (1, 3, 16384), (2, 3, 16383), (300, 3, 64), (1, 1500, 64), (2, 1111, 776),
    (16, 640, 776), (1, 4100, 1001)]                            # sums through the workspace


@pytest.mark.parametrize("B,T,p", BACK)
@pytest.mark.parametrize("dtype,params,pad,offset", [("f32", "f32", 0, 0), ("bf16", "f32", 0, 0), ("bf16", "bf16", 8, 0), ("f32", "f32", 3, 1),
                                                     ("bf16", "f32", 5, 3)])
def test_layernorm_backward(B, T, p, dtype, params, pad, offset):
    dt, pt = DT[dtype], DT[params]
    x = tensor((B, T, p), dt, p + T, mean=0.3, pitch=p + pad, offset=offset)
    g = tensor((B, T, p), dt, p + T + 1, std=1e-2, pitch=p + pad, offset=offset)
    gain = tensor((1, p), pt, p + 2, 0.3, 1.0)[0]
    _, _, m, r = O.layernorm(f64(x), eps=1e-5)
    mean, rstd = (torch.from_numpy(v).float().cuda().contiguous() for v in (m, r))
    dx = tensor((B, T, p), dt, 9, pitch=p + pad, offset=offset)
    gs, ss = torch.full((B, p), 7.0, device="cuda"), torch.full((B, p), 7.0, device="cuda")
    sq = torch.full((B,), 0.5, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    dp.dp_layernorm_backward(g, x, gain, mean, rstd, dX=dx, gain_sums=gs, shift_sums=ss, sq=sq, dev_status=st)
    assert int(st.item()) == 0
    m, r = f64(mean), f64(rstd)
    wdx, wgs, wss, wsq = O.layernorm_backward(f64(g), f64(x), f64(gain), m, r)
    hat = (f64(x) - m[..., None]) * r[..., None]
    hat_err = 2 * U * (np.abs(f64(x)) + np.abs(m)[..., None]) * r[..., None] + U * np.abs(hat)
    u = np.abs(f64(g) * f64(gain))
    s = 45 * U
    m1, m2 = s * u.mean(-1, keepdims=True), (s * u * np.abs(hat) + u * hat_err).mean(-1, keepdims=True)
    size = u + u.mean(-1, keepdims=True) + np.abs(hat) * (u * np.abs(hat)).mean(-1, keepdims=True)
    close(dx, wdx, r[..., None] * (m1 + np.abs(hat) * m2 + hat_err * (u * np.abs(hat)).mean(-1, keepdims=True) + 6 * U * size), dt)
    # a group adds its rows, then 8 groups, then 16 parts (or up to 300 through the workspace) follow
    n = min(T, 400) + 8 + 16
    gs_err = n * U * (np.abs(f64(g)) * (np.abs(hat) + hat_err)).sum(1) + (np.abs(f64(g)) * hat_err).sum(1)
    ss_err = n * U * np.abs(f64(g)).sum(1)
    close(gs, wgs, gs_err)
    close(ss, wss, ss_err)
    sq_err = (2 * np.abs(wgs) * gs_err + gs_err ** 2 + 2 * np.abs(wss) * ss_err + ss_err ** 2).sum(-1) + (p / 128 + 45) * U * wsq
    close(sq, wsq + 0.5, sq_err + U)
    surroundings_untouched(dx, p + pad, offset)


@pytest.mark.parametrize("B,T,p", [(16, 640, 776), (1, 4100, 1001), (16, 640, 2048), (1, 4100, 100)])
def test_layernorm_backward_sums_through_the_workspace_repeat_bit_for_bit(B, T, p):
    """Launches behind one another, clusters that begin while the launch before still runs."""
    assert dp.dp_layernorm_backward_ws_bytes(B, T, p) > 0
    x, g = tensor((B, T, p), torch.bfloat16, 1), tensor((B, T, p), torch.bfloat16, 2, 1e-2)
    mean, rstd = torch.zeros(B, T, device="cuda"), torch.ones(B, T, device="cuda")
    ws = torch.empty(dp.dp_layernorm_backward_ws_bytes(B, T, p), dtype=torch.uint8, device="cuda")
    outs = [(torch.zeros(B, p, device="cuda"), torch.zeros(B, p, device="cuda"), torch.zeros(B, device="cuda")) for _ in range(40)]
    for gs, ss, sq in outs:
        dp.dp_layernorm_backward(g, x, None, mean, rstd, gain_sums=gs, shift_sums=ss, sq=sq, ws=ws)
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))
    gs, ss, sq = (f64(t) for t in outs[0])
    # p squares of either sum, a thread's at most 16 one after the other, then a tree over 128 threads and 8 CTAs
    assert np.abs(sq / ((gs ** 2).sum(-1) + (ss ** 2).sum(-1)) - 1).max() < (32 + 7 + 8 + 3) * U


def test_layernorm_backward_parts_of_the_outputs():
    B, T, p = 3, 37, 264
    x, g = tensor((B, T, p), torch.bfloat16, 1), tensor((B, T, p), torch.bfloat16, 2, 1e-2)
    gain = tensor((1, p), torch.float32, 3)[0]
    hat, mean, rstd = torch.empty_like(x), torch.empty(B, T, device="cuda"), torch.empty(B, T, device="cuda")
    dp.dp_layernorm(x, gain, None, 1e-5, X_hat=hat, mean=mean, rstd=rstd)
    dx, gs, ss, sq = torch.empty_like(x), torch.empty(B, p, device="cuda"), torch.empty(B, p, device="cuda"), torch.zeros(B, device="cuda")
    dp.dp_layernorm_backward(g, x, gain, mean, rstd, dX=dx, gain_sums=gs, shift_sums=ss, sq=sq)
    for k in range(4):
        part = [torch.full_like(dx, 5), torch.full_like(gs, 5), torch.full_like(ss, 5), torch.zeros_like(sq)]
        dp.dp_layernorm_backward(g, x, gain, mean, rstd, **{n: t for j, (n, t) in enumerate(zip(("dX", "gain_sums", "shift_sums", "sq"), part))
                                                            if j == k})
        assert torch.equal(part[k], (dx, gs, ss, sq)[k])
    for alias in (g, x):                                             # dX in the place of an input
        a, b = (t.clone() for t in (g, x))
        out = a if alias is g else b
        again = torch.empty_like(gs)
        dp.dp_layernorm_backward(a, b, gain, mean, rstd, dX=out, gain_sums=again)
        assert torch.equal(out, dx) and torch.equal(again, gs)


@pytest.mark.parametrize("p", [7, 768, 1001, 2049])
def test_layernorm_backward_by_differences(p):
    """dX, gain and shift sums against differences of the forward pass along random directions."""
    B, T, step = 2, 5, 2.0 ** -5
    x, g = tensor((B, T, p), torch.float32, 1, 1.0, 0.3), tensor((B, T, p), torch.float32, 2)
    gain, shift = tensor((1, p), torch.float32, 3, 0.3, 1.0)[0], tensor((1, p), torch.float32, 4)[0]
    mean, rstd = torch.empty(B, T, device="cuda"), torch.empty(B, T, device="cuda")

    def value(x, gain, shift):
        y = torch.empty_like(x)
        dp.dp_layernorm(x, gain, shift, 1e-5, Y=y, mean=mean, rstd=rstd)
        return (y.double() * g.double()).sum(-1)
    value(x, gain, shift)
    dx, gs, ss = torch.empty_like(x), torch.empty(B, p, device="cuda"), torch.empty(B, p, device="cuda")
    dp.dp_layernorm_backward(g, x, gain, mean, rstd, dX=dx, gain_sums=gs, shift_sums=ss)
    size = rstd.double()
    dirs = [tensor(t.shape, torch.float32, 5 + k) for k, t in enumerate((x, gain[None], shift[None]))]
    d, dg, db = dirs[0], dirs[1][0], dirs[2][0]
    y_size = float((g.abs().double().sum(-1)).max()) * 8                # sums of |g| |y|
    up, down = value(x + step * d, gain, shift), value(x - step * d, gain, shift)
    # roundings of y (45 U of its size at most) over the step; the third derivative of a norm, below 15 |d rstd|^3 sqrt(p)'s share of each row
    bend = 15 * step ** 2 / 6 * (d.double().abs().amax(-1) * size) ** 3 * g.double().abs().sum(-1) * float(gain.abs().max())
    got = (dx.double() * d.double()).sum(-1)
    assert ((up - down) / (2 * step) - got).abs().le(bend + 45 * U * y_size / step).all()
    # y is linear in gain and shift
    up, down = value(x, gain + step * dg, shift + step * db), value(x, gain - step * dg, shift - step * db)
    got = (gs.double() * dg.double() + ss.double() * db.double()).sum(-1)
    assert (((up - down) / (2 * step)).sum(-1) - got).abs().max() <= T * 45 * U * y_size / step + 100 * U * T * y_size


@pytest.mark.parametrize("B,T,p,dtype", [(8, 300, 768, "bf16"), (2, 500, 4096, "f32"), (1, 4100, 64, "f32"), (3, 40, 7, "bf16")])
def test_layernorm_wait_limit_leaves_the_context_usable(B, T, p, dtype):
    """Waits that run out are reported, or the result is right; the same call is right afterwards."""
    x, g = tensor((B, T, p), DT[dtype], 1), tensor((B, T, p), DT[dtype], 2)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")

    def run():
        y, dx, mean, rstd = torch.zeros_like(x), torch.zeros_like(x), torch.zeros(B, T, device="cuda"), torch.zeros(B, T, device="cuda")
        gs, ss = torch.zeros(B, p, device="cuda"), torch.zeros(B, p, device="cuda")
        dp.dp_layernorm(x, None, None, 1e-5, Y=y, mean=mean, rstd=rstd, dev_status=st)
        dp.dp_layernorm_backward(g, x, None, mean, rstd, dX=dx, gain_sums=gs, shift_sums=ss, dev_status=st)
        torch.cuda.synchronize()
        return y, dx, mean, rstd, gs, ss
    want = run()
    assert int(st.item()) == 0
    L = dp.load()
    before = L.dp_debug_set_wait_limit(0)
    try:
        got = run()
    finally:
        L.dp_debug_set_wait_limit(before)
    assert int(st.item()) == dp.DP_DEV_TIMEOUT or all(torch.equal(a, b) for a, b in zip(got, want))
    st.zero_()
    assert all(torch.equal(a, b) for a, b in zip(run(), want)) and int(st.item()) == 0


def test_layernorm_sums_are_the_vectors_of_the_clipped_step():
    """The norms and the clipped sums of gains and shifts, as dp_vector_norms and dp_clip_accumulate_vectors make them of G and X."""
    B, T, p, C = 5, 50, 320, 0.4
    x, g = tensor((B, T, p), torch.float32, 1, 2.0), tensor((B, T, p), torch.float32, 2, 1e-2)
    gain = tensor((1, p), torch.float32, 3)[0]
    hat, mean, rstd = torch.empty_like(x), torch.empty(B, T, device="cuda"), torch.empty(B, T, device="cuda")
    dp.dp_layernorm(x, gain, None, 1e-5, X_hat=hat, mean=mean, rstd=rstd)
    gs, ss, sq = torch.empty(B, p, device="cuda"), torch.empty(B, p, device="cuda"), torch.zeros(B, device="cuda")
    dp.dp_layernorm_backward(g, x, gain, mean, rstd, gain_sums=gs, shift_sums=ss, sq=sq)
    outs = [torch.empty(p, device="cuda") for _ in range(2)]
    dp.dp_clip_accumulate_vectors([dp.Vector(gs.view(B, 1, p)), dp.Vector(ss.view(B, 1, p))], B, 1, sq, C, outs)
    vec = [dp.Vector(g, hat), dp.Vector(g)]
    sq2, outs2 = torch.zeros(B, device="cuda"), [torch.empty(p, device="cuda") for _ in range(2)]
    dp.dp_vector_norms(vec, B, T, sq2)
    dp.dp_clip_accumulate_vectors(vec, B, T, sq2, C, outs2)
    # both add up T terms of |g| (|h| + 1), a rounding of h on one side
    room = (2 * T + 60) * U
    assert (np.abs(f64(sq) / f64(sq2) - 1) < 2 * room * T ** 0.5 * 4).all()
    for a, b in zip(outs, outs2):
        assert np.abs(f64(a) - f64(b)).max() < 4 * room * float((g.abs() * (hat.abs() + 1)).sum((0, 1)).max())


# ------------------------------------------------------------------------------------- preference loss
def pref_inputs(B, T, V, dtype, seed, pad=0, offset=0, std=2.0):
    x = tensor((B, 2 * T, V), DT[dtype], seed, std, pitch=V + pad, offset=offset)
    rng = np.random.default_rng(seed)
    t = rng.integers(0, V, size=(B, 2, T))
    first, last = rng.integers(0, T // 2 + 1, size=(B, 1, 1)), rng.integers(T // 2, T + 1, size=(B, 2, 1))
    at = np.arange(T)
    t[(at < first) | (at >= last)] = -1
    ref = (-(t >= 0).sum(-1) * math.log(V) + rng.normal(size=(B, 2)) * 2).astype(np.float32)
    return x, torch.from_numpy(t.astype(np.int32)).cuda(), torch.from_numpy(ref).cuda()


def check_pref(x, t, ref, beta, smoothing, scale, loss, logp, G, dtype):
    B, _, T = t.shape
    V = x.shape[-1]
    wl, wp, wg = O.preference_loss(f64(x), t.cpu().numpy(), None if ref is None else f64(ref), beta, smoothing, scale)
    spread = float((x.float().amax(-1) - x.float().amin(-1)).nan_to_num(0, 0, 0).max()) * 1.4427 + math.log2(V) + 2
    # an exponential; a row's sum (a thread's terms, then a tree) and its logarithm; a token
    e = spread * (U + 2 ** -26) + 2 ** -22
    row = e + (V / 500 + 40) * U + 4 * U * spread
    l_err = (t >= 0).sum(-1).cpu().numpy() * row
    close(logp, wp, l_err)
    h_err = beta * (l_err.sum(-1) + 2 * U * (np.abs(wp).sum(-1) + (0 if ref is None else np.abs(f64(ref)).sum(-1))))
    close(loss, wl, h_err + 2 * U * wl)
    if G is not None:
        # softmax, onehot - softmax; the factor's slope in h is beta / 4 of scale at most
        c = np.abs(scale) * beta
        err = np.abs(wg) * (2 * row + 4 * U) + c * U * 2 + (np.abs(scale) * beta * h_err / 4)[:, None, None] * (np.abs(wg) / max(c, 1e-30) + (wg != 0) * 0)
        close_rows(G, wg, err, c, h_err, dtype)


def close_rows(G, wg, err, c, h_err, dtype):
    # a factor that is small itself (a pair far on the right side) has h_err relative to its own size, e^-h
    err = err + np.abs(wg) * (np.expm1(h_err))[:, None, None]
    close(G, wg, err, dtype)


# short rows take a warp each where there are many (the last three on a B200), others a CTA each
PREF = [(1, 1, 1), (1, 1, 2), (2, 3, 7), (3, 5, 8), (1, 16, 1000), (4, 7, 1003), (2, 33, 300), (2, 9, 50257), (1, 70, 4099), (17, 2, 640), (3, 50, 50257), (40, 3, 50257), (1, 3000, 1500), (300, 20, 1200), (3, 1000, 8192)]


@pytest.mark.parametrize("B,T,V", PREF)
@pytest.mark.parametrize("dtype,pad,offset,smoothing", [("f32", 0, 0, 0.0), ("bf16", 0, 0, 0.1), ("bf16", 7, 0, 0.0), ("f32", 1, 1, 0.1),
                                                        ("bf16", 3, 5, 0.0)])
def test_preference_loss(B, T, V, dtype, pad, offset, smoothing):
    x, t, ref = pref_inputs(B, T, V, dtype, B + T + V, pad, offset)
    loss, logp = torch.empty(B, device="cuda"), torch.empty(B, 2, device="cuda")
    G = tensor((B, 2 * T, V), DT[dtype], 3, pitch=V + pad, offset=offset)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    dp.dp_preference_loss(x, t, ref, 0.3, loss=loss, logp=logp, G=G, smoothing=smoothing, scale=0.5, dev_status=st)
    check_pref(x, t, ref, 0.3, smoothing, 0.5, loss, logp, G, DT[dtype])
    assert int(st.item()) == 0
    surroundings_untouched(G, V + pad, offset)
    rows = (t < 0).reshape(B, 2 * T)
    assert not G[rows].any()                                          # rows that do not count
    again = torch.empty(B, 2, device="cuda")                          # without a gradient, and one sequence's sums for a reference
    dp.dp_preference_loss(x, t, None, 0.3, logp=again)
    assert torch.equal(again, logp)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_preference_loss_other_alignment_of_the_gradient_and_in_place(dtype):
    B, T, V = 2, 6, 777
    x, t, ref = pref_inputs(B, T, V, dtype, 5, pad=3, offset=2)
    loss = torch.empty(B, device="cuda")
    G = [tensor((B, 2 * T, V), DT[dtype], 3, pitch=V + pad, offset=offset) for pad, offset in ((3, 2), (7, 1), (0, 0))]
    for g in G:
        dp.dp_preference_loss(x, t, ref, 0.1, loss=loss, G=g)
    z = tensor((B, 2 * T, V), DT[dtype], 3, pitch=V + 3, offset=2)
    z.copy_(x)
    dp.dp_preference_loss(z, t, ref, 0.1, G=z)
    assert torch.equal(G[0], G[1]) and torch.equal(G[0], G[2]) and torch.equal(G[0], z)
    surroundings_untouched(z, V + 3, 2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,V", [(1, 9, 1), (1, 9, 7), (1, 9, 8), (1, 9, 16), (1, 9, 17), (1, 9, 33), (1, 9, 40), (40, 20, 100), (40, 20, 1001),
                                   (1, 9, 5003)])
def test_preference_gradient_where_rows_of_logits_and_gradient_lie_differently(dtype, B, T, V):
    """Every difference of the two within 16 bytes."""
    x, t, ref = pref_inputs(B, T, V, dtype, 5, pad=5)
    want = torch.empty(B, 2 * T, V + 5, dtype=DT[dtype], device="cuda")[..., :V]
    dp.dp_preference_loss(x, t, ref, 0.1, G=want)
    for pad in range(8):
        g = tensor((B, 2 * T, V), DT[dtype], 3, pitch=V + pad, offset=pad)
        dp.dp_preference_loss(x, t, ref, 0.1, G=g)
        assert torch.equal(g, want), pad
        surroundings_untouched(g, V + pad, pad)


def test_preference_loss_alone_and_in_place_on_long_rows():
    """Rows of a whole CTA: loss and log-probabilities are the same without a gradient, the gradient the same in place."""
    B, T, V = 4, 40, 50257
    x, t, ref = pref_inputs(B, T, V, "bf16", 3, pad=7)
    G, loss, logp = torch.empty_like(x), torch.empty(B, device="cuda"), torch.empty(B, 2, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    alone = [torch.empty(B, device="cuda"), torch.empty(B, 2, device="cuda")]
    dp.dp_preference_loss(x, t, ref, 0.1, loss=loss, logp=logp, G=G, dev_status=st)
    dp.dp_preference_loss(x, t, ref, 0.1, loss=alone[0], logp=alone[1], dev_status=st)
    assert int(st.item()) == 0 and torch.equal(loss, alone[0]) and torch.equal(logp, alone[1])
    check_pref(x, t, ref, 0.1, 0.0, 1.0, loss, logp, G, torch.bfloat16)
    dp.dp_preference_loss(x, t, ref, 0.1, loss=loss, G=x)             # in place
    assert torch.equal(x, G)


def test_preference_loss_masked_rows_and_masked_vocabulary():
    B, T, V = 3, 4, 130
    x, t, ref = pref_inputs(B, T, V, "f32", 8)
    t[:] = torch.randint(0, 50, (B, 2, T), dtype=torch.int32)
    t[0, 1], t[2], t[1, 0, 1] = -1, -100, V + 5                       # a sequence, a pair without tokens; a target outside
    x[:, :, 100:] = torch.finfo(torch.float32).min                    # words that are ruled out
    x[:, :, 120:] = float("-inf")
    clean = x.clone()
    x[2] = float("nan")                                               # in rows that do not count
    x[0, T:] = float("inf")
    x[1, 1] = float("nan")
    loss, logp, G = torch.empty(B, device="cuda"), torch.empty(B, 2, device="cuda"), torch.full_like(x, 3.0)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    dp.dp_preference_loss(x, t, ref, 0.1, loss=loss, logp=logp, G=G, dev_status=st)
    assert int(st.item()) == dp.DP_DEV_BAD_ID
    clean[:, :, 100:] = -1e4                                          # the same softmax, with numbers whose range is a number
    wl, wp, wg = O.preference_loss(f64(clean), t.cpu().numpy(), f64(ref), 0.1)
    assert np.abs(f64(G) - wg).max() < 1e-6 and np.abs(f64(logp) - wp).max() < 1e-4 and np.abs(f64(loss) - wl).max() < 1e-5
    assert not G[2].any() and not G[0, T:].any() and not G[1, 1].any() and not logp[2].any() and logp[0, 1] == 0
    assert not G[:, :, 100:].any()


def test_preference_loss_numbers_that_are_not_finite_stay_in_their_pair():
    x, t, ref = pref_inputs(3, 4, 50, "f32", 9)
    t[:] = 3
    good = [torch.empty(3, device="cuda"), torch.empty(3, 2, device="cuda"), torch.empty_like(x)]
    dp.dp_preference_loss(x, t, ref, 0.1, loss=good[0], logp=good[1], G=good[2])
    x[1, 2, 7] = float("nan")
    x[2, 1] = float("-inf")
    bad = [torch.empty_like(v) for v in good]
    dp.dp_preference_loss(x, t, ref, 0.1, loss=bad[0], logp=bad[1], G=bad[2])
    assert torch.equal(good[2][0], bad[2][0]) and torch.equal(good[0][0], bad[0][0])
    assert torch.isnan(bad[0][1]) and torch.isnan(bad[2][1]).all() and torch.isnan(bad[0][2])


@pytest.mark.parametrize("V", [50, 20000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("smoothing", [0.0, 0.1, 1.0])
def test_preference_loss_of_answers_that_cannot_be(dtype, smoothing, V):
    """A target whose logit is -inf: loss 0 or inf as the definition has it, gradients that are numbers, other pairs as they were."""
    x, t, ref = pref_inputs(3, 4, V, dtype, 10)
    t[:] = 3
    x[1, 6, 3] = x[2, 1, 3] = float("-inf")                           # the other answer, the preferred one
    loss, logp, G = torch.empty(3, device="cuda"), torch.empty(3, 2, device="cuda"), torch.empty_like(x)
    dp.dp_preference_loss(x, t, ref, 0.3, loss=loss, logp=logp, G=G, smoothing=smoothing)
    wl, wp, wg = O.preference_loss(f64(x), t.cpu().numpy(), f64(ref), 0.3, smoothing)
    assert (f64(loss)[1:] == wl[1:]).all() and {0.0: wl[1] == 0, 1.0: wl[2] == 0}.get(smoothing, True)
    assert (np.isneginf(f64(logp)) == np.isneginf(wp)).all() and np.isneginf(wp).sum() == 2
    # a logit's exponent is 20 log2 e at most: 29 U, twice for its row's sum, and as in check_pref otherwise; the factor is beta or 0
    # where h is infinite, and has the rounding of 8 tokens and of ref else
    e = 29 * (U + 2 ** -26) + 2 ** -22
    row = e + (V / 500 + 40) * U + 4 * U * 29
    h_err = 0.3 * (8 * row + 2 * U * (np.abs(wp[0]).sum() + np.abs(f64(ref[0])).sum()))
    assert abs(f64(loss)[0] - wl[0]) <= h_err + 2 * U * wl[0]
    room = np.abs(wg) * (2 * row + 4 * U + np.array([np.expm1(h_err), 0, 0])[:, None, None]) + 0.3 * 2 * U
    close(G, wg, room, DT[dtype])


@pytest.mark.parametrize("dtype,room", [("f32", 3e-8), ("bf16", 1.2e-7)])
@pytest.mark.parametrize("V", [4099, 16384, 50257])
def test_preference_loss_token_errors_do_not_add_up(dtype, room, V):
    """The mean error of a token's log-probability, which every token of a sequence has alike, read from the loss of a pair whose other sequence
    and reference leave h small.  A row's sum is joined by exact powers of two, so that it has ex2's mean error only: on 2^20
    arguments -0.8e-8 between -0.5 and 0.5 (what fp32 logits give it), -5.1e-8 below 0 (bf16 ones), and 1.3e-8 of a logit's distance from the mean logit (4 at
    most here) from log2 e in one term; around it 5e-8 a token, 3e-9 of 300."""
    B, T, beta = 6, 300, 100.0
    x = tensor((B, 2 * T, V), DT[dtype], 40, std=1.5)
    t = torch.full((B, 2, T), -1, dtype=torch.int32)
    t[:, 0] = torch.randint(0, V, (B, T), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    rows = torch.log_softmax(x[:, :T].double(), -1)
    want = rows.gather(2, t[:, 0, :, None].long().cuda())[..., 0].sum(-1)
    ref = torch.zeros(B, 2, device="cuda")
    ref[:, 0] = want.float()
    loss = torch.empty(B, device="cuda")
    dp.dp_preference_loss(x, t.cuda(), ref, beta, loss=loss)
    got = -torch.log(torch.expm1(loss.double())) / beta + ref[:, 0].double()         # loss = log(1 + exp(-h))
    assert ((got - want) / T).abs().max() < room, ((got - want) / T).tolist()


@pytest.mark.parametrize("shift", [3e4, -2e5])
def test_preference_loss_large_logits(shift):
    """The maximum's rounding cancels: logits far from zero give what the same logits near zero give, as far as they are the same."""
    B, T, V = 1, 3, 500
    x, t, ref = pref_inputs(B, T, V, "f32", 11)
    t[:] = 5
    far = x + shift
    near = (far.double() - shift).float()                             # exact: the values that `far` holds
    out = []
    for v in (far, near):
        loss, G = torch.empty(B, device="cuda"), torch.empty_like(x)
        dp.dp_preference_loss(v, t, ref, 0.1, loss=loss, G=G)
        out.append((f64(loss), f64(G)))
    # an exponent's rounding is relative to what is left after the maximum (16 at most here); log2 e's own, 2^-26 relative, cancels too
    assert np.abs(out[0][0] - out[1][0]).max() < 0.1 * 2 * T * 1e-5
    assert np.abs(out[0][1] - out[1][1]).max() < 1e-6


@pytest.mark.parametrize("V", [50, 20000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [1e6, -1e6, 3e7, -3e7, 7e8, -7e8])
def test_preference_loss_of_huge_logits(dtype, top, V):
    """Two words alike at the top, a step of the type below it and far below: probabilities of the logits as they are held."""
    x, t, ref = pref_inputs(2, 3, V, dtype, 12)
    t[:] = 5
    x.copy_((x.float() + top * (2 if top < 0 else 0.5)).to(DT[dtype]))
    peak = torch.tensor(top, dtype=DT[dtype])
    x[..., 5], x[..., V - 1] = peak, peak
    x[1, 2, 5] = torch.nextafter(peak.float(), torch.tensor(-1e38)) if dtype == "f32" else peak - abs(peak) * 2.0 ** -7
    loss, logp, G = torch.empty(2, device="cuda"), torch.empty(2, 2, device="cuda"), torch.empty_like(x)
    beta = 1e-9                                                        # (a step below the top is up to 5e6)
    dp.dp_preference_loss(x, t, None, beta, loss=loss, logp=logp, G=G)
    wl, wp, wg = O.preference_loss(f64(x), t.cpu().numpy(), None, beta)
    # a row's reference is off by 2^-24 of itself, 64 at most, and so exponents at the top are up to 64, rounded by 64 U; log2 e in one term is
    # 1.4e-8 off, of the distance from the top
    close(logp, wp, 3 * (64 * U + 2 ** -20) + 2e-8 * np.abs(wp))
    close(loss, wl, beta * 1e-3 + beta * 2e-8 * np.abs(wp).sum(-1) + 4 * U)
    close(G, wg, beta * 1e-4, DT[dtype])


@pytest.mark.parametrize("V", [50, 20000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_preference_loss_past_the_logits_it_takes_is_nan_in_its_pair(dtype, V):
    lowest = torch.finfo(DT[dtype]).min
    x, t, ref = pref_inputs(9, 3, V, dtype, 13)
    t[:] = 5
    good = [torch.empty(9, device="cuda"), torch.empty(9, 2, device="cuda"), torch.empty_like(x)]
    dp.dp_preference_loss(x, t, ref, 0.1, loss=good[0], logp=good[1], G=good[2])
    for i, v in enumerate((1e12, -1e12, 1e20, -1e30, 3e38, lowest, float("-inf"), float("inf"))):
        x[i, 1] = v
    x[7, 1, : V // 2] = lowest
    loss, logp, G = (torch.empty_like(v) for v in good)
    dp.dp_preference_loss(x, t, ref, 0.1, loss=loss, logp=logp, G=G)
    assert torch.isnan(loss[:8]).all() and torch.isnan(logp[:8, 0]).all() and torch.isnan(G[:8]).all()
    assert torch.equal(loss[8], good[0][8]) and torch.equal(logp[8], good[1][8]) and torch.equal(G[8], good[2][8])


def test_preference_gradient_by_differences():
    B, T, V = 2, 3, 40
    x, t, ref = pref_inputs(B, T, V, "f32", 21)
    t[:] = torch.randint(0, V, (B, 2, T), dtype=torch.int32)
    G, d = torch.empty_like(x), torch.randn(x.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    dp.dp_preference_loss(x, t, ref, 0.5, G=G)
    step, f = 2.0 ** -4, []
    for s in (step, -step):
        loss = torch.empty(B, device="cuda")
        dp.dp_preference_loss(x + s * d, t, ref, 0.5, loss=loss)
        f.append(loss.double().sum().item())
    slope = (G.double() * d.double()).sum().item()
    # differences in fp32: 2 step^2 / 6 of the third derivative (beta^3 |d|^3 of a logistic, < 0.1 each) and roundings of the losses
    assert abs((f[0] - f[1]) / (2 * step) - slope) < 2e-2 * max(1.0, abs(slope))


# ------------------------------------------------------------------------------------- orthogonalised updates
def rel_norm(got, want):
    return np.linalg.norm(f64(got) - want) / max(np.linalg.norm(want), 1e-300)


def ns_room(shapes, out_dtype):
    k = max(max(s) for s in shapes)
    return 90 * (3 * 2.0 ** -22 + math.ceil(k / 16) * 2.0 ** -24) + half(out_dtype)


NS_SETS = [
    [(1, 1)], [(1, 9)], [(9, 1)], [(7, 5)], [(64, 64)], [(65, 64)], [(64, 130)], [(200, 72)], [(129, 257)],
    [(64, 64), (65, 63), (1, 5), (300, 20)],                    # one call, every kind
    [(64, 256), (256, 64), (63, 255), (1, 256), (30, 30), (254, 3)],   # a CTA each
    [(257, 2)], [(2, 3), (2, 257)],                             # just too long for that
    [(256, 256)] * 3 + [(768, 256), (256, 1024)], [(768, 768)],
]


@pytest.mark.parametrize("shapes", NS_SETS)
@pytest.mark.parametrize("dtype,out,pad", [("f32", "f32", 0), ("bf16", "bf16", 0), ("f32", "bf16", 3), ("bf16", "f32", 1)])
def test_orthogonalize(shapes, dtype, out, pad):
    mats = [tensor(s, DT[dtype], 10 + k, 0.7, pitch=s[1] + pad, offset=pad) for k, s in enumerate(shapes)]
    outs = [tensor(s, DT[out], 1, pitch=s[1] + pad, offset=pad) for s in shapes]
    scales = [1.0 + 0.25 * k for k in range(len(shapes))]
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    dp.dp_orthogonalize(mats, outs, scales=scales, dev_status=st)
    assert int(st.item()) == 0
    for m, o, s in zip(mats, outs, scales):
        assert rel_norm(o, O.orthogonalize(f64(m), QUINTIC, 1e-7, s)) < ns_room([m.shape], DT[out]), m.shape
        surroundings_untouched(o, o.shape[1] + pad, pad)


def test_orthogonalize_many_matrices_take_pairs_and_several_launches():
    """Enough tiles for CTA pairs, more matrices than one launch holds, and the same values alone."""
    shapes = [(320, 272)] * 60 + [(40, 300)] * 41
    mats = [tensor(s, torch.float32, k) for k, s in enumerate(shapes)]
    outs = [torch.empty(s, device="cuda") for s in shapes]
    dp.dp_orthogonalize(mats, outs)
    for k in (0, 37, 59, 60, 95, 96, 100):
        want = O.orthogonalize(f64(mats[k]), QUINTIC)
        assert rel_norm(outs[k], want) < ns_room([shapes[k]], torch.float32)
        alone = torch.empty(shapes[k], device="cuda")
        dp.dp_orthogonalize([mats[k]], [alone])
        assert rel_norm(alone, want) < ns_room([shapes[k]], torch.float32)


@pytest.mark.parametrize("coefs", [((1.5, -0.5, 0.0),) * 8, ((1.875, -1.25, 0.375),) * 6, ((4.0, -6.0, 3.0), (2.0, -1.5, 0.5), (1.5, -0.5, 0.0)),
                                   ((2.0, 0.0, 0.0),), ((0.0, 0.0, 0.0),), ((1.9, -1.0, 0.02),) * 2, ((1.5, 0.0, -0.4),)])
def test_orthogonalize_other_polynomials(coefs):
    m = tensor((96, 160), torch.float32, 4)
    o = torch.empty_like(m)
    dp.dp_orthogonalize([m], [o], coefs=coefs)
    want = O.orthogonalize(f64(m), coefs)
    assert np.linalg.norm(f64(o) - want) <= 2 * ns_room([m.shape], torch.float32) * np.linalg.norm(want)


@pytest.mark.parametrize("steps", [1, 16, 17])
def test_orthogonalize_many_small_matrices_and_many_steps(steps):
    """Small matrices take a CTA each, in several launches; with more steps than a launch holds, the tiles of larger ones."""
    mats = [tensor((33, 60), torch.float32, k) for k in range(100)]
    outs = [torch.empty_like(m) for m in mats]
    coefs = ((1.5, -0.5, 0.0),) * steps
    dp.dp_orthogonalize(mats, outs, coefs=coefs)
    for k in (0, 50, 95, 96, 99):
        want = O.orthogonalize(f64(mats[k]), coefs)
        assert np.linalg.norm(f64(outs[k]) - want) <= 2 * ns_room([(33, 60)], torch.float32) * np.linalg.norm(want)


def test_orthogonalize_extreme_inputs():
    """Zeros, tiny and huge values (whose squares fp32 does not hold), rank one, NaN; in place."""
    base = tensor((48, 80), torch.float32, 6)
    one = base[:, :1] @ base[:1]
    mats = [torch.zeros_like(base), base * 1e-30, base * 1e30, one, base.clone()]
    mats[4][3, 4] = float("nan")
    outs = [torch.full_like(m, 9.0) for m in mats]
    dp.dp_orthogonalize(mats, outs, eps=0.0 or 1e-37)
    assert not outs[0].any() and torch.isnan(outs[4]).any()
    for k in (1, 2, 3):
        assert rel_norm(outs[k], O.orthogonalize(f64(mats[k]), QUINTIC, 1e-37)) < ns_room([(48, 80)], torch.float32), k
    z = base.clone()
    dp.dp_orthogonalize([z], [z])
    fresh = torch.empty_like(base)
    dp.dp_orthogonalize([base], [fresh])
    assert torch.equal(z, fresh)


# Closer bounds.  An accumulator of the products holds 64 of K in twelve MMAs, whose sums are truncated by 2^-23 at most each, and is added to
# nearest to the others'; two terms hold 22 bits of each operand, and the product of the low ones is left out.  Relative to the sum of the terms'
# magnitudes:
def product_error(K):
    return 3 * 2.0 ** -22 + 12 * 2.0 ** -23 + math.ceil(K / 64) * U


def dominated_room(shape, at_once):
    """Error of the quintic's result, relative to its norm, on a matrix with one direction of singular value near 1 and others so small that
    all steps amplify them by a = 3.4445.  With e = product_error: A is e off to begin with; A' = B A B is off by a^2 times that and by its
    three products, a^2 e each (B's goes through b A B, less than that).  B, which is a I there, is off by |b| times A's error and its own e.
    X and every X' = B X are off by e beside the large direction, which the steps left amplify.  The result's norm is 0.68 at least."""
    a, b = QUINTIC[0][0], abs(QUINTIC[0][1])
    e, total, left = product_error(max(shape)), 0.0, sum(at_once)
    off = 2.0 ** -22 * a ** left                                       # X in two terms
    for n in at_once:
        err = e
        for _ in range(n):
            total += (b * err + e) / a
            err = a * a * (err + 3 * e)
        left -= n
        off += e * a ** (left + n)
    return total + off / 0.68


def beyond_rounding(got, want):
    """Norm of what `got` differs from `want` by beyond half a step of its type, relative to want's."""
    bits = -math.log2(torch.finfo(got.dtype).eps)
    got = f64(got)
    top = np.floor(np.log2(np.maximum(np.maximum(np.abs(got), np.abs(want)), 1e-300)))
    return np.linalg.norm(np.maximum(np.abs(got - want) - 2.0 ** (top - bits - 1), 0)) / np.linalg.norm(want)


def dominated(shape, rest, seed):
    """One direction, and noise whose norm is `rest` of its."""
    rng = np.random.default_rng(seed)
    u, v, x = rng.normal(size=(shape[0], 1)), rng.normal(size=(1, shape[1])), rng.normal(size=shape)
    return torch.from_numpy(u @ v / (np.linalg.norm(u) * np.linalg.norm(v)) + rest * x / np.linalg.norm(x)).float().cuda()


@pytest.mark.parametrize("rest", [0.1, 0.01, 1e-3])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("shapes", [[(300, 1000)], [(1500, 512)], [(700, 2100), (640, 640)]])
def test_orthogonalize_one_dominant_direction(shapes, out, rest):
    """What the steps amplify beside a dominant direction keeps its digits: bf16 updates are right to their rounding."""
    mats = [dominated(s, rest, k) for k, s in enumerate(shapes)]
    outs = [torch.empty_like(m, dtype=DT[out]) for m in mats]
    dp.dp_orthogonalize(mats, outs)
    for m, o in zip(mats, outs):
        want = O.orthogonalize(f64(m), QUINTIC)
        # no type takes more than three steps at once
        assert beyond_rounding(o, want) < dominated_room(m.shape, (3, 2)), (m.shape, beyond_rounding(o, want))


# Sets of matrices and how they run in fp32 and in bf16 out: (CTA pairs, steps at once).  test_host_operators.py checks the same on the host.
NS_FORMS = {
    "single": ([(200, 330), (330, 200)], (False, 1), (False, 1)),
    "single, bf16 three at once": ([(300, 1000)] * 3 + [(1000, 301)] * 2, (False, 1), (False, 3)),
    "single, two and three at once": ([(700, 2100), (640, 640)], (False, 2), (False, 3)),
    "pairs": ([(1001, 500)] * 10 + [(505, 2000)] * 12, (True, 1), (True, 3)),
    "pairs, two and three at once": ([(650, 2100)] * 6 + [(2100, 651)] * 4 + [(700, 700)] * 2, (True, 2), (True, 3)),
    "pairs, one size": ([(700, 1301)] * 8, (True, 2), (True, 3)),
}


def ns_form(mats, out, coefs=QUINTIC):
    """(CTA pairs, steps at once) of a call; None: a CTA per matrix."""
    flat = [c for step in coefs for c in step]
    arr = (dp._MatrixDesc * len(mats))()
    for D, m in zip(arr, mats):
        D.p, D.d = m
    f = dp.load().dp_debug_orthogonalize_form(arr, len(mats), {torch.float32: dp.DP_F32, torch.bfloat16: dp.DP_BF16}[out],
                                              (ctypes.c_float * len(flat))(*flat), len(coefs))
    assert f >= 0
    return (bool(f & 1), f >> 1) if f else None


def plain_products(m, coefs=QUINTIC):
    """The iterate with products in fp32."""
    x = m.float()
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    x = x / x.double().square().sum().sqrt().float()
    for a, b, c in coefs:
        A = x @ x.T
        x = a * x + (b * A + c * (A @ A)) @ x
    return x.T if tall else x


@pytest.mark.parametrize("name", NS_FORMS)
@pytest.mark.parametrize("dtype,out,pad", [("f32", "f32", 0), ("f32", "bf16", 0), ("bf16", "f32", 3), ("bf16", "bf16", 1)])
def test_orthogonalize_in_every_form(name, dtype, out, pad):
    """Single CTAs and pairs, steps one by one and several at once: as near to the definition as products in fp32 are.

    Operands of 22 bits, where fp32 has 24, are off by 2^-22, and planes are rounded so twice a step and matrix; fp32 products round
    K times a product by 2^-24.  With K of 300 at least, errors that add up as independent ones do, that is 2^-22 sqrt(2) against 2^-24 sqrt(300):
    a third.  Two steps at once bring A's error times |B|^2 = 11.8 beside singular values that are left small; with the products' slope near one
    (1.8, twice) that is 3.3 times the error of steps one by one.  2.5 holds both; three at once are for bf16, whose rounding is taken out."""
    shapes, *forms = NS_FORMS[name]
    assert ns_form(shapes, DT[out]) == forms[out == "bf16"]
    mats = [tensor(s, DT[dtype], 30 + k, 0.7, pitch=s[1] + pad, offset=pad) for k, s in enumerate(shapes)]
    outs = [tensor(s, DT[out], 1, pitch=s[1] + pad, offset=pad) for s in shapes]
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    dp.dp_orthogonalize(mats, outs, dev_status=st)
    assert int(st.item()) == 0
    for k in {0, 1, len(shapes) // 2, len(shapes) - 1}:
        want = O.orthogonalize(f64(mats[k]), QUINTIC)
        assert beyond_rounding(outs[k], want) < 2.5 * rel_norm(plain_products(mats[k]), want), shapes[k]
        surroundings_untouched(outs[k], shapes[k][1] + pad, pad)
    again = [torch.empty_like(o) for o in outs]
    dp.dp_orthogonalize(mats, again)
    assert all(torch.equal(a, b) for a, b in zip(outs, again))


@pytest.mark.parametrize("name", ["single, bf16 three at once", "single, two and three at once", "pairs, one size"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("coefs", [((1.5, -0.5, 0.0),) * 8, ((1.875, -1.25, 0.375),) * 6, ((1.9, -1.0, 0.02),) * 3,
                                   ((1.9, -1.0, 0.02), QUINTIC[0], (1.5, -0.5, 0.0), (1.875, -1.25, 0.375), (1.5, 0.0, -0.4)),
                                   (QUINTIC[0], (1.5, 0.0, -0.4), (2.0, 0.0, 0.0), (0.4, 0.1, 0.1))])
def test_orthogonalize_other_polynomials_in_steps_at_once(name, out, coefs):
    """Polynomials with and without a diagonal's copy, in each other's company."""
    shapes = NS_FORMS[name][0]
    mats = [tensor(s, torch.float32, 60 + k) for k, s in enumerate(shapes)]
    outs = [torch.empty(s, device="cuda", dtype=DT[out]) for s in shapes]
    dp.dp_orthogonalize(mats, outs, coefs=coefs)
    for k in (0, len(shapes) - 1):
        want = O.orthogonalize(f64(mats[k]), coefs)
        assert beyond_rounding(outs[k], want) < 2 * ns_room([shapes[k]], torch.float32)


@pytest.mark.parametrize("name", ["single", "single, bf16 three at once", "pairs, one size"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("coefs", [((1e-3, 0.0, 0.0),) * 8, ((1e-2, 1e-3, 1e-3),) * 10, ((0.0, 1e-2, 0.0),), ((1e-3, 0.0, 0.0),) * 3 + ((1e3, 0.0, 0.0),) * 3])
def test_orthogonalize_polynomials_that_shrink(name, out, coefs):
    """Results down to 1e-27 have the digits that others have."""
    shapes = NS_FORMS[name][0]
    mats = [tensor(s, torch.float32, 70 + k) for k, s in enumerate(shapes)]
    outs = [torch.empty(s, device="cuda", dtype=DT[out]) for s in shapes]
    dp.dp_orthogonalize(mats, outs, coefs=coefs)
    for k in (0, len(shapes) - 1):
        want = O.orthogonalize(f64(mats[k]), coefs)
        # a product's error is at most that of the powers that it takes of A, three of them here
        assert 1e-35 < np.linalg.norm(want) and beyond_rounding(outs[k], want) < 3 * ns_room([shapes[k]], torch.float32)


EXTREME = {"a CTA": [(48, 80)], "single": [(200, 330)], "single, tall": [(330, 200)], "at once": [(300, 1000)], "at once, in fp32 too": [(700, 1301)]}


@pytest.mark.parametrize("where", EXTREME)
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("eps", [0.0, 1e-37])
def test_orthogonalize_extreme_inputs_in_every_form(where, out, eps):
    """Zeros, tiny and huge values (whose squares fp32 does not hold), low rank, an infinity, NaN; in place."""
    shape = EXTREME[where][0]
    base = tensor(shape, torch.float32, 6)
    m = [torch.zeros_like(base), base * 1e-30, base * 1e30, base[:, :1] @ base[:1], base[:, :3] @ base[:3], base.clone(), base.clone(), base]
    m[5][3, 4], m[6][7, 1] = float("inf"), float("nan")
    outs = [torch.full_like(v, 9.0, dtype=DT[out]) for v in m]
    dp.dp_orthogonalize(m, outs, eps=eps)
    assert torch.isnan(outs[0]).all() if eps == 0 else not outs[0].any()           # 0 / 0, 0 / eps
    assert torch.isnan(outs[5]).any() and torch.isnan(outs[6]).any()
    for k in (1, 2, 3, 4, 7):
        want = O.orthogonalize(f64(m[k]), QUINTIC, eps)
        assert beyond_rounding(outs[k], want) < dominated_room(shape, (3, 2)), k
    # the finite ones do not know of the others
    some = [torch.empty_like(outs[0]) for _ in m]
    fresh = [v if k in (1, 2, 3, 4, 7) else base for k, v in enumerate(m)]
    dp.dp_orthogonalize(fresh, some, eps=eps)
    assert all(torch.equal(some[k], outs[k]) for k in (1, 2, 3, 4, 7)) and torch.equal(some[0], some[7])
    if out == "f32":
        z = [v.clone() for v in fresh]
        dp.dp_orthogonalize(z, z, eps=eps)
        assert all(torch.equal(a, b) for a, b in zip(z, some))


@pytest.mark.parametrize("name", ["pairs", "pairs, one size"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_orthogonalize_wait_limit_on_pairs(name, out):
    shapes = NS_FORMS[name][0]
    assert ns_form(shapes, DT[out])[0]
    mats = [tensor(s, torch.float32, k) for k, s in enumerate(shapes)]
    want, got = ([torch.empty_like(m, dtype=DT[out]) for m in mats] for _ in range(2))
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    dp.dp_orthogonalize(mats, want, dev_status=st)
    assert int(st.item()) == 0
    L = dp.load()
    before = L.dp_debug_set_wait_limit(0)
    try:
        dp.dp_orthogonalize(mats, got, dev_status=st)
        torch.cuda.synchronize()
    finally:
        L.dp_debug_set_wait_limit(before)
    # a wait may still end at its one try, which the hardware may hold for a while: reported, or right
    assert int(st.item()) == dp.DP_DEV_TIMEOUT or all(torch.equal(a, b) for a, b in zip(got, want))
    st.zero_()
    dp.dp_orthogonalize(mats, got, dev_status=st)
    assert int(st.item()) == 0 and all(torch.equal(a, b) for a, b in zip(got, want))


def test_orthogonalize_singular_values():
    m = tensor((200, 500), torch.float32, 7)
    o = torch.empty_like(m)
    dp.dp_orthogonalize([m], [o])
    s = np.linalg.svd(f64(o), compute_uv=False)
    assert s.min() > 0.6 and s.max() < 1.3


@pytest.mark.parametrize("shapes", [[(100, 150)], [(128, 130)] * 3, [(70, 192), (260, 20)]])
def test_orthogonalize_wait_limit_with_sums_no_longer_than_the_stages(shapes):
    """Sums of three K steps at most: the copying warps have issued all before any other role's wait runs out."""
    mats = [tensor(s, torch.float32, k) for k, s in enumerate(shapes)]
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    want, got = ([torch.empty_like(m) for m in mats] for _ in range(2))
    dp.dp_orthogonalize(mats, want, dev_status=st)
    assert int(st.item()) == 0
    L = dp.load()
    before = L.dp_debug_set_wait_limit(0)
    try:
        dp.dp_orthogonalize(mats, got, dev_status=st)
        torch.cuda.synchronize()
    finally:
        L.dp_debug_set_wait_limit(before)
    # a wait may still end at its one try, which the hardware may hold for a while: reported, or right
    assert int(st.item()) == dp.DP_DEV_TIMEOUT or all(torch.equal(a, b) for a, b in zip(got, want))
    st.zero_()
    dp.dp_orthogonalize(mats, got, dev_status=st)
    assert int(st.item()) == 0 and all(torch.equal(a, b) for a, b in zip(got, want))


def test_orthogonalize_wait_limit_leaves_the_context_usable():
    m = tensor((300, 300), torch.float32, 8)
    o, st = torch.empty_like(m), torch.zeros(1, dtype=torch.int32, device="cuda")
    L = dp.load()
    before = L.dp_debug_set_wait_limit(0)
    try:
        dp.dp_orthogonalize([m], [o], dev_status=st)
        torch.cuda.synchronize()
    finally:
        L.dp_debug_set_wait_limit(before)
    # a wait may still end at its one try, which the hardware may hold for a while: reported, or right
    assert int(st.item()) == dp.DP_DEV_TIMEOUT or rel_norm(o, O.orthogonalize(f64(m), QUINTIC)) < ns_room([m.shape], torch.float32)
    st.zero_()
    dp.dp_orthogonalize([m], [o], dev_status=st)
    assert int(st.item()) == 0 and rel_norm(o, O.orthogonalize(f64(m), QUINTIC)) < ns_room([m.shape], torch.float32)


# ------------------------------------------------------------------------------------- streams, graphs, repeats
def every_operator(seed=0):
    """Calls of each operator on inputs of their own and what they write."""
    B, T, p, V = 3, 20, 136, 311
    x, g = tensor((B, T, p), torch.bfloat16, seed + 1), tensor((B, T, p), torch.bfloat16, seed + 2, 1e-2)
    gain = tensor((1, p), torch.float32, seed + 3)[0]
    y, mean, rstd, dx = torch.empty_like(x), torch.empty(B, T, device="cuda"), torch.empty(B, T, device="cuda"), torch.empty_like(x)
    gs, ss, sq = torch.empty(B, p, device="cuda"), torch.empty(B, p, device="cuda"), torch.zeros(B, device="cuda")
    logits, t, ref = pref_inputs(B, T, V, "bf16", seed + 4)
    loss, G = torch.empty(B, device="cuda"), torch.empty_like(logits)
    mats = [tensor((100, 70), torch.float32, seed + 5), tensor((64, 64), torch.float32, seed + 6)]
    outs = [torch.empty_like(m) for m in mats]
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (dp.dp_preference_loss_ws_bytes(B, T), dp.dp_orthogonalize_ws_bytes(mats))]

    def run(stream=None):
        dp.dp_layernorm(x, gain, None, 1e-5, Y=y, mean=mean, rstd=rstd, stream=stream)
        dp.dp_layernorm_backward(g, x, gain, mean, rstd, dX=dx, gain_sums=gs, shift_sums=ss, stream=stream)
        dp.dp_preference_loss(logits, t, ref, 0.1, loss=loss, G=G, ws=ws[0], stream=stream)
        dp.dp_orthogonalize(mats, outs, ws=ws[1], stream=stream)
    return run, [y, mean, rstd, dx, gs, ss, loss, G, *outs]


def test_operators_repeat_bit_for_bit_on_streams_and_in_graphs():
    run, out = every_operator()
    run()
    torch.cuda.synchronize()
    want = [o.clone() for o in out]
    side = torch.cuda.Stream()
    for o in out:
        o.fill_(5)
    side.wait_stream(torch.cuda.current_stream())
    run(side)                                                        # a stream by argument
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for o in out:
            o.fill_(5)
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_workspaces_of_the_calls_themselves_outlive_other_streams():
    """No workspace given, another stream: its memory is not handed out again while the kernels run."""
    m = [tensor((512, 512), torch.float32, k) for k in range(2)]
    outs = [torch.empty_like(v) for v in m]
    want = [torch.empty_like(v) for v in m]
    dp.dp_orthogonalize(m, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(5):
        dp.dp_orthogonalize(m, outs, stream=side)
        torch.full((1 << 24,), float("nan"), device="cuda")          # would land in freed memory
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_binding_refuses_what_would_be_misread():
    x = tensor((2, 6, 32), torch.bfloat16, 1)
    f = lambda *s: torch.empty(*s, device="cuda")
    for kw in (dict(Y=f(2, 6, 32)), dict(Y=torch.empty(2, 5, 32, dtype=torch.bfloat16, device="cuda")), dict(mean=f(11)),
               dict(Y=torch.empty_like(x).transpose(0, 1)), dict(mean=f(12).double()), dict(Y=x.cpu())):
        with pytest.raises(dp.DpGhostError):
            dp.dp_layernorm(x, None, None, 1e-5, **kw)
    with pytest.raises(dp.DpGhostError):
        dp.dp_layernorm(x, f(31), None, 1e-5, Y=torch.empty_like(x))
    with pytest.raises(dp.DpGhostError):
        dp.dp_layernorm(x, f(32), f(32).bfloat16(), 1e-5, Y=torch.empty_like(x))
    with pytest.raises(dp.DpGhostError):
        dp.dp_layernorm_backward(x, x, None, f(12), f(12), gain_sums=f(2, 31))
    t = torch.zeros(2, 2, 3, dtype=torch.int32, device="cuda")
    for kw in (dict(targets=t.long()), dict(V=33), dict(loss=f(3)), dict(G=f(2, 6, 32)), dict(ref_logp=f(2)), dict(targets=t[:, :, :2])):
        with pytest.raises(dp.DpGhostError):
            dp.dp_preference_loss(**dict(dict(logits=x, targets=t, ref_logp=None, beta=0.1, loss=f(2)), **kw))
    m = f(8, 6)
    for mats, outs, kw in (([m], [f(6, 8)], {}), ([m], [f(8, 6).half()], {}), ([m, m.bfloat16()], [f(8, 6)] * 2, {}), ([m.t()], [f(6, 8)], {}),
                           ([m], [m], dict(scales=[1.0, 2.0])), ([m], [m], dict(coefs=((1.0, 2.0),))),
                           ([m], [m], dict(ws=torch.empty(8, dtype=torch.uint8, device="cuda")))):
        with pytest.raises(dp.DpGhostError):
            dp.dp_orthogonalize(mats, outs, **kw)
    torch.cuda.synchronize()


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("call", ["preference", "orthogonalize", "backward", "norms"])
def test_workspaces_of_the_calls_themselves_are_not_in_use_on_another_stream(call, raw):
    """A tensor freed while the current stream has yet to read it, then a call on another stream without a workspace of the same size."""
    side = torch.cuda.Stream()
    stream = side.cuda_stream if raw else side
    if call == "preference":
        B, T, V = 40, 500, 64
        x, t, ref = pref_inputs(B, T, V, "f32", 1)
        loss = torch.empty(B, device="cuda")
        need, run = dp.dp_preference_loss_ws_bytes(B, T), lambda s: dp.dp_preference_loss(x, t, ref, 0.1, loss=loss, stream=s)
        out = [loss]
    elif call == "orthogonalize":
        m = [tensor((200, 200), torch.float32, 1)]
        out = [torch.empty_like(m[0])]
        need, run = dp.dp_orthogonalize_ws_bytes(m), lambda s: dp.dp_orthogonalize(m, out, stream=s)
    elif call == "backward":
        B, T, p = 16, 640, 776
        x, g = tensor((B, T, p), torch.bfloat16, 1), tensor((B, T, p), torch.bfloat16, 2)
        mean, rstd = torch.zeros(B, T, device="cuda"), torch.ones(B, T, device="cuda")
        out = [torch.empty(B, p, device="cuda")]
        need = dp.dp_layernorm_backward_ws_bytes(B, T, p)
        run = lambda s: dp.dp_layernorm_backward(g, x, None, mean, rstd, gain_sums=out[0], stream=s)
    else:
        B, T = 32, 256
        layers = [dp.Linear(tensor((B, T, 512), torch.bfloat16, 1), tensor((B, T, 512), torch.bfloat16, 2))]
        out = [torch.zeros(B, device="cuda")]
        need = dp.dp_ghost_norms_ws_bytes(layers, B, T)

        def run(s):
            with torch.cuda.stream(side):
                out[0].zero_()
            dp.dp_ghost_norms(layers, B, T, out[0], stream=s)
    assert need > 0
    run(stream)                                                       # the allocator's pools and the kernels are set up
    torch.cuda.synchronize()
    want = [o.clone() for o in out]
    for o in out:
        o.fill_(5)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    bait = torch.full((need,), 7, dtype=torch.uint8, device="cuda")
    kept = torch.empty_like(bait)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)                                    # some 100 ms
    kept.copy_(bait)
    del bait
    run(stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    torch.cuda.synchronize()
    assert (kept == 7).all()


@pytest.mark.parametrize("stream", [0, "default", "current"])
def test_workspaces_of_the_calls_themselves_on_the_default_stream(stream):
    """The default stream, by its number and as an object, while another one is current and while not."""
    m = tensor((200, 300), torch.float32, 1)
    want, got = torch.empty_like(m), torch.empty_like(m)
    dp.dp_orthogonalize([m], [want])
    torch.cuda.synchronize()
    s = {0: 0, "default": torch.cuda.default_stream(), "current": torch.cuda.current_stream()}[stream]
    for current in (torch.cuda.default_stream(), torch.cuda.Stream()):
        got.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(current):
            dp.dp_orthogonalize([m], [got], stream=s)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


FIRST_CALLS = """
import threading, torch
from paper_2609_40335_b200 import binding as dp
errors = []

def at_once(calls):
    gate = threading.Barrier(len(calls))

    def run(call):
        gate.wait()
        try:
            call()
        except Exception as e:
            errors.append(repr(e))
    threads = [threading.Thread(target=run, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()

for dtype in (torch.float32, torch.bfloat16):
    for p in (64, 65, 512, 1024, 1025, 4096, 16384):
        x = torch.ones(6, p, device="cuda", dtype=dtype)
        outs = [torch.empty_like(x) for _ in range(6)]
        at_once([lambda o=o: dp.dp_layernorm(x, None, None, 1e-5, Y=o) for o in outs])
for n in (40, 300):
    m = torch.eye(n, device="cuda")
    outs = [torch.empty_like(m) for _ in range(6)]
    work = [torch.empty(dp.dp_orthogonalize_ws_bytes([m]), dtype=torch.uint8, device="cuda") for _ in outs]
    at_once([lambda o=o, w=w: dp.dp_orthogonalize([m], [o], ws=w) for o, w in zip(outs, work)])
torch.cuda.synchronize()
print("errors", len(errors), errors[:2])
"""


def test_first_calls_of_several_threads():
    """A kernel's set-up is done before any thread launches it."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], env=dict(os.environ, PYTHONPATH=root), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "errors 0 " in r.stdout, (r.stdout + r.stderr)[-1500:]
