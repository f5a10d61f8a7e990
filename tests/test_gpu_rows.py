"""GPU parity of the row operators against the oracle in 64 bits: 8-bit checkpoints (bit for bit), the gated activation and
the residual join with their backward passes; odd sizes, strides, non-finite values, empty inputs, refusals, streams."""
import numpy as np
import pytest
import torch

from oracle import rows as R
from paper_2605_01255_b200 import binding as B
from paper_2605_01255_b200 import inputs as I

from _harness import raw_bits, to_device, to_host

pytestmark = pytest.mark.gpu

TDT = {"bf16": torch.bfloat16, "f32": torch.float32}
NAN = float("nan")


def new(*shape, dt):
    return torch.full(shape, 77 if dt is torch.int8 else NAN, dtype=dt, device="cuda")


def q8_new(rows, cols):
    return new(rows, cols, dt=torch.int8), new(rows, -(-cols // 128), dt=torch.float32)


def close(name, got, want, dtype, acc):
    """One rounding to the output's type (half a unit of bfloat16 is at most 2^-8 of the value) and `acc`, an absolute bound on
    the fp32 arithmetic before it."""
    got = to_host(got)
    assert got.shape == want.shape, name
    bound = acc + (2.0 ** -8 * (np.abs(want) + acc) if dtype == "bf16" else 0.0)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (name, int(bad.sum()), float(np.nanmax(np.abs(got - want))), np.argwhere(bad)[:3].tolist())


def act(rows, cols, seed, dtype, std=1.0):
    x = I.gaussian((rows, cols), seed, std) * np.exp(0.5 * I.gaussian((rows, 1), seed + 1))
    x[:, ::64] *= 8
    return I.round_to_dtype(x, dtype)


# one group, a partly filled group, several, ragged rows, one row, a row longer than one block's share
SHAPES = [(1, 8), (3, 120), (5, 128), (777, 136), (64, 896), (1027, 1000), (33, 4864), (9, 16392)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [0, 40])
def test_q8_store_and_load(rows, cols, dtype, pad):
    wide = act(rows, cols + pad, rows + cols, dtype)
    xd = to_device(wide, dtype)
    X, x = xd[:, :cols], wide[:, :cols]
    d = B.make_rows_desc(rows, cols, dtype)
    codes, scales = q8_new(rows, cols)
    B.acx_q8_store(d, X, codes, scales)
    want_c, want_s = R.q8_encode(x)
    assert np.array_equal(codes.cpu().numpy(), want_c)
    assert np.array_equal(raw_bits(scales), want_s.view(np.uint32))
    back = new(rows, cols + pad, dt=TDT[dtype])
    B.acx_q8_load(d, codes, scales, back[:, :cols])
    close("q8", back[:, :cols], R.q8_decode(want_c, want_s), dtype, 2.0 ** -24 * np.abs(x).max())
    assert torch.isnan(back[:, cols:].float()).all()      # nothing beside the slice is written


def test_q8_corner_values():
    x = np.zeros((8, 264), np.float32)
    x[1, 3], x[1, 200] = 2.0 ** -101, 2.0 ** -100
    x[2, 0], x[3, 130], x[4, 263] = np.inf, np.nan, -np.inf
    x[5] = np.finfo(np.float32).max
    x[6, :5] = (127, 0.5, 1.5, -2.5, -127)
    x[7] = -1e-45
    d = B.make_rows_desc(8, 264, "f32")
    codes, scales = q8_new(8, 264)
    B.acx_q8_store(d, to_device(x, "f32"), codes, scales)
    back = new(8, 264, dt=torch.float32)
    B.acx_q8_load(d, codes, scales, back)
    wc, ws = R.q8_encode(x)
    want = R.q8_decode(wc, ws)
    got = to_host(back)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(want).any()
    ok = ~np.isnan(want)
    assert np.array_equal(codes.cpu().numpy()[ok], wc[ok])
    assert np.allclose(got[ok], want[ok], rtol=2.0 ** -23, atol=0)


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("stacked", [False, True])
def test_swiglu(rows, cols, dtype, stacked):
    gu = act(rows, 2 * cols, 3 * rows + cols, dtype, 1.5)
    dh = I.gaussian((rows, cols), 5, 0.1, dtype)
    gud = to_device(gu, dtype)
    g, u = gu[:, :cols], gu[:, cols:]
    G, U = (gud[:, :cols], gud[:, cols:]) if stacked else (gud[:, :cols].contiguous(), gud[:, cols:].contiguous())
    d = B.make_rows_desc(rows, cols, dtype)
    H, H2, dGU = new(rows, cols, dt=TDT[dtype]), new(rows, cols, dt=TDT[dtype]), new(rows, 2 * cols, dt=TDT[dtype])
    qG, qU = q8_new(rows, cols), q8_new(rows, cols)
    B.acx_swiglu_fwd(d, G, U, H, *qG, *qU)
    B.acx_swiglu_fwd(d, G, U, H2)
    assert torch.equal(H, H2)
    for q, x in ((qG, g), (qU, u)):
        wc, ws = R.q8_encode(x)
        assert np.array_equal(q[0].cpu().numpy(), wc) and np.array_equal(raw_bits(q[1]), ws.view(np.uint32))
    # exp: 2 units in the last place and, in the hardware's form, the rounding of g * log2(e): |g| * 2^-23; then a quotient
    # and two products.  Relative to |g s u|; where g is very negative s itself is tiny and so is the product.
    e32 = 2.0 ** -23
    close("H", H, R.swiglu_fwd(g, u), dtype, e32 * (8 + 2 * np.abs(g)) * np.abs(R.swiglu_fwd(g, u)) + 1e-36)
    if stacked:
        dG, dU = dGU[:, :cols], dGU[:, cols:]
    else:
        dG, dU = new(rows, cols, dt=TDT[dtype]), new(rows, cols, dt=TDT[dtype])
    B.acx_swiglu_bwd(d, to_device(dh, dtype), *qG, *qU, dG, dU)
    gq, uq = R.q8_values(g), R.q8_values(u)
    want_g, want_u = R.swiglu_bwd(dh, gq, uq)
    s = 1 / (1 + np.exp(-gq))
    close("dU", dU, want_u, dtype, e32 * (10 + 2 * np.abs(gq)) * np.abs(want_u) + 1e-36)
    # 1 + g (1 - s): the error of s (absolute 2^-23 * (8 + 2 |g|) * s) enters through 1 - s too
    close("dG", dG, want_g, dtype, e32 * (16 + 4 * np.abs(gq)) * np.abs(dh * uq) * s * (1 + np.abs(gq)) + 1e-36)


def test_swiglu_extreme_gates():
    g = np.array([[-1e4, -200, -100, -88, -87.5, -80, 0, -0.0, 80, 88.8, 100, 1e4, -1.2784645, 1, -1, 20]], np.float32)
    u = np.full_like(g, 2)
    d = B.make_rows_desc(1, 16, "f32")
    for dtype in ("f32", "bf16"):
        gr = I.round_to_dtype(g, dtype)
        H = new(1, 16, dt=TDT[dtype])
        B.acx_swiglu_fwd(B.make_rows_desc(1, 16, dtype), to_device(gr, dtype), to_device(u, dtype), H)
        want = R.swiglu_fwd(gr, u)
        close("H", H, want, dtype, 2.0 ** -23 * (8 + 2 * np.abs(gr)) * np.abs(want) + 1e-34)
    G = to_device(np.array([[np.nan, np.inf] + [0] * 6], np.float32), "f32")
    H = new(1, 8, dt=torch.float32)
    B.acx_swiglu_fwd(B.make_rows_desc(1, 8, "f32"), G, torch.ones_like(G), H)
    assert torch.isnan(H[0, 0]) and torch.isinf(H[0, 1]) and not H[0, 2:].any()


def _exact_values(rows, cols, seed):
    """Values that an 8-bit checkpoint holds without loss: whole multiples of 2^-6 with 127 * 2^-6 in every group."""
    x = np.round(I.gaussian((rows, cols), seed, 30.0)).clip(-127, 127)
    x[:, ::128] = 127
    return (x * 2.0 ** -6).astype(np.float32)


def test_swiglu_gradient_against_differences():
    rows, cols, eps = 7, 264, 2.0 ** -10
    g, u, dh = _exact_values(rows, cols, 1), _exact_values(rows, cols, 2), I.gaussian((rows, cols), 3)
    d = B.make_rows_desc(rows, cols, "f32")
    dir_g, dir_u = (np.sign(I.gaussian((rows, cols), s)).astype(np.float32) for s in (4, 5))

    def value(a, b):
        H = new(rows, cols, dt=torch.float32)
        B.acx_swiglu_fwd(d, to_device(a, "f32"), to_device(b, "f32"), H)
        return np.sum(to_host(H) * dh)

    qG, qU = q8_new(rows, cols), q8_new(rows, cols)
    B.acx_swiglu_fwd(d, to_device(g, "f32"), to_device(u, "f32"), new(rows, cols, dt=torch.float32), *qG, *qU)
    dG, dU = new(rows, cols, dt=torch.float32), new(rows, cols, dt=torch.float32)
    B.acx_swiglu_bwd(d, to_device(dh, "f32"), *qG, *qU, dG, dU)
    # second differences: eps^2 / 6 * |f'''| <= 2^-20 / 6 per element of size |dh u|; roundings 2^-22 * |H| / eps
    scale = np.sum(np.abs(dh) * (np.abs(u) + np.abs(g)))
    tol = scale * (eps * eps / 6 + 2.0 ** -21 / eps / np.sqrt(rows * cols))
    assert abs(np.sum(to_host(dG) * dir_g) - (value(g + eps * dir_g, u) - value(g - eps * dir_g, u)) / (2 * eps)) <= tol
    assert abs(np.sum(to_host(dU) * dir_u) - (value(g, u + eps * dir_u) - value(g, u - eps * dir_u)) / (2 * eps)) <= tol


VARIANTS = [(False, False, False), (True, False, False), (True, True, False), (True, False, True), (True, True, True)]
# below a warp, one vector per thread, two, four; ragged last vectors and groups; more rows than resident blocks
NORM_SHAPES = [(1, 8), (5, 264), (1500, 896), (2500, 1000), (67, 4096), (41, 4872), (11, 8200), (3, 32768)]
WIDE_SHAPES = [(650, 5640), (700, 12296), (301, 16384), (90, 28672)]    # rows shared by several blocks, more of them than run at once


def _norm_inputs(rows, cols, dtype, join, post, gate, exact=False):
    mk = (lambda s: _exact_values(rows, cols, s)) if exact else (lambda s: act(rows, cols, s + cols, dtype))
    a = {"h": mk(1), "b": mk(2) if join else None, "w_pre": I.round_to_dtype(1 + 0.2 * I.gaussian((cols,), 3), dtype),
         "w_post": I.round_to_dtype(1 + 0.2 * I.gaussian((cols,), 4), dtype) if post else None,
         "gate": I.round_to_dtype(0.5 + 0.2 * I.gaussian((cols,), 5), dtype) if gate else None}
    return a, {k: None if v is None else to_device(v, dtype) for k, v in a.items()}


def _norm_fwd(desc, dv, dtype, alpha, keep=True, eps=1e-5):
    rows, cols, t = desc.rows, desc.cols, TDT[dtype]
    o = {"y": new(rows, cols, dt=t), "h_out": new(rows, cols, dt=t) if dv["b"] is not None else None}
    k = dict(Hq=None, Hs=None, Bq=None, Bs=None, rstd_post=None, rstd_pre=None)
    if keep:
        k["Hq"], k["Hs"] = q8_new(rows, cols)
        k["rstd_pre"] = new(rows, dt=torch.float32)
        if dv["b"] is not None:
            k["Bq"], k["Bs"] = q8_new(rows, cols)
        if dv["w_post"] is not None:
            k["rstd_post"] = new(rows, dt=torch.float32)
    B.acx_norm_join_fwd(desc, dv["h"], dv["b"], dv["w_post"], dv["gate"], dv["w_pre"], o["h_out"], o["y"], **k, alpha=alpha, eps=eps)
    return o, k


@pytest.mark.parametrize("rows,cols", NORM_SHAPES + WIDE_SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("join,post,gate", VARIANTS)
def test_norm_join(rows, cols, dtype, join, post, gate):
    alpha, eps = 0.7 if join else 1.0, 1e-5
    a, dv = _norm_inputs(rows, cols, dtype, join, post, gate)
    desc = B.make_rows_desc(rows, cols, dtype)
    o, k = _norm_fwd(desc, dv, dtype, alpha)
    o2, _ = _norm_fwd(desc, dv, dtype, alpha, keep=False)
    assert torch.equal(o["y"], o2["y"])
    t, y, r_b, r_t = R.norm_join_fwd(a["h"], a["b"], a["w_post"], a["gate"], a["w_pre"], alpha, eps)
    # fp32 arithmetic: a sum of squares over the row (a tree of at most 32 * 40 additions: under 40 units), the inverse root
    # (2 units), a few products; relative to the largest term of each sum
    e32 = 2.0 ** -24 * 64
    mag = np.abs(a["h"]) + (np.abs(t - a["h"]) if join else 0)
    close("y", o["y"], y, dtype, e32 * mag * r_t * np.abs(a["w_pre"]))
    if join:
        close("h_out", o["h_out"], t, dtype, e32 * mag)
    checks = [("H", a["h"])] + ([("B", a["b"])] if join else [])
    for n, x in checks:
        wc, ws = R.q8_encode(x)
        assert np.array_equal(k[n + "q"].cpu().numpy(), wc) and np.array_equal(raw_bits(k[n + "s"]), ws.view(np.uint32))
    np.testing.assert_allclose(to_host(k["rstd_pre"]), r_t[:, 0], rtol=2 * e32)
    if post:
        np.testing.assert_allclose(to_host(k["rstd_post"]), r_b[:, 0], rtol=e32)

    dy, dn = (I.gaussian((rows, cols), s, 0.1, dtype) for s in (8, 9))
    for with_next in (True, False):
        outs = []
        for _ in range(2):
            z = dict(dh=new(rows, cols, dt=TDT[dtype]), db=new(rows, cols, dt=TDT[dtype]) if join else None,
                     dw_post=new(cols, dt=torch.float32) if post else None, dgate=new(cols, dt=torch.float32) if gate else None,
                     dw_pre=new(cols, dt=torch.float32))
            B.acx_norm_join_bwd(desc, to_device(dy, dtype), to_device(dn, dtype) if with_next else None, dv["w_post"], dv["gate"], dv["w_pre"],
                                k["Hq"], k["Hs"], k["Bq"], k["Bs"], k["rstd_post"], k["rstd_pre"], **z, alpha=alpha,
                                ws=B.alloc_rows_workspace(desc, B.ACX_OP_NORM_BWD))
            outs.append(z)
        for n in z:
            assert z[n] is None or np.array_equal(raw_bits(outs[0][n]), raw_bits(outs[1][n])), n
        hq, bq = R.q8_values(a["h"]), R.q8_values(a["b"]) if join else None
        want = R.norm_join_bwd(dy, dn if with_next else None, hq, bq, a["w_post"], a["gate"], a["w_pre"], r_b, r_t, alpha)
        z = outs[0]
        bh = (bq * (r_b if post else 1.0)) if join else 0.0
        kk = alpha * (a["w_post"] if post else 1.0) * (a["gate"] if gate else 1.0)
        th = (hq + (kk * bh if join else 0)) * r_t
        tm = (np.abs(hq) + (np.abs(kk * bh) if join else 0)) * r_t      # magnitudes of the terms of that
        v = np.abs(dy * a["w_pre"])
        m1 = np.mean(v * tm, axis=1, keepdims=True)
        dm = (np.abs(dn) if with_next else 0) + r_t * (v + tm * m1)      # and of dh
        close("dh", z["dh"], want["dh"], dtype, e32 * dm)
        if join:
            p = np.abs(kk) * dm
            pm = r_b * (p + np.abs(bh) * np.mean(p * np.abs(bh), axis=1, keepdims=True)) if post else p
            close("db", z["db"], want["db"], dtype, 2 * e32 * pm)
        # column sums: a block adds its rows one after the other, then 32 strips of blocks: relative to the sum of magnitudes,
        # (rows per block + blocks / 32 + 32) roundings at worst
        chain = 2.0 ** -24 * (rows / 100 + 100)
        close("dw_pre", z["dw_pre"], want["dw_pre"], "f32", (e32 + chain) * np.sum(np.abs(dy) * tm, axis=0))
        cm = np.abs(alpha) * np.sum(dm * np.abs(bh), axis=0) if join else 0
        if post:
            close("dw_post", z["dw_post"], want["dw_post"], "f32", (e32 + chain) * cm * (np.abs(a["gate"]) if gate else 1.0))
        if gate:
            close("dgate", z["dgate"], want["dgate"], "f32", (e32 + chain) * cm * (np.abs(a["w_post"]) if post else 1.0))


def test_norm_join_gradients_against_differences():
    rows, cols, alpha, eps = 5, 264, 0.7, 2.0 ** -9
    a, dv = _norm_inputs(rows, cols, "f32", True, True, True, exact=True)
    desc = B.make_rows_desc(rows, cols, "f32")
    dy, dn = I.gaussian((rows, cols), 8), I.gaussian((rows, cols), 9)
    _, k = _norm_fwd(desc, dv, "f32", alpha)
    f = torch.float32
    z = dict(dh=new(rows, cols, dt=f), db=new(rows, cols, dt=f), dw_post=new(cols, dt=f), dgate=new(cols, dt=f), dw_pre=new(cols, dt=f))
    B.acx_norm_join_bwd(desc, to_device(dy, "f32"), to_device(dn, "f32"), dv["w_post"], dv["gate"], dv["w_pre"], k["Hq"], k["Hs"], k["Bq"],
                        k["Bs"], k["rstd_post"], k["rstd_pre"], **z, alpha=alpha, ws=B.alloc_rows_workspace(desc, B.ACX_OP_NORM_BWD))

    def value(name, x):
        q = {**dv, name: to_device(x.astype(np.float32), "f32")}
        o, _ = _norm_fwd(desc, q, "f32", alpha, keep=False)
        return np.sum(to_host(o["y"]) * dy) + np.sum(to_host(o["h_out"]) * dn)

    for grad, name in (("dh", "h"), ("db", "b"), ("dw_post", "w_post"), ("dgate", "gate"), ("dw_pre", "w_pre")):
        d = np.sign(I.gaussian(a[name].shape, 11)).astype(np.float32)
        quot = (value(name, a[name] + eps * d) - value(name, a[name] - eps * d)) / (2 * eps)
        n = d.size
        # outputs of size one: their roundings (2^-22 each, random) over eps, and the third derivative's eps^2
        tol = np.sqrt(rows * cols) * 4 * 2.0 ** -22 / eps + 8 * n * eps * eps
        assert abs(np.sum(to_host(z[grad]) * d) - quot) <= tol, (grad, quot, tol)


def test_rows_of_zeros_and_of_nan():
    desc = B.make_rows_desc(4, 264, "bf16")
    h = torch.randn(4, 264, device="cuda").bfloat16()
    b = torch.randn(4, 264, device="cuda").bfloat16()
    h[1], b[1] = 0, 0
    h[2, 7] = NAN
    w = torch.ones(264, device="cuda").bfloat16()
    dv = {"h": h, "b": b, "w_pre": w, "w_post": w, "gate": None}
    o, k = _norm_fwd(desc, dv, "bf16", 1.0)
    assert not o["y"][1].any() and torch.isnan(o["y"][2]).all()
    assert torch.isfinite(o["y"][[0, 1, 3]]).all()
    z = [new(4, 264, dt=torch.bfloat16) for _ in range(2)]
    B.acx_norm_join_bwd(desc, torch.ones_like(h), None, w, None, w, k["Hq"], k["Hs"], k["Bq"], k["Bs"], k["rstd_post"], k["rstd_pre"], *z,
                        None, None, None, alpha=1.0, ws=B.alloc_rows_workspace(desc, B.ACX_OP_NORM_BWD))
    assert torch.isfinite(z[0][[0, 1, 3]]).all() and torch.isfinite(z[1][[0, 1, 3]]).all() and torch.isnan(z[0][2].float()).any()


def test_empty_inputs_and_refusals():
    e = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    d0 = B.make_rows_desc(0, 64, "bf16")
    q = B.q8_empty(0, 64)
    launches = B.acx_kernel_launches()
    B.acx_q8_store(d0, e, *q)
    B.acx_q8_load(d0, *q, e)
    B.acx_swiglu_fwd(d0, e, e, e, *q, *q)
    B.acx_swiglu_bwd(d0, e, *q, *q, e, e)
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    g = [torch.full((64,), 5.0, device="cuda") for _ in range(3)]
    r = torch.empty(0, device="cuda")
    B.acx_norm_join_fwd(d0, e, e, w, w, w, e, e, *q, *q, r, r)
    B.acx_norm_join_bwd(d0, e, e, w, w, w, *q, *q, r, r, e, e, *g)
    assert B.acx_kernel_launches() == launches and not any(x.any() for x in g)
    d = B.make_rows_desc(4, 64, "bf16")
    X = torch.ones(4, 64, dtype=torch.bfloat16, device="cuda")
    q = B.q8_empty(4, 64)
    with pytest.raises(ValueError):
        B.acx_q8_store(d, X.float(), *q)
    with pytest.raises(ValueError):
        B.acx_q8_store(d, torch.ones(64, 4, dtype=torch.bfloat16, device="cuda").t(), *q)
    bad = torch.ones(4, 68, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B.AcxError) as err:
        B.acx_q8_store(d, bad[:, :64], *q)          # a stride that is not a multiple of 8
    assert err.value.status == B.ACX_ERR_UNSUPPORTED_SHAPE
    with pytest.raises(B.AcxError) as err:
        B.acx_q8_store(d, torch.ones(4, 72, dtype=torch.bfloat16, device="cuda")[:, 4:68], *q)   # 8-byte aligned
    assert err.value.status == B.ACX_ERR_ALIGNMENT
    with pytest.raises(B.AcxError) as err:
        B.acx_swiglu_fwd(d, X, X, X.clone(), q[0], q[1], None, None)     # half a checkpoint
    assert err.value.status == B.ACX_ERR_INVALID_ARG
    with pytest.raises(B.AcxError) as err:
        B.acx_norm_join_fwd(d, X, None, w, None, w, None, X.clone())     # a norm behind a block that is not there
    assert err.value.status == B.ACX_ERR_INVALID_ARG
    rstd = torch.ones(4, device="cuda")
    with pytest.raises(B.AcxError) as err:
        B.acx_norm_join_bwd(d, X, None, None, None, w, *q, None, None, None, rstd, X.clone(), None, None, None, None)
    assert err.value.status == B.ACX_ERR_WORKSPACE
    assert B.acx_kernel_launches() == launches


def test_rows_on_two_streams_and_in_a_graph():
    rows, cols = 3000, 1032
    desc = B.make_rows_desc(rows, cols, "bf16")
    GU = torch.randn(rows, 2 * cols, device="cuda").bfloat16()
    dH = torch.randn(rows, cols, device="cuda").bfloat16()
    bufs = lambda: dict(H=new(rows, cols, dt=torch.bfloat16), q=(*q8_new(rows, cols), *q8_new(rows, cols)), dGU=new(rows, 2 * cols, dt=torch.bfloat16))  # noqa: E731

    def step(o, stream=None):
        B.acx_swiglu_fwd(desc, GU[:, :cols], GU[:, cols:], o["H"], *o["q"], stream=stream)
        B.acx_swiglu_bwd(desc, dH, *o["q"], o["dGU"][:, :cols], o["dGU"][:, cols:], stream=stream)

    ref = bufs()
    step(ref)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream(), torch.cuda.Stream()], [bufs(), bufs()]
    torch.cuda.synchronize()
    for s, o in zip(streams, outs):
        step(o, s)
    graphed = bufs()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        step(graphed)
    g.replay()
    torch.cuda.synchronize()
    for o in outs + [graphed]:
        assert torch.equal(o["H"], ref["H"]) and torch.equal(o["dGU"], ref["dGU"])


@pytest.mark.parametrize("rows,cols", [(3, 8), (37, 264), (9, 2056), (5, 3000)])
def test_fp32_matrices_that_start_between_two_32_byte_boundaries(rows, cols):
    """The same bits wherever the matrices start: 16-byte alignment is all that is asked for, 32 bytes take the wide accesses."""
    n, vec, one = rows * cols, (cols,), torch.float32

    def at(offset, *shape):     # a dense fp32 matrix `offset` elements behind a 32-byte boundary, with a guard behind it
        flat = torch.full((offset + int(np.prod(shape)) + 8,), NAN, dtype=one, device="cuda")
        assert flat.data_ptr() % 32 == 0
        return flat, flat[offset:offset + int(np.prod(shape))].view(shape)

    d = B.make_rows_desc(rows, cols, "f32")
    src = [to_device(act(rows, cols, 11 + k, "f32"), "f32") for k in range(4)]
    w = [to_device(1 + I.gaussian((1, cols), 20 + k, 0.2), "f32")[0] for k in range(3)]
    ws = B.alloc_rows_workspace(d, B.ACX_OP_NORM_BWD)
    results = []
    for offset in (0, 4):
        ins = []
        for t in src + w:
            v = at(offset, *t.shape)[1]
            v.copy_(t)
            ins.append(v)
        x, b, dy, dn, w_post, gate, w_pre = ins
        flats, outs = zip(*[at(offset, rows, cols) for _ in range(8)])
        H, dG, dU, h_out, y, dh, db, back = outs
        q = [q8_new(rows, cols) for _ in range(4)]
        r = [new(rows, dt=one) for _ in range(2)]
        g = [new(*vec, dt=one) for _ in range(3)]
        B.acx_swiglu_fwd(d, x, b, H, *q[0], *q[1])
        B.acx_swiglu_bwd(d, dy, *q[0], *q[1], dG, dU)
        B.acx_norm_join_fwd(d, x, b, w_post, gate, w_pre, h_out, y, *q[2], *q[3], *r, alpha=0.5)
        B.acx_norm_join_bwd(d, dy, dn, w_post, gate, w_pre, *q[2], *q[3], *r, dh, db, *g, alpha=0.5, ws=ws)
        B.acx_q8_load(d, *q[2], back)
        for flat in flats:
            assert torch.isnan(flat[:offset]).all() and torch.isnan(flat[offset + n:]).all()
        results.append([t.clone() for t in (*outs, *g, *r, *(t for pair in q for t in pair))])
    for a, c in zip(*results):
        assert torch.equal(a, c) and not torch.isnan(a.float()).any()
