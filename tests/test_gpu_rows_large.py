"""The row operators on matrices of more than 2^31 elements: the rows around that element and the last ones come out as they do in a
small call on those rows alone (rows do not depend on one another)."""
import pytest
import torch

from paper_2605_01255_b200 import binding as B

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _blocks(rows, cols):
    edge = (1 << 31) // cols
    assert edge + 40 < rows < edge + 4000
    return [slice(0, 70), slice(edge // 2 - 5, edge // 2 + 60), slice(edge - 40, edge + 40), slice(rows - 70, rows)]


def _rand(rows, cols, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(rows, cols, generator=g, device="cuda", dtype=BF)


def _new(rows, cols, dt=BF):
    return torch.empty(rows, cols, dtype=dt, device="cuda")


def test_checkpoints_and_gated_activation():
    rows, cols = 262_100, 8200
    big = B.make_rows_desc(rows, cols, BF)
    G, U = _rand(rows, cols, 1), _rand(rows, cols, 2)
    qG, qU, H, back = B.q8_empty(rows, cols), B.q8_empty(rows, cols), _new(rows, cols), _new(rows, cols)
    B.acx_swiglu_fwd(big, G, U, H, *qG, *qU)
    q = B.q8_empty(rows, cols)
    B.acx_q8_store(big, G, *q)
    assert torch.equal(q[0], qG[0]) and torch.equal(q[1], qG[1])
    B.acx_q8_load(big, *q, back)
    dH, dG, dU = H, _new(rows, cols), _new(rows, cols)
    B.acx_swiglu_bwd(big, dH, *qG, *qU, dG, dU)
    for s in _blocks(rows, cols):
        n = s.stop - s.start
        d = B.make_rows_desc(n, cols, BF)
        a, b, h, x, dg, du = B.q8_empty(n, cols), B.q8_empty(n, cols), _new(n, cols), _new(n, cols), _new(n, cols), _new(n, cols)
        B.acx_swiglu_fwd(d, G[s], U[s], h, *a, *b)
        B.acx_q8_load(d, *a, x)
        B.acx_swiglu_bwd(d, dH[s], *a, *b, dg, du)
        for large, small in ((qG[0], a[0]), (qG[1], a[1]), (qU[0], b[0]), (qU[1], b[1]), (H, h), (back, x), (dG, dg), (dU, du)):
            assert torch.equal(large[s], small)


@pytest.mark.parametrize("rows,cols", [(262_300, 8192), (262_100, 8200)])      # a row in one block, and shared by several
def test_norm_join(rows, cols):
    big = B.make_rows_desc(rows, cols, BF)
    h, b, dy, dn = (_rand(rows, cols, k) for k in (1, 2, 3, 4))
    w = [(1 + 0.2 * torch.randn(cols, device="cuda")).to(BF) for _ in range(3)]
    grads = lambda: [torch.empty(cols, device="cuda") for _ in range(3)]  # noqa: E731

    def step(desc, h, b, dy, dn):
        n = desc.rows
        h_out, y, dh, db = (_new(n, cols) for _ in range(4))
        q, r, g = B.q8_empty(n, cols) + B.q8_empty(n, cols), [torch.empty(n, device="cuda") for _ in range(2)], grads()
        B.acx_norm_join_fwd(desc, h, b, *w, h_out, y, *q, *r, alpha=0.5)
        B.acx_norm_join_bwd(desc, dy, dn, *w, *q, *r, dh, db, *g, alpha=0.5, ws=B.alloc_rows_workspace(desc, B.ACX_OP_NORM_BWD))
        return [h_out, y, dh, db, *q, *r], g

    outs, g = step(big, h, b, dy, dn)
    for s in _blocks(rows, cols):
        small, _ = step(B.make_rows_desc(s.stop - s.start, cols, BF), h[s], b[s], dy[s], dn[s])
        for x, z in zip(outs, small):
            assert torch.equal(x[s], z)
    # the vectors' gradients: those of the parts add up to them
    parts = [0.0, 0.0, 0.0]
    size = [0.0, 0.0, 0.0]
    for r0 in range(0, rows, 40_000):
        s = slice(r0, min(rows, r0 + 40_000))
        _, p = step(B.make_rows_desc(s.stop - s.start, cols, BF), h[s], b[s], dy[s], dn[s])
        parts, size = [a + x.double() for a, x in zip(parts, p)], [a + x.double().square() for a, x in zip(size, p)]
    for x, a, z in zip(g, parts, size):
        # sums of rows / 200 terms each, in fp32: relative to the root of the sum of squares that the parts have
        assert bool(((x.double() - a).abs() <= 2.0 ** -24 * (rows / 100 + 100) * z.sqrt().amax()).all())
    assert B.acx_last_device_status() == B.ACX_OK
