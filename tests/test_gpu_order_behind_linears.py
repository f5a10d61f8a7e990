"""What follows acx_linear_bwd on its stream finds dX complete.  The call's last launch is the gradient factor, which starts
beside dX and needs nothing of it; the row operators line up behind that launch and wait for it alone, so the factor may not
end before dX.  The shapes give dX few tiles with a long contraction and the factor many short ones, which then runs to its
end on the SMs that dX leaves free."""
import pytest
import torch

from paper_2605_01255_b200 import binding as B

pytestmark = pytest.mark.gpu

# tokens, d_in, d_out, r: the factor unsplit, split in clusters, narrow and wide
SHAPES = [(64, 896, 9728, 64), (256, 896, 19456, 128), (512, 896, 9728, 64), (512, 136, 9728, 16), (300, 1032, 16392, 192)]


class Chain:
    """acx_linear_bwd and, right behind it, a row operator that reads its dX."""

    def __init__(self, m, d_in, d_out, r, reader):
        g = torch.Generator(device="cuda").manual_seed(m + d_out)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.desc = B.make_desc(m, d_in, d_out, r, 0, "bf16")
        self.G, self.W = rnd(m, d_out).bfloat16(), (rnd(d_out, d_in) * d_out ** -0.5).bfloat16()
        self.XS, self.A = rnd(m, r).bfloat16(), torch.empty(d_out, r, device="cuda")
        self.dX = torch.empty(m, d_in, dtype=torch.bfloat16, device="cuda")
        self.ws = B.alloc_workspace(self.desc, B.ACX_OP_BWD)
        self.rows, self.reader = B.make_rows_desc(m, d_in, "bf16"), reader
        if reader == "q8":
            self.out = B.q8_empty(m, d_in)
        else:
            self.qG, self.qU = B.q8_empty(m, d_in), B.q8_empty(m, d_in)
            for q in (self.qG, self.qU):
                B.acx_q8_store(self.rows, rnd(m, d_in).bfloat16(), *q)
            self.out = torch.empty_like(self.dX), torch.empty_like(self.dX)
            if reader == "norm":
                self.w, self.rstd = torch.ones(d_in, dtype=torch.bfloat16, device="cuda"), torch.ones(m, device="cuda")
                self.out = self.out[0], torch.empty(d_in, device="cuda")
                self.ws_norm = B.alloc_rows_workspace(self.rows, B.ACX_OP_NORM_BWD)

    def linear(self):
        B.acx_linear_bwd(self.desc, self.G, self.W, self.XS, self.dX, self.A, self.ws)

    def read(self):
        if self.reader == "q8":
            B.acx_q8_store(self.rows, self.dX, *self.out)
        elif self.reader == "swiglu":
            B.acx_swiglu_bwd(self.rows, self.dX, *self.qG, *self.qU, *self.out)
        else:
            B.acx_norm_join_bwd(self.rows, self.dX, None, None, None, self.w, *self.qG, None, None, None, self.rstd, self.out[0], None,
                                None, None, self.out[1], ws=self.ws_norm)


@pytest.mark.parametrize("m,d_in,d_out,r", SHAPES)
@pytest.mark.parametrize("reader", ["q8", "swiglu", "norm"])
def test_readers_right_behind_the_backward_see_all_of_dx(m, d_in, d_out, r, reader):
    c = Chain(m, d_in, d_out, r, reader)
    c.linear()
    torch.cuda.synchronize()
    c.read()
    want = [t.clone() for t in c.out]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        c.linear()
        c.read()

    def once():
        c.linear()
        c.read()

    for run in (once, graph.replay):
        for _ in range(40):
            c.dX.zero_()             # what a reader that comes too early finds
            for t in c.out:
                t.zero_()
            run()
            for a, b in zip(c.out, want):
                assert torch.equal(a, b)
    assert B.acx_last_device_status() == B.ACX_OK
