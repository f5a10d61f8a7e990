"""What the training step says it keeps between forward and backward is what its backward pass reads: every tensor that the calls are
given there and that is neither a weight, a gradient, a descriptor nor scratch."""
import torch

from paper_2605_01255_b200 import binding as B
from paper_2605_01255_b200 import build as acx_build
from paper_2605_01255_b200 import mlp_lm as M


def test_kept_bytes_are_the_bytes_the_backward_reads(monkeypatch):
    acx_build.build()
    s = M.Sizes(tokens=96, d=64, inter=128, vocab=100, layers=2, r=16)
    model = M.MlpLm(s, device="cpu")
    h0, y = M.synthetic_batch(s, device="cpu")
    read = {}

    def record(written):
        """Notes the tensors of a call up to its first output."""
        def call(desc, *args, **kw):
            named = [kw[k] for k in ("loss", "weight", "denom") if kw.get(k) is not None]
            for i, t in enumerate(args):
                if isinstance(t, torch.Tensor) and i not in written:
                    read[t.untyped_storage().data_ptr()] = t.untyped_storage().nbytes()
            for t in named:
                read[t.untyped_storage().data_ptr()] = t.untyped_storage().nbytes()
        return call

    nothing = lambda *a, **k: None  # noqa: E731
    for name in ("acx_norm_join_fwd", "acx_linear_fwd", "acx_swiglu_fwd", "acx_linear_ce_fwd"):
        monkeypatch.setattr(B, name, nothing)
    model.forward(h0, y)
    monkeypatch.setattr(B, "acx_linear_ce_bwd", record({4, 5}))
    monkeypatch.setattr(B, "acx_norm_join_bwd", record({11, 12, 13, 14, 15}))
    monkeypatch.setattr(B, "acx_linear_bwd", record({3, 4, 5}))
    monkeypatch.setattr(B, "acx_swiglu_bwd", record({5, 6}))
    model.backward()
    known = [model.head, *model.w_pre, *model.w_post, *model.gate, *(w for lw in model.w for w in lw.values()),        # weights
             model.dy, model.db, model.dgu, model.dhid, *model.dh, y]                                                 # gradients, the batch
    for t in known:
        read.pop(t.untyped_storage().data_ptr(), None)
    assert model.kept_bytes()["kept"] == sum(read.values())
