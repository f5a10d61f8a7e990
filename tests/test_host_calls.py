"""What the compiled argument checks in front of the row operators and the cross entropy refuse, and that nothing of a refused
call runs.  The checks come before any CUDA call, so the refusals of tensors that are not on a GPU are tested without one."""
import pytest
import torch

from paper_2605_01255_b200 import binding as B
from paper_2605_01255_b200 import build as acx_build


@pytest.fixture(scope="module", autouse=True)
def built():
    acx_build.build()


def calls(device):
    """Every operator with complete arguments: name, function, arguments by name in order, keywords."""
    bf16, f32 = torch.bfloat16, torch.float32
    rows, cols, tokens, d, vocab = 4, 136, 5, 64, 40
    m = lambda: torch.ones(rows, cols, dtype=bf16, device=device)  # noqa: E731
    v = lambda dt=bf16: torch.ones(cols, dtype=dt, device=device)  # noqa: E731
    q = lambda: torch.zeros(rows, cols, dtype=torch.int8, device=device)  # noqa: E731
    s = lambda: torch.ones(rows, 2, dtype=f32, device=device)  # noqa: E731
    r = lambda n=rows: torch.ones(n, dtype=f32, device=device)  # noqa: E731
    rd, cd = B.make_rows_desc(rows, cols, bf16), B.make_ce_desc(tokens, d, vocab)
    ws = lambda desc, op, need: torch.empty(need(desc, op), dtype=torch.uint8, device=device)  # noqa: E731
    X, W = torch.ones(tokens, d, dtype=bf16, device=device), torch.ones(vocab, d, dtype=bf16, device=device)
    y = torch.arange(tokens, device=device)
    one = torch.ones(1, device=device)
    norm_ws = {"ws": ws(rd, B.ACX_OP_NORM_BWD, B.acx_rows_workspace_bytes)} if device == "cuda" else {}
    fwd_ws = ({"ws": ws(cd, B.ACX_OP_CE_FWD, B.acx_ce_workspace_bytes)}) if device == "cuda" else {}
    bwd_ws = ({"ws": ws(cd, B.ACX_OP_CE_BWD, B.acx_ce_workspace_bytes)}) if device == "cuda" else {}
    return [
        (B.acx_q8_store, rd, dict(X=m(), codes=q(), scales=s()), {}),
        (B.acx_q8_load, rd, dict(codes=q(), scales=s(), X=m()), {}),
        (B.acx_swiglu_fwd, rd, dict(G=m(), U=m(), H=m(), Gq=q(), Gs=s(), Uq=q(), Us=s()), {}),
        (B.acx_swiglu_bwd, rd, dict(dH=m(), Gq=q(), Gs=s(), Uq=q(), Us=s(), dG=m(), dU=m()), {}),
        (B.acx_norm_join_fwd, rd, dict(h=m(), b=m(), w_post=v(), gate=v(), w_pre=v(), h_out=m(), y=m(), Hq=q(), Hs=s(), Bq=q(), Bs=s(),
                                       rstd_post=r(), rstd_pre=r()), dict(eps=1e-5, alpha=0.5)),
        (B.acx_norm_join_bwd, rd, dict(dy=m(), dh_next=m(), w_post=v(), gate=v(), w_pre=v(), Hq=q(), Hs=s(), Bq=q(), Bs=s(), rstd_post=r(),
                                       rstd_pre=r(), dh=m(), db=m(), dw_post=v(f32), dgate=v(f32), dw_pre=v(f32)), dict(alpha=0.5, **norm_ws)),
        (B.acx_linear_ce_fwd, cd, dict(X=X, W=W, targets=y, loss=r(tokens), lse=r(tokens), total=r(2), weight=r(tokens)), fwd_ws),
        (B.acx_linear_ce_bwd, cd, dict(X=X, W=W, targets=y, lse=r(tokens), dX=torch.empty_like(X), dW=torch.empty_like(W)),
         dict(weight=r(tokens), denom=one, scale=1.0, **bwd_ws)),
    ]


OPS = list(range(8))
STRIDED = {"acx_q8_store": ("X",), "acx_q8_load": ("X",), "acx_swiglu_fwd": ("G", "U"), "acx_swiglu_bwd": ("dG", "dU")}


@pytest.mark.parametrize("op", OPS)
def test_tensors_that_are_not_on_a_gpu_are_refused(op):
    f, desc, args, kw = calls("cpu")[op]
    first = next(iter(args)) if op != 1 else "codes"
    with pytest.raises(ValueError, match="cpu"):
        f(desc, *args.values(), **kw)
    with pytest.raises(ValueError, match=first + r"|codes of X"):
        f(desc, "text", *list(args.values())[1:], **kw)


@pytest.mark.parametrize("op", OPS)
def test_descriptor_of_another_operator(op):
    f, desc, args, kw = calls("cpu")[op]
    other = B.make_desc(4, 64, 64, 16, 0, "bf16")
    with pytest.raises(TypeError):
        f(other, *args.values(), **kw)
    with pytest.raises(TypeError):
        f(None, *args.values(), **kw)


def test_missing_matrix_and_unbound_numbers():
    d = B.make_rows_desc(4, 64, "bf16")
    with pytest.raises(ValueError, match="X must be"):
        B.acx_q8_store(d, None, None, None)
    with pytest.raises(TypeError):
        B._calls().q8_store(d)
    with pytest.raises(TypeError):
        B._calls().bind((1, 2))


@pytest.mark.gpu
@pytest.mark.parametrize("op", OPS)
def test_wrong_type_shape_or_order_of_each_argument(op):
    f, desc, args, kw = calls("cuda")[op]
    f(desc, *args.values(), **kw)
    torch.cuda.synchronize()
    launches = B.acx_kernel_launches()
    for name, t in args.items():
        bad = [t.double(), t[:-1].clone(), t.cpu(), t.to_sparse()]
        if t.dim() == 2:
            bad.append(torch.empty_strided(t.shape, (1, t.shape[0]), dtype=t.dtype, device="cuda"))     # columns first
            if name not in STRIDED.get(f.__name__, ()):
                bad.append(torch.empty(t.shape[0], t.shape[1] + 16, dtype=t.dtype, device="cuda")[:, :t.shape[1]])
        else:
            bad.append(torch.empty(2 * t.numel(), dtype=t.dtype, device="cuda")[::2])
        for x in bad:
            if x.dtype == t.dtype and x.layout is torch.strided and x.is_cuda and x.shape == t.shape and x.is_contiguous():
                continue
            with pytest.raises(ValueError):
                f(desc, *[x if k == name else a for k, a in args.items()], **kw)
    if "ws" in kw:
        with pytest.raises(B.AcxError) as err:
            f(desc, *args.values(), **dict(kw, ws=None))
        assert err.value.status == B.ACX_ERR_WORKSPACE
        with pytest.raises(ValueError):
            f(desc, *args.values(), **dict(kw, ws=kw["ws"].cpu()))
        with pytest.raises(B.AcxError) as err:
            f(desc, *args.values(), **dict(kw, ws=kw["ws"][:kw["ws"].numel() // 2]))
        assert err.value.status == B.ACX_ERR_WORKSPACE
    with pytest.raises(AttributeError):
        f(desc, *args.values(), **dict(kw, stream=3))
    assert B.acx_kernel_launches() == launches


@pytest.mark.gpu
def test_parameters_and_streams():
    d = B.make_rows_desc(3, 64, "f32")
    X = torch.nn.Parameter(torch.randn(3, 64, device="cuda"))
    codes, scales = B.q8_empty(3, 64)
    want = [t.clone() for t in (codes, scales)]
    B.acx_q8_store(d, X, *want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.acx_q8_store(d, X, codes, scales, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(codes, want[0]) and torch.equal(scales, want[1])
    codes.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.acx_q8_store(d, X, codes, scales)
    side.synchronize()
    assert torch.equal(codes, want[0])
