"""What attention, the embedding table and the clipping refuse.  All refusals come before any CUDA call, so those of the C entries
and of tensors that are not on a GPU are tested without one."""
import ctypes

import pytest
import torch

from paper_2605_01255_b200 import binding as B
from paper_2605_01255_b200 import build as acx_build

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def built():
    acx_build.build()


# ------------------------------------------------------------------------------------------------------------- C entries
P = 1 << 20      # an aligned address that no refused call reads


def attn_desc(**kw):
    d = B.make_attn_desc(256, 4, 2, 64, 3)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def attn_calls(d, **kw):
    """The three entries with arguments that are in order, those of `kw` replaced."""
    room = 1 << 40
    a = dict(offsets=P, prefix=None, plan=P, plan_bytes=room, Q=P, ldq=256, K=P, ldk=128, V=P, ldv=128, slopes=None, O=P, ldo=256, lse=P, dO=P, lddo=256,
             dQ=P, lddq=256, dK=P, lddk=128, dV=P, lddv=128, ws=P, ws_bytes=room)
    a.update(kw)
    take = lambda *names: [ctypes.c_void_p(a[n]) if a[n] is None or not n.startswith("ld") and not n.endswith("bytes") else a[n] for n in names]  # noqa: E731
    L, ref = B.lib(), ctypes.byref(d)
    mats = ("Q", "ldq", "K", "ldk", "V", "ldv", "slopes", "plan", "plan_bytes")
    return {
        "plan": lambda: L.acx_attn_plan(ref, *take("offsets", "prefix", "plan", "plan_bytes"), None),
        "fwd": lambda: L.acx_attn_fwd(ref, *take(*mats, "O", "ldo"), ctypes.c_void_p(a["lse"]), None),
        "bwd": lambda: L.acx_attn_bwd(ref, *take(*mats, "O", "ldo", "dO", "lddo"), ctypes.c_void_p(a["lse"]),
                                      *take("dQ", "lddq", "dK", "lddk", "dV", "lddv", "ws", "ws_bytes"), None),
    }


BAD_ATTN = [(dict(struct_size=8), B.ACX_ERR_INVALID_ARG), (dict(io_dtype=B.ACX_F32), B.ACX_ERR_INVALID_ARG), (dict(io_dtype=7), B.ACX_ERR_INVALID_ARG),
            (dict(causal=2), B.ACX_ERR_INVALID_ARG), (dict(scale=0.0), B.ACX_ERR_INVALID_ARG), (dict(scale=-1.0), B.ACX_ERR_INVALID_ARG),
            (dict(scale=NAN), B.ACX_ERR_INVALID_ARG), (dict(scale=INF), B.ACX_ERR_INVALID_ARG), (dict(softcap=-1.0), B.ACX_ERR_INVALID_ARG),
            (dict(softcap=NAN), B.ACX_ERR_INVALID_ARG), (dict(softcap=INF), B.ACX_ERR_INVALID_ARG), (dict(tokens=-1), B.ACX_ERR_UNSUPPORTED_SHAPE),
            (dict(tokens=(1 << 24) + 1), B.ACX_ERR_UNSUPPORTED_SHAPE), (dict(docs=0), B.ACX_ERR_UNSUPPORTED_SHAPE),
            (dict(docs=(1 << 24) + 1), B.ACX_ERR_UNSUPPORTED_SHAPE), (dict(heads=0), B.ACX_ERR_UNSUPPORTED_SHAPE),
            (dict(heads=5), B.ACX_ERR_UNSUPPORTED_SHAPE), (dict(heads=4098), B.ACX_ERR_UNSUPPORTED_SHAPE), (dict(kv_heads=0), B.ACX_ERR_UNSUPPORTED_SHAPE),
            (dict(kv_heads=-2), B.ACX_ERR_UNSUPPORTED_SHAPE), (dict(head_dim=0), B.ACX_ERR_UNSUPPORTED_SHAPE),
            (dict(head_dim=60), B.ACX_ERR_UNSUPPORTED_SHAPE), (dict(head_dim=136), B.ACX_ERR_UNSUPPORTED_SHAPE),
            (dict(heads=4096, tokens=1 << 24, docs=1 << 20), B.ACX_ERR_UNSUPPORTED_SHAPE)]


@pytest.mark.parametrize("change,status", BAD_ATTN, ids=lambda x: str(x))
def test_attention_descriptors(change, status):
    d = attn_desc(**change)
    for f in attn_calls(d).values():
        assert f() == status
    assert B.acx_attn_workspace_bytes(d, B.ACX_OP_ATTN_PLAN) == 0 and B.acx_attn_workspace_bytes(d, B.ACX_OP_ATTN_BWD) == 0


@pytest.mark.parametrize("name", ["plan", "fwd", "bwd"])
def test_attention_arguments(name):
    d = attn_desc()
    wanted = {"plan": ("offsets",), "fwd": ("Q", "K", "V", "O"), "bwd": ("Q", "K", "V", "O", "dO", "lse", "dQ", "dK", "dV")}[name]
    for k in wanted:
        assert attn_calls(d, **{k: None})[name]() == B.ACX_ERR_INVALID_ARG, k
        assert attn_calls(d, **{k: P + 2})[name]() == B.ACX_ERR_ALIGNMENT, k
    if name == "plan":
        assert attn_calls(d, prefix=P + 2)[name]() == B.ACX_ERR_ALIGNMENT
        assert attn_calls(attn_desc(causal=0), prefix=P)[name]() == B.ACX_ERR_INVALID_ARG
    else:
        assert attn_calls(d, slopes=P + 2)[name]() == B.ACX_ERR_ALIGNMENT
        for k in ("ldq", "ldk", "ldv", "ldo") + (("lddo", "lddq", "lddk", "lddv") if name == "bwd" else ()):
            least = 256 if k[-1] in "qo" else 128
            for bad in (least - 8, least + 4, 0, -256, 1 << 40):
                assert attn_calls(d, **{k: bad})[name]() == B.ACX_ERR_UNSUPPORTED_SHAPE, (k, bad)
    need = B.acx_attn_workspace_bytes(d, B.ACX_OP_ATTN_PLAN)
    assert attn_calls(d, plan=None)[name]() == B.ACX_ERR_WORKSPACE
    assert attn_calls(d, plan_bytes=need - 1)[name]() == B.ACX_ERR_WORKSPACE
    assert attn_calls(d, plan=P + 8)[name]() == B.ACX_ERR_ALIGNMENT
    if name == "bwd":
        assert attn_calls(d, ws=None)[name]() == B.ACX_ERR_WORKSPACE
        assert attn_calls(d, ws_bytes=B.acx_attn_workspace_bytes(d, B.ACX_OP_ATTN_BWD) - 1)[name]() == B.ACX_ERR_WORKSPACE


def test_no_tokens_is_no_work():
    calls = attn_calls(attn_desc(tokens=0), Q=None, K=None, V=None, O=None, dO=None, lse=None, dQ=None, dK=None, dV=None, ws=None, ws_bytes=0)
    assert calls["fwd"]() == B.ACX_OK and calls["bwd"]() == B.ACX_OK


def embed_call(fwd, change=None, ids=P, E=P, Y=P, beta=0.0, ws=P, ws_bytes=1 << 40):
    d = B.make_embed_desc(100, 64, 1000, "bf16", "f32")
    for k, v in (change or {}).items():
        setattr(d, k, v)
    p = ctypes.c_void_p
    if fwd:
        return B.lib().acx_embed_fwd(ctypes.byref(d), p(ids), p(E), p(Y), None)
    return B.lib().acx_embed_bwd(ctypes.byref(d), p(ids), p(Y), p(E), beta, p(ws), ws_bytes, None)


def test_embedding_refusals():
    for change, status in [(dict(struct_size=0), B.ACX_ERR_INVALID_ARG), (dict(io_dtype=9), B.ACX_ERR_INVALID_ARG), (dict(grad_dtype=-1), B.ACX_ERR_INVALID_ARG),
                           (dict(scale=NAN), B.ACX_ERR_INVALID_ARG), (dict(scale=INF), B.ACX_ERR_INVALID_ARG), (dict(tokens=-1), B.ACX_ERR_UNSUPPORTED_SHAPE),
                           (dict(tokens=(1 << 28) + 1), B.ACX_ERR_UNSUPPORTED_SHAPE), (dict(d=0), B.ACX_ERR_UNSUPPORTED_SHAPE),
                           (dict(d=60), B.ACX_ERR_UNSUPPORTED_SHAPE), (dict(d=65544), B.ACX_ERR_UNSUPPORTED_SHAPE),
                           (dict(vocab=0), B.ACX_ERR_UNSUPPORTED_SHAPE), (dict(vocab=(1 << 22) + 1), B.ACX_ERR_UNSUPPORTED_SHAPE)]:
        for fwd in (True, False):
            assert embed_call(fwd, change) == status, change
    for fwd in (True, False):
        for name, step in (("ids", 4), ("E", 8), ("Y", 8)):
            assert embed_call(fwd, **{name: None}) == B.ACX_ERR_INVALID_ARG, name
            assert embed_call(fwd, **{name: P + step}) == B.ACX_ERR_ALIGNMENT, name
    assert embed_call(False, beta=NAN) == B.ACX_ERR_INVALID_ARG
    assert embed_call(False, ws=None) == B.ACX_ERR_WORKSPACE
    need = B.acx_embed_workspace_bytes(B.make_embed_desc(100, 64, 1000, "bf16", "f32"), B.ACX_OP_EMBED_BWD)
    assert need > 0 and embed_call(False, ws_bytes=need - 1) == B.ACX_ERR_WORKSPACE
    assert embed_call(True, dict(tokens=0), ids=None, E=None, Y=None) == B.ACX_OK
    assert embed_call(False, dict(tokens=0), ids=None, Y=None, beta=1.0, ws=None, ws_bytes=0) == B.ACX_OK


def describe(*items):
    """items: (src, dst, n, weight, types)"""
    arr = (B.acx_grad * max(1, len(items)))()
    for i, (src, dst, n, w, (a, b)) in enumerate(items):
        arr[i] = B.acx_grad(src, dst, n, w, a, b, 0)
    d = B.acx_grad_desc()
    return B.lib().acx_grad_describe(arr, len(items), ctypes.byref(d)), d, arr


F, H = B.ACX_F32, B.ACX_BF16


def test_lists_of_gradients():
    ok, d, arr = describe((P, P, 10, 1.0, (F, F)), (2 * P, 3 * P, 5, 0.0, (H, F)), (None, None, 0, 1.0, (F, H)))
    assert ok == B.ACX_OK and d.tensors == 3 and d.chunks == 2
    for item, status in [((P, P, 10, -1.0, (F, F)), B.ACX_ERR_INVALID_ARG), ((P, P, 10, NAN, (F, F)), B.ACX_ERR_INVALID_ARG),
                         ((P, P, 10, INF, (F, F)), B.ACX_ERR_INVALID_ARG), ((P, P, 10, 1.0, (5, F)), B.ACX_ERR_INVALID_ARG),
                         ((P, P, 10, 1.0, (F, H)), B.ACX_ERR_INVALID_ARG), ((None, P, 10, 1.0, (F, F)), B.ACX_ERR_INVALID_ARG),
                         ((P, None, 10, 1.0, (F, F)), B.ACX_ERR_INVALID_ARG), ((P + 4, P, 10, 1.0, (F, F)), B.ACX_ERR_ALIGNMENT),
                         ((P, 2 * P + 8, 10, 1.0, (F, F)), B.ACX_ERR_ALIGNMENT), ((P, P, -1, 1.0, (F, F)), B.ACX_ERR_UNSUPPORTED_SHAPE),
                         ((P, P, (1 << 40) + 1, 1.0, (F, F)), B.ACX_ERR_UNSUPPORTED_SHAPE)]:
        assert describe((4 * P, 4 * P, 8, 1.0, (F, F)), item)[0] == status, item
    L, p = B.lib(), ctypes.c_void_p
    assert L.acx_grad_describe(None, 1, ctypes.byref(d)) == B.ACX_ERR_INVALID_ARG and L.acx_grad_describe(arr, 1, None) == B.ACX_ERR_INVALID_ARG
    assert L.acx_grad_describe(arr, -1, ctypes.byref(d)) == B.ACX_ERR_INVALID_ARG
    ok, d, arr = describe((P, P, 10, 1.0, (F, F)))
    need = L.acx_grad_workspace_bytes(ctypes.byref(d), B.ACX_OP_GRAD_PLAN)
    assert L.acx_grad_plan(ctypes.byref(d), arr, p(P), need - 1, None) == B.ACX_ERR_WORKSPACE
    assert L.acx_grad_plan(ctypes.byref(d), arr, None, need, None) == B.ACX_ERR_WORKSPACE
    assert L.acx_grad_plan(ctypes.byref(d), arr, p(P + 8), need, None) == B.ACX_ERR_ALIGNMENT
    clip = lambda max_norm=1.0, total=P, plan=P, plan_bytes=need, ws=P, ws_bytes=1 << 30: L.acx_grad_clip(  # noqa: E731
        ctypes.byref(d), p(plan), plan_bytes, max_norm, p(total), p(ws), ws_bytes, None)
    for bad in (0.0, -1.0, NAN):
        assert clip(max_norm=bad) == B.ACX_ERR_INVALID_ARG
    assert clip(total=None) == B.ACX_ERR_INVALID_ARG and clip(total=P + 2) == B.ACX_ERR_ALIGNMENT
    assert clip(plan=None) == B.ACX_ERR_WORKSPACE and clip(plan_bytes=need - 1) == B.ACX_ERR_WORKSPACE and clip(plan=P + 8) == B.ACX_ERR_ALIGNMENT
    assert clip(ws=None) == B.ACX_ERR_WORKSPACE and clip(ws_bytes=8) == B.ACX_ERR_WORKSPACE
    d.chunks += 1
    assert L.acx_grad_plan(ctypes.byref(d), arr, p(P), 1 << 20, None) == B.ACX_ERR_INVALID_ARG     # another list's descriptor
    d.reserved = 1
    assert clip(plan_bytes=1 << 20) == B.ACX_ERR_INVALID_ARG


@pytest.mark.parametrize("items,ok", [
    ([(P, P, 100, 1.0, (F, F)), (P + 400, P + 400, 8, 1.0, (F, F))], True),                       # neighbours
    ([(P, P, 100, 1.0, (F, F)), (P, P, 100, 1.0, (F, F))], False),                                # one tensor twice, in place
    ([(P, P, 100, 1.0, (F, F)), (P + 384, P + 384, 8, 1.0, (F, F))], False),                      # the last four elements
    ([(P, 2 * P, 100, 1.0, (F, F)), (P, 3 * P, 100, 1.0, (F, F))], True),                         # read twice
    ([(P, 2 * P, 100, 1.0, (F, F)), (2 * P, 3 * P, 100, 1.0, (F, F))], False),                    # an output is another one's input
    ([(P, P + 16, 100, 1.0, (F, F))], False),                                                     # shifted
    ([(P, 2 * P, 100, 1.0, (F, H)), (3 * P, 2 * P + 208, 100, 1.0, (F, H))], True),
    ([(P, 2 * P, 100, 1.0, (F, H)), (3 * P, 2 * P + 192, 100, 1.0, (F, H))], False),
    ([(P, P, 0, 1.0, (F, F)), (P, P, 100, 1.0, (F, F))], True),                                   # nothing of an empty one is there
])
def test_outputs_that_overlap(items, ok):
    assert describe(*items)[0] == (B.ACX_OK if ok else B.ACX_ERR_INVALID_ARG)


# ------------------------------------------------------------------------------------------- the compiled argument checks
def calls(device):
    """Every operator with complete arguments: name, function, descriptor, arguments by name in order, keywords."""
    T, H, K, d, docs, vocab = 7, 4, 2, 16, 2, 30
    m = lambda h: torch.ones(T, h, d, dtype=BF, device=device)  # noqa: E731
    ad, ed = B.make_attn_desc(T, H, K, d, docs), B.make_embed_desc(T, 64, vocab, BF, F32)
    room = lambda n: torch.zeros(n, dtype=torch.uint8, device=device)  # noqa: E731
    plan = room(B.acx_attn_workspace_bytes(ad, B.ACX_OP_ATTN_PLAN))
    lse = torch.zeros(H, T, device=device)
    offsets = torch.tensor([0, 3, T], dtype=I32, device=device)
    slopes = torch.ones(H, device=device)
    ids = torch.arange(T, device=device)
    rows = lambda n, dt=BF: torch.ones(n, 64, dtype=dt, device=device)  # noqa: E731
    return [
        (B.acx_attn_plan, ad, dict(offsets=offsets, plan=plan), dict(prefix=torch.ones(docs, dtype=I32, device=device))),
        (B.acx_attn_fwd, ad, dict(Q=m(H), K=m(K), V=m(K), plan=plan, O=m(H), lse=lse), dict(slopes=slopes)),
        (B.acx_attn_bwd, ad, dict(Q=m(H), K=m(K), V=m(K), plan=plan, O=m(H), dO=m(H), lse=lse, dQ=m(H), dK=m(K), dV=m(K)),
         dict(slopes=slopes, ws=room(B.acx_attn_workspace_bytes(ad, B.ACX_OP_ATTN_BWD)))),
        (B.acx_embed_fwd, ed, dict(ids=ids, E=rows(vocab), Y=rows(T)), {}),
        (B.acx_embed_bwd, ed, dict(ids=ids, dY=rows(T), dE=rows(vocab, F32)), dict(beta=0.5, ws=room(B.acx_embed_workspace_bytes(ed, B.ACX_OP_EMBED_BWD)))),
    ]


OPS = list(range(5))


@pytest.mark.parametrize("op", OPS)
def test_tensors_that_are_not_on_a_gpu_are_refused(op):
    f, desc, args, kw = calls("cpu")[op]
    with pytest.raises(ValueError, match="cpu"):
        f(desc, *args.values(), **kw)
    with pytest.raises(ValueError, match=next(iter(args))):
        f(desc, "text", *list(args.values())[1:], **kw)


@pytest.mark.parametrize("op", OPS)
def test_descriptor_of_another_operator(op):
    f, desc, args, kw = calls("cpu")[op]
    for other in (B.make_rows_desc(4, 64, "bf16"), None, 3):
        with pytest.raises(TypeError):
            f(other, *args.values(), **kw)


def test_lists_that_are_not_on_a_gpu_are_refused():
    with pytest.raises(ValueError, match="cpu"):
        B.make_grad_list([torch.ones(3)])
    with pytest.raises(ValueError):
        B.make_grad_list([])
    with pytest.raises(ValueError):
        B.make_grad_list([torch.ones(3)], weights=[1.0, 2.0])


@pytest.mark.gpu
@pytest.mark.parametrize("op", OPS)
def test_wrong_type_shape_or_order_of_each_argument(op):
    f, desc, args, kw = calls("cuda")[op]
    if op in (1, 2):
        B.acx_attn_plan(desc, calls("cuda")[0][2]["offsets"], args["plan"])
    f(desc, *args.values(), **kw)
    torch.cuda.synchronize()
    launches = B.acx_kernel_launches()
    tensors = {**args, **{k: v for k, v in kw.items() if isinstance(v, torch.Tensor) and k != "ws"}}
    for name, t in tensors.items():
        bad = [t.cpu(), t.to_sparse()]
        if name != "plan":
            bad += [t.double(), t[:-1].clone()]
            bad.append(torch.empty(2 * t.numel(), dtype=t.dtype, device="cuda")[::2] if t.dim() == 1
                       else t.transpose(-1, -2).contiguous().transpose(-1, -2))     # columns first
        for x in bad:
            if x.dtype == t.dtype and x.layout is torch.strided and x.is_cuda and x.shape == t.shape and x.is_contiguous():
                continue
            with pytest.raises(ValueError):
                f(desc, *[x if k == name else a for k, a in args.items()], **{k: x if k == name else v for k, v in kw.items()})
    if "plan" in args:
        with pytest.raises(B.AcxError) as err:
            f(desc, *[a[:64].clone() if k == "plan" else a for k, a in args.items()], **kw)
        assert err.value.status == B.ACX_ERR_WORKSPACE
    if "ws" in kw:
        for ws in (None, kw["ws"][:kw["ws"].numel() // 2]):
            with pytest.raises(B.AcxError) as err:
                f(desc, *args.values(), **dict(kw, ws=ws))
            assert err.value.status == B.ACX_ERR_WORKSPACE
        with pytest.raises(ValueError):
            f(desc, *args.values(), **dict(kw, ws=kw["ws"].cpu()))
    with pytest.raises(AttributeError):
        f(desc, *args.values(), **dict(kw, stream=3))
    assert B.acx_kernel_launches() == launches


@pytest.mark.gpu
def test_clip_arguments():
    g = torch.ones(100, device="cuda")
    lst = B.make_grad_list([g])
    total, ws = torch.zeros(2, device="cuda"), B.alloc_grad_workspace(lst)
    launches = B.acx_kernel_launches()
    for bad in (total.cpu(), total.double(), total[:1].clone(), torch.zeros(4, device="cuda")[::2]):
        with pytest.raises(ValueError):
            B.acx_grad_clip(lst, 1.0, bad, ws=ws)
    for kw in (dict(ws=None), dict(ws=ws[:16])):
        with pytest.raises(B.AcxError) as err:
            B.acx_grad_clip(lst, 1.0, total, **kw)
        assert err.value.status == B.ACX_ERR_WORKSPACE
    for bad in (0.0, -1.0, NAN):
        with pytest.raises(B.AcxError):
            B.acx_grad_clip(lst, bad, total, ws=ws)
    with pytest.raises(B.AcxError):
        B.make_grad_list([g, g])                       # the same gradient twice
    with pytest.raises(B.AcxError):
        B.make_grad_list([g[:50], g[48:]])             # two that share elements
    for bad in (g.double(), g[::2], g.to_sparse(), g.half()):
        with pytest.raises(ValueError):
            B.make_grad_list([bad])
    with pytest.raises(ValueError):
        B.make_grad_list([g], out=[torch.empty(99, device="cuda")])
    assert B.acx_kernel_launches() == launches and float(g.sum()) == 100.0
