"""Refusals and sizes of the full-rank operators that need no GPU: every one returns before anything is enqueued."""
import ctypes as C

import pytest

from paper_2602_04396_amd import lordo


@pytest.fixture(scope="module")
def lib():
    return lordo.load()


def _tensors(*shapes):
    arr = (lordo.Tensor * len(shapes))()
    for a, sh in zip(arr, shapes):
        a.rows, a.cols, a.decay, a.reserved = (tuple(sh) + (1, 0))[:4] if len(sh) < 4 else sh
    return arr


def _bytes(lib, shapes, hp):
    size = C.c_size_t(0)
    return lib.lordo_adamw_workspace_bytes(_tensors(*shapes), len(shapes), C.byref(hp), C.byref(size)), size.value


def test_struct_layout():
    assert C.sizeof(lordo.Tensor) == 24 and C.sizeof(lordo.Grad) == 48 and C.sizeof(lordo.AdamWHParams) == 48
    assert lordo.Grad.slots.offset == 32 and lordo.Grad.dtype.offset == 40


def test_workspace_holds_the_moments(lib):
    shapes = [(1000, 513), (1, 7), (1, 129)]
    padded = sum((p * q + 127) // 128 * 128 for p, q in shapes)
    rc, full = _bytes(lib, shapes, lordo.adamw_hparams())
    assert rc == lordo.OK and 8 * padded <= full <= 8 * padded + 4096
    rc, small = _bytes(lib, shapes, lordo.adamw_hparams(state_dtype=lordo.Q8))
    assert rc == lordo.OK and 2 * padded + padded // 64 <= small <= 2 * padded + padded // 64 + 4096


@pytest.mark.parametrize("shapes", [[(0, 4)], [(4, 0)], [(-1, 4)], [(1 << 20, (1 << 18) + 1)], [(1 << 39, 1)], [(1 << 18, 1 << 18)], [(1 << 17, 1 << 18), (1 << 17, 1 << 18)], [(4, 4, 2, 0)], [(4, 4, 1, 1)]])
def test_bad_shapes(lib, shapes):
    assert _bytes(lib, shapes, lordo.adamw_hparams())[0] == lordo.EINVAL


@pytest.mark.parametrize("bad", [dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=-1e-8), dict(eps=1e-31), dict(eps=float("inf")),
                                 dict(weight_decay=-0.1), dict(weight_decay=float("nan")), dict(param_dtype=2), dict(state_dtype=1), dict(state_dtype=3)])
def test_bad_hyper_parameters(lib, bad):
    assert _bytes(lib, [(4, 4)], lordo.adamw_hparams(**bad))[0] == lordo.EINVAL


def test_null_contexts(lib):
    hp, size, t = lordo.adamw_hparams(), C.c_size_t(0), C.c_int64(0)
    p = C.c_void_p()
    one = _tensors((4, 4))
    assert lib.lordo_adamw_workspace_bytes(None, 1, C.byref(hp), C.byref(size)) == lordo.EINVAL
    assert lib.lordo_adamw_workspace_bytes(one, 0, C.byref(hp), C.byref(size)) == lordo.EINVAL
    assert lib.lordo_adamw_workspace_bytes(one, 1, None, C.byref(size)) == lordo.EINVAL
    assert lib.lordo_adamw_workspace_bytes(one, 1, C.byref(hp), None) == lordo.EINVAL
    assert lib.lordo_adamw_init(None, one, 1, C.byref(hp), C.c_void_p(256), 1 << 20, None) == lordo.EINVAL
    assert lib.lordo_adamw_init(C.byref(p), one, 1, C.byref(hp), None, 1 << 20, None) == lordo.EINVAL
    assert lib.lordo_adamw_init(C.byref(p), one, 1, C.byref(hp), C.c_void_p(128), 1 << 20, None) == lordo.EINVAL
    assert lib.lordo_adamw_init(C.byref(p), one, 1, C.byref(hp), C.c_void_p(256), 64, None) == lordo.ENOMEM and not p.value
    assert lib.lordo_adamw_step(None, None, None, 1e-3, 1.0, None, None) == lordo.EINVAL
    assert lib.lordo_adamw_sync_payload(None, C.byref(p), C.byref(size)) == lordo.EINVAL
    assert lib.lordo_adamw_export_moments(None, None, None) == lordo.EINVAL
    assert lib.lordo_adamw_import_moments(None, None, None) == lordo.EINVAL
    assert lib.lordo_adamw_get_step(None, C.byref(t)) == lordo.EINVAL
    assert lib.lordo_adamw_set_step(None, 1) == lordo.EINVAL
    assert lib.lordo_adamw_poll_status(None, None) == lordo.EINVAL
    lib.lordo_adamw_destroy(None)


def _grad(data=4096, index=None, rows=4, cols=4, slots=0, dtype=lordo.F32, reserved=0):
    arr = (lordo.Grad * 1)()
    arr[0].data, arr[0].index, arr[0].rows, arr[0].cols = data, index, rows, cols
    arr[0].slots, arr[0].dtype, arr[0].reserved = slots, dtype, reserved
    return arr


@pytest.mark.parametrize("bad", [dict(data=None), dict(data=4097), dict(data=4098), dict(data=4097, dtype=lordo.BF16), dict(rows=0), dict(cols=0),
                                 dict(rows=1 << 30, cols=1 << 9), dict(dtype=lordo.Q8), dict(reserved=1), dict(slots=1), dict(index=4097, slots=1),
                                 dict(index=4096, slots=-1), dict(index=4096, slots=lordo.MAX_TOKENS + 1), dict(index=4096, rows=(1 << 22) + 1),
                                 dict(index=4096, data=None, slots=1)])
def test_bad_gradients(lib, bad):
    ws, out = C.c_void_p(1 << 20), C.c_void_p(4096)
    assert lib.lordo_grad_norm(_grad(**bad), 1, 1.0, out, ws, lordo.NORM_WORKSPACE_BYTES, None) == lordo.EINVAL


def test_bad_norm_arguments(lib):
    g, ws, out, n = _grad(), C.c_void_p(1 << 20), C.c_void_p(4096), lordo.NORM_WORKSPACE_BYTES
    assert lib.lordo_grad_norm(None, 1, 1.0, out, ws, n, None) == lordo.EINVAL
    assert lib.lordo_grad_norm(g, 0, 1.0, out, ws, n, None) == lordo.EINVAL
    for bad in (0.0, -1.0, float("nan")):
        assert lib.lordo_grad_norm(g, 1, bad, out, ws, n, None) == lordo.EINVAL
    assert lib.lordo_grad_norm(g, 1, 1.0, None, ws, n, None) == lordo.EINVAL
    assert lib.lordo_grad_norm(g, 1, 1.0, C.c_void_p(4098), ws, n, None) == lordo.EINVAL
    assert lib.lordo_grad_norm(g, 1, 1.0, out, None, n, None) == lordo.EINVAL
    assert lib.lordo_grad_norm(g, 1, 1.0, out, C.c_void_p(128), n, None) == lordo.EINVAL
    assert lib.lordo_grad_norm(g, 1, 1.0, out, ws, n - 1, None) == lordo.ENOMEM


GOOD = dict(ids=4096, ids_dtype=lordo.I64, tokens=8, dy=4096, dy_dtype=lordo.F32, vocab=10, cols=6, scale=1.0)
BAD = [dict(ids=None), dict(ids=4100), dict(ids_dtype=lordo.F32), dict(tokens=-1), dict(tokens=lordo.MAX_TOKENS + 1), dict(dy=None), dict(dy=4098),
       dict(dy_dtype=lordo.Q8), dict(vocab=0), dict(vocab=lordo.MAX_VOCAB + 1), dict(cols=0), dict(cols=(1 << 20) + 1), dict(scale=float("inf")),
       dict(scale=float("nan"))]


@pytest.mark.parametrize("bad", BAD + [dict(out=None), dict(out=4098), dict(out_dtype=5)])
def test_bad_lookups(lib, bad):
    a = {**GOOD, "out": 8192, "out_dtype": lordo.F32, **bad}
    assert lib.lordo_embed_lookup(a["dy"], a["dy_dtype"], a["vocab"], a["cols"], a["ids"], a["ids_dtype"], a["tokens"], a["scale"], a["out"],
                                  a["out_dtype"], None) == lordo.EINVAL


BAD_OUT = BAD + [dict(out=None), dict(out=4098), dict(out_dtype=5), dict(ws=None), dict(ws=128)]


@pytest.mark.parametrize("rows, bad", [(False, b) for b in BAD_OUT + [dict(accumulate=2)]] + [(True, b) for b in BAD_OUT + [dict(index=None), dict(index=4098)]])
def test_bad_embedding_gradients(lib, rows, bad):
    a = {**GOOD, "out": 8192, "out_dtype": lordo.F32, "ws": 1 << 20, "accumulate": 0, "index": 4096, **bad}
    head = (a["ids"], a["ids_dtype"], a["tokens"], a["dy"], a["dy_dtype"], a["vocab"], a["cols"], a["scale"], -1)
    if rows:
        rc = lib.lordo_embed_gradient_rows(*head, a["out"], a["out_dtype"], a["index"], a["ws"], 1 << 20, None)
    else:
        rc = lib.lordo_embed_gradient(*head, a["accumulate"], a["out"], a["out_dtype"], a["ws"], 1 << 20, None)
    assert rc == lordo.EINVAL


@pytest.mark.parametrize("scale", [1e39, -1e39, 3.5e38])
def test_a_scale_beyond_fp32(lib, scale):
    """Infinite in fp32, where it would make the zero rows of padding NaN."""
    ws = C.c_void_p(1 << 20)
    assert lib.lordo_embed_lookup(4096, lordo.F32, 10, 6, 4096, lordo.I64, 8, scale, 8192, lordo.F32, None) == lordo.EINVAL
    assert lib.lordo_embed_gradient(4096, lordo.I64, 8, 4096, lordo.F32, 10, 6, scale, -1, 0, 8192, lordo.F32, ws, 1 << 20, None) == lordo.EINVAL
    assert lib.lordo_embed_gradient_rows(4096, lordo.I64, 8, 4096, lordo.F32, 10, 6, scale, -1, 8192, lordo.F32, 4096, ws, 1 << 20, None) == lordo.EINVAL


def test_embedding_workspace(lib):
    size = C.c_size_t(0)
    assert lib.lordo_embed_workspace_bytes(8, 10, 6, C.byref(size)) == lordo.OK and size.value > 0
    a = GOOD
    for call, more in ((lib.lordo_embed_gradient, (0, 8192, lordo.F32)), (lib.lordo_embed_gradient_rows, (8192, lordo.F32, 4096))):
        assert call(a["ids"], a["ids_dtype"], 8, a["dy"], a["dy_dtype"], 10, 6, 1.0, -1, *more, 1 << 20, size.value - 1, None) == lordo.ENOMEM
    for bad in ((-1, 10, 6), (lordo.MAX_TOKENS + 1, 10, 6), (8, 0, 6), (8, 10, 0), (8, lordo.MAX_VOCAB + 1, 6)):
        assert lib.lordo_embed_workspace_bytes(*bad, C.byref(size)) == lordo.EINVAL
    assert lib.lordo_embed_workspace_bytes(8, 10, 6, None) == lordo.EINVAL
    # no tokens, nothing to do
    assert lib.lordo_embed_lookup(None, lordo.F32, 10, 6, None, lordo.I64, 0, 1.0, None, lordo.F32, None) == lordo.OK


def test_without_a_gpu(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    p, ctx = C.c_void_p(1 << 20), C.c_void_p()
    assert lib.lordo_adamw_init(C.byref(ctx), _tensors((4, 4)), 1, C.byref(lordo.adamw_hparams()), p, 1 << 20, None) == lordo.EHIP and not ctx.value
    assert lib.lordo_grad_norm(_grad(), 1, 1.0, 4096, p, lordo.NORM_WORKSPACE_BYTES, None) == lordo.EHIP
    assert lib.lordo_embed_lookup(4096, lordo.F32, 10, 6, 4096, lordo.I64, 8, 1.0, 8192, lordo.F32, None) == lordo.EHIP
    assert lib.lordo_embed_gradient(4096, lordo.I64, 8, 4096, lordo.F32, 10, 6, 1.0, -1, 0, 8192, lordo.F32, p, 1 << 20, None) == lordo.EHIP


def test_binding_refuses_host_tensors():
    import torch
    with pytest.raises(ValueError):
        lordo.grad_list([torch.zeros(4)])
    with pytest.raises(ValueError):
        lordo.grad_list([])
    with pytest.raises(ValueError):
        lordo.grad_list([torch.zeros(4, 4).t()[1:]])
    with pytest.raises(ValueError):
        lordo.embed_lookup(torch.zeros(4, 4), torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        lordo.RowGrad(torch.zeros(2, 4), torch.zeros(5, dtype=torch.int32), 4)
