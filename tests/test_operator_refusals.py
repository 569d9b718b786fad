"""What the operators around the time-step loop refuse, on the host: no call here reaches a GPU."""
import ctypes
import math

import pytest
import torch

from paper_2412_07752_amd import api

P = ctypes.c_void_p(4096)   # an aligned address that nothing reads: every call here is refused before a launch


def _embedding(**kw):
    d = dict(tokens=4, vocab=10, width=8, table_dtype=0, io_dtype=1, index_dtype=3, scale=1.0)
    d.update(kw)
    return ctypes.byref(api.flashrnn_embedding_desc_t(*d.values()))


def _norm(**kw):
    d = dict(rows_outer=2, rows_inner=3, x_stride=24, groups=1, width=8, x_dtype=0, io_dtype=1, dx_dtype=0, param_dtype=0, eps=1e-5)
    d.update(kw)
    return ctypes.byref(api.flashrnn_layer_norm_desc_t(*d.values()))


def _loss(**kw):
    d = dict(rows=4, logits_stride=10, dlogits_stride=10, classes=10, io_dtype=0, index_dtype=3, grad_scale=1.0)
    d.update(kw)
    return ctypes.byref(api.flashrnn_cross_entropy_desc_t(*d.values()))


@pytest.mark.parametrize("bad", [dict(tokens=-1), dict(vocab=0), dict(vocab=-5), dict(width=0), dict(table_dtype=2), dict(io_dtype=-1), dict(index_dtype=0), dict(index_dtype=4)])
def test_embedding_descriptors(bad):
    L = api.lib()
    assert L.flashrnn_embedding_workspace_bytes(_embedding(**bad)) == 0
    assert L.flashrnn_embedding_fwd(_embedding(**bad), P, P, P, None) == api.FLASHRNN_ERR_SHAPE
    assert L.flashrnn_embedding_bwd(_embedding(**bad), P, P, P, 0, P, None) == api.FLASHRNN_ERR_SHAPE


def test_embedding_pointers():
    L = api.lib()
    assert L.flashrnn_embedding_fwd(None, P, P, P, None) == api.FLASHRNN_ERR_NULL
    assert L.flashrnn_embedding_bwd(None, P, P, P, 0, P, None) == api.FLASHRNN_ERR_NULL
    assert L.flashrnn_embedding_workspace_bytes(None) == 0
    for i in range(3):
        args = [None if i == k else P for k in range(3)]
        assert L.flashrnn_embedding_fwd(_embedding(), *args, None) == api.FLASHRNN_ERR_NULL
        assert L.flashrnn_embedding_bwd(_embedding(), *args, 0, P, None) == api.FLASHRNN_ERR_NULL
    for ws in (None, ctypes.c_void_p(4096 + 16)):
        assert L.flashrnn_embedding_bwd(_embedding(), P, P, P, 0, ws, None) == api.FLASHRNN_ERR_WORKSPACE
    for at, off in ((0, 2), (1, 4), (2, 1)):
        args = [ctypes.c_void_p(4096 + off) if at == k else P for k in range(3)]
        assert L.flashrnn_embedding_fwd(_embedding(), *args, None) == api.FLASHRNN_ERR_UNSUPPORTED
    assert L.flashrnn_embedding_bwd(_embedding(), P, ctypes.c_void_p(4097), P, 0, P, None) == api.FLASHRNN_ERR_UNSUPPORTED
    assert L.flashrnn_embedding_bwd(_embedding(tokens=1 << 31), P, P, P, 0, P, None) == api.FLASHRNN_ERR_UNSUPPORTED
    assert L.flashrnn_embedding_fwd(_embedding(tokens=0), None, None, None, None) == api.FLASHRNN_OK
    sizes = [api.flashrnn_embedding_workspace_bytes(n, 50000, 64) for n in (0, 1, 4096, 1 << 20)]
    assert 0 < sizes[0] <= sizes[1] < sizes[2] < sizes[3]


@pytest.mark.parametrize("bad", [dict(rows_outer=-1), dict(rows_inner=-1), dict(x_stride=-8), dict(groups=0), dict(width=0), dict(x_dtype=2), dict(io_dtype=3), dict(dx_dtype=9),
                                 dict(param_dtype=-1), dict(eps=-1e-5), dict(eps=math.nan)])
def test_layer_norm_descriptors(bad):
    L = api.lib()
    assert L.flashrnn_layer_norm_workspace_bytes(_norm(**bad)) == 0
    assert L.flashrnn_layer_norm_fwd(_norm(**bad), P, P, P, P, P, P, None) == api.FLASHRNN_ERR_SHAPE
    assert L.flashrnn_layer_norm_bwd(_norm(**bad), P, P, P, P, P, P, P, P, P, None) == api.FLASHRNN_ERR_SHAPE


def test_layer_norm_pointers():
    L = api.lib()
    assert L.flashrnn_layer_norm_fwd(None, P, P, P, P, P, P, None) == api.FLASHRNN_ERR_NULL
    assert L.flashrnn_layer_norm_bwd(None, P, P, P, P, P, P, P, P, P, None) == api.FLASHRNN_ERR_NULL
    for i in (0, 3, 4, 5):   # x, y; one of the two statistics without the other
        args = [None if i == k else P for k in range(6)]
        assert L.flashrnn_layer_norm_fwd(_norm(), *args, None) == api.FLASHRNN_ERR_NULL
    for i in (0, 1, 3, 4, 5):
        args = [None if i == k else P for k in range(9)]
        assert L.flashrnn_layer_norm_bwd(_norm(), *args, None) == api.FLASHRNN_ERR_NULL
    for ws in (None, ctypes.c_void_p(4096 + 64)):
        assert L.flashrnn_layer_norm_bwd(_norm(), P, P, P, P, P, P, P, None, ws, None) == api.FLASHRNN_ERR_WORKSPACE
    for i, off in ((0, 2), (1, 2), (2, 1), (3, 1), (4, 2), (5, 2)):
        args = [ctypes.c_void_p(4096 + off) if i == k else P for k in range(6)]
        assert L.flashrnn_layer_norm_fwd(_norm(), *args, None) == api.FLASHRNN_ERR_UNSUPPORTED, i
    for i, off in ((0, 1), (1, 2), (2, 2), (3, 2), (4, 2), (5, 2), (6, 2), (7, 1)):
        args = [ctypes.c_void_p(4096 + off) if i == k else P for k in range(8)]
        assert L.flashrnn_layer_norm_bwd(_norm(), *args, P, None) == api.FLASHRNN_ERR_UNSUPPORTED, i
    assert L.flashrnn_layer_norm_fwd(_norm(rows_outer=1 << 40, rows_inner=1 << 20), P, P, P, P, P, P, None) == api.FLASHRNN_ERR_UNSUPPORTED
    assert L.flashrnn_layer_norm_fwd(_norm(rows_inner=0), None, None, None, None, None, None, None) == api.FLASHRNN_OK


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(classes=0), dict(logits_stride=9), dict(dlogits_stride=9), dict(io_dtype=2), dict(index_dtype=1)])
def test_cross_entropy_descriptors(bad):
    assert api.lib().flashrnn_cross_entropy(_loss(**bad), P, P, P, P, P, P, None) == api.FLASHRNN_ERR_SHAPE


def test_cross_entropy_pointers():
    L = api.lib()
    assert L.flashrnn_cross_entropy(None, P, P, P, P, P, P, None) == api.FLASHRNN_ERR_NULL
    for i in (0, 1, 3):
        assert L.flashrnn_cross_entropy(_loss(), *[None if i == k else P for k in range(6)], None) == api.FLASHRNN_ERR_NULL
    for i, off in ((0, 2), (1, 4), (2, 2), (3, 1), (4, 2), (5, 1)):
        assert L.flashrnn_cross_entropy(_loss(), *[ctypes.c_void_p(4096 + off) if i == k else P for k in range(6)], None) == api.FLASHRNN_ERR_UNSUPPORTED, i
    assert L.flashrnn_cross_entropy(_loss(dlogits_stride=0, rows=0), None, None, None, None, None, None, None) == api.FLASHRNN_OK
    assert L.flashrnn_cross_entropy(_loss(rows=1 << 61, logits_stride=1 << 20), P, P, P, P, P, None, None) == api.FLASHRNN_ERR_UNSUPPORTED


def test_clip_arguments():
    L = api.lib()

    def call(count=2, grads=(4096, 8192), out=(4096, 8192), sizes=(3, 5), dtypes=(0, 1), max_norm=1.0, norm=P, ws=P):
        arr = lambda t, v: None if v is None else (t * len(v))(*v)
        return L.flashrnn_grad_clip(count, arr(ctypes.c_void_p, grads), arr(ctypes.c_void_p, out), arr(ctypes.c_longlong, sizes), arr(ctypes.c_int, dtypes), max_norm, norm, ws, None)

    assert call(count=-1) == api.FLASHRNN_ERR_SHAPE and api.lib().flashrnn_grad_clip_workspace_bytes(-1) == 0
    for bad in (-1.0, math.nan):
        assert call(max_norm=bad) == api.FLASHRNN_ERR_SHAPE
    assert call(sizes=(3, -1)) == api.FLASHRNN_ERR_SHAPE and call(dtypes=(0, 2)) == api.FLASHRNN_ERR_SHAPE
    for kw in (dict(norm=None), dict(grads=None), dict(sizes=None), dict(dtypes=None), dict(grads=(4096, 0)), dict(out=(0, 8192))):
        assert call(**kw) == api.FLASHRNN_ERR_NULL, kw
    for ws in (None, ctypes.c_void_p(4096 + 8)):
        assert call(ws=ws) == api.FLASHRNN_ERR_WORKSPACE
    for kw in (dict(grads=(4098, 8192)), dict(out=(4096, 8193)), dict(norm=ctypes.c_void_p(4098)), dict(sizes=(3, 1 << 50))):
        assert call(**kw) == api.FLASHRNN_ERR_UNSUPPORTED, kw
    assert L.flashrnn_grad_clip_workspace_bytes(0) > 0
    assert L.flashrnn_grad_clip_workspace_bytes(10_000) >= L.flashrnn_grad_clip_workspace_bytes(1)


def test_host_tensors_are_refused():
    f, t = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: api.flashrnn_embedding_fwd(f, t), lambda: api.flashrnn_embedding_bwd(t, f, 9), lambda: api.flashrnn_layer_norm_fwd(f),
                 lambda: api.flashrnn_layer_norm_bwd(f, f, t.float(), t.float()), lambda: api.flashrnn_cross_entropy(f, t), lambda: api.flashrnn_grad_clip([f], 1.0)):
        with pytest.raises(ValueError, match="device tensor"):
            call()


def test_rows_of_strided_tensors():
    """Blocks, dense rows per block and the blocks' distance, for every view that one strided axis describes; the others are refused."""
    base = torch.zeros(6, 4, 5, 8)
    assert api._rows_of(base, 1) == (1, 120, 0)
    assert api._rows_of(base[1:, 0], 1) == (5, 5, 160) and api._rows_of(base[1:, 0], 2) == (5, 1, 160)
    assert api._rows_of(base[::2], 1) == (3, 20, 320)
    assert api._rows_of(base[:, :, 2], 1) == (24, 1, 40)
    assert api._rows_of(base[2, 1, 3], 1) == (1, 1, 0)
    assert api._rows_of(base[:1, :1], 1) == (1, 5, 0)
    assert api._rows_of(torch.zeros(8).expand(7, 8), 1) == (7, 1, 0)
    assert api._rows_of(torch.zeros(3, 0, 8), 1) == (0, 0, 0)
    for bad, inner in ((base.transpose(0, 1), 1), (base[..., ::2], 1), (base.transpose(2, 3), 1), (base[:, ::2, ::2], 1), (base.transpose(2, 3), 2)):
        with pytest.raises(ValueError, match="dense"):
            api._rows_of(bad, inner)


@pytest.mark.gpu
def test_shapes_and_types_that_do_not_fit_are_refused():
    f, b, t = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 8, device="cuda", dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64, device="cuda")
    s, n8, n4 = torch.zeros(4, device="cuda"), torch.zeros(8, device="cuda"), torch.zeros(1, device="cuda")
    refused = [
        lambda: api.flashrnn_embedding_fwd(f, t, out=torch.zeros(4, 7, device="cuda")),
        lambda: api.flashrnn_embedding_fwd(f.t(), t),
        lambda: api.flashrnn_embedding_fwd(f, t.float()),
        lambda: api.flashrnn_embedding_fwd(f.double(), t),
        lambda: api.flashrnn_embedding_fwd(f, t[::2]),
        lambda: api.flashrnn_embedding_fwd(f, t.cpu()),
        lambda: api.flashrnn_embedding_bwd(t, f[:3], 9),
        lambda: api.flashrnn_embedding_bwd(t, f, 9, accumulate=True),
        lambda: api.flashrnn_embedding_bwd(t, f, 9, dtable=torch.zeros(9, 8, device="cuda", dtype=torch.bfloat16)),
        lambda: api.flashrnn_embedding_bwd(t, f, 9, workspace=torch.zeros(16, device="cuda")),
        lambda: api.flashrnn_layer_norm_fwd(f, n8[:7]),
        lambda: api.flashrnn_layer_norm_fwd(f, n8, n8.bfloat16()),
        lambda: api.flashrnn_layer_norm_fwd(f, torch.zeros(3, 8, device="cuda")),
        lambda: api.flashrnn_layer_norm_fwd(f, torch.zeros(1, 4, 8, device="cuda")),
        lambda: api.flashrnn_layer_norm_fwd(f.half()),
        lambda: api.flashrnn_layer_norm_fwd(f.t()),
        lambda: api.flashrnn_layer_norm_fwd(f, y=f[:3]),
        lambda: api.flashrnn_layer_norm_fwd(f, mean=n8),
        lambda: api.flashrnn_layer_norm_fwd(f, eps=-1.0),
        lambda: api.flashrnn_layer_norm_bwd(f[:, :7], f, s, s),
        lambda: api.flashrnn_layer_norm_bwd(f, f, s[:3], s),
        lambda: api.flashrnn_layer_norm_bwd(f, f, s, s.double()),
        lambda: api.flashrnn_layer_norm_bwd(f, f, s, s, out=(f, n8[:4], n8)),
        lambda: api.flashrnn_layer_norm_bwd(f, f, s, s, workspace=torch.zeros(1, device="cuda")),
        lambda: api.flashrnn_cross_entropy(f, t[:3]),
        lambda: api.flashrnn_cross_entropy(f, s),
        lambda: api.flashrnn_cross_entropy(f.t(), torch.zeros(8, dtype=torch.int64, device="cuda")),
        lambda: api.flashrnn_cross_entropy(f, t, dlogits=b),
        lambda: api.flashrnn_cross_entropy(f, t, dlogits=f[:1].expand(4, 8)),
        lambda: api.flashrnn_cross_entropy(f, t, dloss=n8),
        lambda: api.flashrnn_cross_entropy(f, t, loss=n8),
        lambda: api.flashrnn_grad_clip([f, f.double()], 1.0),
        lambda: api.flashrnn_grad_clip([f.t()], 1.0),
        lambda: api.flashrnn_grad_clip([f], 1.0, out=[b]),
        lambda: api.flashrnn_grad_clip([f], 1.0, out=[]),
        lambda: api.flashrnn_grad_clip([f], -1.0),
        lambda: api.flashrnn_grad_clip([], 1.0),
        lambda: api.flashrnn_grad_clip([f], 1.0, norm=n8),
        lambda: api.flashrnn_grad_clip([f], 1.0, workspace=n4),
    ]
    for i, call in enumerate(refused):
        with pytest.raises((ValueError, TypeError, api.FlashRNNError)):
            call()
            print(f"call {i} was taken", flush=True)
    torch.cuda.synchronize()
