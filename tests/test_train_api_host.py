"""Argument checks of the operators around the encoder: found on the host, before anything is launched."""
import ctypes as C
import os

import pytest
import torch

import paper_2404_00509_amd as mae
from paper_2404_00509_amd import binding as bi

FAKE = 0x10000  # never dereferenced


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(mae.LIB_PATH):
        from paper_2404_00509_amd.build import build_hip
        build_hip()
    return mae.load()


def _with(d, fields, over):
    for k, v in {**fields, **over}.items():
        setattr(d, k, v)
    return d


def _norm(**over):
    return _with(bi.MaeNormDesc(), dict(M=8, D=768, x=FAKE, weight=FAKE, bias=FAKE, eps=1e-6, x_dtype=1, y_dtype=1), over)


def _drop(**over):
    return _with(bi.MaeDropoutDesc(), dict(M=8, D=768, x=FAKE, residual=FAKE, dtype=1, p=0.1), over)


def _class(**over):
    return _with(bi.MaeClassDesc(), dict(M=8, D=768, V=1000, tokens=FAKE, weight=FAKE, bias=FAKE, labels=FAKE,
                                         smoothing=0.1, grad_scale=1.0), over)


def _embed(**over):
    return _with(bi.MaeEmbedDesc(), dict(M=8, D=768, E=768, L=196, visible=FAKE, ids_keep=FAKE, weight=FAKE, bias=FAKE,
                                         pos=FAKE, out_dtype=1), over)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("over,status", [
    (dict(x=None), bi.MAE_ERR_NULL), (dict(M=0), bi.MAE_ERR_SHAPE), (dict(M=-1), bi.MAE_ERR_SHAPE),
    (dict(D=0), bi.MAE_ERR_SHAPE), (dict(D=8193), bi.MAE_ERR_RANGE), (dict(M=(1 << 28) + 1), bi.MAE_ERR_RANGE),
    (dict(eps=-1.0), bi.MAE_ERR_RANGE), (dict(eps=NAN), bi.MAE_ERR_RANGE), (dict(eps=INF), bi.MAE_ERR_RANGE),
    (dict(x_dtype=2), bi.MAE_ERR_DTYPE), (dict(y_dtype=-1), bi.MAE_ERR_DTYPE), (dict(x=FAKE + 1), bi.MAE_ERR_RANGE),
    (dict(x=FAKE + 2, x_dtype=0), bi.MAE_ERR_RANGE), (dict(weight=FAKE + 2), bi.MAE_ERR_RANGE),
    (dict(bias=FAKE + 3), bi.MAE_ERR_RANGE)])
def test_layer_norm_rejects_bad_descriptors(lib, over, status):
    d = _norm(**over)
    assert lib.mae_layer_norm(C.byref(d), FAKE, FAKE, FAKE, None) == status
    assert lib.mae_layer_norm_grad(C.byref(d), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 30, None) == status
    assert lib.mae_layer_norm_workspace_bytes(C.byref(d)) == 0


def test_layer_norm_rejects_bad_arguments(lib):
    d = _norm()
    ref = C.byref(d)
    need = lib.mae_layer_norm_workspace_bytes(ref)
    assert need > 0
    assert lib.mae_layer_norm(ref, None, None, None, None) == bi.MAE_ERR_NULL
    assert lib.mae_layer_norm(None, FAKE, None, None, None) == bi.MAE_ERR_NULL
    assert lib.mae_layer_norm(ref, FAKE + 1, None, None, None) == bi.MAE_ERR_RANGE
    assert lib.mae_layer_norm(ref, FAKE, FAKE + 2, None, None) == bi.MAE_ERR_RANGE
    grad = lambda *a, ws=FAKE, n=need: lib.mae_layer_norm_grad(ref, *a, ws, n, None)  # noqa: E731
    assert grad(None, FAKE, FAKE, FAKE, FAKE, FAKE) == bi.MAE_ERR_NULL
    assert grad(FAKE, None, FAKE, FAKE, FAKE, FAKE) == bi.MAE_ERR_NULL
    assert grad(FAKE, FAKE, None, FAKE, FAKE, FAKE) == bi.MAE_ERR_NULL
    assert grad(FAKE, FAKE, FAKE, None, None, None) == bi.MAE_ERR_NULL
    assert grad(FAKE, FAKE, FAKE, FAKE + 1, None, None) == bi.MAE_ERR_RANGE
    assert grad(FAKE, FAKE, FAKE, None, FAKE, None, n=need - 1) == bi.MAE_ERR_WORKSPACE
    assert grad(FAKE, FAKE, FAKE, None, None, FAKE, ws=None) == bi.MAE_ERR_WORKSPACE
    assert grad(FAKE, FAKE, FAKE, None, FAKE, None, ws=FAKE + 128) == bi.MAE_ERR_WORKSPACE


@pytest.mark.parametrize("over,status", [
    (dict(x=None), bi.MAE_ERR_NULL), (dict(M=0), bi.MAE_ERR_SHAPE), (dict(D=-4), bi.MAE_ERR_SHAPE),
    (dict(M=(1 << 28) + 1), bi.MAE_ERR_RANGE), (dict(D=8193), bi.MAE_ERR_RANGE), (dict(dtype=3), bi.MAE_ERR_DTYPE),
    (dict(p=-0.1), bi.MAE_ERR_RANGE), (dict(p=1.1), bi.MAE_ERR_RANGE), (dict(p=NAN), bi.MAE_ERR_RANGE),
    (dict(rows_per_draw=-1), bi.MAE_ERR_RANGE), (dict(row_base=(1 << 48) + 1), bi.MAE_ERR_RANGE),
    (dict(x=FAKE + 1), bi.MAE_ERR_RANGE), (dict(x=FAKE + 2, dtype=0), bi.MAE_ERR_RANGE),
    (dict(residual=FAKE + 1), bi.MAE_ERR_RANGE)])
def test_dropout_rejects_bad_descriptors(lib, over, status):
    assert lib.mae_dropout(C.byref(_drop(**over)), FAKE, None) == status


def test_dropout_rejects_bad_outputs(lib):
    assert lib.mae_dropout(C.byref(_drop()), None, None) == bi.MAE_ERR_NULL
    assert lib.mae_dropout(C.byref(_drop()), FAKE + 1, None) == bi.MAE_ERR_RANGE
    assert lib.mae_dropout(None, FAKE, None) == bi.MAE_ERR_NULL


@pytest.mark.parametrize("over,status", [
    (dict(tokens=None), bi.MAE_ERR_NULL), (dict(weight=None), bi.MAE_ERR_NULL), (dict(labels=None), bi.MAE_ERR_NULL),
    (dict(M=0), bi.MAE_ERR_SHAPE), (dict(D=0), bi.MAE_ERR_SHAPE), (dict(V=0), bi.MAE_ERR_SHAPE),
    (dict(D=772), bi.MAE_ERR_SHAPE), (dict(D=8200), bi.MAE_ERR_RANGE), (dict(M=(1 << 24) + 1), bi.MAE_ERR_RANGE),
    (dict(V=(1 << 20) + 1), bi.MAE_ERR_RANGE), (dict(M=1 << 24, V=1 << 20), bi.MAE_ERR_RANGE),
    (dict(smoothing=-0.1), bi.MAE_ERR_RANGE), (dict(smoothing=1.5), bi.MAE_ERR_RANGE),
    (dict(smoothing=NAN), bi.MAE_ERR_RANGE), (dict(grad_scale=NAN), bi.MAE_ERR_RANGE),
    (dict(grad_scale=INF), bi.MAE_ERR_RANGE), (dict(tokens=FAKE + 8), bi.MAE_ERR_RANGE),
    (dict(weight=FAKE + 8), bi.MAE_ERR_RANGE), (dict(bias=FAKE + 2), bi.MAE_ERR_RANGE),
    (dict(labels=FAKE + 2), bi.MAE_ERR_RANGE)])
def test_class_loss_rejects_bad_descriptors(lib, over, status):
    d = _class(**over)
    assert lib.mae_class_loss(C.byref(d), FAKE, FAKE, FAKE, FAKE, None, FAKE, 1 << 60, None) == status
    for grad in (0, 1):
        assert lib.mae_class_loss_workspace_bytes(C.byref(d), grad) == 0


def test_class_loss_rejects_bad_arguments(lib):
    d = _class()
    ref = C.byref(d)
    small, large = (lib.mae_class_loss_workspace_bytes(ref, g) for g in (0, 1))
    assert 0 < small < large
    call = lambda *a, n=large, ws=FAKE: lib.mae_class_loss(ref, *a, ws, n, None)  # noqa: E731
    assert call(None, FAKE, FAKE, FAKE, FAKE) == bi.MAE_ERR_NULL
    assert lib.mae_class_loss(None, FAKE, None, None, None, None, FAKE, large, None) == bi.MAE_ERR_NULL
    assert call(FAKE, None, FAKE + 8, None, None) == bi.MAE_ERR_RANGE
    assert call(FAKE, None, None, FAKE + 8, None) == bi.MAE_ERR_RANGE
    assert call(FAKE, None, None, None, FAKE + 2) == bi.MAE_ERR_RANGE
    assert call(FAKE, None, FAKE, None, None, n=large - 1) == bi.MAE_ERR_WORKSPACE
    assert call(FAKE, None, None, None, None, n=small - 1) == bi.MAE_ERR_WORKSPACE
    assert call(FAKE, None, None, None, None, ws=None) == bi.MAE_ERR_WORKSPACE
    assert call(FAKE, None, None, None, None, ws=FAKE + 64) == bi.MAE_ERR_WORKSPACE
    d.bias = None
    assert call(FAKE, None, None, None, FAKE) == bi.MAE_ERR_NULL


def test_class_loss_workspace_stays_far_below_the_logits(lib):
    d = _class(M=1 << 20, D=768, V=1 << 17, bias=None)
    logits = 4 * (1 << 20) * (1 << 17)
    assert lib.mae_class_loss_workspace_bytes(C.byref(d), 1) < logits / 16


@pytest.mark.parametrize("over,status", [
    (dict(visible=None), bi.MAE_ERR_NULL), (dict(weight=None), bi.MAE_ERR_NULL), (dict(ids_keep=None), bi.MAE_ERR_NULL),
    (dict(M=0), bi.MAE_ERR_SHAPE), (dict(D=770), bi.MAE_ERR_SHAPE), (dict(E=0), bi.MAE_ERR_SHAPE),
    (dict(E=8193), bi.MAE_ERR_RANGE), (dict(L=8193), bi.MAE_ERR_RANGE), (dict(out_dtype=0), bi.MAE_ERR_DTYPE),
    (dict(visible=FAKE + 8), bi.MAE_ERR_RANGE)])
def test_embed_grad_rejects_bad_descriptors(lib, over, status):
    d = _embed(**over)
    assert lib.mae_patch_embed_grad(C.byref(d), FAKE, FAKE, FAKE, None, FAKE, 1 << 60, None) == status
    assert lib.mae_patch_embed_grad_workspace_bytes(C.byref(d)) == 0


def test_embed_grad_rejects_bad_arguments(lib):
    d = _embed()
    ref = C.byref(d)
    need = lib.mae_patch_embed_grad_workspace_bytes(ref)
    call = lambda *a, n=need, ws=FAKE: lib.mae_patch_embed_grad(ref, *a, ws, n, None)  # noqa: E731
    assert call(None, FAKE, FAKE, FAKE) == bi.MAE_ERR_NULL
    assert call(FAKE, None, None, None) == bi.MAE_ERR_NULL
    assert call(FAKE + 8, FAKE, None, None) == bi.MAE_ERR_RANGE
    assert call(FAKE, FAKE + 4, None, None) == bi.MAE_ERR_RANGE
    assert call(FAKE, FAKE, None, None, n=need - 1) == bi.MAE_ERR_WORKSPACE
    assert call(FAKE, FAKE, None, None, ws=FAKE + 8) == bi.MAE_ERR_WORKSPACE
    d.pos = None
    assert call(FAKE, FAKE, None, FAKE) == bi.MAE_ERR_NULL


def test_binding_refuses_tensors_it_cannot_pass_on():
    host = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        mae.make_norm_desc(host)
    with pytest.raises(ValueError):
        mae.make_dropout_desc(host, p=0.1)
    with pytest.raises(ValueError):
        mae.make_class_desc(host.to(torch.bfloat16), torch.zeros(4, dtype=torch.int32), host.to(torch.bfloat16))
    with pytest.raises(TypeError):
        mae.make_norm_desc(None)


def test_binding_refuses_another_device(monkeypatch):
    class Elsewhere:
        device = torch.device("cuda", 1)

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="cuda:1"):
        bi._one_device(Elsewhere())
    with pytest.raises(ValueError, match="stream"):
        bi._one_device(stream=Elsewhere())
    here = Elsewhere()
    here.device = torch.device("cuda", 0)
    bi._one_device(here, None, stream=here)


def test_binding_refuses_counts_that_a_field_would_cut_off(monkeypatch):
    monkeypatch.setattr(bi, "_check", lambda *a, **k: None)
    wide = torch.empty(1, (1 << 32) + 8, dtype=torch.bfloat16, device="meta")  # the low 32 bits say 8
    tall = torch.empty((1 << 32) + 8, 8, dtype=torch.bfloat16, device="meta")
    labels = torch.empty(1, dtype=torch.int32, device="meta")
    rows = torch.empty(4, 8, dtype=torch.bfloat16, device="meta")
    with pytest.raises(ValueError, match="D = 4294967304"):
        mae.make_norm_desc(wide)
    with pytest.raises(ValueError, match="D = 4294967304"):
        mae.make_dropout_desc(wide, p=0.1)
    with pytest.raises(ValueError, match="D = 4294967304"):
        mae.make_class_desc(wide, labels, wide)
    with pytest.raises(ValueError, match="V = 4294967304"):
        mae.make_class_desc(rows, labels, tall)
    for over in (dict(rows_per_draw=1 << 32), dict(rows_per_draw=-1), dict(layer=1 << 32), dict(layer=-1),
                 dict(row_base=-1), dict(row_base=1 << 64)):
        with pytest.raises(ValueError, match=next(iter(over))):
            mae.make_dropout_desc(rows, p=0.1, **over)
    d = mae.make_dropout_desc(rows, p=0.1, rows_per_draw=(1 << 31) - 1, layer=(1 << 32) - 1, row_base=1 << 48)
    assert (d.rows_per_draw, d.layer, d.row_base) == ((1 << 31) - 1, (1 << 32) - 1, 1 << 48)
