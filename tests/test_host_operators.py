"""What the loss head without logits and the rows kept in 8 bits refuse.  No GPU: every refusal comes before the first launch."""
from __future__ import annotations

import ctypes as C

import pytest
import torch

import paper_2308_10087_amd as g
from paper_2308_10087_amd.binding import lib

BUF = (C.c_char * 8192)()
AT = (C.addressof(BUF) + 255) // 256 * 256  # a 256-byte aligned address that is never read


def _head(h=AT, ld_h=64, W=AT, dtype=1, bias=None, labels=AT, mask=None, rows=10, d=64, n_classes=5, row_loss=AT, dh=None, ld_dh=64, dW=None,
          db=None, ws=AT, size=1 << 40):
    return lib.gnntrain_head_xent(h, ld_h, W, dtype, bias, labels, mask, rows, d, n_classes, 1.0, row_loss, dh, ld_dh, dW, db, ws, size, None)


@pytest.mark.parametrize("bad,code", [(dict(rows=-1), -1), (dict(rows=1 << 41), -1), (dict(d=0), -1), (dict(d=65537), -1), (dict(n_classes=0), -1),
                                      (dict(n_classes=(1 << 24) + 1), -1), (dict(dtype=2), -1), (dict(dtype=-1), -1), (dict(ld_h=63), -1),
                                      (dict(dh=AT, ld_dh=63), -1), (dict(h=None), -1), (dict(W=None), -1), (dict(labels=None), -1),
                                      (dict(row_loss=None), -1), (dict(ws=None), -1), (dict(ws=AT + 16), -1), (dict(size=0), -4),
                                      (dict(dW=AT, size=1000), -4), (dict(dh=AT), -1), (dict(d=65535), -1),
                                      (dict(d=1024, ld_h=1024, n_classes=1 << 24), -1)])
def test_head_refuses(bad, code):
    assert _head(**bad) == code
    assert "gnntrain_head_xent" in lib.gnntrain_last_error(None).decode()


def test_head_of_no_rows_is_nothing_to_do():
    assert _head(rows=0, h=None, W=None, labels=None, row_loss=None, ws=None, size=0) == 0


def test_head_workspace_sizes():
    size = lambda *a: lib.gnntrain_head_xent_workspace_size(*a)
    for bad in ((-1, 64, 5, 1, 1), (10, 0, 5, 1, 1), (10, 64, 0, 1, 1), (10, 64, 5, 7, 1)):
        assert size(*bad) == 0
    with pytest.raises(g.GnnStageError):
        g.gnntrain_head_xent_workspace_size(10, 0, 5, g.GNNSTAGE_F32)
    assert size(10, 64, 5, 1, 0) <= size(10, 64, 5, 1, 1)
    # no room for the logits of all rows and classes (fp32: 4e11 bytes here), nor for the rows themselves twice over
    assert size(1000000, 256, 100000, 1, 1) < 4e9
    assert size(1000000, 256, 100000, 0, 1) < 4e9


def _store(x=AT, dtype=1, ld_x=100, rows=10, d=100, q=AT, ld_q=128, scale=AT, ld_s=4):
    return lib.gnnstage_rows8_store(x, dtype, ld_x, rows, d, q, ld_q, scale, ld_s, None)


def _load(q=AT, ld_q=128, scale=AT, ld_s=4, rows=10, d=100, x=AT, dtype=1, ld_x=100):
    return lib.gnnstage_rows8_load(q, ld_q, scale, ld_s, rows, d, x, dtype, ld_x, None)


def _grad(q=AT, ld_q=128, scale=AT, ld_s=4, dY=AT, dtype=1, ld_dy=64, rows=10, d=100, d_out=64, dW=AT, dbias=None, ws=AT, size=1 << 40):
    return lib.gnnstage_rows8_weight_grad(q, ld_q, scale, ld_s, dY, dtype, ld_dy, rows, d, d_out, dW, dbias, ws, size, None)


SHARED = [dict(dtype=2), dict(rows=-1), dict(rows=1 << 41), dict(d=0), dict(q=None), dict(q=AT + 8), dict(ld_q=120), dict(ld_q=96), dict(scale=None),
          dict(ld_s=3)]


@pytest.mark.parametrize("bad", SHARED + [dict(x=None), dict(ld_x=99)])
def test_store_and_load_refuse(bad):
    for call in (_store, _load):
        assert call(**bad) == -1
        assert "gnnstage_rows8" in lib.gnnstage_last_error(None).decode()


@pytest.mark.parametrize("bad,code", [(b, -1) for b in SHARED] + [(dict(dY=None), -1), (dict(dW=None), -1), (dict(d_out=0), -1), (dict(ld_dy=63), -1),
                                                                  (dict(ld_dy=1 << 31), -1), (dict(ws=None), -1), (dict(ws=AT + 1), -1), (dict(size=64), -4)])
def test_weight_gradient_refuses(bad, code):
    assert _grad(**bad) == code
    assert "gnnstage_rows8_weight_grad" in lib.gnnstage_last_error(None).decode()


def test_no_rows_are_nothing_to_do():
    assert _store(rows=0, x=None, q=None, scale=None) == 0
    assert _load(rows=0, x=None, q=None, scale=None) == 0
    assert _grad(rows=0, dY=None, dW=None, q=None, scale=None, ws=None, size=0) == 0


def test_tensors_are_checked_before_anything_else():
    f = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t)
    h, W, y, loss, ws = f(6, 8), f(8, 3), f(6, t=torch.int32), f(6), f(64, t=torch.uint8)
    calls = [
        lambda: g.gnntrain_head_xent(h, W, None, y, None, 1.0, loss, ws),                              # on the CPU
        lambda: g.gnntrain_head_xent(h.double(), W, None, y, None, 1.0, loss, ws),
        lambda: g.gnntrain_head_xent(h, W.bfloat16(), None, y, None, 1.0, loss, ws),
        lambda: g.gnntrain_head_xent(h, W[:7], None, y, None, 1.0, loss, ws),
        lambda: g.gnntrain_head_xent(h, f(3, 8).t(), None, y, None, 1.0, loss, ws),
        lambda: g.gnntrain_head_xent(f(8, 6).t(), W, None, y, None, 1.0, loss, ws),
        lambda: g.gnntrain_head_xent(f(1, 8).expand(6, 8), W, None, y, None, 1.0, loss, ws),
        lambda: g.gnntrain_head_xent(h, W, f(4), y, None, 1.0, loss, ws),
        lambda: g.gnntrain_head_xent(h, W, None, y.long(), None, 1.0, loss, ws),
        lambda: g.gnntrain_head_xent(h, W, None, y, f(6, t=torch.bool), 1.0, loss, ws),
        lambda: g.gnntrain_head_xent(h, W, None, y, None, 1.0, loss[:5], ws),
        lambda: g.gnntrain_head_xent(h, W, None, y, None, 1.0, loss, ws.float()),
        lambda: g.gnntrain_head_xent(h, W, None, y, None, 1.0, loss, ws, dh=f(6, 8, t=torch.bfloat16)),
        lambda: g.gnntrain_head_xent(h, W, None, y, None, 1.0, loss, ws, dW=f(3, 8)),
        lambda: g.gnntrain_head_xent(h, W, None, y, None, 1.0, loss, ws, db=f(3, t=torch.bfloat16)),
        lambda: g.gnnstage_rows8_store(h, f(6, 32, t=torch.int8), f(6, 1, t=torch.uint8)),             # on the CPU
        lambda: g.gnnstage_rows8_store(h, f(6, 64, t=torch.int8), f(6, 2, t=torch.uint8)),
        lambda: g.gnnstage_rows8_store(h, f(6, 32, t=torch.int8), f(6, 2, t=torch.uint8)),
        lambda: g.gnnstage_rows8_store(h, f(6, 32, t=torch.uint8), f(6, 1, t=torch.uint8)),
        lambda: g.gnnstage_rows8_load(f(6, 32, t=torch.int8), f(6, 1, t=torch.uint8), h.half()),
        lambda: g.gnnstage_rows8_weight_grad(f(6, 32, t=torch.int8), f(6, 1, t=torch.uint8), f(6, 4), f(33, 4), ws),
        lambda: g.gnnstage_rows8_weight_grad(f(6, 32, t=torch.int8), f(6, 1, t=torch.uint8), f(5, 4), f(8, 4), ws),
        lambda: g.gnnstage_rows8_weight_grad(f(6, 32, t=torch.int8), f(6, 1, t=torch.uint8), f(6, 4), f(8, 4), ws, dbias=f(5)),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(g.GnnStageError) as e:
            call()
        assert e.value.code == -1, i


def test_refusals_of_threads_keep_apart():
    """A message is the calling thread's: another one's refusal neither replaces nor frees it."""
    import threading
    assert _head(d=0) == -1 and _store(ld_x=99) == -1
    mine = lib.gnntrain_last_error(None), lib.gnnstage_last_error(None)
    others = []

    def refused():
        before = lib.gnntrain_last_error(None), lib.gnnstage_last_error(None)
        assert _head(ld_h=63) == -1 and _store(rows=-1) == -1
        others.append((before, (lib.gnntrain_last_error(None), lib.gnnstage_last_error(None))))

    t = threading.Thread(target=refused)
    t.start()
    t.join()
    assert (lib.gnntrain_last_error(None), lib.gnnstage_last_error(None)) == mine
    (before, after), = others
    assert before == (b"", b"") and b"leading dimension" in after[0] and b"rows" in after[1]
