"""RMSNorm, clipping of gradients and the cross-entropy of a linear layer without a GPU: bound, and refusing bad arguments before anything is launched (the addresses
below are never read)."""
import ctypes as C

import pytest

import paper_2405_10951_amd as P

INVALID = -1
A = 1 << 20                     # an aligned address
BIG = (1 << 30) + 1


def call(name, good, **bad):
    """`good` is an ordered dict of valid arguments; any of them replaced"""
    args = dict(good, **bad)
    return getattr(P.load_library(), name)(*args.values())


def refused(name, good, **bad):
    assert call(name, good, **bad) == INVALID
    text = P.load_library().bsr_last_error(None).decode()
    assert text.startswith(name) and len(text) > len(name) + 8


RF = dict(x=A, ldx=64, res=2 * A, ldr=64, type=0, M=4, D=64, gamma=A, eps=1e-6, sum=3 * A, lds=64, y=4 * A, ldy=64, values=None, scales=None, rstd=A, stream=None)
RB = dict(dy=A, lddy=64, x=2 * A, ldx=64, res=3 * A, ldr=64, type=1, M=4, D=64, rstd=A, gamma=A, dx=4 * A, lddx=64, dgamma=A, ws=A, ws_floats=1 << 20, stream=None)
CF = dict(x=A, ldx=64, w=2 * A, ldw=64, type=0, rows=4, width=64, classes=10, bias=None, labels=A, loss=A, stats=A, ws=A, ws_bytes=1 << 40, stream=None)
CB = dict(x=A, ldx=64, w=2 * A, ldw=64, type=0, rows=4, width=64, classes=10, bias=A, labels=A, stats=A, row_grad=None, scale=1.0, dx=3 * A, lddx=64, dw=4 * A, lddw=64, dw_type=1, db=A,
          ws=A, ws_bytes=1 << 40, stream=None)
CFB = dict(x=A, ldx=64, w=2 * A, ldw=64, type=0, rows=4, width=64, classes=10, bias=A, labels=A, loss=A, row_grad=None, scale=1.0, dx=3 * A, lddx=64, dw=4 * A, lddw=64, dw_type=1, db=A,
           ws=A, ws_bytes=1 << 40, stream=None)
CE_BAD = [dict(x=None), dict(x=A + 1), dict(ldx=63), dict(w=None), dict(ldw=9), dict(type=2), dict(rows=-1), dict(rows=(1 << 22) + 1), dict(type=1, dw_type=1, rows=(1 << 21) + 1), dict(width=0), dict(width=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21,
          lddx=1 << 21, lddw=1 << 21), dict(rows=1 << 22, width=2049, ldx=2049, ldw=2049, lddx=2049, lddw=2049), dict(classes=0), dict(classes=BIG), dict(bias=A + 2), dict(labels=None),
          dict(labels=A + 1), dict(ws=None), dict(ws=A + 128), dict(ws_bytes=100)]
CE_GRADS = [dict(row_grad=A + 1), dict(dx=None, dw=None, db=None), dict(dw_type=2), dict(type=1, dw_type=0), dict(dx=3 * A + 1), dict(lddx=5), dict(dw=4 * A + 2), dict(lddw=60), dict(db=A + 2),
            dict(dx=A), dict(dx=2 * A), dict(dw=2 * A), dict(dw=A), dict(dx=4 * A)]
CASES = [
    ("bsr_linear_ce_forward", CF, [{k: v for k, v in bad.items() if k in CF} for bad in CE_BAD] + [dict(loss=None, stats=None), dict(loss=A + 2), dict(stats=A + 4)]),
    ("bsr_linear_ce_forward_backward", CFB, CE_BAD + CE_GRADS + [dict(loss=None), dict(loss=A + 2)]),
    ("bsr_linear_ce_backward", CB, CE_BAD + CE_GRADS + [dict(stats=None), dict(stats=A + 4)]),
    ("bsr_rmsnorm_forward", RF, [dict(x=None), dict(x=A + 1), dict(ldx=63), dict(res=2 * A + 1), dict(ldr=8), dict(type=2), dict(M=-1), dict(D=0),
                                 dict(D=BIG, ldx=BIG, ldr=BIG, lds=BIG, ldy=BIG), dict(gamma=None), dict(gamma=A + 4), dict(eps=-1.0), dict(eps=float("nan")),
                                 dict(sum=3 * A + 1), dict(lds=2), dict(res=None), dict(y=None), dict(ldy=5), dict(values=A), dict(scales=A), dict(values=A + 8, scales=A), dict(rstd=A + 2),
                                 dict(sum=4 * A), dict(y=A, ldy=72), dict(sum=A, lds=72), dict(y=2 * A, ldy=72), dict(sum=2 * A, lds=80)]),
    ("bsr_rmsnorm_backward", RB, [dict(dy=None), dict(x=A + 2), dict(lddy=1), dict(ldr=8), dict(type=7), dict(M=-5), dict(D=0), dict(rstd=None), dict(rstd=A + 2), dict(gamma=None),
                                  dict(dx=None, dgamma=None), dict(ws=None), dict(ws=A + 4), dict(ws_floats=100), dict(lddx=60), dict(dgamma=A + 1),
                                  dict(dx=A, lddx=72), dict(dx=2 * A, lddx=72), dict(dx=3 * A, lddx=72), dict(D=BIG, lddy=BIG, ldx=BIG, ldr=BIG, lddx=BIG, ws_floats=1 << 50)]),
]


@pytest.mark.parametrize("name,good,bad", [(n, g, b) for n, g, bads in CASES for b in bads])
def test_refused_before_a_launch(name, good, bad):
    refused(name, good, **bad)


def test_no_rows_no_launch():
    assert call("bsr_rmsnorm_forward", RF, M=0) == 0
    assert call("bsr_rmsnorm_backward", RB, M=0, dgamma=None) == 0
    assert call("bsr_linear_ce_forward", CF, rows=0, ws=None, ws_bytes=0) == 0


def table(kind, *values):
    return (kind * len(values))(*values)


def clip_args(grads=(A, 2 * A), types=(0, 1), lengths=(10, 20), out=(3 * A, 4 * A), **more):
    good = dict(grads=table(C.c_void_p, *grads), types=table(C.c_int32, *types), lengths=table(C.c_int64, *lengths), count=len(grads), max_norm=1.0,
                out=None if out is None else table(C.c_void_p, *out), norm=A, ws=A, ws_bytes=1 << 20, stream=None)
    return dict(good, **more)


@pytest.mark.parametrize("bad", [
    dict(count=0), dict(count=-3), dict(grads=(None, A)), dict(grads=(A + 1, A)), dict(grads=(A, 2 * A + 2)), dict(types=(0, 2)), dict(lengths=(10, -1)), dict(lengths=(10, (1 << 36) + 1)),
    dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(out=(None, A)), dict(out=(3 * A, 4 * A + 2)), dict(out=None, norm=None), dict(norm=A + 2), dict(ws=None), dict(ws=A + 4),
    dict(ws_bytes=100), dict(out=(A, A)), dict(out=(A + 2, 4 * A)), dict(out=(2 * A, A)), dict(out=(3 * A, 3 * A + 16)), dict(grads=(A, A), types=(1, 1), out=(A, A)),
    dict(grads=(A, A), types=(1, 1), out=(A, 3 * A)), dict(out=(2 * A + 76, 4 * A))])
def test_clip_refused_before_a_launch(bad):
    """among them results that lie on one another or on another tensor's gradient"""
    good = clip_args(**{k: v for k, v in bad.items() if k in ("grads", "types", "lengths", "out")})
    refused("bsr_clip_grads", good, **{k: v for k, v in bad.items() if k not in ("grads", "types", "lengths", "out")})


def test_clip_without_tables():
    for name in ("grads", "types", "lengths"):
        refused("bsr_clip_grads", clip_args(), **{name: None})


def test_workspaces():
    lib = P.load_library()
    assert lib.bsr_rmsnorm_workspace_floats(0) == 0 and lib.bsr_rmsnorm_workspace_floats(768) >= 768
    assert lib.bsr_clip_workspace_bytes(0) == lib.bsr_clip_workspace_bytes(-4) == 0
    assert lib.bsr_linear_ce_workspace_bytes(0, 0, 64, 10, 0) == lib.bsr_linear_ce_workspace_bytes(2, 4, 64, 10, 0) == 0
    for kind in (0, 1):
        for rows, width, classes in ((1, 1, 1), (4096, 4096, 131072), ((1 << 22) >> kind, 64, 1 << 30), (33, 1 << 20, 100), (1, 64, 1 << 30)):
            one = [lib.bsr_linear_ce_workspace_bytes(kind, rows, width, classes, what) for what in (0, 1, 2)]
            assert min(one) > 0 and one[2] >= max(one) and lib.bsr_linear_ce_workspace_bytes(kind, rows, width, classes, 3) == 0
    assert 0 < lib.bsr_clip_workspace_bytes(1) <= lib.bsr_clip_workspace_bytes(1000)


def test_the_binding_refuses():
    import torch
    x, g = torch.zeros(4, 64), torch.zeros(64)
    with pytest.raises(ValueError, match="GPU"):
        P.bsr_rmsnorm_forward(x, g)
    with pytest.raises(ValueError, match="GPU"):
        P.bsr_clip_grads([x], 1.0)
    with pytest.raises(ValueError, match="no gradients"):
        P.bsr_grad_norm([])
