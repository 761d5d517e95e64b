"""The operators on a caller's own tensors without a GPU: exported, bound, and refusing bad arguments before anything is launched (the
addresses below are never read)."""
import copy
import ctypes as C
import pickle

import pytest

import paper_2405_10951_amd as P
from reference8 import blocks8, exponent, to_e4m3

INVALID = -1
A = 1 << 20                     # an aligned address


def test_bound_under_their_c_names():
    for n in ("bsr_layernorm_forward", "bsr_layernorm_forward8", "bsr_layernorm_backward", "bsr_quantize8_rows", "bsr_quantize8_weight",
              "bsr_linear8_forward", "bsr_linear8_dgrad", "bsr_distill_forward", "bsr_distill_forward_backward", "bsr_distill_backward"):
        assert hasattr(P, n)


@pytest.mark.parametrize("k,ldv,lds", [(0, 0, 0), (1, 128, 4), (128, 128, 4), (129, 256, 4), (512, 512, 4), (513, 640, 8), (768, 768, 8)])
def test_strides_of_8_bit_rows(k, ldv, lds):
    v, s = C.c_int64(-1), C.c_int64(-1)
    P.load_library().bsr_block8_strides(k, C.byref(v), C.byref(s))
    assert (v.value, s.value) == (ldv, lds)


def test_workspaces():
    lib = P.load_library()
    assert lib.bsr_layernorm_workspace_floats(0) == 0 and lib.bsr_layernorm_workspace_floats(768) >= 2 * 768
    assert lib.bsr_linear8_workspace_bytes(1, 4096) == 0 and lib.bsr_linear8_workspace_bytes(0, 64) == 0
    assert lib.bsr_linear8_workspace_bytes(6304, 768) >= 6304 * (768 + 8)


def call(name, good, **bad):
    """`good` is an ordered dict of valid arguments; any of them replaced"""
    args = dict(good, **bad)
    return getattr(P.load_library(), name)(*args.values())


LN = dict(x=A, type=0, M=4, D=64, ldx=64, gamma=A, beta=A, eps=1e-6, y=A, ldy=64, values=None, scales=None, mean=A, rstd=A, stream=None)
LNB = dict(dy=A, lddy=64, x=A, ldx=64, res=None, ldr=0, type=1, M=4, D=64, mean=A, rstd=A, gamma=A, dx=A, lddx=64, dgamma=A, dbeta=A, ws=A,
           ws_floats=1 << 20, stream=None)
QR = dict(x=A, type=0, M=4, K=64, ldx=64, values=A, scales=A, stream=None)
QW = dict(w=A, type=0, n_in=64, n_out=32, ldw=32, values=A, scales=A, values_back=A, scales_back=A, stream=None)
LF = dict(x=A, x_type=0, ldx=64, x_scales=None, M=400, n_in=64, n_out=32, values=A, scales=A, bias=None, act=0, u=None, res=None, y=A, y_type=0, ws=A,
          ws_bytes=1 << 20, stream=None)
LD = dict(dy=A, type=0, lddy=32, dy_scales=None, M=400, n_in=64, n_out=32, values=A, scales=A, u=None, dx=A, dx_type=0, ws=A, ws_bytes=1 << 20, stream=None)
DF = dict(z=A, type=0, rows=4, classes=10, ldz=10, index=A, ldi=3, logits=A, logits_type=1, ldt=3, top=3, labels=None, T=1.0, a=0.0, loss=A, stats=A,
          row_grad=None, scale=1.0, dz=None, ldd=0, ws=None, ws_floats=0, stream=None)
DB = dict(z=A, type=0, rows=4, classes=10, ldz=10, index=A, ldi=3, logits=A, logits_type=1, ldt=3, top=3, labels=None, T=1.0, a=0.0, stats=A,
          row_grad=None, scale=1.0, dz=2 * A, ldd=10, stream=None)
REFUSED = [
    ("bsr_layernorm_forward", LN, [dict(x=None), dict(x=A + 1), dict(type=2), dict(M=-1), dict(D=0), dict(ldx=63), dict(gamma=A + 4), dict(beta=None),
                                   dict(eps=float("nan")), dict(y=None), dict(ldy=8), dict(values=A), dict(scales=A), dict(values=A + 8, scales=A), dict(mean=A + 2)]),
    ("bsr_layernorm_backward", LNB, [dict(dy=None), dict(x=A + 2), dict(lddy=1), dict(res=A, ldr=8), dict(type=7), dict(M=-5), dict(mean=None), dict(gamma=None),
                                     dict(dgamma=None), dict(dx=None, dgamma=None, dbeta=None), dict(ws=None), dict(ws_floats=100), dict(lddx=60)]),
    ("bsr_quantize8_rows", QR, [dict(x=None), dict(type=3), dict(M=-1), dict(K=0), dict(ldx=10), dict(values=None), dict(values=A + 8), dict(scales=None)]),
    ("bsr_quantize8_weight", QW, [dict(w=None), dict(n_in=0), dict(n_out=-1), dict(ldw=31), dict(values=None), dict(scales_back=None), dict(values_back=A + 1)]),
    ("bsr_linear8_forward", LF, [dict(x=None), dict(x_type=5), dict(ldx=63), dict(M=-1), dict(n_in=0), dict(n_out=0), dict(values=None), dict(scales=None), dict(act=2),
                                 dict(y=None), dict(y=A + 2), dict(y_type=9), dict(ws=None), dict(ws_bytes=10), dict(res=A + 4), dict(act=1, u=A + 8),
                                 dict(x_scales=A, x=A + 4), dict(bias=A + 2)]),
    ("bsr_linear8_dgrad", LD, [dict(dy=None), dict(lddy=16), dict(u=A + 2), dict(dx=None), dict(ws_bytes=0), dict(values=A + 4), dict(dx_type=-1)]),
    ("bsr_distill_forward", DF, [dict(z=None), dict(z=A + 1), dict(type=4), dict(logits_type=4), dict(rows=-1), dict(rows=1 << 31), dict(classes=0), dict(ldz=9), dict(top=0),
                                 dict(top=1025, ldi=1025, ldt=1025), dict(index=None), dict(ldi=2), dict(logits=None), dict(T=0.0), dict(T=float("inf")), dict(T=float("nan")),
                                 dict(a=-0.1), dict(a=1.1), dict(a=float("nan")), dict(loss=None, stats=None), dict(loss=A + 2), dict(labels=A + 1), dict(dz=A, ldd=11),
                                 dict(dz=2 * A, ldd=4), dict(ws=A + 2, ws_floats=100), dict(classes=1 << 20, ldz=1 << 20, ws=A, ws_floats=3)]),
    ("bsr_distill_backward", DB, [dict(stats=None), dict(dz=None), dict(row_grad=A + 1), dict(ldd=9)]),
]


@pytest.mark.parametrize("name,good,bad", [(n, g, b) for n, g, bads in REFUSED for b in bads])
def test_refused_before_a_launch(name, good, bad):
    assert call(name, good, **bad) == INVALID
    text = P.load_library().bsr_last_error(None).decode()
    assert text.startswith(name) and len(text) > len(name) + 8


@pytest.mark.parametrize("name,good,rows", [(n, g, "rows" if "distill" in n else "M") for n, g, _ in REFUSED if "M" in g or "rows" in g])
def test_no_rows_no_launch(name, good, rows):
    """(the backward of a LayerNorm zeroes its sums, which is a launch: dx alone here)"""
    more = dict(dgamma=None, dbeta=None) if name == "bsr_layernorm_backward" else {}
    assert call(name, good, **{rows: 0}, **more) == 0


def test_the_reference_of_8_bit_blocks():
    """the numpy form that the GPU tests compare with, on values worked out by hand"""
    assert [exponent(v) for v in (0.0, 448.0, 448.1, 1.0, 1.75, 1.7500001, 3.4e38, 1e-45)] == [0, 0, 1, -8, -8, -7, 120, -127]
    assert list(to_e4m3([17.0, 19.0, 21.0, 2 ** -10, 3 * 2 ** -10, -17.0, 448.0, 0.0])) == [16.0, 20.0, 20.0, 0.0, 2 ** -8, -16.0, 448.0, 0.0]
    v, e = blocks8([[896.0, 1.0, 3.1]], 1, 128)
    assert e[0, 0] == 1 and list(v[0]) == [896.0, 1.0, 3.0]


BIG, WIDE = (1 << 30) + 1, (1 << 23) + 1


@pytest.mark.parametrize("name,good,bad", [
    ("bsr_layernorm_forward", LN, dict(D=BIG, ldx=BIG, ldy=BIG)), ("bsr_layernorm_backward", LNB, dict(D=BIG, lddy=BIG, ldx=BIG, lddx=BIG, ws_floats=1 << 50)),
    ("bsr_quantize8_rows", QR, dict(K=BIG, ldx=BIG)), ("bsr_quantize8_weight", QW, dict(n_in=WIDE)), ("bsr_quantize8_weight", QW, dict(n_out=WIDE, ldw=WIDE)),
    ("bsr_linear8_forward", LF, dict(n_in=WIDE, ldx=WIDE, ws_bytes=1 << 50)), ("bsr_linear8_forward", LF, dict(n_out=WIDE)),
    ("bsr_linear8_dgrad", LD, dict(n_out=WIDE, lddy=WIDE, ws_bytes=1 << 50)), ("bsr_linear8_dgrad", LD, dict(n_in=WIDE)),
    ("bsr_distill_forward", DF, dict(classes=BIG, ldz=BIG)), ("bsr_distill_backward", DB, dict(classes=BIG, ldz=BIG, ldd=BIG))])
def test_lengths_past_their_limits(name, good, bad):
    test_refused_before_a_launch(name, good, bad)


@pytest.mark.parametrize("name,good,bad", [("bsr_linear8_forward", LF, dict(y_type=1 | 256)), ("bsr_linear8_dgrad", LD, dict(dx_type=1 | 256)),
                                           ("bsr_linear8_forward", LF, dict(x_type=256)), ("bsr_linear8_forward", LF, dict(y_type=2 | 256))])
def test_cut_sums_are_for_bf16_results(name, good, bad):
    assert P.BSR_SUMS_CUT == 256
    test_refused_before_a_launch(name, good, bad)


@pytest.mark.parametrize("rows", [4, 400, 0])
def test_a_stored_input_needs_its_gelu(rows):
    """u_out would stay as it was"""
    test_refused_before_a_launch("bsr_linear8_forward", LF, dict(M=rows, act=0, u=A))


def blocks(rows, cols, rows_per_scale, **how):
    import torch
    how = dict(dict(dtype=torch.uint8), **how)
    return torch.zeros(rows, -(-cols // 128) * 128, **how), torch.zeros(-(-rows // rows_per_scale), -(-cols // 512) * 4, **how)


def test_parts_of_a_layer_are_looked_at():
    """tensors of other shapes, types or strides would be read past their ends"""
    import torch
    v, s = blocks(300, 200, 128)
    vb, sb = blocks(200, 300, 128)
    layer = P.Weight8(v, s, vb, sb, 200, 300)
    assert layer.values is v and layer.scales_back is sb and (layer.n_in, layer.n_out) == (200, 300)
    assert P.Weight8(v, s, None, None, 200, 300).values_back is None
    for bad in ((v[:299], s, vb, sb), (v[:, :128], s, vb, sb), (v, s[:2], vb, sb), (v, s[:, :2], vb, sb), (v.view(torch.int8), s, vb, sb), (v, s.int(), vb, sb),
                (v.t(), s, vb, sb), (v, s, v, sb), (v, s, vb, s), (v, s, vb, None), (v, s, None, sb), (v, s, vb.to("meta"), sb),
                (torch.zeros(600, 256, dtype=torch.uint8)[::2], s, vb, sb)):
        with pytest.raises(ValueError):
            P.Weight8(*bad, 200, 300)
    for n_in, n_out in ((0, 300), (200, 0), (300, 200), (257, 300), (200, 385)):
        with pytest.raises(ValueError):
            P.Weight8(v, s, vb, sb, n_in, n_out)
    with pytest.raises(AttributeError):
        layer.values = v[:10]
    for again in (copy.copy(layer), copy.deepcopy(layer), pickle.loads(pickle.dumps(layer))):
        assert again.n_out == 300 and again.values.shape == v.shape and torch.equal(again.scales_back, sb)


@pytest.mark.parametrize("call", ["forward", "dgrad"])
def test_rows_in_8_bits_are_looked_at(call):
    import torch
    v, s = blocks(20, 200, 1)
    layer = P.Weight8(*blocks(200, 200, 128), *blocks(200, 200, 128), 200, 200)
    product = P.bsr_linear8_forward if call == "forward" else P.bsr_linear8_dgrad
    for bad in ((v[:, :128], s), (v[::2], s[::2]), (v, s[:19]), (v, s[:, :2]), (v, s.view(torch.int8)), (v.short(), s), (v.view(-1), s), (v[0, 0], s),
                (torch.zeros(20, 512, dtype=torch.uint8)[:, :256], s)):
        with pytest.raises(ValueError, match="(values|scales): contiguous"):
            product(P.Rows8(*bad, 200), layer)
    with pytest.raises(ValueError, match="GPU"):
        product(P.Rows8(v, s, 200), layer)


def test_lengths_past_32_bits_are_refused_not_wrapped():
    """the library's columns, and the rows of its products, are 32-bit numbers (tensors without memory: nothing is launched)"""
    import torch

    def big(*shape, dtype=torch.bfloat16):
        return torch.empty(*shape, dtype=dtype, device="meta")

    wrapped = (1 << 32) + 64                    # 64 in 32 bits
    v64 = big(64, dtype=torch.float32)
    layer = P.Weight8(*blocks(48, 64, 128), *blocks(64, 48, 128), 64, 48)
    for call in (lambda: P.bsr_quantize8_rows(big(4, wrapped)), lambda: P.bsr_quantize8_weight(big(wrapped, 64)), lambda: P.bsr_quantize8_weight(big(64, wrapped)),
                 lambda: P.bsr_linear8_forward(big(wrapped, 64), layer), lambda: P.bsr_linear8_dgrad(big(wrapped, 48), layer),
                 lambda: P.bsr_linear8_forward(P.Rows8(big(wrapped, 128, dtype=torch.uint8), big(wrapped, 4, dtype=torch.uint8), 64), layer),
                 lambda: P.bsr_layernorm_forward(big(4, wrapped), v64, v64), lambda: P.bsr_layernorm_forward8(big(4, wrapped), v64, v64),
                 lambda: P.binding._distill_args(big(4, wrapped), big(4, 3, dtype=torch.int32), big(4, 3), None, 1.0, 0.0),
                 lambda: P.binding._distill_args(big(4, 64), big(4, wrapped, dtype=torch.int32), big(4, wrapped), None, 1.0, 0.0)):
        with pytest.raises(ValueError, match="2147483647"):
            call()


@pytest.mark.parametrize("name,good,bad", [
    ("bsr_layernorm_forward", LN, dict(y=A, ldx=80, ldy=72)), ("bsr_layernorm_backward", LNB, dict(dy=A, lddy=72, x=2 * A, dx=A, lddx=64)),
    ("bsr_layernorm_backward", LNB, dict(dy=2 * A, x=2 * A, res=A, ldr=72, dx=A)), ("bsr_layernorm_backward", LNB, dict(dy=2 * A, x=A, ldx=72, dx=A))])
def test_results_in_the_place_of_an_input_need_its_stride(name, good, bad):
    """rows would be written over others that have not been read yet"""
    test_refused_before_a_launch(name, good, bad)


@pytest.mark.parametrize("name,good", [("bsr_distill_forward", DF), ("bsr_distill_backward", DB)])
@pytest.mark.parametrize("T", [1e-39, 1e-45, 2e19, 3e38])
def test_temperatures_whose_square_or_reciprocal_overflows(name, good, T):
    """their losses and gradients would be 0 times infinity"""
    test_refused_before_a_launch(name, good, dict(T=T))
