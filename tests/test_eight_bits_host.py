"""Refusals of the operators on matrices held in 8 bits, on the CPU: sizes, types and combinations that no kernel may see."""
import ctypes as C

import pytest
import torch

import paper_1806_00187_amd as A
from paper_1806_00187_amd import binding as B

P = 1 << 20          # an address that is never read: every call here is refused before it launches anything
E4M3 = torch.float8_e4m3fn


def refused(rc, code=A.NMT_EINVAL, says=None):
    msg = A.load().nmt_last_error().decode()
    assert rc == code, (rc, msg)
    assert says is None or says in msg, msg


QUANTIZE = dict(x=P, ld_x=300, rows=200, d=300, type=0, square=0, codes=P, ld_codes=300, scales=P, ld_scales=200, codes_t=P, ld_codes_t=200, scales_t=P,
                ld_scales_t=300)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=2 ** 31 - 1), dict(d=0), dict(d=2 ** 31 - 1), dict(type=3), dict(x=None), dict(ld_x=299), dict(ld_codes=299),
                                 dict(ld_scales=199), dict(ld_codes_t=199), dict(ld_scales_t=299), dict(codes=None), dict(scales=None), dict(codes_t=None),
                                 dict(scales_t=None), dict(codes=None, scales=None, codes_t=None, scales_t=None), dict(square=1, ld_scales=1),
                                 dict(square=1, ld_scales_t=2), dict(rows=2 ** 30, d=2 ** 30, ld_x=2 ** 30, ld_codes=2 ** 30)])
def test_quantize_refuses(bad):
    refused(A.load().nmt_op_quantize8(*dict(QUANTIZE, **bad).values(), None), says="nmt_op_quantize8")


def norm(**kw):
    base = dict(rows=4, d=300, type=A.NMT_F16, kind=A.NMT_NORM_RMS, eps=1e-5, resid_scale=1.0, ld_x=300, ld_y=300, ld_h=300, ld_n=300, ld_codes=300, ld_scales=4,
                d_x=P, d_y=P, d_gain=P, d_shift=P, d_h=P, d_n=P, d_codes=P, d_scales=P, d_stats=P)
    base.update(kw)
    return B.nmt_norm8(**base)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=2 ** 31 - 1), dict(d=0), dict(d=16385), dict(type=3), dict(kind=2), dict(eps=0.0), dict(eps=float("nan")),
                                 dict(resid_scale=float("inf")), dict(ld_x=299), dict(ld_y=299), dict(ld_h=299), dict(ld_n=299), dict(ld_codes=299), dict(ld_scales=3),
                                 dict(d_x=None), dict(d_gain=None), dict(d_codes=None), dict(d_scales=None), dict(d_y=None), dict(d_y=None, d_h=None, resid_scale=0.5), dict(ld_h=301), dict(ld_n=301)])
def test_norm_refuses(bad):
    refused(A.load().nmt_op_norm8(C.byref(norm(**bad)), None), says="nmt_op_norm8")


def gemm(**kw):
    base = dict(M=200, N=300, K=400, batch=2, type=A.NMT_F16, a_square=0, b_square=1, lda=400, ldb=400, ldc=300, ld_add=300, ld_sa=200, ld_sb=3,
                stride_a=80000, stride_b=120000, stride_c=60000, stride_add=60000, stride_bias=300, stride_sa=800, stride_sb=12,
                d_a=P, d_b=P, d_sa=P, d_sb=P, d_bias=P, d_add=P, d_c=P, d_ranges=None, d_scratch=P, scratch_floats=1 << 40)
    base.update(kw)
    return B.nmt_gemm8(**base)


@pytest.mark.parametrize("bad", [dict(M=-1), dict(N=-1), dict(K=-1), dict(M=2 ** 31 - 1), dict(batch=-1), dict(batch=1025), dict(type=3), dict(lda=399), dict(lda=408), dict(lda=384),
                                 dict(ldb=384), dict(lda=2 ** 22 + 16), dict(ldb=2 ** 22 + 16), dict(ldc=299), dict(ld_add=299), dict(ld_sa=199), dict(ld_sb=2),
                                 dict(a_square=1, ld_sa=1), dict(b_square=0), dict(d_a=None), dict(d_b=None), dict(d_sa=None), dict(d_sb=None), dict(d_c=None),
                                 dict(d_a=P + 8), dict(d_b=P + 8), dict(stride_a=8), dict(stride_b=-16), dict(stride_c=0), dict(stride_c=-1), dict(stride_bias=-1),
                                 dict(stride_sa=-1), dict(ldc=301), dict(stride_add=0), dict(d_ranges=P, a_square=1), dict(d_scratch=P + 4)])
def test_gemm_refuses(bad):
    refused(A.load().nmt_op_gemm8(C.byref(gemm(**bad)), None), says="nmt_op_gemm8")


def test_gemm_wants_the_scratch_it_asks_for():
    need = A.nmt_op_gemm8_scratch(128, 128, 100000)
    assert need > 0
    a = dict(M=128, N=128, K=100000, batch=1, lda=100000, ldb=100000, ldc=128, ld_add=128, ld_sa=128, ld_sb=1)
    for bad in (dict(d_scratch=None), dict(scratch_floats=need - 1)):
        refused(A.load().nmt_op_gemm8(C.byref(gemm(**a, **bad)), None), A.NMT_ENOMEM, str(need))
    assert A.nmt_op_gemm8_scratch(128, 128, 100000, 1, True) == 0      # (rows of experts are not cut along k)
    for bad in ((-1, 8, 8), (8, -1, 8), (8, 8, -1), (8, 8, 8, 1025), (8, 8, 8, -1)):
        with pytest.raises(A.NmtError):
            A.nmt_op_gemm8_scratch(*bad)


def test_gemm_forms_are_named_and_bad_ones_refused():
    assert A.nmt_debug_gemm8_form(1, 1, 1, torch.float16) == (64, 1)
    assert A.nmt_debug_gemm8_form(1 << 20, 1 << 12, 1 << 10, torch.float16) == (256, 1)
    assert A.nmt_debug_gemm8_form(1 << 20, 1 << 12, 1 << 10, torch.float16, b_square=False)[0] == 128
    for bad in ((-1, 8, 8), (8, 8, 8, torch.float16, 1025)):
        with pytest.raises(A.NmtError):
            A.nmt_debug_gemm8_form(*bad[:3], *(bad[3:] or [torch.float16]))
    with pytest.raises(A.NmtError):
        A.nmt_debug_gemm8_form(8, 8, 8, torch.float64)


def layer(**kw):
    base = dict(tokens=4, k=2, experts=8, d=200, ff=300, type=A.NMT_F16, act=A.NMT_ACT_SILU_GATE, ld_x=200, ld_add=200, ld_out=200, ld_up=208, stride_up=208 * 600,
                ld_up_scales=5, stride_up_scales=10, ld_down=304, stride_down=304 * 200, ld_down_scales=2, stride_down_scales=6, d_x=P, d_expert=P, d_weights=P,
                d_up=P, d_up_scales=P, d_down=P, d_down_scales=P, d_add=P, d_out=P, d_scratch=P, scratch_floats=1 << 30)
    base.update(kw)
    return B.nmt_expert_layer8(**base)


@pytest.mark.parametrize("bad", [dict(tokens=-1), dict(tokens=65), dict(k=0), dict(k=65), dict(experts=0), dict(experts=1025), dict(d=0), dict(ff=0), dict(d=2 ** 20 + 1),
                                 dict(ff=2 ** 20 + 1), dict(type=3), dict(act=2), dict(ld_x=199), dict(ld_add=199), dict(ld_out=199), dict(ld_add=201), dict(ld_up=192),
                                 dict(ld_up=200), dict(ld_down=288), dict(ld_down=300), dict(stride_up=8), dict(stride_down=-16), dict(stride_up_scales=-1),
                                 dict(stride_down_scales=-1), dict(ld_up_scales=4), dict(ld_down_scales=1), dict(d_x=None), dict(d_expert=None), dict(d_up=None),
                                 dict(d_up_scales=None), dict(d_down=None), dict(d_down_scales=None), dict(d_out=None), dict(d_up=P + 8), dict(d_down=P + 1),
                                 dict(d_scratch=P + 4)])
def test_layer_refuses(bad):
    refused(A.load().nmt_op_expert_layer8(C.byref(layer(**bad)), None), says="nmt_op_expert_layer8")


def test_layer_wants_the_scratch_it_asks_for():
    need = A.nmt_op_expert_layer8_scratch(4, 2, 8, 200, 300)
    for bad in (dict(d_scratch=None), dict(scratch_floats=need - 1)):
        refused(A.load().nmt_op_expert_layer8(C.byref(layer(**bad)), None), A.NMT_ENOMEM, str(need))
    for bad in ((65, 2, 8, 16, 16), (4, 0, 8, 16, 16), (4, 2, 0, 16, 16), (4, 2, 8, 0, 16), (4, 2, 8, 16, 0)):
        with pytest.raises(A.NmtError):
            A.nmt_op_expert_layer8_scratch(*bad)


def test_null_structs_and_calls_of_nothing():
    lib = A.load()
    refused(lib.nmt_op_norm8(None, None))
    refused(lib.nmt_op_gemm8(None, None))
    refused(lib.nmt_op_expert_layer8(None, None))
    # (nothing is launched)
    assert lib.nmt_op_quantize8(*dict(QUANTIZE, rows=0).values(), None) == A.NMT_OK
    assert lib.nmt_op_norm8(C.byref(norm(rows=0)), None) == A.NMT_OK
    for none in (dict(M=0), dict(N=0), dict(batch=0)):
        assert lib.nmt_op_gemm8(C.byref(gemm(**none)), None) == A.NMT_OK
    assert lib.nmt_op_expert_layer8(C.byref(layer(tokens=0)), None) == A.NMT_OK


# ---- what the binding sees before the library does ------------------------------------------------
def zeros(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype)


def codes(*shape):
    return torch.zeros(*shape, dtype=torch.uint8).view(E4M3)


H = torch.float16


@pytest.mark.parametrize("change", [dict(x=zeros(4, 300, dtype=torch.float64)), dict(x=zeros(300, dtype=H)), dict(x=zeros(300, 4, dtype=H).t()), dict(codes=codes(4, 299)),
                                    dict(codes=zeros(4, 300, dtype=torch.uint8)), dict(scales=zeros(3, 3)), dict(scales=zeros(2, 4)), dict(scales=zeros(4, 3).t()),
                                    dict(codes_t=codes(300, 3)), dict(scales_t=zeros(2, 300)), dict(square=True), dict(scales=zeros(3, 4, dtype=H)), {}])
def test_quantize_binding_refuses(change):
    a = dict(x=zeros(4, 300, dtype=H), codes=codes(4, 300), scales=zeros(3, 4), codes_t=codes(300, 4), scales_t=zeros(1, 300))
    a.update(change)
    with pytest.raises(A.NmtError) as e:
        A.nmt_op_quantize8(**a)
    assert e.value.code == A.NMT_EINVAL


@pytest.mark.parametrize("change", [dict(y=zeros(4, 299, dtype=H)), dict(y=zeros(4, 300)), dict(h=zeros(1, 300, dtype=H).expand(4, 300)), dict(codes=codes(5, 300)),
                                    dict(scales=zeros(4, 3)), dict(gain=zeros(300)), dict(shift=zeros(299, dtype=H)), dict(kind="l2"), dict(stats=zeros(4, 3)),
                                    dict(n=zeros(4, 300)), {}])
def test_norm_binding_refuses(change):
    r, v = zeros(4, 300, dtype=H), zeros(300, dtype=H)
    a = dict(x=r, y=r, h=r, codes=codes(4, 300), scales=zeros(3, 4), gain=v, shift=v, n=r, stats=zeros(4, 4))
    a.update(change)
    with pytest.raises(A.NmtError) as e:
        A.nmt_op_norm8(**a)
    assert e.value.code == A.NMT_EINVAL


@pytest.mark.parametrize("change", [dict(a=codes(200, 384)), dict(a=zeros(200, 400, dtype=H)), dict(b=codes(299, 400)), dict(b=codes(2, 300, 400)), dict(c=zeros(200, 300, dtype=torch.float64)),
                                    dict(c=None), dict(a_scales=zeros(4, 199)), dict(a_scales=zeros(3, 200)), dict(b_scales=zeros(4, 4)), dict(b_scales=zeros(4)),
                                    dict(bias=zeros(300)), dict(bias=zeros(299, dtype=H)), dict(add=zeros(200, 300)), dict(ranges=zeros(2, 2, dtype=torch.int32)),
                                    dict(ranges=zeros(2), b=codes(2, 300, 400), b_scales=zeros(2, 4, 3)), dict(scratch=zeros(8, dtype=H)),
                                    dict(c=zeros(2, 200, 300, dtype=H)), dict(a=codes(400, 200).t()), {}])
def test_gemm_binding_refuses(change):
    a = dict(a=codes(200, 400), a_scales=zeros(4, 200), b=codes(300, 400), b_scales=zeros(4, 3), c=zeros(200, 300, dtype=H), bias=zeros(300, dtype=H),
             add=zeros(200, 300, dtype=H), scratch=zeros(1))
    a.update(change)
    with pytest.raises(A.NmtError) as e:
        A.nmt_op_gemm8(**a)
    assert e.value.code == A.NMT_EINVAL


@pytest.mark.parametrize("change", [dict(expert=zeros(4, 2)), dict(expert=zeros(3, 2, dtype=torch.int32)), dict(weights=zeros(4, 1)), dict(up=codes(8, 300, 256)), dict(down=codes(7, 256, 304)),
                                    dict(up=codes(600, 256)), dict(down_scales=zeros(8, 2, 2)), dict(up_scales=zeros(8, 2, 4)), dict(out=zeros(4, 256)),
                                    dict(act="gelu"), dict(act="relu"), dict(scratch=zeros(8, dtype=H)), dict(add=zeros(4, 255, dtype=H)), {}])
def test_layer_binding_refuses(change):
    a = dict(x=zeros(4, 256, dtype=H), expert=zeros(4, 2, dtype=torch.int32), weights=zeros(4, 2), up=codes(8, 608, 256), up_scales=zeros(8, 2, 5), down=codes(8, 256, 304),
             down_scales=zeros(8, 3, 2), out=zeros(4, 256, dtype=H), scratch=zeros(1 << 16), act="silu_gate")
    a.update(change)
    with pytest.raises(A.NmtError) as e:
        A.nmt_op_expert_layer8(**a)
    assert e.value.code == A.NMT_EINVAL


def test_sizes_that_32_bits_do_not_hold_are_refused():
    big, one = 2 ** 32 + 4, zeros(1, 1, dtype=H)
    for call in (lambda: A.nmt_op_quantize8(one.expand(big, 16)), lambda: A.nmt_op_norm8(one.expand(big, 16), None, None, None, None, None),
                 lambda: A.nmt_op_gemm8_scratch(big, 8, 8), lambda: A.nmt_op_gemm8_scratch(8, 8, big), lambda: A.nmt_op_expert_layer8_scratch(big, 2, 8, 16, 16),
                 lambda: A.nmt_op_gemm8(codes(1, 1).expand(big, 16), zeros(1, 1), codes(8, 16), zeros(1, 8), one.expand(big, 8))):
        with pytest.raises(A.NmtError, match="32 bits"):
            call()
