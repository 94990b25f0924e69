"""Refusals of the operators around a gated, sparse block, on the CPU: sizes, types and combinations that no kernel may see."""
import ctypes as C

import pytest
import torch

import paper_1806_00187_amd as A
from paper_1806_00187_amd import binding as B

P = 1 << 20          # an address that is never read: every call here is refused before it launches anything


def refused(rc, code=A.NMT_EINVAL, says=None):
    msg = A.load().nmt_last_error().decode()
    assert rc == code, (rc, msg)
    assert says is None or says in msg, msg


def block(**kw):
    base = dict(rows=4, d=16, type=A.NMT_F16, kind=A.NMT_NORM_LAYER, eps=1e-5, resid_scale=1.0, rows_per_gate=4, ld_x=16, ld_y=16, ld_h=16, ld_n=16,
                d_x=P, d_y=P, d_post_gain=P, d_post_shift=P, d_gate=P, d_pre_gain=P, d_pre_shift=P, d_h=P, d_n=P, d_stats=P)
    base.update(kw)
    return B.nmt_gated_norm(**base)


def grads(**kw):
    base = dict(ld_dh=16, ld_dn=16, ld_dx=16, ld_dy=16, d_dh=P, d_dn=P, d_dx=P, d_dy=P, d_dpost_gain=P, d_dpost_shift=P, d_dgate=P, d_dpre_gain=P,
                d_dpre_shift=P, d_scratch=P, scratch_floats=1 << 20)
    base.update(kw)
    return B.nmt_gated_norm_grad(**base)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=2 ** 31 - 1), dict(d=0), dict(d=16385), dict(type=3), dict(kind=2), dict(eps=0.0), dict(eps=float("nan")),
                                 dict(resid_scale=float("inf")), dict(rows_per_gate=0), dict(ld_x=15), dict(ld_y=15), dict(ld_h=15), dict(ld_n=15),
                                 dict(d_x=None), dict(d_h=None), dict(d_n=None), dict(d_pre_gain=None), dict(d_post_gain=None),
                                 dict(d_y=None), dict(d_y=None, d_post_gain=None, d_post_shift=None, d_gate=None),
                                 dict(d_y=None, d_post_gain=None, d_post_shift=None, d_gate=None, d_h=None, d_n=None, d_pre_gain=None, d_pre_shift=None)])
def test_gated_norm_refuses(bad):
    refused(A.load().nmt_op_gated_norm_fwd(C.byref(block(**bad)), None), says="nmt_op_gated_norm_fwd")


@pytest.mark.parametrize("bad,worse", [(dict(d=0), {}), (dict(type=-1), {}), (dict(rows_per_gate=0), {}), (dict(ld_y=15), {}), (dict(ld_h=15), {}),
                                       (dict(d_stats=None), {}), (dict(d_pre_gain=None), {}), (dict(d_h=None), {}), (dict(d_gate=None), {}),
                                       (dict(d_post_gain=None, d_post_shift=None), {}), (dict(d_post_gain=None), {}), (dict(d_y=None), {}),
                                       ({}, dict(ld_dh=15)), ({}, dict(ld_dn=15)), ({}, dict(ld_dx=15)), ({}, dict(ld_dy=15)), ({}, dict(d_dx=None)),
                                       ({}, dict(d_dy=None)), ({}, dict(d_dh=None, d_dn=None)), ({}, dict(d_dn=None)), ({}, dict(d_scratch=P + 4))])
def test_gated_norm_backward_refuses(bad, worse):
    refused(A.load().nmt_op_gated_norm_bwd(C.byref(block(**bad)), C.byref(grads(**worse)), None), says="nmt_op_gated_norm_bwd")


def test_gated_norm_backward_wants_the_scratch_it_asks_for():
    need = A.nmt_op_gated_norm_bwd_scratch(4, 16, 4)
    lib = A.load()
    for g in (grads(d_scratch=None), grads(scratch_floats=need - 1)):
        refused(lib.nmt_op_gated_norm_bwd(C.byref(block()), C.byref(g), None), A.NMT_ENOMEM, str(need))
    for bad in ((-1, 16, 4), (4, 0, 4), (4, 16385, 4)):
        with pytest.raises(A.NmtError):
            A.nmt_op_gated_norm_bwd_scratch(*bad)
    assert A.nmt_op_gated_norm_bwd_scratch(0, 16) == 0
    assert A.nmt_op_gated_norm_bwd_scratch(1000, 64, 10) > A.nmt_op_gated_norm_bwd_scratch(1000, 64) > 0


def test_null_structs_are_refused():
    lib = A.load()
    refused(lib.nmt_op_gated_norm_fwd(None, None))
    refused(lib.nmt_op_gated_norm_bwd(None, C.byref(grads()), None))
    refused(lib.nmt_op_gated_norm_bwd(C.byref(block()), None, None))
    refused(lib.nmt_adamw_step(None, 1e-3, 0.9, 0.98, 1e-8, 1, 1.0, None, None))
    refused(lib.nmt_adamw_create(0, None, 32, 0, 0, None, 0, None, None))


DISPATCH = dict(expert=P, tokens=4, k=2, experts=8, capacity=0, x=P, ld_x=16, d=16, type=0, rows=P, ld_rows=16, slot=P, ranges=P, scratch=P, scratch_ints=1 << 20)


@pytest.mark.parametrize("bad", [dict(tokens=-1), dict(k=0), dict(k=65), dict(experts=0), dict(experts=1025), dict(capacity=-1), dict(capacity=2 ** 28),
                                 dict(tokens=2 ** 30), dict(d=0), dict(type=3), dict(ld_x=15), dict(ld_rows=15), dict(x=None), dict(rows=None),
                                 dict(expert=None), dict(slot=None), dict(ranges=None)])
def test_dispatch_refuses(bad):
    a = dict(DISPATCH, **bad)
    refused(A.load().nmt_op_expert_dispatch(*a.values(), None), says="nmt_op_expert_dispatch")


def test_dispatch_wants_the_scratch_it_asks_for():
    need = A.nmt_op_expert_dispatch_scratch(4, 2, 8)
    for bad in (dict(scratch=None), dict(scratch_ints=need - 1)):
        a = dict(DISPATCH, **bad)
        refused(A.load().nmt_op_expert_dispatch(*a.values(), None), A.NMT_ENOMEM, str(need))


COMBINE = dict(rows=P, ld_rows=16, n_rows=8, slot=P, weights=P, add=P, ld_add=16, out=P, ld_out=16, tokens=4, k=2, d=16, type=0)


@pytest.mark.parametrize("bad", [dict(rows=None), dict(ld_rows=15), dict(n_rows=-1), dict(slot=None), dict(ld_add=15), dict(out=None), dict(ld_out=15),
                                 dict(tokens=-1), dict(k=0), dict(d=0), dict(d=2 ** 20 + 1), dict(type=7)])
def test_combine_refuses(bad):
    a = dict(COMBINE, **bad)
    refused(A.load().nmt_op_expert_combine(*a.values(), None), says="nmt_op_expert_combine")


COMBINE_BWD = dict(dout=P, ld_dout=16, rows=P, ld_rows=16, n_rows=8, slot=P, weights=P, drows=P, ld_drows=16, dweights=P, ranges=P, experts=8, capacity=1,
                   tokens=4, k=2, d=16, type=0)


@pytest.mark.parametrize("bad", [dict(dout=None), dict(ld_dout=15), dict(rows=None), dict(dweights=None), dict(ld_rows=15), dict(n_rows=9), dict(n_rows=-1),
                                 dict(slot=None), dict(drows=None), dict(ld_drows=15), dict(ranges=None), dict(experts=7), dict(capacity=2),
                                 dict(capacity=-1), dict(tokens=-1), dict(k=65), dict(d=0), dict(type=3)])
def test_combine_backward_refuses(bad):
    a = dict(COMBINE_BWD, **bad)
    refused(A.load().nmt_op_expert_combine_bwd(*a.values(), None), says="nmt_op_expert_combine_bwd")


def test_dispatch_scratch_grows_with_the_choices_and_refuses_what_dispatch_refuses():
    sizes = [A.nmt_op_expert_dispatch_scratch(t, 2, 64) for t in (0, 1, 1000, 10000, 100000)]
    assert sizes == sorted(sizes) and sizes[0] == 0
    for bad in ((-1, 2, 8), (4, 0, 8), (4, 2, 0), (4, 2, 1025), (2 ** 30, 2, 8)):
        with pytest.raises(A.NmtError):
            A.nmt_op_expert_dispatch_scratch(*bad)


def tensor_of(**kw):
    base = dict(n=100, weight_decay=0.01, lr_factor=1.0, d_master=P, d_m=P, d_v=P, d_m_scale=None, d_v_scale=None, d_grad=P, d_weights=P)
    base.update(kw)
    return B.nmt_adamw_tensor(**base)


@pytest.mark.parametrize("bad,bits,says", [(dict(n=-1), 32, "elements"), (dict(weight_decay=-0.1), 32, "decay"), (dict(lr_factor=float("nan")), 32, "factor"),
                                           (dict(d_master=None), 32, "null"), (dict(d_m=None), 32, "null"), (dict(d_v=None), 32, "null"), (dict(d_grad=None), 32, "null"),
                                           (dict(d_m_scale=P), 32, "scales"), ({}, 8, "scales"), (dict(d_m_scale=P), 8, "scales"),
                                           (dict(d_master=P + 2), 32, "multiple"), (dict(d_grad=P + 1), 32, "multiple"), (dict(d_weights=P + 1), 32, "multiple"),
                                           (dict(d_v=P + 2), 32, "multiple"), (dict(d_m_scale=P + 2, d_v_scale=P), 8, "multiple"), ({}, 16, "bits")])
def test_adamw_create_refuses(bad, bits, says):
    arr, out = (B.nmt_adamw_tensor * 1)(tensor_of(**bad)), C.c_void_p()
    refused(A.load().nmt_adamw_create(1, arr, bits, A.NMT_F16, A.NMT_F16, P, 1 << 20, None, C.byref(out)), says=says)
    assert not out.value


def test_adamw_create_wants_the_table_it_asks_for():
    lib, arr, out = A.load(), (B.nmt_adamw_tensor * 2)(tensor_of(n=5000), tensor_of(n=1)), C.c_void_p()
    need = lib.nmt_adamw_table_bytes(2, arr)
    assert need > 0 and lib.nmt_adamw_table_bytes(1, arr) < need and lib.nmt_adamw_table_bytes(0, None) == 0
    refused(lib.nmt_adamw_create(2, arr, 32, 0, 0, P, need - 1, None, C.byref(out)), A.NMT_ENOMEM, str(need))
    refused(lib.nmt_adamw_create(2, arr, 32, 0, 0, None, need, None, C.byref(out)), A.NMT_ENOMEM)
    refused(lib.nmt_adamw_create(2, arr, 32, 0, 0, P + 8, need, None, C.byref(out)), says="aligned")
    refused(lib.nmt_adamw_create(2, arr, 32, 3, 0, P, need, None, C.byref(out)), says="type")
    refused(lib.nmt_adamw_create(2, None, 32, 0, 0, P, need, None, C.byref(out)))


def test_adamw_over_nothing_is_a_plan_whose_steps_do_nothing():
    lib, out = A.load(), C.c_void_p()
    arr = (B.nmt_adamw_tensor * 2)(tensor_of(n=0, d_master=None, d_grad=None), tensor_of(n=0))
    for n, a in ((0, None), (2, arr)):
        assert lib.nmt_adamw_create(n, a, 32, 0, 0, None, 0, None, C.byref(out)) == A.NMT_OK and out.value
        assert lib.nmt_adamw_step(out, 1e-3, 0.9, 0.98, 1e-8, 1, 1.0, None, None) == A.NMT_OK
        for bad in ((float("nan"), 0.9, 0.98, 1e-8, 1, 1.0), (-1.0, 0.9, 0.98, 1e-8, 1, 1.0), (1e-3, 1.0, 0.98, 1e-8, 1, 1.0), (1e-3, 0.9, -0.1, 1e-8, 1, 1.0),
                    (1e-3, 0.9, 0.98, 0.0, 1, 1.0), (1e-3, 0.9, 0.98, 1e-8, 0, 1.0), (1e-3, 0.9, 0.98, 1e-8, 1, float("inf"))):
            refused(lib.nmt_adamw_step(out, *bad, None, None), says="nmt_adamw_step")
        lib.nmt_adamw_destroy(out)


# ---- what the binding sees before the library does ------------------------------------------------
def rows(n, d, dtype=torch.float16):
    return torch.zeros(n, d, dtype=dtype)


@pytest.mark.parametrize("change", [dict(y=rows(4, 17)), dict(y=rows(5, 16)), dict(y=rows(4, 16, torch.float32)), dict(y=rows(16, 4).t()), dict(h=rows(1, 16).expand(4, 16)),
                                    dict(gate=torch.zeros(2, 16, dtype=torch.float16)), dict(gate=rows(1, 16), rows_per_gate=2), dict(kind="l2"),
                                    dict(post=(torch.zeros(15, dtype=torch.float16), None)), dict(pre=(torch.zeros(16), None)), dict(stats=torch.zeros(4, 3)),
                                    dict(stats=torch.zeros(4, 4, dtype=torch.float64)), dict(x=rows(4, 16, torch.float64)), dict(x=torch.zeros(16, dtype=torch.float16)),
                                    {}])        # (the last: tensors of the CPU)
def test_gated_norm_binding_refuses(change):
    v = torch.ones(16, dtype=torch.float16)
    a = dict(x=rows(4, 16), y=rows(4, 16), h=rows(4, 16), n=rows(4, 16), stats=torch.zeros(4, 4), post=(v, v), gate=rows(1, 16), pre=(v, None))
    a.update(change)
    with pytest.raises(A.NmtError) as e:
        A.nmt_op_gated_norm_fwd(**a)
    assert e.value.code == A.NMT_EINVAL


@pytest.mark.parametrize("change,code", [(dict(expert=torch.zeros(4, 2, dtype=torch.int64)), -1), (dict(expert=torch.zeros(8, dtype=torch.int32)), -1),
                                         (dict(rows=rows(7, 16)), -1), (dict(capacity=2), -1), (dict(x=rows(5, 16)), -1), (dict(x=None), -1),
                                         (dict(slot=torch.zeros(4, 1, dtype=torch.int32)), -1), (dict(ranges=torch.zeros(8, dtype=torch.int32)), -1),
                                         (dict(scratch=torch.zeros(8)), -1), (dict(experts=2000), -1), ({}, -1)])
def test_dispatch_binding_refuses(change, code):
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)
    a = dict(expert=i(4, 2), experts=8, capacity=0, x=rows(4, 16), rows=rows(8, 16), slot=i(4, 2), ranges=i(8, 2), scratch=i(4096))
    a.update(change)
    with pytest.raises(A.NmtError) as e:
        A.nmt_op_expert_dispatch(**a)
    assert e.value.code == code


@pytest.mark.parametrize("change", [dict(m=torch.zeros(99)), dict(grad=torch.zeros(100, dtype=torch.float64)), dict(master=torch.zeros(100, dtype=torch.float16)),
                                    dict(m=torch.zeros(100, dtype=torch.float8_e4m3fn)), dict(v=torch.zeros(200)[::2]), dict(weights=torch.zeros(50)), {}])
def test_adamw_binding_refuses(change):
    t = dict(master=torch.zeros(100), m=torch.zeros(100), v=torch.zeros(100), grad=torch.zeros(100, dtype=torch.float16), weights=torch.zeros(100))
    t.update(change)
    with pytest.raises(A.NmtError) as e:
        A.nmt_adamw_create([t], torch.zeros(1 << 16, dtype=torch.uint8))
    assert e.value.code == A.NMT_EINVAL


def far(n, d, dtype=torch.float16):
    """A tensor of a size that is no int32 and of no memory."""
    return torch.zeros(1, 1, dtype=dtype).expand(n, d)


def test_sizes_that_32_bits_do_not_hold_are_refused():
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)
    big = 2 ** 32 + 4
    for call in (lambda: A.nmt_op_gated_norm_fwd(far(big, 16), far(big, 16), None, far(big, 16), pre=(rows(1, 16), None)),
                 lambda: A.nmt_op_gated_norm_bwd(None, None, None, None, None, far(big, 16), None, None),
                 lambda: A.nmt_op_gated_norm_bwd_scratch(big, 16), lambda: A.nmt_op_gated_norm_bwd_scratch(4, big), lambda: A.nmt_op_gated_norm_bwd_scratch(4, 16, big),
                 lambda: A.nmt_op_expert_dispatch_scratch(big, 2, 8), lambda: A.nmt_op_expert_dispatch_scratch(4, 2, big),
                 lambda: A.nmt_op_expert_dispatch(i(4, 2), 8, 2 ** 32, None, None, i(4, 2), i(8, 2), i(4096)),
                 lambda: A.nmt_op_expert_combine(far(big, 16), i(4, 2), None, rows(4, 16)),
                 lambda: A.nmt_op_expert_combine_bwd(rows(4, 16), None, i(4, 2), None, far(big, 16), None),
                 lambda: A.nmt_op_expert_combine_bwd(rows(4, 16), None, i(4, 2), None, rows(8, 16), None, i(8, 2), 2 ** 32 + 1)):
        with pytest.raises(A.NmtError, match="32 bits"):
            call()


def test_slots_in_place_of_the_choices_are_refused():
    """Every work-group of a sort reads all choices."""
    refused(A.load().nmt_op_expert_dispatch(P, 4, 2, 8, 0, None, 0, 0, 0, None, 0, P, P + 4096, P + 8192, 1 << 20, None), says="in place")


AT = dict(d_master=P, d_m=P + 0x1000, d_v=P + 0x2000, d_grad=P + 0x3000, d_weights=P + 0x4000)      # of a tensor of 100 elements


@pytest.mark.parametrize("other", [{}, dict(d_master=P + 396), dict(d_m=P + 0x1000), dict(d_v=P + 0x3000 + 196), dict(d_weights=P + 0x4000 + 198), dict(d_grad=P + 398),
                                   dict(d_weights=P + 0x8000 + 100), dict(d_m=P - 396)])
def test_adamw_refuses_what_it_would_write_twice(other):
    """One tensor twice, or buffers that share a few bytes: what a step leaves there would depend on an order that nothing fixes."""
    second = {f: p + 0x8000 for f, p in AT.items()}
    second.update(other or AT)
    lib, arr, out = A.load(), (B.nmt_adamw_tensor * 2)(tensor_of(**AT), tensor_of(**second)), C.c_void_p()
    for pair in (arr, (B.nmt_adamw_tensor * 2)(arr[1], arr[0])):
        refused(lib.nmt_adamw_create(2, pair, 32, A.NMT_F16, A.NMT_F16, P << 8, 1 << 20, None, C.byref(out)), says="overlaps")
        assert not out.value


def test_adamw_step_refuses_what_32_bits_make_zero_or_infinite():
    lib, out = A.load(), C.c_void_p()
    assert lib.nmt_adamw_create(0, None, 32, 0, 0, None, 0, None, C.byref(out)) == A.NMT_OK
    refused(lib.nmt_adamw_step(out, 1e39, 0.9, 0.98, 1e-8, 1, 1.0, None, None), says="learning rate")
    refused(lib.nmt_adamw_step(out, 1e-3, 0.9, 0.98, 1e-50, 1, 1.0, None, None), says="eps")
    lib.nmt_adamw_destroy(out)


def test_the_norm_before_the_first_block_has_no_residual_scale():
    """Without a block's output h is x itself: a scale that the forward call left out and the backward call put into dx would be no gradient of it."""
    alone = dict(d_y=None, d_post_gain=None, d_post_shift=None, d_gate=None, d_h=None, resid_scale=0.9)
    refused(A.load().nmt_op_gated_norm_fwd(C.byref(block(**alone)), None), says="resid_scale")


@pytest.mark.parametrize("per", [1, 27, 2 ** 31 - 2])
def test_no_rows_have_no_gates_per_group_of_rows(per):
    """ceil(0 / rows_per_gate) gates: their gradient is an array of nothing, wherever it begins.  (Nothing is launched.)"""
    g = grads(d_dpost_gain=None, d_dpost_shift=None, d_dpre_gain=None, d_dpre_shift=None)
    for gate in (P, None):
        assert A.load().nmt_op_gated_norm_bwd(C.byref(block(rows=0, rows_per_gate=per, d_gate=gate)), C.byref(g), None) == A.NMT_OK


@pytest.mark.parametrize("per", [1, 27, None, 0])
@pytest.mark.parametrize("gates", [0, 1])
def test_binding_takes_the_gates_of_no_rows(gates, per):
    """None, or the one that all rows share; more do not belong to no rows."""
    e, v = rows(0, 16), torch.ones(16, dtype=torch.float16)
    a = dict(post=(v, None), pre=(v, None), rows_per_gate=per)
    with pytest.raises(A.NmtError, match="not on a GPU"):
        A.nmt_op_gated_norm_fwd(e, e, e, e, torch.zeros(0, 4), gate=rows(gates, 16), **a)
    with pytest.raises(A.NmtError, match="not on a GPU"):
        A.nmt_op_gated_norm_bwd(e, e, e, e, torch.zeros(0, 4), e, e, None, gate=rows(gates, 16), dgate=rows(gates, 16), **a)
    with pytest.raises(A.NmtError, match="gate"):
        A.nmt_op_gated_norm_fwd(e, e, e, e, torch.zeros(0, 4), gate=rows(2, 16), **a)
    with pytest.raises(A.NmtError, match="gate"):
        A.nmt_op_gated_norm_bwd(e, e, e, e, torch.zeros(0, 4), e, e, None, gate=rows(gates, 16), dgate=rows(1 - gates, 16), **a)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("d", [1, 64, 100, 256, 512, 1024, 2048, 4096, 4100, 8192, 8200, 12289, 16384])
def test_forward_grids_have_less_than_2_to_the_32_threads(d, dtype):
    """A launch of as many is refused.  Rows around all multiples of 2^22, where a run gets another row, and the most there may be."""
    most = 2 ** 31 - 1 - 65536
    for rows in {max(1, min(most, (m << 22) + off)) for m in range(513) for off in (-2, -1, 0, 1, 2)}:
        groups, threads = A.nmt_debug_gated_norm_grid(rows, d, dtype)
        assert groups * threads < 2 ** 32, (rows, groups, threads)


# ---- sessions ------------------------------------------------------------------------------------
@pytest.mark.parametrize("optimizer", [True, False])
@pytest.mark.parametrize("bad", [dict(state_bits=16), dict(state_bits=0), dict(weight_decay=-0.01), dict(weight_decay=float("nan")), dict(weight_decay=float("inf")),
                                 dict(weight_decay=1e39)])
def test_sessions_refuse_bad_optimizer_settings_before_they_make_anything(bad, optimizer, monkeypatch):
    import nmt_inputs as I
    from paper_1806_00187_amd import session
    made = []
    monkeypatch.setattr(session.nmt, "nmt_create", lambda **cfg: made.append(cfg))
    with pytest.raises(ValueError):
        session.Session(I.MODELS["tiny"], {}, device="cpu", optimizer=optimizer, **bad)
    assert not made


def test_sessions_name_moments_of_8_bits():
    from paper_1806_00187_amd.session import Session
    s = object.__new__(Session)
    s.layout = {"w": (0, 2, 3), "b": (8, 1, 4)}
    flat = torch.arange(-6, 6).float().to(torch.float8_e4m3fn)
    named = s.named(flat)
    assert named["w"].shape == (2, 3) and named["w"].tolist() == [[-6, -5, -4], [-3, -2, -1]] and named["b"].tolist() == [2, 3, 4, 5]


def test_adamw_plans_keep_the_tensors_they_were_made_for(monkeypatch):
    """Whatever becomes of the caller's list and its dicts: the device table holds those tensors' addresses."""
    import weakref
    monkeypatch.setattr(B, "_call", lambda *args, **kw: None)      # (of tensors on the CPU)
    t = dict(master=torch.zeros(100), m=torch.zeros(100), v=torch.zeros(100), grad=torch.zeros(100), weights=torch.zeros(100))
    seen, tensors = [weakref.ref(x) for x in t.values()], [t]
    plan = A.nmt_adamw_create(tensors, torch.zeros(1 << 16, dtype=torch.uint8))
    for name in ("grad", "weights"):
        t[name] = None
    t.clear(), tensors.clear()
    assert all(ref() is not None for ref in seen)
    A.nmt_adamw_destroy(plan)
    assert all(ref() is None for ref in seen)


@pytest.mark.parametrize("at", [P, P + 0x2000 + 384, P - 16, P + 0x3000, P + 0x4000])
def test_adamw_refuses_a_table_among_its_buffers(at):
    """The kernel takes its addresses from the table, which neither a step nor a backward pass may write over."""
    lib, arr, out = A.load(), (B.nmt_adamw_tensor * 1)(tensor_of(**AT)), C.c_void_p()
    refused(lib.nmt_adamw_create(1, arr, 32, A.NMT_F16, A.NMT_F16, at, lib.nmt_adamw_table_bytes(1, arr), None, C.byref(out)), says="overlaps")
    assert not out.value
