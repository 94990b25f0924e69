"""The operators around a gated, sparse block against plain implementations in 64 bits: norms with gate and residual scale, tokens sorted by
expert and back, AdamW over many tensors.

Tolerances.  Every output is rounded once to its type: half a step, u = eps / 2, of its value.  What comes before is fp32 (U32 = 2^-24): a sum over a
row is at most 16 additions in a lane, 6 across lanes and 15 across wavefronts, so a row's mean is off by at most 37 U32 of the mean magnitude, and what
is formed from it by a handful of roundings more: 64 U32 of the largest terms that enter."""
import pytest
import torch

import paper_1806_00187_amd as A
from tests import operators_plain as R
from tests.operators_plain import D, U32, half_step

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
TYPES = [F16, BF16, F32]
GUARD = 12345.0


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def guarded(rows, d, dtype, fill, ld=None, shift=0):
    """A [rows, d] view, rows `ld` apart and `shift` elements off any alignment, in a buffer of guard values, and a check that those are untouched."""
    ld = ld or d
    buf = torch.full((rows * ld + shift + 8,), GUARD, dtype=dtype, device=DEV)
    view = buf[shift:shift + rows * ld].view(rows, ld)[:, :d] if rows else buf[:0].view(0, d)
    if fill is not None:
        view.copy_(fill)

    def untouched():
        mask = torch.ones_like(buf, dtype=torch.bool)
        if rows:
            mask[shift:shift + rows * ld].view(rows, ld)[:, :d] = False
        return bool((buf[mask] == GUARD).all())
    return view, untouched


def within(got, want, bound, what):
    # below the type's smallest normal number its values lie smallest_normal * eps apart whatever their size, so a rounding is off by up to half of that there (fp16: 2^-25)
    bound = bound + torch.finfo(got.dtype).smallest_normal * half_step(got.dtype) if got.dtype in TYPES else bound
    got = got.to(D)
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), what
    over = (got - want).abs() / bound.clamp(min=1e-300)
    over = torch.where((got - want) == 0, 0.0, over)
    worst = float(over.max()) if over.numel() else 0.0
    assert worst <= 1.0, (what, "largest error / bound", worst)


# ---- norms around a gated block --------------------------------------------------------------------
def norm_inputs(rows, d, dtype, kind, per, seed, shifts=True):
    g = gen(seed)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)
    gates = 1 if per is None or per >= rows else -(-rows // per)
    s = dict(x=3 * r(rows, d) + .3, y=2 * r(rows, d) - .5, dh=r(rows, d), dn=r(rows, d), gate=.5 + .3 * r(gates, d), post_g=1 + .2 * r(d), post_s=.1 * r(d),
             pre_g=1 + .2 * r(d), pre_s=.1 * r(d))
    s = {k: v.to(dtype) for k, v in s.items()}
    s["post"], s["pre"] = (s["post_g"], s["post_s"] if shifts else None), (s["pre_g"], s["pre_s"] if shifts else None)
    return s


def wide(v):
    return None if v is None else tuple(wide(x) for x in v) if isinstance(v, tuple) else v.to(D)


def row_terms(a, kind):
    """Per row: (largest + mean) magnitude over the deviation, what an error of the statistics is measured in."""
    n, mean, rstd = R.norm(a, kind, 1e-5)
    return (a.abs().amax(1, keepdim=True) + a.abs().mean(1, keepdim=True)) * rstd


def check_forward(rows, d, dtype, kind, per, resid, parts, seed, ld=None, shift=0, in_place=False):
    s = norm_inputs(rows, d, dtype, kind, per, seed, "s" in parts)
    post, gate, pre = s["post"] if "p" in parts else None, s["gate"] if "g" in parts else None, s["pre"] if "n" in parts else None
    with_y = "y" in parts
    x, ux = guarded(rows, d, dtype, s["x"], ld, shift)
    y, uy = guarded(rows, d, dtype, s["y"], ld, shift) if with_y else (None, lambda: True)
    h, uh = (x, ux) if in_place else guarded(rows, d, dtype, None, ld, shift)
    n, un = (y, uy) if in_place else guarded(rows, d, dtype, None, ld, shift)
    if not with_y:
        h, uh = None, ux
    stats = torch.full((rows, 4), GUARD, device=DEV)
    A.nmt_op_gated_norm_fwd(x, y, h, n if pre else None, stats, post=post, gate=gate, pre=pre, kind=kind, rows_per_gate=per, resid_scale=resid)
    torch.cuda.synchronize()
    X, Y = s["x"].to(D), s["y"].to(D) if with_y else None
    want_h, want_n = R.gated_norm(X, Y, wide(post), wide(gate), wide(pre), kind, per, resid)
    u = half_step(dtype)
    zero = torch.zeros(rows, d, dtype=D, device=DEV)
    mag = zero
    if with_y:
        G = torch.ones_like(zero) if gate is None else R.gates_of(gate.to(D), rows, per or rows).abs()
        z = Y.abs() if post is None else post[0].to(D).abs() * row_terms(Y, kind) + (post[1].to(D).abs() if post[1] is not None else 0)
        mag = abs(resid) * X.abs() + G * z
        within(h, want_h, u * want_h.abs() + 64 * U32 * mag, "h")
    if pre:
        rstd = R.norm(want_h, kind, 1e-5)[2]
        # an error of h moves h's normalised value by its own size over the deviation, and that of the whole row through the statistics
        moved = row_terms(want_h, kind) + 2 * (mag.amax(1, keepdim=True) if with_y else 0) * rstd * (1 + R.norm(want_h, kind, 1e-5)[0].abs())
        bound = u * want_n.abs() + 64 * U32 * (pre[0].to(D).abs() * moved + (pre[1].to(D).abs() if pre[1] is not None else 0))
        within(n, want_n, bound, "n")
    assert ux() and uy() and uh() and un()
    for col, a, there in ((0, Y, post is not None), (2, want_h, pre is not None)):
        if there:
            _, mean, rstd = R.norm(a, kind, 1e-5)
            size = a.abs().amax(1, keepdim=True) + (mag.amax(1, keepdim=True) if col and with_y else 0)
            within(stats[:, col:col + 1], mean, 64 * U32 * size + 1e-30, "mean")
            within(stats[:, col + 1:col + 2], rstd, rstd * (64 * U32 * (1 + 4 * (size * rstd) ** 2)), "rstd")
        else:
            assert (stats[:, col] == 0).all() and (stats[:, col + 1] == 1).all()


WIDTHS = [1, 7, 64, 100, 128, 129, 512, 520, 777, 1024, 1030, 2048, 2056, 4096, 5000, 8192, 9000, 16384]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_gated_norm_forward_of_any_width(d, dtype):
    if d == 1:      # (LayerNorm of one column is 0 / sqrt(eps) and nothing but its shift)
        check_forward(19, 1, dtype, "rms", None, 0.9, "ypgns", 3)
        return
    for kind, rows, per in (("layer", 37, None), ("rms", 21, 1), ("layer", 33, 5)):
        check_forward(rows, d, dtype, kind, per, 0.9, "ypgns", d)


@pytest.mark.parametrize("parts", ["y", "yp", "ypg", "yg", "yn", "ypgn", "ypn", "n", "ns", "ygns", "yps"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_gated_norm_forward_with_any_of_its_parts(parts, kind):
    check_forward(50, 256, F16, kind, 7, 1.0, parts, 5)


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 64, 65, 4097, 9001])
def test_gated_norm_forward_of_any_number_of_rows(rows):
    check_forward(rows, 64, F16, "layer", None, 1.0, "ypgns", rows)
    check_forward(rows, 640, BF16, "rms", 27, 2.5, "ypgn", rows)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,ld,shift", [(64, 65, 1), (100, 131, 3), (512, 777, 5), (1024, 1025, 7), (2049, 2051, 1)])
def test_gated_norm_forward_of_rows_anywhere(d, ld, shift, dtype):
    check_forward(23, d, dtype, "layer", None, 1.0, "ypgns", 1, ld, shift)
    check_forward(23, d, dtype, "rms", 4, 1.0, "ypgns", 1, ld, shift, in_place=True)


@pytest.mark.parametrize("d", [530, 700, 1030, 1600, 2500, 5000, 9000])
@pytest.mark.parametrize("parts", ["y", "yg", "yp", "yn"])
def test_gated_norm_forward_in_place_of_its_inputs(d, parts):
    """Rows held by several wavefronts, some of whose lanes take the same columns."""
    check_forward(300, d, F16, "rms", 9, 0.9, parts, d, in_place=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d", [(32769 * 4, 5), (65600, 64), (65537, 50), (32801, 100), (16387, 256), (8193, 512), (8195, 300), (4097, 1024), (4099, 1030), (2049, 2048), (2051, 1500), (1027, 4000),
                                    (1025, 4096), (515, 8192), (513, 5000), (515, 9000), (517, 16384)])
def test_gated_norm_forward_of_two_rows_a_worker(rows, d, dtype):
    """The second row is in flight while the first is worked on, in place of its inputs too; an odd number leaves the last worker one."""
    check_forward(rows, d, dtype, "layer", None, 0.9, "ypgns", d, in_place=True)
    check_forward(rows, d, dtype, "rms", 7, 1.0, "ypgn", d + 1)


@pytest.mark.parametrize("rows,d,dtype", [(530001, 64, F16), (270001, 127, BF16), (140001, 125, F32), (33001, 1030, BF16), (22001, 777, F32), (8301, 4100, F16), (2101, 8200, F32), (2101, 16384, BF16)])
def test_gated_norm_forward_past_the_caches(rows, d, dtype):
    """Results of 64 MB and more, in place and apart, rows of whole vectors and others."""
    assert rows * d * dtype.itemsize >= 64 << 20
    check_forward(rows, d, dtype, "layer", None, 0.9, "ypgns", d)
    check_forward(rows, d, dtype, "rms", 27, 0.9, "ypgn", d, in_place=True)
    check_forward(rows, d, dtype, "layer", None, 0.9, "yg", d, in_place=True)
    check_forward(rows, d, dtype, "layer", None, 1.0, "ns", d)


def check_backward(rows, d, dtype, kind, per, resid, parts, seed, ld=None, shift=0, in_place=False):
    s = norm_inputs(rows, d, dtype, kind, per, seed, "s" in parts)
    post, gate, pre = s["post"] if "p" in parts else None, s["gate"] if "g" in parts else None, s["pre"] if "n" in parts else None
    with_y, with_dh = "y" in parts, "h" in parts
    H, Y = s["x"].to(D), s["y"].to(D)
    stats = torch.tensor([0., 1., 0., 1.], dtype=D, device=DEV).repeat(rows, 1)
    if post and with_y:
        stats[:, 0:2] = torch.cat(R.norm(Y, kind, 1e-5)[1:], 1)
    if pre:
        stats[:, 2:4] = torch.cat(R.norm(H, kind, 1e-5)[1:], 1)
    h, _ = guarded(rows, d, dtype, s["x"], ld, shift)
    y, _ = guarded(rows, d, dtype, s["y"], ld, shift) if with_y else (None, None)
    dh, ud = guarded(rows, d, dtype, s["dh"], ld, shift) if with_dh else (None, lambda: True)
    dn, un = guarded(rows, d, dtype, s["dn"], ld, shift) if pre else (None, lambda: True)
    dx, ux = (dh, ud) if in_place and with_dh else guarded(rows, d, dtype, None, ld, shift)
    dy, uy = ((dn, un) if in_place and pre else guarded(rows, d, dtype, None, ld, shift)) if with_y else (None, lambda: True)
    like = lambda v: None if v is None else torch.full_like(v, GUARD)
    dpost, dgate, dpre = (like(post[0]), like(post[1])) if post else None, like(gate), (like(pre[0]), like(pre[1])) if pre else None
    scratch = torch.full((A.nmt_op_gated_norm_bwd_scratch(rows, d, per if gate is not None else None),), float("nan"), device=DEV)
    A.nmt_op_gated_norm_bwd(dh, dn, y, h, stats.float(), dx, dy, scratch, post=post, gate=gate, pre=pre, dpost=dpost, dgate=dgate, dpre=dpre, kind=kind,
                            rows_per_gate=per if gate is not None else None, resid_scale=resid)
    torch.cuda.synchronize()
    # the formula, and the magnitudes of its terms
    u, layer = half_step(dtype), kind == "layer"
    mean = lambda a: a.mean(1, keepdim=True)
    zero = torch.zeros(rows, d, dtype=D, device=DEV)
    G, size = (s["dh"].to(D), s["dh"].to(D).abs()) if with_dh else (zero, zero)
    if pre:
        hh, mu, r = (H - stats[:, 2:3]) * stats[:, 3:4], stats[:, 2:3], stats[:, 3:4]
        hs = row_terms(H, kind)                                     # (what a rounding of h - mean is, in deviations)
        t = s["dn"].to(D) * pre[0].to(D)
        G = G + r * (t - (mean(t) if layer else 0) - hh * mean(t * hh))
        size = size + r * (t.abs() + mean(t.abs()) * (1 + hs) + hs * mean(t.abs() * hs))
    within(dx, resid * G, u * (resid * G).abs() + 64 * U32 * abs(resid) * size, "dx")
    if with_y:
        yh, ys = (Y - stats[:, 0:1]) * stats[:, 1:2], row_terms(Y, kind) if post else Y.abs()
        gt = torch.ones_like(zero) if gate is None else R.gates_of(gate.to(D), rows, per or rows)
        dz, zs = gt * G, gt.abs() * size
        want, ws = dz, zs
        if post:
            r, t, ts = stats[:, 1:2], dz * post[0].to(D), zs * post[0].to(D).abs()
            want = r * (t - (mean(t) if layer else 0) - yh * mean(t * yh))
            ws = r * (ts + mean(ts) * (1 + ys) + ys * mean(ts * ys))
        within(dy, want, u * want.abs() + 64 * U32 * ws, "dy")
    # sums over rows: at most 512 additions in a row at these sizes, of terms as exact as the above
    sums = lambda got, terms, sizes, what: within(got, terms.sum(0), u * terms.sum(0).abs() + 576 * U32 * sizes.sum(0), what)
    if post and with_y:
        sums(dpost[0], dz * yh, zs * (1 + ys), "gain after")
        if post[1] is not None:
            sums(dpost[1], dz, zs, "shift after")
    if pre:
        a = s["dn"].to(D)
        sums(dpre[0], a * hh, a.abs() * (1 + hs), "gain before")
        if pre[1] is not None:
            sums(dpre[1], a, a.abs(), "shift before")
    if gate is not None:
        z, zz = (Y, Y.abs()) if post is None else (yh * post[0].to(D) + (0 if post[1] is None else post[1].to(D)),
                                                   ys * post[0].to(D).abs() + (0 if post[1] is None else post[1].to(D).abs()))
        of = torch.arange(rows, device=DEV) // (per or rows)
        gathered = lambda a: torch.zeros(gate.shape[0], d, dtype=D, device=DEV).index_add_(0, of, a)
        within(dgate, gathered(G * z), u * gathered(G * z).abs() + 576 * U32 * gathered(size * zz), "gate")
    assert ud() and un() and ux() and uy()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", WIDTHS[1:])
def test_gated_norm_backward_of_any_width(d, dtype):
    for kind, rows, per in (("layer", 37, None), ("rms", 21, 1), ("layer", 33, 5)):
        check_backward(rows, d, dtype, kind, per, 0.9, "yhpgns", d)


@pytest.mark.parametrize("parts", ["yh", "yhp", "yhpg", "yhg", "yn", "ypgn", "yhpn", "n", "hns", "ygns", "yhps"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_gated_norm_backward_with_any_of_its_parts(parts, kind):
    check_backward(50, 256, F16, kind, 7, 1.0, parts, 5)


@pytest.mark.parametrize("rows,per", [(1, None), (1, 1), (2, 1), (15, 4), (16, 16), (17, 16), (65, 64), (4097, None), (4097, 1), (4097, 2), (4097, 100), (9001, 27),
                                      (9001, 8999), (9001, 9001), (9001, 10 ** 6), (20011, 3), (20011, 6000)])
def test_gated_norm_backward_of_any_rows_and_gates(rows, per):
    check_backward(rows, 64, F16, "layer", per, 1.0, "yhpgns", rows)
    check_backward(rows, 648, BF16, "rms", per, 2.5, "yhpgn", rows)


@pytest.mark.parametrize("rows,d,per", [(26001, 1024, 27), (26001, 1024, 40), (26001, 1024, 52), (26001, 1024, 53), (3584, 512, 7), (3584, 512, 15), (52000, 64, 13), (52000, 64, 15),
                                        (2001, 8192, 16), (2001, 8192, 17)])
def test_gated_norm_backward_of_gates_on_both_sides_of_a_run(rows, d, per):
    """Rows a gate up to twice a worker's run, which is then rounded to whole gates, and beyond, where two workers share a gate.  A sum has less than 128 additions in a row."""
    check_backward(rows, d, F16, "layer", per, 0.9, "yhpgns", per)
    check_backward(rows, d, BF16, "rms", per, 0.9, "yhpgn", per, in_place=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,ld,shift", [(64, 65, 1), (100, 131, 3), (512, 777, 5), (1024, 1025, 7), (2049, 2051, 1)])
def test_gated_norm_backward_of_rows_anywhere(d, ld, shift, dtype):
    check_backward(23, d, dtype, "layer", None, 1.0, "yhpgns", 1, ld, shift)
    check_backward(23, d, dtype, "rms", 4, 1.0, "yhpgns", 1, ld, shift, in_place=True)


@pytest.mark.parametrize("d", [530, 700, 1030, 1600, 2500, 5000, 9000])
@pytest.mark.parametrize("parts", ["yh", "yhg", "yhp", "yhn", "hn"])
def test_gated_norm_backward_in_place_of_its_inputs(d, parts):
    check_backward(300, d, F16, "rms", 9, 0.9, parts, d, in_place=True)
    check_backward(300, d, F32, "layer", 9, 0.9, parts, d, in_place=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [8193, 10007, 12288, 12289, 14000, 16384])
def test_gated_norm_of_very_wide_rows(d, dtype):
    """Some of the column sums are in LDS; more rows than work-groups, gates that two of those share, in place and apart."""
    for parts, per, kind, place in (("yhpgns", 700, "layer", False), ("yhpgns", 7, "rms", True), ("yhpgn", None, "layer", True), ("hns", None, "rms", False),
                                    ("yhps", None, "layer", False), ("yhg", 3, "rms", True)):
        check_backward(530, d, dtype, kind, per, 0.9, parts, d, in_place=place)
    check_backward(5, d, dtype, "layer", 2, 1.0, "yhpgns", 1, d + 3, 1)
    check_forward(300, d, dtype, "layer", 9, 0.9, "ypgns", d, in_place=True)


def test_gated_norm_scratch_serves_fewer_rows():
    for d in (64, 512, 777, 1024, 2048, 8192):
        for per in (None, 7):
            sizes = [A.nmt_op_gated_norm_bwd_scratch(n, d, per) for n in (1, 10, 63, 500, 1023, 1024, 1025, 4096, 4097, 50000, 10 ** 6)]
            assert sizes == sorted(sizes)
    check_backward(1023, 64, F16, "rms", 7, 1.0, "yhpgns", 1)


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_gated_norm_gradients_are_the_differences_of_its_values(kind):
    """Central differences along a random direction, in fp32.  The outputs' roundings, U32 of some 3 each over 64 * 96 * 2 of them, weigh 2 sqrt(12288) 3 U32 / (2 eps) at
    random signs, and eps^2 / 6 times the third derivative (of the size of the value itself): together below 2e-3 of the gradient's norm at eps = 2^-7."""
    rows, d, per, eps = 64, 96, 9, 2.0 ** -7
    s = {k: v for k, v in norm_inputs(rows, d, F32, kind, per, 11).items() if torch.is_tensor(v)}
    names = ["x", "y", "gate", "post_g", "post_s", "pre_g", "pre_s"]
    g = gen(12)
    way = {k: torch.randn(s[k].shape, generator=g, device=DEV) for k in names}

    def forward(p):
        h, n, stats = torch.empty(rows, d, device=DEV), torch.empty(rows, d, device=DEV), torch.empty(rows, 4, device=DEV)
        A.nmt_op_gated_norm_fwd(p["x"], p["y"], h, n, stats, post=(p["post_g"], p["post_s"]), gate=p["gate"], pre=(p["pre_g"], p["pre_s"]), kind=kind,
                                rows_per_gate=per, resid_scale=0.9)
        return h, n, stats

    value = lambda p: sum((a.to(D) * b.to(D)).sum() for a, b in zip(forward(p)[:2], (s["dh"], s["dn"])))
    h, _, stats = forward(s)
    out = {k: torch.empty_like(s[k]) for k in names}
    scratch = torch.empty(A.nmt_op_gated_norm_bwd_scratch(rows, d, per), device=DEV)
    A.nmt_op_gated_norm_bwd(s["dh"], s["dn"], s["y"], h, stats, out["x"], out["y"], scratch, post=(s["post_g"], s["post_s"]), gate=s["gate"],
                            pre=(s["pre_g"], s["pre_s"]), dpost=(out["post_g"], out["post_s"]), dgate=out["gate"], dpre=(out["pre_g"], out["pre_s"]), kind=kind,
                            rows_per_gate=per, resid_scale=0.9)
    for k in names:
        moved = lambda e: {**s, k: s[k] + e * way[k]}
        slope = float((value(moved(eps)) - value(moved(-eps))) / (2 * eps))
        want = float((out[k].to(D) * way[k].to(D)).sum())
        assert abs(slope - want) <= 2e-3 * float(out[k].norm() * way[k].norm()) / way[k].numel() ** 0.5 + 2e-3, (k, slope, want)


def norm_alone(x, a, dtype, kind, s):
    """Gradient at x of h = a x and n = pre(h), from the library: the caller forms h, which is a product by a power of two and exact."""
    h = a * x
    n, stats, dx = torch.empty_like(h), torch.empty(*h.shape[:1], 4, device=DEV), torch.empty_like(h)
    A.nmt_op_gated_norm_fwd(h, None, None, n, stats, pre=s["pre"], kind=kind)
    scratch = torch.empty(A.nmt_op_gated_norm_bwd_scratch(*h.shape), device=DEV)
    A.nmt_op_gated_norm_bwd(s["dh"], s["dn"], None, h, stats, dx, None, scratch, pre=s["pre"], kind=kind, resid_scale=a)
    return dx


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("d", [64, 777, 2056, 9000])
def test_gradient_of_a_norm_without_a_block(d, kind, dtype):
    """Against the derivative, in 64 bits, of the plain form.  The statistics are the forward call's, off by up to 64 U32 of a row's terms over its deviation: once in the factor
    of all terms, twice in the normalised values; with the 64 U32 of the backward pass itself 256 U32 of the magnitudes."""
    s = norm_inputs(37, d, dtype, kind, None, d)
    for a in (1.0, 2.0):
        X = s["x"].to(D).requires_grad_()
        H, N = R.gated_norm(a * X, pre=wide(s["pre"]), kind=kind)
        ((H * s["dh"].to(D)).sum() + (N * s["dn"].to(D)).sum()).backward()
        H, t = H.detach(), (s["dn"].to(D) * s["pre"][0].to(D)).abs()
        hs, r = row_terms(H, kind), R.norm(H, kind, 1e-5)[2]
        mean = lambda v: v.mean(1, keepdim=True)
        size = s["dh"].to(D).abs() + r * hs * (t + mean(t) * (1 + hs) + hs * mean(t * hs))
        within(norm_alone(s["x"], a, dtype, kind, s), X.grad, half_step(dtype) * X.grad.abs() + 256 * U32 * a * size, f"dx, {a} x")


def test_gated_norm_keeps_rows_apart():
    """Infinities and NaN in one row reach that row's outputs alone."""
    s = norm_inputs(40, 512, F16, "layer", None, 2)
    def run():
        h, n, stats = torch.empty_like(s["x"]), torch.empty_like(s["x"]), torch.empty(40, 4, device=DEV)
        A.nmt_op_gated_norm_fwd(s["x"], s["y"], h, n, stats, post=s["post"], gate=s["gate"], pre=s["pre"])
        dx, dy = torch.empty_like(h), torch.empty_like(h)
        scratch = torch.empty(A.nmt_op_gated_norm_bwd_scratch(40, 512), device=DEV)
        A.nmt_op_gated_norm_bwd(s["dh"], s["dn"], s["y"], h, stats, dx, dy, scratch, post=s["post"], gate=s["gate"], pre=s["pre"])
        return h, n, dx, dy
    clean = run()
    s["x"][3, 7], s["y"][11, 500], s["dn"][20, 0] = float("nan"), float("inf"), float("-inf")
    dirty = run()
    keep = torch.ones(40, dtype=torch.bool, device=DEV)
    keep[[3, 11, 20]] = False
    for a, b in zip(clean, dirty):
        assert torch.equal(a[keep], b[keep])
    assert not torch.isfinite(dirty[1][3]).any() and not torch.isfinite(dirty[1][11]).any() and not torch.isfinite(dirty[2][20]).any()


def test_gated_norm_of_constant_rows():
    """No variance: eps alone under the root, no division by zero."""
    y = torch.full((5, 256), 3.0, dtype=F16, device=DEV)
    h, n, stats = torch.empty_like(y), torch.empty_like(y), torch.empty(5, 4, device=DEV)
    one, zero = torch.ones(256, dtype=F16, device=DEV), torch.zeros(5, 256, dtype=F16, device=DEV)
    A.nmt_op_gated_norm_fwd(zero, y, h, n, stats, post=(one, None), pre=(one, one), kind="layer")
    assert (h == 0).all() and (n == 1).all() and (stats[:, 0] == 3).all()
    A.nmt_op_gated_norm_fwd(zero, torch.zeros_like(y), h, n, stats, post=(one, None), pre=(one, None), kind="rms")
    assert (h == 0).all() and (n == 0).all() and torch.isfinite(stats).all()


def test_gated_norm_of_no_rows_leaves_zero_gradients():
    e = torch.empty(0, 64, dtype=F16, device=DEV)
    v = [torch.full((64,), GUARD, dtype=F16, device=DEV) for _ in range(4)]
    gate, dgate = torch.ones(1, 64, dtype=F16, device=DEV), torch.full((1, 64), GUARD, dtype=F16, device=DEV)
    one = torch.ones(64, dtype=F16, device=DEV)
    stats = torch.empty(0, 4, device=DEV)
    A.nmt_op_gated_norm_fwd(e, e, e, e, stats, post=(one, one), gate=gate, pre=(one, one))
    A.nmt_op_gated_norm_bwd(e, e, e, e, stats, e, e, None, post=(one, one), gate=gate, pre=(one, one), dpost=v[:2], dgate=dgate, dpre=v[2:])
    torch.cuda.synchronize()
    assert all((x == 0).all() for x in v) and (dgate == 0).all()


@pytest.mark.parametrize("per,gates", [(1, 0), (27, 0), (27, 1), (None, 1), (None, 0)])
def test_gated_norm_of_no_rows_leaves_what_lies_behind_its_gates(per, gates):
    """The gradient of no gates is an empty stretch of a larger buffer; that of the one that all rows share is zero."""
    e, one, stats = torch.empty(0, 64, dtype=F16, device=DEV), torch.ones(64, dtype=F16, device=DEV), torch.empty(0, 4, device=DEV)
    flat = torch.full((320,), GUARD, dtype=F16, device=DEV)
    dgate, v = flat[128:128 + 64 * gates].view(gates, 64), [torch.full((64,), GUARD, dtype=F16, device=DEV) for _ in range(4)]
    a = dict(post=(one, one), gate=torch.ones(gates, 64, dtype=F16, device=DEV), pre=(one, one), rows_per_gate=per)
    A.nmt_op_gated_norm_fwd(e, e, e, e, stats, **a)
    A.nmt_op_gated_norm_bwd(e, e, e, e, stats, e, e, None, dpost=v[:2], dgate=dgate, dpre=v[2:], **a)
    torch.cuda.synchronize()
    assert all((x == 0).all() for x in v) and (dgate == 0).all()
    assert (flat[:128] == GUARD).all() and (flat[128 + 64 * gates:] == GUARD).all()


def test_gated_norm_of_rows_more_than_32_bits_apart():
    """Rows 2^30 + 5 elements apart: the third begins behind 2^31 elements."""
    ld, d = 2 ** 30 + 5, 520
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    s = norm_inputs(3, d, F16, "layer", None, 9)
    far = lambda t: torch.empty(2 * ld + d, dtype=F16, device=DEV).as_strided((3, d), (ld, 1)).copy_(t) if t is not None else \
        torch.empty(2 * ld + d, dtype=F16, device=DEV).as_strided((3, d), (ld, 1))
    x, y, h = far(s["x"]), far(s["y"]), far(None)
    n, n2, h2 = torch.empty(3, d, dtype=F16, device=DEV), torch.empty(3, d, dtype=F16, device=DEV), torch.empty(3, d, dtype=F16, device=DEV)
    A.nmt_op_gated_norm_fwd(x, y, h, n, None, post=s["post"], gate=s["gate"], pre=s["pre"])
    A.nmt_op_gated_norm_fwd(s["x"], s["y"], h2, n2, None, post=s["post"], gate=s["gate"], pre=s["pre"])
    assert torch.equal(h, h2) and torch.equal(n, n2)
    stats = torch.zeros(3, 4, device=DEV)
    A.nmt_op_gated_norm_fwd(s["x"], s["y"], h2, n2, stats, post=s["post"], gate=s["gate"], pre=s["pre"])
    grads = []
    for yy, hh, ddx in ((y, h, x), (s["y"], h2, torch.empty_like(h2))):
        ddy = torch.empty_like(h2)
        scratch = torch.empty(A.nmt_op_gated_norm_bwd_scratch(3, d), device=DEV)
        A.nmt_op_gated_norm_bwd(s["dh"], s["dn"], yy, hh, stats, ddx, ddy, scratch, post=s["post"], gate=s["gate"], pre=s["pre"])
        grads.append((ddx.clone(), ddy))
    assert torch.equal(grads[0][0], grads[1][0]) and torch.equal(grads[0][1], grads[1][1])


# ---- tokens to their experts and back -----------------------------------------------------------------
def choices(tokens, k, experts, seed, dropped=0.0, skew=1.0):
    g = gen(seed)
    p = torch.exp(skew * torch.randn(experts, generator=g, device=DEV))
    ids = torch.multinomial(p.expand(max(tokens, 1), experts), k, replacement=True, generator=g).int()[:tokens]
    if dropped:
        lost = torch.rand(ids.shape, generator=g, device=DEV) < dropped
        ids = torch.where(lost, torch.where(torch.rand(ids.shape, generator=g, device=DEV) < .5, -1, experts).int(), ids)
    return ids.contiguous()


def dispatched(ids, experts, capacity, x=None, rows=None):
    T, k = ids.shape
    i = lambda *s: torch.full(s, -77, dtype=torch.int32, device=DEV)
    slot, ranges, scratch = i(T, k), i(experts, 2), i(A.nmt_op_expert_dispatch_scratch(T, k, experts))
    A.nmt_op_expert_dispatch(ids, experts, capacity, x, rows, slot, ranges, scratch)
    return slot, ranges


SORTS = [(1, 1, 1, 0), (1, 2, 8, 0), (5, 2, 8, 0), (7, 3, 3, 2), (64, 1, 64, 0), (65, 2, 256, 1), (130, 2, 1000, 1), (1000, 4, 16, 100), (1024, 1, 2, 0), (1025, 2, 1024, 0),
         (3584, 2, 16, 560), (3585, 2, 17, 0), (5000, 8, 128, 0), (8191, 2, 5, 0), (8193, 2, 5, 1000), (9000, 2, 33, 0), (20000, 8, 256, 600), (70001, 1, 7, 0), (300, 64, 9, 0)]


@pytest.mark.parametrize("tokens,k,experts,capacity", SORTS)
def test_dispatch_sorts(tokens, k, experts, capacity):
    for seed, dropped, skew in ((1, 0.0, 0.5), (2, 0.2, 2.0)):
        ids = choices(tokens, k, experts, seed, dropped, skew)
        slot, ranges = dispatched(ids, experts, capacity)
        want_slot, want_ranges = R.dispatch(ids.cpu(), experts, capacity)
        assert torch.equal(ranges.cpu(), want_ranges)
        assert torch.equal(slot.cpu(), want_slot)


@pytest.mark.parametrize("capacity", [0, 3])
def test_dispatch_of_one_sided_choices(capacity):
    """Everything to one expert, to the last one, to none; ids far outside; the same expert twice."""
    for experts in (1, 8, 300):
        for ids in (torch.zeros(500, 2), torch.full((500, 2), experts - 1), torch.full((500, 2), -1), torch.full((500, 2), 2 ** 31 - 1),
                    torch.full((500, 2), -2 ** 31), torch.full((9000, 1), experts - 1)):
            ids = ids.to(torch.int64).to(torch.int32).to(DEV)
            x = torch.randn(ids.shape[0], 24, device=DEV).half()
            rows = torch.full((experts * capacity or ids.numel(), 24), GUARD, dtype=F16, device=DEV)
            slot, ranges = dispatched(ids, experts, capacity, x, rows)
            want_slot, want_ranges = R.dispatch(ids.cpu(), experts, capacity)
            assert torch.equal(ranges.cpu(), want_ranges) and torch.equal(slot.cpu(), want_slot)
            check_rows(rows, x, slot, capacity)


def check_rows(rows, x, slot, capacity):
    want = torch.full_like(rows, 0.0 if capacity else GUARD)       # (rows behind the last are left as they were)
    k, flat = slot.shape[1], slot.reshape(-1)
    took = (flat >= 0).nonzero().reshape(-1)
    want[flat[took].long()] = x[took // k]
    assert torch.equal(rows, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,k,experts,capacity,d", [(1, 1, 1, 0, 1), (1, 2, 8, 0, 512), (37, 2, 8, 0, 64), (37, 2, 8, 12, 100), (129, 4, 16, 40, 777), (1000, 2, 300, 9, 1024),
                                                         (511, 8, 32, 0, 2056), (50, 2, 4, 0, 6000), (3000, 1, 4, 800, 24), (0, 2, 8, 5, 64), (0, 2, 8, 0, 64)])
def test_tokens_go_to_their_experts_and_back(tokens, k, experts, capacity, d, dtype):
    g = gen(tokens + d)
    ids = choices(tokens, k, experts, d, 0.1)
    n = experts * capacity if capacity else tokens * k
    x, ux = guarded(tokens, d, dtype, torch.randn(tokens, d, generator=g, device=DEV), d + 3, 1)
    rows, ur = guarded(n, d, dtype, torch.full((n, d), GUARD, device=DEV), d + 5, 3)
    slot, ranges = dispatched(ids, experts, capacity, x, rows)
    want_slot, want_ranges = R.dispatch(ids.cpu(), experts, capacity)
    assert torch.equal(ranges.cpu(), want_ranges) and torch.equal(slot.cpu(), want_slot)
    check_rows(rows, x, slot, capacity)
    assert ux() and ur()
    # back, weighted; each product and each sum rounds once: (k + 1) U32 of the magnitudes
    made, _ = guarded(n, d, dtype, torch.randn(n, d, generator=g, device=DEV), d + 1, 5)
    weights = torch.rand(tokens, k, generator=g, device=DEV)
    add, _ = guarded(tokens, d, dtype, torch.randn(tokens, d, generator=g, device=DEV), d + 2, 1)
    u = half_step(dtype)
    for w, a in ((weights, None), (None, None), (weights, add)):
        out, uo = guarded(tokens, d, dtype, None, d + 7, 1)
        A.nmt_op_expert_combine(made, slot, w, out, add=a)
        want = R.combine(made, slot, w, a)
        size = R.combine(made.abs(), slot, None if w is None else w.abs(), None if a is None else a.abs())
        within(out, want, u * want.abs() + (k + 2) * U32 * size, "out")
        assert uo()
    A.nmt_op_expert_combine(made, slot, weights, add, add=add)      # (in place)
    assert torch.equal(add, out)
    # gradients
    dout, _ = guarded(tokens, d, dtype, torch.randn(tokens, d, generator=g, device=DEV), d + 4, 1)
    drows, ur = guarded(n, d, dtype, torch.full((n, d), GUARD, device=DEV), d + 6, 1)
    dweights = torch.full((tokens, k), GUARD, device=DEV)
    A.nmt_op_expert_combine_bwd(dout, made, slot, weights, drows, dweights, ranges, capacity)
    want = torch.full((n, d), 0.0 if capacity else GUARD, dtype=D, device=DEV)
    flat = slot.reshape(-1)
    took = (flat >= 0).nonzero().reshape(-1)
    want[flat[took].long()] = weights.reshape(-1)[took].to(D)[:, None] * dout.to(D)[took // k]
    within(drows, want, (u + 2 * U32) * want.abs(), "drows")
    dw, size = torch.zeros(tokens * k, dtype=D, device=DEV), torch.zeros(tokens * k, dtype=D, device=DEV)
    terms = dout.to(D)[took // k] * made.to(D)[flat[took].long()]
    dw[took], size[took] = terms.sum(1), terms.abs().sum(1)
    chain = -(-d // 64) + 64                                         # additions in a lane (at worst one column in 64), then across lanes
    within(dweights.reshape(-1), dw, chain * U32 * size, "dweights")
    assert ur()
    plain = torch.full((n, d), GUARD, dtype=dtype, device=DEV)       # without weights and their gradient
    A.nmt_op_expert_combine_bwd(dout, None, slot, None, plain, None, ranges, capacity)
    check_rows(plain, dout, slot, capacity)
    if tokens:                                                       # in place of the experts' rows
        A.nmt_op_expert_combine_bwd(dout, made, slot, weights, made, dweights, ranges, capacity)
        assert torch.equal(made[flat[took].long()], drows[flat[took].long()])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,k,experts,capacity,d", [(1, 8, 64, 0, 8192), (1, 1, 2, 0, 2049), (3, 5, 8, 0, 4099), (17, 2, 8, 40, 2057), (2, 64, 9, 0, 4100), (40, 3, 5, 7, 20000),
                                                         (2200, 1, 7, 0, 2100), (8191, 2, 4, 0, 1111), (8192, 2, 4, 0, 1111), (8192, 1, 4, 2100, 2051)])
def test_few_tokens_of_wide_rows(tokens, k, experts, capacity, d, dtype):
    """Several wavefronts take a token; in place too, where rows of no whole number of vectors end in single elements."""
    test_tokens_go_to_their_experts_and_back(tokens, k, experts, capacity, d, dtype)
    g = gen(d)
    ids = choices(tokens, k, experts, d, 0.1)
    n = experts * capacity if capacity else tokens * k
    slot, ranges = dispatched(ids, experts, capacity)
    made, um = guarded(n, d, dtype, torch.randn(n, d, generator=g, device=DEV), d + 1, 1)
    dout, weights = torch.randn(tokens, d, generator=g, device=DEV).to(dtype), torch.rand(tokens, k, generator=g, device=DEV)
    first, dweights = torch.full((n, d), GUARD, dtype=dtype, device=DEV), torch.full((tokens, k), GUARD, device=DEV)
    flat = slot.reshape(-1)
    took = (flat >= 0).nonzero().reshape(-1)
    terms = dout.to(D)[took // k] * made.to(D)[flat[took].long()]
    A.nmt_op_expert_combine_bwd(dout, None, slot, weights, first, None, ranges, capacity)
    A.nmt_op_expert_combine_bwd(dout, made, slot, weights, made, dweights, ranges, capacity)
    assert torch.equal(made[flat[took].long()], first[flat[took].long()])
    dw, size = torch.zeros(tokens * k, dtype=D, device=DEV), torch.zeros(tokens * k, dtype=D, device=DEV)
    dw[took], size[took] = terms.sum(1), terms.abs().sum(1)
    within(dweights.reshape(-1), dw, (-(-d // 64) + 64) * U32 * size, "dweights in place")     # (additions in a lane, then across lanes)
    assert um()


@pytest.mark.parametrize("tokens,k,experts,capacity,d", [(8, 2, 64, 512, 1024), (0, 1, 3, 5000, 777), (300, 2, 8, 4000, 100), (1, 1, 1024, 64, 8), (16384, 1, 16, 3000, 64)])
def test_much_room_for_few_tokens(tokens, k, experts, capacity, d):
    """Rows that no token took are set to zero by more work-groups than there are choices for."""
    g = gen(d)
    ids = choices(tokens, k, experts, 5, 0.1)
    x = torch.randn(tokens, d, generator=g, device=DEV).half()
    rows, ur = guarded(experts * capacity, d, F16, torch.full((experts * capacity, d), GUARD, device=DEV), d + 3, 1)
    slot, ranges = dispatched(ids, experts, capacity, x, rows)
    want_slot, want_ranges = R.dispatch(ids.cpu(), experts, capacity)
    assert torch.equal(ranges.cpu(), want_ranges) and torch.equal(slot.cpu(), want_slot)
    check_rows(rows, x, slot, capacity)
    assert ur()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,k,experts,capacity,d", [(16385, 1, 16, 0, 1), (8200, 2, 8, 0, 64), (8193, 2, 16, 1200, 100), (9000, 2, 300, 0, 41), (9001, 2, 300, 70, 100),
                                                         (20000, 1, 1024, 0, 24), (4100, 4, 7, 3000, 777), (300, 64, 9, 0, 2056), (260, 64, 500, 50, 4100), (17000, 1, 3, 6000, 520)])
def test_many_tokens_go_to_their_experts_and_back(tokens, k, experts, capacity, d, dtype):
    """More choices than one launch takes: counts of segments, added up where they are used or by a scan, and rows copied by a launch of their own."""
    test_tokens_go_to_their_experts_and_back(tokens, k, experts, capacity, d, dtype)


@pytest.mark.parametrize("tokens,k,experts,capacity,d,dtype", [(25001, 2, 8, 0, 1030, F16), (25001, 2, 8, 7000, 1030, BF16), (13003, 4, 128, 0, 1024, F16), (24600, 1, 5, 0, 1027, F32),
                                                               (5000, 5, 64, 0, 2057, F16), (6200, 2, 3, 4500, 2052, F32), (8191, 3, 400, 0, 2051, BF16)])
def test_rows_past_the_caches_go_to_their_experts_and_back(tokens, k, experts, capacity, d, dtype):
    """96 MB of the experts' rows and more."""
    assert tokens * k * d * dtype.itemsize >= 96 << 20
    test_tokens_go_to_their_experts_and_back(tokens, k, experts, capacity, d, dtype)


@pytest.mark.parametrize("skew", ["all", "nine tenths"])
@pytest.mark.parametrize("capacity", [0, 500])
def test_many_one_sided_choices(capacity, skew):
    """One expert's list spans every segment."""
    T, k, E, d = 30000, 2, 12, 72
    ids = torch.full((T, k), 7, dtype=torch.int32, device=DEV)
    if skew != "all":
        ids = torch.where(torch.rand(T, k, generator=gen(3), device=DEV) < 0.9, ids, choices(T, k, E, 4, 0.1))
    x, rows = torch.randn(T, d, generator=gen(5), device=DEV).half(), torch.full((E * capacity or T * k, d), GUARD, dtype=F16, device=DEV)
    slot, ranges = dispatched(ids, E, capacity, x, rows)
    want_slot, want_ranges = R.dispatch(ids.cpu(), E, capacity)
    assert torch.equal(ranges.cpu(), want_ranges) and torch.equal(slot.cpu(), want_slot)
    check_rows(rows, x, slot, capacity)


def test_dropped_choices_weigh_nothing():
    """NaN weights of dropped choices, and NaN in rows that no token took, reach nothing; a token without an expert gets zeros."""
    ids = torch.tensor([[0, -1], [-1, -1], [1, 0], [0, 0]], dtype=torch.int32, device=DEV)
    slot, ranges = dispatched(ids, 2, 2)
    assert slot.tolist() == [[0, -1], [-1, -1], [2, 1], [-1, -1]] and ranges.tolist() == [[0, 2], [2, 1]]
    rows = torch.ones(4, 40, dtype=F16, device=DEV)
    rows[3] = float("nan")
    w = torch.tensor([[1.0, float("nan")], [float("inf")] * 2, [2.0, 3.0], [float("nan")] * 2], device=DEV)
    out = torch.empty(4, 40, dtype=F16, device=DEV)
    A.nmt_op_expert_combine(rows, slot, w, out)
    assert out[:, 0].tolist() == [1.0, 0.0, 5.0, 0.0] and (out == out[:, :1]).all()
    drows, dw = torch.full_like(rows, GUARD), torch.full((4, 2), GUARD, device=DEV)
    A.nmt_op_expert_combine_bwd(out, rows, slot, w, drows, dw, ranges, 2)
    assert dw.tolist() == [[40.0, 0.0], [0.0, 0.0], [200.0, 200.0], [0.0, 0.0]]
    assert drows[:, 0].tolist() == [1.0, 15.0, 10.0, 0.0]
    odd = torch.tensor([[7, 2 ** 31 - 1], [4, -5], [2, 3], [0, 1]], dtype=torch.int32, device=DEV)   # slots outside the rows are no slots
    A.nmt_op_expert_combine(rows[:3], odd, None, out)
    assert out[:, 0].tolist() == [0.0, 0.0, 1.0, 2.0]
    keep = drows.clone()
    A.nmt_op_expert_combine_bwd(out[:2], None, odd[:2].contiguous(), None, drows[:3], None)
    assert torch.equal(drows, keep)


def test_experts_rows_behind_32_bits_of_elements():
    n, d = 70000, 32768
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GB")
    rows = torch.empty(n, d, dtype=F16, device=DEV)
    x = torch.randn(2, d, device=DEV).half()
    rows[69999], rows[65537] = x[0], x[1]
    slot = torch.tensor([[69999], [65537]], dtype=torch.int32, device=DEV)
    out = torch.empty_like(x)
    A.nmt_op_expert_combine(rows, slot, None, out)
    assert torch.equal(out, x)
    rows[69999], rows[65537] = 0, 0
    A.nmt_op_expert_combine_bwd(x, None, slot, None, rows, None)
    assert torch.equal(rows[69999], x[0]) and torch.equal(rows[65537], x[1])
    del rows
    ids = torch.tensor([[0], [1]], dtype=torch.int32, device=DEV)      # the second expert's rows begin behind 2^31 elements
    big = torch.empty(2 * 70000, d // 2, dtype=F16, device=DEV)
    slot, _ = dispatched(ids, 2, 70000, x[:, :d // 2], big)
    assert slot.tolist() == [[0], [70000]] and torch.equal(big[70000], x[1, :d // 2])
    assert float(big[139999].abs().max()) == 0 and float(big[1].abs().max()) == 0


# ---- AdamW -----------------------------------------------------------------------------------------
HYPER = dict(lr=3e-3, b1=0.9, b2=0.98, eps=1e-8)


def adamw_tensors(sizes, bits, grad, weights, seed, shift=0, start="running"):
    g = gen(seed)
    r = lambda n: torch.randn(n, generator=g, device=DEV)
    out, checks = [], []

    def place(values, dtype):
        v, ok = guarded(1, values.numel(), dtype, None, None, shift)
        v.view(torch.uint8).copy_(values.to(dtype).view(1, -1).view(torch.uint8)) if dtype == torch.float8_e4m3fn else v.copy_(values.view(1, -1))
        checks.append(ok)
        return v.view(-1)
    for i, n in enumerate(sizes):
        t = dict(weight_decay=0.01 * (i % 3), lr_factor=1.0 - 0.25 * (i % 2))
        t["master"], t["grad"] = place(0.1 * r(n), F32), place(0.02 * r(n) * torch.exp(r(n)), grad)
        t["weights"] = None if weights is None or i % 5 == 4 else place(torch.zeros(n, device=DEV), weights)
        zero = 0.0 if start == "zero" else 1.0
        m, v = zero * 0.01 * r(n), zero * (0.02 * torch.exp(r(n))) ** 2
        if bits == 32:
            t["m"], t["v"] = place(m, F32), place(v, F32)
        else:
            for name, x in (("m", m), ("v", v.sqrt())):
                pad = torch.nn.functional.pad(x, (0, -n % 256)).view(-1, 256)
                scale = pad.abs().amax(1) / 448
                code = (pad / scale.clamp(min=1e-30)[:, None]).to(torch.float8_e4m3fn).view(-1)[:n]
                t[name] = torch.empty(n + shift, dtype=torch.float8_e4m3fn, device=DEV)[shift:]
                t[name].view(torch.uint8).copy_(code.view(torch.uint8))
                t[name + "_scale"] = place(scale, F32)
        out.append(t)
    return out, lambda: all(c() for c in checks)


def states(t, bits):
    """(m, v) as 64-bit values"""
    if bits == 32:
        return t["m"].to(D), t["v"].to(D)
    n = t["m"].numel()
    spread = lambda name: t[name].float().to(D) * t[name + "_scale"].to(D).repeat_interleave(256)[:n]
    return spread("m"), spread("v") ** 2


def check_step(tensors, bits, t, plan, grad_scale=1.0):
    h = HYPER
    want = []
    for x in tensors:
        m, v = states(x, bits)
        g = x["grad"].to(D) * grad_scale
        w, m2, v2 = R.adamw(x["master"].to(D), m, v, g, h["lr"], h["b1"], h["b2"], h["eps"], t, x["weight_decay"], x["lr_factor"])
        want.append((x["master"].to(D), m, v, g, w, m2, v2))
    A.nmt_adamw_step(plan, h["lr"], h["b1"], h["b2"], h["eps"], t, grad_scale=grad_scale)
    torch.cuda.synchronize()
    for i, (x, (w0, m, v, g, w, m2, v2)) in enumerate(zip(tensors, want)):
        # a product or sum rounds once, so do the constants: 6 U32 of the terms (8 bits: two more for the state's scale, squared in v).  The step m / sqrt(v): those of m and
        # half of v's, and five of its own: 24 U32 of the terms of m over the root; the master weight: one of its own, of each term
        ms, vs = h["b1"] * m.abs() + (1 - h["b1"]) * g.abs(), v2
        den = torch.sqrt(v2 / (1 - h["b2"] ** t)) + h["eps"]
        rate = h["lr"] * x["lr_factor"]
        step = ms / (1 - h["b1"] ** t) / den
        within(x["master"], w, U32 * (2 * w.abs() + 24 * rate * step + 6 * rate * x["weight_decay"] * w0.abs()) + 1e-40, f"master {i}")
        if x["weights"] is not None:
            assert torch.equal(x["weights"], x["master"].to(x["weights"].dtype)), i
        if bits == 32:
            within(x["m"], m2, 8 * U32 * ms + 1e-44, f"m {i}")
            within(x["v"], v2, 8 * U32 * vs + 1e-44, f"v {i}")
            continue
        n = w.numel()
        for name, value in (("m", m2), ("v", v2.sqrt())):
            pad = torch.nn.functional.pad(value, (0, -n % 256)).view(-1, 256)
            scale = pad.abs().amax(1) / 448
            within(x[name + "_scale"], scale, 12 * U32 * pad.abs().amax(1) / 100, f"{name} scale {i}")
            s = x[name + "_scale"].to(D).repeat_interleave(256)[:n]
            q = torch.where(s > 0, value / s.clamp(min=1e-300), 0.0)
            half = R.e4m3_half_step(q)
            code = x[name].float().to(D)
            if name == "v":       # what is not zero is not rounded to zero
                assert ((code > 0) == (value > 0)).all(), i
                half = torch.where((value > 0) & (q < 2.0 ** -10), 2.0 ** -9, half)
            within(code, q, half + 24 * U32 * (q.abs() + (ms / s.clamp(min=1e-300) if name == "m" else 0)), f"{name} codes {i}")


SIZES = [1, 3, 4, 255, 256, 257, 1000, 1023, 1024, 1025, 5000, 70001, 0, 2]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad,weights", [(F16, F16), (BF16, BF16), (F32, F32), (F32, F16), (F16, None), (BF16, F16)])
def test_adamw_over_tensors_of_all_sizes(bits, grad, weights):
    for shift, start in ((0, "running"), (1, "running"), (3, "zero")):
        tensors, ok = adamw_tensors(SIZES, bits, grad, weights, 5, shift, start)
        table = torch.empty(A.nmt_adamw_table_bytes(tensors), dtype=torch.uint8, device=DEV)
        plan = A.nmt_adamw_create(tensors, table)
        for t in ((1, 2, 3) if start == "zero" else (50, 51)):
            check_step(tensors, bits, t, plan, grad_scale=0.5)
        A.nmt_adamw_destroy(plan)
        assert ok()


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_over_more_pieces_than_work_groups(bits):
    tensors, _ = adamw_tensors([70_000_003, 513], bits, F16, F16, 6)
    plan = A.nmt_adamw_create(tensors, torch.empty(A.nmt_adamw_table_bytes(tensors), dtype=torch.uint8, device=DEV))
    check_step(tensors, bits, 9, plan)
    A.nmt_adamw_destroy(plan)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sizes", [[(16 << 20) - 1], [(16 << 20) - 514, 513], [16 << 20], [(16 << 20) - 513, 514]])
def test_adamw_through_the_caches_and_past_them(sizes, bits):
    """Lists of 2^24 elements and more go past the caches, with a last piece that is not whole, those of one less through them."""
    tensors, ok = adamw_tensors(sizes, bits, F16, F16, 9)
    plan = A.nmt_adamw_create(tensors, torch.empty(A.nmt_adamw_table_bytes(tensors), dtype=torch.uint8, device=DEV))
    check_step(tensors, bits, 9, plan)
    A.nmt_adamw_destroy(plan)
    assert ok()


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_skips_on_the_flag_and_repeats_in_a_graph(bits):
    tensors, _ = adamw_tensors([1000, 70001], bits, F16, F16, 7)
    twin, _ = adamw_tensors([1000, 70001], bits, F16, F16, 7)
    make = lambda ts: A.nmt_adamw_create(ts, torch.empty(A.nmt_adamw_table_bytes(ts), dtype=torch.uint8, device=DEV))
    plan, other = make(tensors), make(twin)
    bits_of = lambda ts: [x[k].view(torch.uint8).clone() for x in ts for k in ("master", "m", "v", "weights")]
    flag = torch.ones(1, dtype=torch.int32, device=DEV)
    before = bits_of(tensors)
    A.nmt_adamw_step(plan, 1e-3, 0.9, 0.98, 1e-8, 3, flag=flag)
    assert all(torch.equal(a, b) for a, b in zip(before, bits_of(tensors)))
    flag.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.nmt_adamw_step(plan, 1e-3, 0.9, 0.98, 1e-8, 3, flag=flag)
    for _ in range(3):
        graph.replay()
        A.nmt_adamw_step(other, 1e-3, 0.9, 0.98, 1e-8, 3)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(bits_of(twin), bits_of(tensors)))
    for p in (plan, other):
        A.nmt_adamw_destroy(p)
    with pytest.raises(A.NmtError):
        A.nmt_adamw_step(plan, 1e-3, 0.9, 0.98, 1e-8, 3)


def test_adamw_plans_cannot_be_made_while_capturing():
    tensors, _ = adamw_tensors([1000], 32, F16, F16, 7)
    table = torch.empty(A.nmt_adamw_table_bytes(tensors), dtype=torch.uint8, device=DEV)
    x = torch.zeros(4, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.add_(1)
        with pytest.raises(A.NmtError) as e:
            A.nmt_adamw_create(tensors, table)
    assert e.value.code == A.NMT_EINVAL and "captured" in str(e.value)
    graph.replay()
    torch.cuda.synchronize()
    assert x.tolist() == [1.0] * 4


def test_adamw_of_8_bits_keeps_what_is_not_finite_to_its_element():
    tensors, _ = adamw_tensors([600], 8, F32, F16, 8)
    clean, _ = adamw_tensors([600], 8, F32, F16, 8)
    x, c = tensors[0], clean[0]
    # (two elements that do not hold their block's largest magnitude)
    x["grad"][10], x["grad"][300] = float("nan"), float("inf")
    c["grad"][10], c["grad"][300] = 0, 0
    for ts in (tensors, clean):
        plan = A.nmt_adamw_create(ts, torch.empty(A.nmt_adamw_table_bytes(ts), dtype=torch.uint8, device=DEV))
        A.nmt_adamw_step(plan, 1e-3, 0.9, 0.98, 1e-8, 3)
        A.nmt_adamw_destroy(plan)
    keep = torch.ones(600, dtype=torch.bool, device=DEV)
    keep[[10, 300]] = False
    for k in ("master", "m", "v", "weights"):
        a, b = x[k].float(), c[k].float()
        assert torch.equal(a[keep], b[keep]), k
        if k in ("m", "v"):
            assert torch.isnan(a[~keep]).all(), k
    assert torch.equal(x["m_scale"], c["m_scale"]) and torch.equal(x["v_scale"], c["v_scale"])


def test_adamw_of_8_bits_never_divides_by_eps_alone():
    """An element whose v falls below what its block's scale resolves keeps the smallest code, so that the next step stays of ordinary size."""
    n = 256
    x = dict(master=torch.zeros(n, device=DEV), grad=torch.full((n,), 1e-9, device=DEV), weights=None, weight_decay=0.0, lr_factor=1.0,
             m=torch.zeros(n, device=DEV).to(torch.float8_e4m3fn), v=torch.zeros(n, device=DEV).to(torch.float8_e4m3fn), m_scale=torch.zeros(1, device=DEV),
             v_scale=torch.zeros(1, device=DEV))
    x["grad"][0] = 1.0
    plan = A.nmt_adamw_create([x], torch.empty(A.nmt_adamw_table_bytes([x]), dtype=torch.uint8, device=DEV))
    for t in range(1, 4):
        A.nmt_adamw_step(plan, 1e-3, 0.9, 0.98, 1e-12, t)
    A.nmt_adamw_destroy(plan)
    assert float(x["v"].float().min()) == 2.0 ** -9 and float(x["master"].abs().max()) <= 3.1e-3


def test_adamw_of_8_bits_over_blocks_of_nothing():
    """Zero gradients and states: nothing divides by a scale of zero."""
    tensors, _ = adamw_tensors([700], 8, F16, F16, 8, start="zero")
    x = tensors[0]
    x["grad"].zero_()
    before = x["master"].clone()
    plan = A.nmt_adamw_create(tensors, torch.empty(A.nmt_adamw_table_bytes(tensors), dtype=torch.uint8, device=DEV))
    A.nmt_adamw_step(plan, 1e-3, 0.9, 0.98, 1e-8, 1)
    A.nmt_adamw_destroy(plan)
    assert torch.equal(x["master"], before) and not x["m"].float().any() and not x["v"].float().any()
    assert not x["m_scale"].any() and not x["v_scale"].any()


# ---- streams, graphs, repetition ---------------------------------------------------------------------
class Block:
    """Everything a sparse, gated block calls besides its products: forwards, and back."""

    def __init__(self, seed, tokens=333, d=256, experts=8, k=2, capacity=0, dtype=F16):
        s = norm_inputs(tokens, d, dtype, "layer", 9, seed)
        g = gen(seed + 1)
        self.s, self.ids, self.experts, self.cap = s, choices(tokens, k, experts, seed), experts, capacity
        self.w = torch.rand(tokens, k, generator=g, device=DEV)
        n = experts * capacity if capacity else tokens * k
        e = lambda *shape, t=dtype: torch.zeros(*shape, dtype=t, device=DEV)
        i = lambda *shape: e(*shape, t=torch.int32)
        self.slot, self.ranges, self.scratch = i(tokens, k), i(experts, 2), i(A.nmt_op_expert_dispatch_scratch(tokens, k, experts))
        self.rows, self.out, self.h, self.n, self.stats = e(n, d), e(tokens, d), e(tokens, d), e(tokens, d), e(tokens, 4, t=F32)
        self.dx, self.dy, self.dgate, self.drows, self.dw, self.dt = e(tokens, d), e(tokens, d), torch.zeros_like(s["gate"]), e(n, d), e(tokens, k, t=F32), e(tokens, d)
        self.dpost, self.dpre = (e(d), e(d)), (e(d), e(d))
        self.partial = e(A.nmt_op_gated_norm_bwd_scratch(tokens, d, 9), t=F32)

    def run(self, stream=None):
        s, kw = self.s, dict(post=self.s["post"], gate=self.s["gate"], pre=self.s["pre"], rows_per_gate=9, resid_scale=0.9, stream=stream)
        A.nmt_op_expert_dispatch(self.ids, self.experts, self.cap, s["y"], self.rows, self.slot, self.ranges, self.scratch, stream=stream)
        A.nmt_op_expert_combine(self.rows, self.slot, self.w, self.out, stream=stream)
        A.nmt_op_gated_norm_fwd(s["x"], self.out, self.h, self.n, self.stats, **kw)
        A.nmt_op_gated_norm_bwd(s["dh"], s["dn"], self.out, self.h, self.stats, self.dx, self.dy, self.partial, dpost=self.dpost, dgate=self.dgate, dpre=self.dpre, **kw)
        A.nmt_op_expert_combine_bwd(self.dy, self.rows, self.slot, self.w, self.drows, self.dw, self.ranges, self.cap, stream=stream)
        A.nmt_op_expert_combine(self.drows, self.slot, None, self.dt, stream=stream)

    def outputs(self):
        return [t.clone() for t in (self.slot, self.ranges, self.rows, self.out, self.h, self.n, self.stats, self.dx, self.dy, self.dgate, *self.dpost, *self.dpre, self.drows,
                                    self.dw, self.dt)]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("capacity,tokens", [(0, 333), (90, 333), (0, 9000)])
def test_same_bits_every_time_on_any_stream_and_in_a_graph(capacity, tokens):
    b = Block(21, capacity=capacity, tokens=tokens)
    b.run()
    torch.cuda.synchronize()
    first = b.outputs()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b.run()
    side.synchronize()
    assert same(first, b.outputs())
    b.run(stream=side.cuda_stream)
    side.synchronize()
    assert same(first, b.outputs())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run()
    other = Block(22, capacity=capacity, tokens=tokens)
    other.run()
    torch.cuda.synchronize()
    want = other.outputs()
    for k in range(4):      # replays with the program's own work and new inputs in between
        b.s["y"].copy_(other.s["y"] if k % 2 else b.s["y"])
        for t in (b.rows, b.h, b.dx, b.dgate, b.partial, b.slot):
            t.zero_()
        graph.replay()
        other.run()
        torch.cuda.synchronize()
        assert same(want, other.outputs())
        got = b.outputs()
        b.run()
        torch.cuda.synchronize()
        assert same(got, b.outputs())


def test_calls_on_two_streams_at_once():
    a, b = Block(31, tokens=4000), Block(32, tokens=3000, capacity=900)
    for x in (a, b):
        x.run()
    torch.cuda.synchronize()
    want = a.outputs(), b.outputs()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        a.run(stream=s.cuda_stream)
        b.run(stream=t.cuda_stream)
    torch.cuda.synchronize()
    assert same(want[0], a.outputs()) and same(want[1], b.outputs())


# ---- together ----------------------------------------------------------------------------------------
def test_a_sparse_gated_block_trains():
    """Norm, experts, their products, weighted sum, norm with gate and residual, the next norm; the way back; AdamW over everything.  Against autograd in 64 bits: some ten
    tensors lie in fp16 between a loss and a gradient, each off by at most 2^-11 of its values: 10 * 2^-11 of a gradient's norm, and as much again for the products' fp32."""
    T, d, F, E, k, cap = 240, 64, 128, 4, 2, 200
    g = gen(77)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)
    x, ch, cn = r(T, d).half(), r(T, d).half(), r(T, d).half()
    # (biases of +-6 over products of size 1: no ReLU hangs on a rounding)
    side = torch.where(torch.arange(F, device=DEV) % 2 == 0, 6.0, -6.0)
    P = {f"w1.{e}": r(F, d) / d ** .5 for e in range(E)} | {f"b1.{e}": side + .1 * r(F) for e in range(E)} | {f"w2.{e}": r(d, F) / F ** .5 for e in range(E)} \
        | {"first_g": 1 + .1 * r(d), "first_s": .1 * r(d), "post_g": 1 + .1 * r(d), "post_s": .1 * r(d), "gate": .5 + .1 * r(1, d), "pre_g": 1 + .1 * r(d), "pre_s": .1 * r(d)}
    P = {n: v.half() for n, v in P.items()}
    ids, w = choices(T, k, E, 5, dropped=0.1, skew=0.3), torch.rand(T, k, generator=g, device=DEV)
    new = lambda *s, t=F16: torch.empty(*s, dtype=t, device=DEV)
    I32 = torch.int32
    # forwards
    n0, st0 = new(T, d), new(T, 4, t=F32)
    A.nmt_op_gated_norm_fwd(x, None, None, n0, st0, pre=(P["first_g"], P["first_s"]))
    rows, slot, ranges, scratch = new(E * cap, d), new(T, k, t=I32), new(E, 2, t=I32), new(A.nmt_op_expert_dispatch_scratch(T, k, E), t=I32)
    A.nmt_op_expert_dispatch(ids, E, cap, n0, rows, slot, ranges, scratch)
    assert int(ranges[:, 1].max()) < cap and int((slot < 0).sum()) > 0          # room is left, and some choices are dropped
    hid, made = new(E * cap, F), new(E * cap, d)
    of = lambda t, e: t[e * cap:(e + 1) * cap]
    for e in range(E):
        A.nmt_op_gemm(of(rows, e), 0, d, P[f"w1.{e}"], 0, d, of(hid, e), F, cap, F, d, bias=P[f"b1.{e}"], relu=True)
        A.nmt_op_gemm(of(hid, e), 0, F, P[f"w2.{e}"], 0, F, of(made, e), d, cap, d, F)
    out, h, n1, st1 = new(T, d), new(T, d), new(T, d), new(T, 4, t=F32)
    A.nmt_op_expert_combine(made, slot, w, out)
    parts = dict(post=(P["post_g"], P["post_s"]), gate=P["gate"], pre=(P["pre_g"], P["pre_s"]), resid_scale=0.9)
    A.nmt_op_gated_norm_fwd(x, out, h, n1, st1, **parts)
    # back
    G = {n: torch.empty_like(v) for n, v in P.items()}
    dx, dout, partial = new(T, d), new(T, d), new(A.nmt_op_gated_norm_bwd_scratch(T, d), t=F32)
    A.nmt_op_gated_norm_bwd(ch, cn, out, h, st1, dx, dout, partial, dpost=(G["post_g"], G["post_s"]), dgate=G["gate"], dpre=(G["pre_g"], G["pre_s"]), **parts)
    dmade, dw = new(E * cap, d), new(T, k, t=F32)
    A.nmt_op_expert_combine_bwd(dout, made, slot, w, dmade, dw, ranges, cap)
    dhid, drows = new(E * cap, F), new(E * cap, d)
    for e in range(E):
        A.nmt_op_gemm(of(dmade, e), 0, d, P[f"w2.{e}"], 1, F, of(dhid, e), F, cap, F, d, relu_src=of(hid, e))
        A.nmt_op_gemm(of(dhid, e), 0, F, P[f"w1.{e}"], 1, d, of(drows, e), d, cap, d, F)
        A.nmt_op_wgrad_group([(of(dhid, e), F, of(rows, e), d, G[f"w1.{e}"], d, G[f"b1.{e}"], F, d, cap), (of(dmade, e), d, of(hid, e), F, G[f"w2.{e}"], F, None, d, F, cap)])
    dn0 = new(T, d)
    A.nmt_op_expert_combine(drows, slot, None, dn0)
    A.nmt_op_gated_norm_bwd(dx, dn0, None, x, st0, dx, None, partial, pre=(P["first_g"], P["first_s"]), dpre=(G["first_g"], G["first_s"]))
    torch.cuda.synchronize()
    # the same in 64 bits
    leaf = {n: v.to(D).requires_grad_() for n, v in P.items()}
    X, W = x.to(D).requires_grad_(), w.to(D).requires_grad_()
    N0 = R.gated_norm(X, pre=(leaf["first_g"], leaf["first_s"]))[1]
    Y = torch.zeros(T, d, dtype=D, device=DEV)
    for j in range(k):
        for e in range(E):
            t = ((ids[:, j] == e) & (slot[:, j] >= 0)).nonzero().reshape(-1)
            Y = Y.index_add(0, t, W[t, j, None] * (torch.relu(N0[t] @ leaf[f"w1.{e}"].t() + leaf[f"b1.{e}"]) @ leaf[f"w2.{e}"].t()))
    H, N1 = R.gated_norm(X, Y, (leaf["post_g"], leaf["post_s"]), leaf["gate"], (leaf["pre_g"], leaf["pre_s"]), resid_scale=0.9)
    ((H * ch.to(D)).sum() + (N1 * cn.to(D)).sum()).backward()
    bound = 20 * 2.0 ** -11
    near = lambda got, want, what: None if float((got.to(D) - want.detach()).norm()) <= bound * float(want.detach().norm()) else pytest.fail(
        f"{what}: {float((got.to(D) - want).norm() / want.norm()):.5f}")
    near(h, H, "h"), near(n1, N1, "n"), near(dx, X.grad, "x"), near(dw, W.grad, "weights")
    for n in P:
        near(G[n], leaf[n].grad, n)
    # and the step, from these gradients
    for bits in (32, 8):
        tensors = []
        for n, v in P.items():
            size = v.numel()
            t = dict(master=v.float().reshape(-1), grad=G[n].reshape(-1), weights=v.clone().reshape(-1), weight_decay=0.01 if v.dim() == 2 and v.shape[0] > 1 else 0.0, lr_factor=1.0)
            for s in ("m", "v"):
                t[s] = torch.zeros(size, device=DEV) if bits == 32 else torch.zeros(size, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
                if bits == 8:
                    t[s + "_scale"] = torch.zeros(-(-size // 256), device=DEV)
            tensors.append(t)
        plan = A.nmt_adamw_create(tensors, torch.empty(A.nmt_adamw_table_bytes(tensors), dtype=torch.uint8, device=DEV))
        for t in (1, 2):
            check_step(tensors, bits, t, plan)
        A.nmt_adamw_destroy(plan)


# ---- sessions ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("weight_decay,state_bits", [(0.01, 32), (0.0, 8), (0.05, 8)])
def test_sessions_update_with_adamw(weight_decay, state_bits):
    """Weights after three updates of two sub-batches each, from the accumulated gradients the session itself holds; an update that overflows changes nothing."""
    import nmt_inputs as I
    from paper_1806_00187_amd.session import Session
    model = I.MODELS["tiny"]
    sess = Session(model, I.init_weights(seed=0, **model), max_sentences=8, weight_decay=weight_decay, state_bits=state_bits)
    batches = [sess.to_device(I.tiny_batch(seed=s)) for s in (1001, 1002)]
    of = lambda flat, off, n: flat[off:off + n]

    def pieces():
        out, at = [], 0
        for name, (off, rows, cols) in sess.layout.items():
            n = rows * cols
            t = dict(master=of(sess.master, off, n), m=of(sess.m, off, n), v=of(sess.v, off, n), grad=of(sess.acc, off, n), weights=of(sess.w16, off, n),
                     weight_decay=weight_decay if rows > 1 else 0.0, lr_factor=1.0)
            if state_bits == 8:
                blocks = -(-n // 256)
                t.update(m_scale=of(sess.m_scale, at, blocks), v_scale=of(sess.v_scale, at, blocks))
                at += blocks
            out.append(t)
        return out
    for t in (1, 2, 3):
        before = [dict(master=x["master"].to(D), state=states(x, state_bits)) for x in pieces()]
        _, ntok, flag = sess.update(batches, 128.0, 1e-3, t)
        assert flag == 0
        for x, b in zip(pieces(), before):
            m, v = b["state"]
            w, _, _ = R.adamw(b["master"], m, v, x["grad"].to(D) / (128.0 * ntok), 1e-3, 0.9, 0.98, 1e-8, t, x["weight_decay"])
            step = (w - b["master"]).abs()
            # (as in check_step, 24 U32 of the step's terms, and of the factor 1 / (128 tokens) in fp32 one more; |m| / root v is at most 1 / sqrt(1 - beta2) beyond the step)
            within(x["master"], w, 2 * U32 * w.abs() + 64 * U32 * 1e-3 * (8 + step / 1e-3), "master")
            assert torch.equal(x["weights"], x["master"].half())
    keep = [t.view(torch.uint8).clone() for t in (sess.master, sess.m, sess.v, sess.w16)]
    _, _, flag = sess.update(batches, 128.0 * 2 ** 20, 1e-3, 4)
    assert flag == 1 and all(torch.equal(a, t.view(torch.uint8)) for a, t in zip(keep, (sess.master, sess.m, sess.v, sess.w16)))
    sess.close()


def test_sessions_without_decay_in_32_bits_keep_adam():
    import nmt_inputs as I
    from paper_1806_00187_amd.session import Session
    model = I.MODELS["tiny"]
    sess = Session(model, I.init_weights(seed=0, **model), max_sentences=8)
    assert sess.plan is None and sess.m.dtype == torch.float32
    sess.close()
    with pytest.raises(ValueError):
        Session(model, I.init_weights(seed=0, **model), state_bits=16)


@pytest.mark.parametrize("state_bits", [32, 8])
def test_sessions_of_several_pipes_update_with_adamw(state_bits):
    """The step over the shared accumulator, from what that held: the first update's moments are (1 - beta) g and (1 - beta) g^2."""
    import nmt_inputs as I
    from paper_1806_00187_amd.session import Session
    model = I.MODELS["tiny"]
    sess = Session(model, I.init_weights(seed=0, **model), max_sentences=8, n_pipes=2, auto_streams=False, weight_decay=0.02, state_bits=state_bits)
    batches = [sess.to_device(I.tiny_batch(seed=s)) for s in (1001, 1002, 1003)]
    before = sess.master.to(D)
    _, ntok, flag = sess.update(batches, 128.0, 1e-3, 1)
    assert flag == 0
    for name, (off, rows, cols) in sess.layout.items():
        n = rows * cols
        w0, g = before[off:off + n], sess.acc[off:off + n].to(D) / (128.0 * ntok)
        assert float(g.abs().max()) > 0, name
        w, _, _ = R.adamw(w0, torch.zeros_like(g), torch.zeros_like(g), g, 1e-3, 0.9, 0.98, 1e-8, 1, 0.02 if rows > 1 else 0.0)
        # (as in test_sessions_update_with_adamw; a first step has |m| / root v = 1)
        within(sess.master[off:off + n], w, 2 * U32 * w.abs() + 64 * U32 * 1e-3 * 9, name)
    assert torch.equal(sess.w16, sess.master.half())
    sess.close()
