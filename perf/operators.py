"""The training operators beside the Transformer step, as a user's program calls them: the norms around a gated residual block, tokens
sorted by expert and back, and AdamW over many tensors, forwards and backwards, from calls bound by latency to calls bound by memory.

A case names its operator and sizes; inputs follow from the seed.  `run` computes a case with elementary torch operations in 32 bits,
or, where `own` is set, with the library's entry points."""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"f16": 2, "bf16": 2, "f32": 4}
BLOCK = 256        # elements that share a scale of an 8-bit state
TOP = 448.0        # the largest value of torch.float8_e4m3fn
EPS = 1e-5


def _norm(name, op, rows, d, dtype, kind, gate_rows, resid_scale=1.0):
    # gate_rows: rows that share a row of the gate; 0: one gate for all
    return dict(name=name, op=op, rows=rows, d=d, dtype=dtype, kind=kind, gate_rows=gate_rows, resid_scale=resid_scale)


def _experts(name, op, tokens, k, experts, d, dtype, room, unrouted=0.0):
    # room: rows set aside for each expert, as a multiple of an even share; 0: as many as it gets
    # unrouted: share of tokens that go to no expert (padding)
    return dict(name=name, op=op, tokens=tokens, k=k, experts=experts, d=d, dtype=dtype, room=room, unrouted=unrouted)


def _adamw(name, bits, layers, d, ff, vocab, grad, copy):
    return dict(name=name, op="adamw", bits=bits, layers=layers, d=d, ff=ff, vocab=vocab, grad=grad, copy=copy)


def listed():
    return [
        # the two-layer, 64-wide model on one small sub-batch: a call bound by latency
        _norm("norm_fwd_tiny", "norm_fwd", 136, 64, "f16", "layer", 0),
        # Transformer-big's width over the positions of a whole update, one gate for all
        _norm("norm_fwd_update", "norm_fwd", 52701, 1024, "bf16", "rms", 0, 0.9),
        # one sub-batch of the usual budget at Transformer-base's width
        _norm("norm_bwd_base", "norm_bwd", 3584, 512, "f16", "layer", 0),
        # Transformer-big's width, gates that belong to a sentence of 27 positions each
        _norm("norm_bwd_sentences", "norm_bwd", 26001, 1024, "f16", "rms", 27, 0.9),
        # an odd width in 32 bits, a gate for every element
        _norm("norm_bwd_odd_f32", "norm_bwd", 1531, 777, "f32", "layer", 1),
        # a few tokens, as while one sentence is translated
        _experts("experts_fwd_few", "experts_fwd", 5, 2, 8, 512, "f16", 0.0),
        # one sub-batch of the usual budget, a tenth of it padding, experts of fixed room
        _experts("experts_fwd_room", "experts_fwd", 3584, 2, 16, 512, "f16", 1.25, 0.1),
        # a whole update's positions at Transformer-big's width
        _experts("experts_fwd_update", "experts_fwd", 52701, 2, 64, 1024, "bf16", 0.0),
        # the way back over a quarter of an update, four experts a token
        _experts("experts_bwd_four", "experts_bwd", 13003, 4, 128, 1024, "f16", 0.0),
        # the two-layer model's 65 tensors: a call bound by latency
        _adamw("adamw32_tiny", 32, 2, 64, 256, 1000, "f32", "f16"),
        # Transformer-base's tensors, states in 32 bits
        _adamw("adamw32_base", 32, 6, 512, 2048, 32768, "f32", "f16"),
        # Transformer-big's tensors, states in 8 bits, gradients as the backward pass leaves them
        _adamw("adamw8_big", 8, 6, 1024, 4096, 32768, "f16", "f16"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "experts_fwd", "experts_bwd", "adamw"])
    dtype = rng.choice(["f16", "f16", "bf16", "f32"])
    if op.startswith("norm"):
        d = _log(rng, 40, 5000)
        if rng.random() < 0.6:
            d = -(-d // 64) * 64
        rows = min(_log(rng, 1, 52701), 26001 * 1024 * 2 // (d * SIZE[dtype]))
        gate = rng.choice([0, 0, 1, _log(rng, 2, 300)])
        return _norm("", op, rows, d, dtype, rng.choice(["layer", "rms"]), gate, rng.choice([1.0, 0.9, 2.5]))
    if op.startswith("experts"):
        experts = _log(rng, 2, 256)
        k = min(rng.choice([1, 2, 2, 4, 8]), experts)
        d = _log(rng, 40, 3000)
        if rng.random() < 0.6:
            d = -(-d // 64) * 64
        tokens = min(_log(rng, 1, 52701), 13003 * 4 * 1024 * 2 // (d * k * SIZE[dtype]))
        return _experts("", op, max(tokens, 1), k, experts, d, dtype, rng.choice([0.0, 0.0, 1.0, 1.5]), rng.choice([0.0, 0.0, 0.13]))
    d = 8 * _log(rng, 4, 110)
    return _adamw("", rng.choice([8, 32]), rng.randint(1, 6), d, d * rng.choice([1, 2, 4]), _log(rng, 100, 30000), dtype,
                  rng.choice(["f16", "bf16", "none"]))


# ---- inputs --------------------------------------------------------------------------------------
def _tensors(case):
    """(elements, weight decay, learning-rate factor) of an encoder-decoder's tensors; vectors do not decay."""
    d, ff = case["d"], case["ff"]
    attention = [(3 * d * d, .01, 1.), (3 * d, 0., 1.), (d * d, .01, 1.), (d, 0., 1.)]
    cross = [(d * d, .01, 1.), (d, 0., 1.), (2 * d * d, .01, 1.), (2 * d, 0., 1.), (d * d, .01, 1.), (d, 0., 1.)]
    forward = [(d * ff, .01, 1.), (ff, 0., 1.), (d * ff, .01, 1.), (d, 0., 1.)]
    norm = [(d, 0., 1.), (d, 0., 1.)]
    encoder = attention + norm + forward + norm
    decoder = attention + norm + cross + norm + forward + norm
    return [(case["vocab"] * d, .01, .5)] + case["layers"] * encoder + case["layers"] * decoder


def _room(case):
    return math.ceil(case["room"] * case["tokens"] * case["k"] / case["experts"])


def _slots(ids, experts, room):
    """Where every assignment's row goes ([tokens, k], -1: nowhere), and (first row, rows) of every expert."""
    flat = ids.reshape(-1)
    order = torch.sort(torch.where(flat >= 0, flat, experts), stable=True).indices
    counts = (flat[:, None] == torch.arange(experts, device=DEV, dtype=torch.int32)).sum(0)
    first = counts.cumsum(0) - counts
    at = torch.empty_like(order)
    at[order] = torch.arange(order.numel(), device=DEV)
    expert = flat.clamp(min=0).long()
    rank = at - first[expert]
    if room:
        slot = torch.where((flat >= 0) & (rank < room), expert * room + rank, -1)
        ranges = torch.stack([torch.arange(experts, device=DEV) * room, counts.clamp(max=room)], 1)
    else:
        slot = torch.where(flat >= 0, at, -1)
        ranges = torch.stack([first, counts], 1)
    return slot.int().reshape(ids.shape), ranges.int()


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device=DEV)  # noqa: E731
    s = dict(case)
    if s["op"].startswith("norm"):
        T, rows, d = TYPES[s["dtype"]], s["rows"], s["d"]
        gates = 1 if s["gate_rows"] == 0 else -(-rows // s["gate_rows"])
        s["x"], s["y"] = (3 * normal(rows, d) + 0.3).to(T), (2 * normal(rows, d) - 0.5).to(T)
        s["post"] = ((1 + 0.2 * normal(d)).to(T), (0.1 * normal(d)).to(T) if s["kind"] == "layer" else None)
        s["pre"] = ((1 + 0.2 * normal(d)).to(T), (0.1 * normal(d)).to(T) if s["kind"] == "layer" else None)
        s["gate"] = (0.5 + 0.3 * normal(gates, d)).to(T)
        s["rows_per_gate"] = s["gate_rows"] or rows
        if s["op"] == "norm_bwd":   # what the forward pass left, and the gradients that arrive
            s["y"] = s["y"].contiguous()
            f = _norm_forward(s)
            s["h"], s["stats"] = f["h"], f["stats"].contiguous()
            s["dh"], s["dn"] = normal(rows, d).to(T), normal(rows, d).to(T)
            del s["x"]
        if own:
            import paper_1806_00187_amd as A
            new = lambda like: torch.empty_like(like)  # noqa: E731
            if s["op"] == "norm_fwd":
                s["h"], s["n"], s["stats"] = new(s["x"]), new(s["x"]), torch.empty(rows, 4, device=DEV)
            else:
                s["dx"], s["dy"], s["dgate"] = new(s["h"]), new(s["h"]), new(s["gate"])
                s["dpost"], s["dpre"] = (tuple(None if v is None else new(v) for v in s[p]) for p in ("post", "pre"))
                s["scratch"] = torch.empty(A.nmt_op_gated_norm_bwd_scratch(rows, d, s["rows_per_gate"]), device=DEV)
        return s
    if s["op"].startswith("experts"):
        T, tokens, k, E, d = TYPES[s["dtype"]], s["tokens"], s["k"], s["experts"], s["d"]
        logits = 0.5 * normal(E) - torch.log(-torch.log(torch.rand(tokens, E, generator=gen, device=DEV).clamp(1e-6, 1 - 1e-6)))
        top = logits.topk(k, dim=1)
        s["ids"], s["weights"] = top.indices.int(), torch.softmax(top.values, 1)
        if s["unrouted"]:
            s["ids"][torch.rand(tokens, generator=gen, device=DEV) < s["unrouted"]] = -1
        s["cap"] = _room(s)
        n = E * s["cap"] if s["cap"] else tokens * k
        s["out_rows"] = normal(n, d).to(T)                # what the experts made of their rows
        if s["op"] == "experts_fwd":
            s["x"] = normal(tokens, d).to(T)
            s["rows"] = torch.zeros(n, d, dtype=T, device=DEV)
        else:
            s["slot"], s["ranges"] = _slots(s["ids"], E, s["cap"])
            s["dout"], s["dx_rows"] = normal(tokens, d).to(T), normal(n, d).to(T)
            s["dout_rows"] = torch.zeros(n, d, dtype=T, device=DEV)
        if own:
            import paper_1806_00187_amd as A
            if s["op"] == "experts_fwd":
                s["slot"] = torch.empty(tokens, k, dtype=torch.int32, device=DEV)
                s["ranges"] = torch.empty(E, 2, dtype=torch.int32, device=DEV)
                s["scratch"] = torch.empty(A.nmt_op_expert_dispatch_scratch(tokens, k, E), dtype=torch.int32, device=DEV)
                s["out"] = torch.empty_like(s["x"])
            else:
                s["dweights"], s["dx"] = torch.empty_like(s["weights"]), torch.empty_like(s["dout"])
        return s
    tensors = _tensors(case)
    # flat buffers in which every tensor starts a block of 256 elements
    sizes = torch.tensor([n for n, _, _ in tensors])
    blocks = (sizes + BLOCK - 1) // BLOCK
    first = (blocks.cumsum(0) - blocks) * BLOCK
    total = int(blocks.sum()) * BLOCK
    used = torch.zeros(total, device=DEV)
    for (n, _, _), at in zip(tensors, first.tolist()):
        used[at:at + n] = 1
    sigma = 0.02 * torch.exp(normal(total // BLOCK, 1)).expand(-1, BLOCK).reshape(-1)
    s["t"] = 100
    s["grad_scale"] = 1 / 1024
    s["master"] = 0.05 * normal(total) * used
    s["grad"] = (1024 * sigma * normal(total) * used).to(TYPES[s["grad"]])
    m, r = 0.3 * sigma * normal(total) * used, (sigma * (0.5 + torch.rand(total, generator=gen, device=DEV))) * used
    if s["bits"] == 8:
        for name, x in (("m", m), ("v", r)):
            scale = x.view(-1, BLOCK).abs().amax(1) / TOP
            s[name] = (x.view(-1, BLOCK) / scale[:, None].clamp(min=1e-30)).to(torch.float8_e4m3fn).view(-1)
            s[name + "_scale"] = scale
    else:
        s["m"], s["v"] = m, r * r
    s["weights"] = None if s["copy"] == "none" else s["master"].to(TYPES[s["copy"]])
    per_block = lambda values: torch.repeat_interleave(torch.tensor(values), blocks).to(DEV)[:, None]  # noqa: E731
    s["decay"], s["lr_factor"] = per_block([w for _, w, _ in tensors]), per_block([f for _, _, f in tensors])
    if own:
        import paper_1806_00187_amd as A
        cut = lambda name, at, n: None if s.get(name) is None else s[name][at:at + n]  # noqa: E731
        each = [dict(master=cut("master", at, n), m=cut("m", at, n), v=cut("v", at, n), grad=cut("grad", at, n), weights=cut("weights", at, n),
                     m_scale=cut("m_scale", at // BLOCK, -(-n // BLOCK)), v_scale=cut("v_scale", at // BLOCK, -(-n // BLOCK)),
                     weight_decay=w, lr_factor=f) for (n, w, f), at in zip(tensors, first.tolist())]
        s["table"] = torch.empty(A.nmt_adamw_table_bytes(each), dtype=torch.uint8, device=DEV)
        s["plan"] = _Plan(A, each, s["table"])
    return s


class _Plan:
    """An optimizer's handle, given back when the program drops it."""

    def __init__(self, A, tensors, table):
        self.A, self.handle = A, A.nmt_adamw_create(tensors, table)

    def __del__(self):
        self.A.nmt_adamw_destroy(self.handle)


# ---- one pass ------------------------------------------------------------------------------------
def run(s):
    return {"norm_fwd": _run_norm_fwd, "norm_bwd": _run_norm_bwd, "experts_fwd": _run_experts_fwd, "experts_bwd": _run_experts_bwd,
            "adamw": _run_adamw}[s["op"]](s)


def _normed(a, kind):
    mean = a.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(a[:, :1])
    a = a - mean
    rstd = 1 / torch.sqrt((a * a).mean(1, keepdim=True) + EPS)
    return a * rstd, mean, rstd


def _affine(a, gain, shift):
    return a * gain.float() if shift is None else a * gain.float() + shift.float()


def _gates(s, rows):
    """The gate of every row, in 32 bits."""
    return s["gate"].float() if s["gate"].shape[0] == 1 else s["gate"].float()[torch.arange(rows, device=DEV) // s["rows_per_gate"]]


def _norm_forward(s):
    T = s["x"].dtype
    yhat, mean_y, rstd_y = _normed(s["y"].float(), s["kind"])
    h = s["resid_scale"] * s["x"].float() + _gates(s, s["rows"]) * _affine(yhat, *s["post"])
    hhat, mean_h, rstd_h = _normed(h, s["kind"])
    return {"h": h.to(T), "n": _affine(hhat, *s["pre"]).to(T), "stats": torch.cat([mean_y, rstd_y, mean_h, rstd_h], 1)}


def _run_norm_fwd(s):
    if own:
        import paper_1806_00187_amd as A
        A.nmt_op_gated_norm_fwd(s["x"], s["y"], s["h"], s["n"], s["stats"], post=s["post"], gate=s["gate"], pre=s["pre"], kind=s["kind"],
                                rows_per_gate=s["rows_per_gate"], resid_scale=s["resid_scale"], eps=EPS)
        return {"h": s["h"], "n": s["n"], "stats": s["stats"]}
    return _norm_forward(s)


def _norm_grad(g, xhat, rstd, kind):
    """Gradient at a norm's input from that at its normalised value."""
    m2 = (g * xhat).mean(1, keepdim=True)
    return rstd * (g - g.mean(1, keepdim=True) - xhat * m2) if kind == "layer" else rstd * (g - xhat * m2)


def _run_norm_bwd(s):
    if own:
        import paper_1806_00187_amd as A
        A.nmt_op_gated_norm_bwd(s["dh"], s["dn"], s["y"], s["h"], s["stats"], s["dx"], s["dy"], s["scratch"], post=s["post"], gate=s["gate"],
                                pre=s["pre"], dpost=s["dpost"], dgate=s["dgate"], dpre=s["dpre"], kind=s["kind"],
                                rows_per_gate=s["rows_per_gate"], resid_scale=s["resid_scale"])
        return {"dx": s["dx"], "dy": s["dy"], "dgate": s["dgate"], "dpost": s["dpost"], "dpre": s["dpre"]}
    T, kind, per = s["h"].dtype, s["kind"], s["rows_per_gate"]
    stats, dn, gate = s["stats"], s["dn"].float(), _gates(s, s["rows"])
    hhat = (s["h"].float() - stats[:, 2:3]) * stats[:, 3:4]
    yhat = (s["y"].float() - stats[:, 0:1]) * stats[:, 1:2]
    dh = s["dh"].float() + _norm_grad(dn * s["pre"][0].float(), hhat, stats[:, 3:4], kind)
    dz = gate * dh
    dy = _norm_grad(dz * s["post"][0].float(), yhat, stats[:, 1:2], kind)
    to_gate = dh * _affine(yhat, *s["post"])
    if s["gate"].shape[0] == 1:
        dgate = to_gate.sum(0, keepdim=True)
    else:
        short = s["gate"].shape[0] * per - s["rows"]
        dgate = torch.cat([to_gate, to_gate.new_zeros(short, s["d"])]).view(-1, per, s["d"]).sum(1)
    shift = kind == "layer"
    return {"dx": (s["resid_scale"] * dh).to(T), "dy": dy.to(T), "dgate": dgate.to(T),
            "dpost": ((dz * yhat).sum(0).to(T), dz.sum(0).to(T) if shift else None),
            "dpre": ((dn * hhat).sum(0).to(T), dn.sum(0).to(T) if shift else None)}


def _run_experts_fwd(s):
    if own:
        import paper_1806_00187_amd as A
        A.nmt_op_expert_dispatch(s["ids"], s["experts"], s["cap"], s["x"], s["rows"], s["slot"], s["ranges"], s["scratch"])
        A.nmt_op_expert_combine(s["out_rows"], s["slot"], s["weights"], s["out"])
        return {"rows": s["rows"], "slot": s["slot"], "ranges": s["ranges"], "out": s["out"]}
    slot, ranges = _slots(s["ids"], s["experts"], s["cap"])
    kept = slot >= 0
    at = torch.where(kept, slot, s["rows"].shape[0]).long().reshape(-1)   # (one row more takes what goes nowhere)
    rows = torch.zeros(s["rows"].shape[0] + 1, s["d"], dtype=s["x"].dtype, device=DEV)
    rows[at] = s["x"].repeat_interleave(s["k"], 0)
    back = s["out_rows"].float()[slot.clamp(min=0).long()] * torch.where(kept, s["weights"], 0.0)[:, :, None]
    return {"rows": rows[:-1], "slot": slot, "ranges": ranges, "out": back.sum(1).to(s["x"].dtype)}


def _run_experts_bwd(s):
    if own:
        import paper_1806_00187_amd as A
        A.nmt_op_expert_combine_bwd(s["dout"], s["out_rows"], s["slot"], s["weights"], s["dout_rows"], s["dweights"], s["ranges"], s["cap"])
        A.nmt_op_expert_combine(s["dx_rows"], s["slot"], None, s["dx"])
        return {"dout_rows": s["dout_rows"], "dweights": s["dweights"], "dx": s["dx"]}
    T, slot = s["dout"].dtype, s["slot"]
    kept = (slot >= 0)[:, :, None]
    at, from_ = torch.where(slot >= 0, slot, s["out_rows"].shape[0]).long().reshape(-1), slot.clamp(min=0).long()
    dout = s["dout"].float()
    dout_rows = torch.zeros(s["out_rows"].shape[0] + 1, s["d"], dtype=T, device=DEV)
    dout_rows[at] = (dout[:, None, :] * s["weights"][:, :, None]).to(T).reshape(-1, s["d"])
    dweights = torch.where(kept, dout[:, None, :] * s["out_rows"].float()[from_], 0.0).sum(2)
    dx = torch.where(kept, s["dx_rows"].float()[from_], 0.0).sum(1)
    return {"dout_rows": dout_rows[:-1], "dweights": dweights, "dx": dx.to(T)}


LR, BETAS, ADAM_EPS = 5e-4, (0.9, 0.98), 1e-8


def _to_8_bits(x, keep):
    """Codes and scales of x [blocks, 256]; keep: what is not zero stays so."""
    top = x.abs().amax(1, keepdim=True)
    scale = top * (1 / TOP)
    code = (x * torch.where(top > 2.0 ** -100, torch.ones_like(top) / scale, 0.0)).to(torch.float8_e4m3fn)
    if keep:
        code = torch.where((code.float() == 0) & (x > 0) & (top > 2.0 ** -100), 2.0 ** -9, code.float()).to(torch.float8_e4m3fn)
    return code.view(-1), scale.view(-1)


def _run_adamw(s):
    s["t"] += 1
    if own:
        import paper_1806_00187_amd as A
        A.nmt_adamw_step(s["plan"].handle, LR, BETAS[0], BETAS[1], ADAM_EPS, s["t"], grad_scale=s["grad_scale"])
    else:
        b1, b2 = BETAS
        g = s["grad"].float().view(-1, BLOCK) * s["grad_scale"]
        m, v = s["m"].float().view(-1, BLOCK), s["v"].float().view(-1, BLOCK)
        if s["bits"] == 8:
            m, v = m * s["m_scale"][:, None], v * s["v_scale"][:, None]
            v = v * v
        m = m * b1 + g * (1 - b1)
        v = v * b2 + (g * g) * (1 - b2)
        w = s["master"].view(-1, BLOCK)
        step = (m * (1 / (1 - b1 ** s["t"]))) / (torch.sqrt(v * (1 / (1 - b2 ** s["t"]))) + ADAM_EPS)
        w = w - (s["lr_factor"] * LR) * (step + s["decay"] * w)
        s["master"].copy_(w.view(-1))
        if s["weights"] is not None:
            s["weights"].copy_(w.view(-1))
        if s["bits"] == 8:
            s["m"], s["m_scale"] = _to_8_bits(m, False)
            s["v"], s["v_scale"] = _to_8_bits(torch.sqrt(v), True)
        else:
            s["m"], s["v"] = m.view(-1), v.view(-1)
    out = {"master": s["master"], "m": s["m"], "v": s["v"]}
    if s["weights"] is not None:
        out["weights"] = s["weights"]
    if s["bits"] == 8:
        out["m_scale"], out["v_scale"] = s["m_scale"], s["v_scale"]
    return out


# ---- work and exact values -----------------------------------------------------------------------
def work(case):
    if case["op"].startswith("norm"):
        n, z = case["rows"] * case["d"], SIZE[case["dtype"]]
        gates = (-(-case["rows"] // case["gate_rows"]) if case["gate_rows"] else 1) * case["d"] * z
        if case["op"] == "norm_fwd":   # x, y read; h, n written
            return {"bytes": 4 * n * z + gates + 16 * case["rows"], "flops": 20 * n}
        return {"bytes": 6 * n * z + 2 * gates + 16 * case["rows"], "flops": 40 * n}   # h, y, dh, dn read; dx, dy written
    if case["op"].startswith("experts"):
        z, d = SIZE[case["dtype"]], case["d"]
        routed = case["tokens"] * case["k"] * (1 - case["unrouted"])
        rows = case["experts"] * _room(case) if case["room"] else routed
        kept = min(rows, routed)
        lists = 4 * case["tokens"] * case["k"]
        if case["op"] == "experts_fwd":   # x read, rows written, rows read, out written; ids, weights read, slots written
            return {"bytes": (2 * case["tokens"] + rows + kept) * d * z + 3 * lists, "flops": 2 * kept * d}
        # dout, rows read, rows written, rows read, dx written; slots, weights read, their gradients written
        return {"bytes": (2 * case["tokens"] + rows + 2 * kept) * d * z + 3 * lists, "flops": 4 * kept * d}
    n = sum(t[0] for t in _tensors(case))
    state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * (8 + state + SIZE[case["grad"]] + SIZE.get(case["copy"], 0)), "flops": 20 * n}


def _e4m3(x):
    """The nearest values of four exponent and three mantissa bits, ties to even, in 64 bits."""
    exponent = torch.frexp(x).exponent.clamp(min=-5) - 4    # steps of 2^-9 below 2^-6
    step = torch.ldexp(torch.ones_like(x), exponent)
    return torch.round(x / step) * step


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    D = torch.float64
    if s["op"].startswith("norm"):
        wide = lambda v: None if v is None else v.to(D).requires_grad_()  # noqa: E731
        post, pre, gate, y = [wide(v) for v in s["post"]], [wide(v) for v in s["pre"]], wide(s["gate"]), wide(s["y"])
        per = torch.arange(s["rows"], device=DEV) // s["rows_per_gate"]

        def norm(a, gain, shift):
            mean = a.mean(1, keepdim=True) if s["kind"] == "layer" else a.new_zeros(a.shape[0], 1)
            var = (a - mean).square().mean(1, keepdim=True)
            out = (a - mean) * (var + EPS) ** -0.5 * gain
            return (out if shift is None else out + shift), mean, (var + EPS) ** -0.5

        z, mean_y, rstd_y = norm(y, *post)
        branch = z * gate[per]
        if s["op"] == "norm_fwd":
            h = s["resid_scale"] * s["x"].to(D) + branch
            n, mean_h, rstd_h = norm(h, *pre)
            return {"h": h.detach(), "n": n.detach(), "stats": torch.cat([mean_y, rstd_y, mean_h, rstd_h], 1).detach()}
        # h is an input of the backward pass, as it was stored: what its norm gives back is taken at that value, and goes on through the sum
        h = s["h"].to(D).requires_grad_()
        n = norm(h, *pre)[0]
        n.backward(s["dn"].to(D))
        dh = h.grad + s["dh"].to(D)
        branch.backward(dh)
        return {"dx": s["resid_scale"] * dh, "dy": y.grad, "dgate": gate.grad, "dpost": tuple(None if v is None else v.grad for v in post),
                "dpre": tuple(None if v is None else v.grad for v in pre)}
    if s["op"].startswith("experts"):
        T, E, cap, k = s["tokens"], s["experts"], s["cap"], s["k"]
        ids = s["ids"].reshape(-1).cpu()
        slot, ranges, start = torch.full((T * k,), -1, dtype=torch.int32), torch.zeros(E, 2, dtype=torch.int32), 0
        for e in range(E):
            mine = (ids == e).nonzero().reshape(-1)
            if cap:
                mine, start = mine[:cap], e * cap
            slot[mine] = torch.arange(start, start + len(mine), dtype=torch.int32)
            ranges[e] = torch.tensor([start, len(mine)])
            start += len(mine)
        slot, kept = slot.to(DEV), (slot >= 0).nonzero().reshape(-1).to(DEV)
        token, at = kept // k, slot[kept].long()
        weight = s["weights"].reshape(-1)[kept].to(D)[:, None]
        n, d = s["out_rows"].shape
        if s["op"] == "experts_fwd":
            rows = torch.zeros(n, d, dtype=D, device=DEV)
            rows[at] = s["x"].to(D)[token]
            out = torch.zeros(T, d, dtype=D, device=DEV).index_add_(0, token, weight * s["out_rows"].to(D)[at])
            return {"rows": rows, "slot": slot.view(T, k), "ranges": ranges.to(DEV), "out": out}
        dout = s["dout"].to(D)
        dout_rows = torch.zeros(n, d, dtype=D, device=DEV)
        dout_rows[at] = weight * dout[token]
        dweights = torch.zeros(T * k, dtype=D, device=DEV)
        dweights[kept] = (dout[token] * s["out_rows"].to(D)[at]).sum(1)
        dx = torch.zeros(T, d, dtype=D, device=DEV).index_add_(0, token, s["dx_rows"].to(D)[at])
        return {"dout_rows": dout_rows, "dweights": dweights.view(T, k), "dx": dx}
    t, g = s["t"] + 1, s["grad"].to(D) * s["grad_scale"]
    spread = lambda scale: scale.to(D).repeat_interleave(BLOCK)  # noqa: E731
    m, v = s["m"].to(D), s["v"].to(D)
    if s["bits"] == 8:
        m, v = m * spread(s["m_scale"]), (v * spread(s["v_scale"])) ** 2
    m, v = m + (1 - BETAS[0]) * (g - m), v + (1 - BETAS[1]) * (g ** 2 - v)
    rate = LR * s["lr_factor"].to(D).expand(-1, BLOCK).reshape(-1)
    w = s["master"].to(D) * (1 - rate * s["decay"].to(D).expand(-1, BLOCK).reshape(-1))
    w -= rate * m / (1 - BETAS[0] ** t) / ((v / (1 - BETAS[1] ** t)) ** 0.5 + ADAM_EPS)
    out = {"master": w}
    if s["weights"] is not None:
        out["weights"] = w
    if s["bits"] == 32:
        return {**out, "m": m, "v": v}
    for name, x in (("m", m), ("v", v ** 0.5)):
        scale = x.view(-1, BLOCK).abs().amax(1) / TOP
        code = _e4m3(x / spread(scale).clamp(min=1e-300))
        out[name] = torch.where((code == 0) & (x > 0), 2.0 ** -9, code) if name == "v" else code
        out[name + "_scale"] = scale
    return out
