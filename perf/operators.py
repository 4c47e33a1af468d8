"""The operators of a layer of experts and of 8-bit weights, each on its own: what they compute in plain form, and the
calls a program makes of the library for them.

Two layouts that the operators share, each one allocation of bytes:
  8-bit weights   values (e4m3) [experts, n, Kp], Kp = cols rounded up to 128, zeros behind cols; then fp32 scales
                  [experts, ceil(n / 128), Kp / 128], one per block of 128 x 128
  8-bit rows      values (e4m3) [rows, Kp]; then scale exponents (a byte e stands for 2^(e - 127)) [rows, Kp / 128 rounded up to 4]
and routed slots: pairs of an int32 expert (below 0: an empty slot) and an fp32 weight, [rows, k].
"""
import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 128
MOST_FLOPS = 2 * 32768 * 1024 * 2048       # of one pass: the largest listed product

_streams = {}


def _stream():
    """One stream for all passes, as in a server that answers one request after the other."""
    dev = torch.cuda.current_device()
    if dev not in _streams:
        _streams[dev] = torch.cuda.Stream(device=dev)
    return _streams[dev]


def listed():
    return [
        # a single token's choice among 64 experts: latency
        {"name": "route_b1_e64", "kind": "route", "rows": 1, "experts": 64, "k": 8, "groups": 1, "kept": 1, "sigmoid": False, "bias": False,
         "renorm": True, "top2": False, "scale": 1.0, "masked": 0.0, "dtype": "bf16"},
        # a prompt's tokens, sigmoid scores with a balancing bias, half of the groups kept, a twentieth of the experts switched off
        {"name": "route_4096_e256_groups", "kind": "route", "rows": 4096, "experts": 256, "k": 8, "groups": 8, "kept": 4, "sigmoid": True, "bias": True,
         "renorm": True, "top2": True, "scale": 2.5, "masked": 0.05, "dtype": "f32"},
        # the activation of one token, in front of an 8-bit product
        {"name": "quantize_b1_2048", "kind": "quantize", "rows": 1, "cols": 2048, "dtype": "bf16"},
        # a prompt's activations
        {"name": "quantize_8192x4096", "kind": "quantize", "rows": 8192, "cols": 4096, "dtype": "bf16"},
        # one decode step's product, 8-bit weights against a bf16 activation
        {"name": "f8_b1_2048x2048", "kind": "gemv_f8", "rows": 1, "n": 2048, "cols": 2048, "h": "bf16", "out": "bf16"},
        # odd batch, ragged width and outputs, fp32 result (logits)
        {"name": "f8_b37_1000x520", "kind": "gemv_f8", "rows": 37, "n": 1000, "cols": 520, "h": "bf16", "out": "f32"},
        # a prompt: both operands in 8 bits
        {"name": "f8_4096x4096x4096", "kind": "gemv_f8", "rows": 4096, "n": 4096, "cols": 4096, "h": "f8", "out": "bf16"},
        # one token through 8 of 64 experts, 8-bit weights
        {"name": "experts_b1_e64", "kind": "expert_gemv", "rows": 1, "k": 8, "experts": 64, "n": 1024, "cols": 2048, "w": "f8", "h": "bf16",
         "per_slot": False, "empty": 0.0, "out": "bf16"},
        # a serving batch through bf16 experts, the second product: a row of h for each slot; ragged, with dropped tokens
        {"name": "experts_b64_e32_slots", "kind": "expert_gemv", "rows": 64, "k": 4, "experts": 32, "n": 2048, "cols": 1000, "w": "bf16", "h": "bf16",
         "per_slot": True, "empty": 0.05, "out": "bf16"},
        # a prompt through 64 experts, both operands in 8 bits
        {"name": "experts_4096_e64", "kind": "expert_gemv", "rows": 4096, "k": 8, "experts": 64, "n": 1024, "cols": 2048, "w": "f8", "h": "f8",
         "per_slot": False, "empty": 0.0, "out": "bf16"},
        # the experts' outputs joined, one token
        {"name": "sum_b1_k8", "kind": "expert_sum", "rows": 1, "k": 8, "n": 2048, "dtype": "bf16", "residual": True, "empty": 0.0},
        # and a prompt's
        {"name": "sum_4096_k8", "kind": "expert_sum", "rows": 4096, "k": 8, "n": 2048, "dtype": "bf16", "residual": True, "empty": 0.02},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """A width: the usual multiples, and one in four odd."""
    step = rng.choice([1, 8, 128, 128])
    return max(lo, _log_int(rng, lo, hi) // step * step)


def draw(rng):
    kind = rng.choice(["route", "quantize", "gemv_f8", "gemv_f8", "expert_gemv", "expert_gemv", "expert_gemv", "expert_sum"])
    if kind == "route":
        rows = _log_int(rng, 1, 4096)
        groups = rng.choice([1, 1, 4, 8])
        experts = groups * _log_int(rng, 2, 256 // groups)
        kept = rng.randint(1, groups)
        return {"kind": kind, "rows": rows, "experts": experts, "k": rng.randint(1, min(8, experts // groups * kept)), "groups": groups, "kept": kept,
                "sigmoid": rng.random() < 0.5, "bias": rng.random() < 0.5, "renorm": rng.random() < 0.5, "top2": rng.random() < 0.5,
                "scale": rng.choice([1.0, 2.5]), "masked": rng.choice([0.0, 0.1, 0.5]), "dtype": rng.choice(["f32", "bf16"])}
    if kind == "quantize":
        cols = _size(rng, 64, 8192)
        return {"kind": kind, "rows": _log_int(rng, 1, (8192 * 4096) // cols // 2), "cols": cols, "dtype": rng.choice(["f32", "bf16"])}
    if kind == "expert_sum":
        n, k = _size(rng, 64, 8192), rng.randint(1, 8)
        return {"kind": kind, "rows": _log_int(rng, 1, max(1, (4096 * 8 * 2048) // (n * k * 2))), "k": k, "n": n, "dtype": rng.choice(["f32", "bf16"]),
                "residual": rng.random() < 0.5, "empty": rng.choice([0.0, 0.1])}
    n, cols = _size(rng, 64, 8192), _size(rng, 64, 8192)
    if kind == "gemv_f8":
        return {"kind": kind, "rows": _log_int(rng, 1, min(4096, MOST_FLOPS // (2 * n * cols))), "n": n, "cols": cols,
                "h": rng.choice(["bf16", "f8"]), "out": rng.choice(["bf16", "bf16", "f32"])}
    w = rng.choice(["bf16", "f8", "f8"])
    experts = _log_int(rng, 2, max(2, min(128, (1 << 28) // (n * cols))))
    k = rng.randint(1, min(8, experts))
    return {"kind": kind, "rows": _log_int(rng, 1, max(1, min(4096, MOST_FLOPS // (2 * n * cols * k)))), "k": k, "experts": experts, "n": n, "cols": cols,
            "w": w, "h": "bf16" if w == "bf16" else rng.choice(["bf16", "f8"]), "per_slot": rng.random() < 0.5, "empty": rng.choice([0.0, 0.0, 0.1]),
            "out": rng.choice(["bf16", "bf16", "f32"])}


# ---- the layouts -------------------------------------------------------------------------------------------
def _up(x, to):
    return (x + to - 1) // to * to


def _two_to(e):
    """2^e in fp32, -126 <= e <= 127, exactly: from its bits."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _exponents(amax):
    """Least e in [-126, 127] with amax <= 448 * 2^e: 448 is 0.875 * 2^9."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(-126, 127)
    return torch.where(amax > 0, e, torch.full_like(e, -126))


def _quantized(x):
    """(e4m3 values [rows, Kp], exponent bytes [rows, Kp / 128]) of x [rows, cols]."""
    rows, cols = x.shape
    b = torch.nn.functional.pad(x.float(), (0, _up(cols, BLOCK) - cols)).view(rows, -1, BLOCK)
    finite = torch.isfinite(b)
    e = _exponents(torch.where(finite, b.abs(), torch.zeros_like(b)).amax(-1))
    q = torch.where(finite, b * _two_to(-e).unsqueeze(-1), torch.full_like(b, math.nan)).to(torch.float8_e4m3fn)
    return q.view(rows, -1), (e + 127).to(torch.uint8)


def _pack_rows(x):
    q, e = _quantized(x)
    e = torch.nn.functional.pad(e, (0, _up(e.shape[1], 4) - e.shape[1]), value=127)
    return torch.cat([q.view(torch.uint8).reshape(-1), e.reshape(-1)])


def _rows_parts(buf, rows, cols):
    kp = _up(cols, BLOCK)
    nb = kp // BLOCK
    return buf[:rows * kp].view(torch.float8_e4m3fn).view(rows, kp), buf[rows * kp:].view(rows, _up(nb, 4))[:, :nb]


def _pack_weights(x):
    """8-bit weights of x [experts, n, cols] fp32: per block the scale that takes its largest value to 448."""
    experts, n, cols = x.shape
    np_, kp = _up(n, BLOCK), _up(cols, BLOCK)
    b = torch.nn.functional.pad(x, (0, kp - cols, 0, np_ - n)).view(experts, np_ // BLOCK, BLOCK, kp // BLOCK, BLOCK)
    s = (b.abs().amax((2, 4)) / 448.0).clamp(min=1e-20)
    q = (b / s[:, :, None, :, None]).to(torch.float8_e4m3fn).view(experts, np_, kp)[:, :n]
    return torch.cat([q.contiguous().view(torch.uint8).reshape(-1), s.contiguous().view(torch.uint8).reshape(-1)])


def _weights_parts(buf, experts, n, cols):
    np_, kp = _up(n, BLOCK), _up(cols, BLOCK)
    return (buf[:experts * n * kp].view(torch.float8_e4m3fn).view(experts, n, kp),
            buf[experts * n * kp:].view(torch.float32).view(experts, np_ // BLOCK, kp // BLOCK))


# ---- inputs ------------------------------------------------------------------------------------------------
def _activations(g, rows, cols):
    """Rows of different sizes, a few columns much larger than the rest, as activations have."""
    x = torch.randn(rows, cols, device=DEVICE, generator=g)
    x *= torch.exp(0.5 * torch.randn(rows, 1, device=DEVICE, generator=g))
    x *= torch.where(torch.rand(1, cols, device=DEVICE, generator=g) < 0.01, 8.0, 1.0)
    return x


def _routed(g, rows, k, experts, empty):
    """k different experts a row, some of them more popular than others; weights that sum to one; some slots empty."""
    popular = torch.randn(experts, device=DEVICE, generator=g) * 0.3
    u = torch.rand(rows, experts, device=DEVICE, generator=g).clamp(1e-9, 1 - 1e-7)
    ids = torch.topk(popular - torch.log(-torch.log(u)), k, dim=1).indices.to(torch.int32)
    w = torch.rand(rows, k, device=DEVICE, generator=g) + 0.1
    w /= w.sum(1, keepdim=True)
    if empty:
        gone = torch.rand(rows, k, device=DEVICE, generator=g) < empty
        ids, w = torch.where(gone, -1, ids).to(torch.int32), torch.where(gone, 0.0, w)
    return torch.stack([ids, w.view(torch.int32)], -1).contiguous()


def _make(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    kind, rows, s = case["kind"], case["rows"], {"case": case}
    if kind == "route":
        x = torch.randn(rows, case["experts"], device=DEVICE, generator=g) * 1.5
        if case["masked"]:
            x = torch.where(torch.rand(x.shape, device=DEVICE, generator=g) < case["masked"], -math.inf, x)
        s["scores"] = x.to(DTYPES[case["dtype"]])
        s["bias"] = torch.randn(case["experts"], device=DEVICE, generator=g) * 0.05 if case["bias"] else None
    elif kind == "quantize":
        s["x"] = _activations(g, rows, case["cols"]).to(DTYPES[case["dtype"]])
    elif kind == "expert_sum":
        s["z"] = torch.randn(rows, case["k"], case["n"], device=DEVICE, generator=g).to(DTYPES[case["dtype"]])
        s["routed"] = _routed(g, rows, case["k"], 64, case["empty"])
        s["x"] = torch.randn(rows, case["n"], device=DEVICE, generator=g).to(DTYPES[case["dtype"]]) if case["residual"] else None
    else:
        experts = case.get("experts", 1)
        w = torch.randn(experts, case["n"], case["cols"], device=DEVICE, generator=g) * 0.02
        s["w"] = w.to(torch.bfloat16) if case.get("w") == "bf16" else _pack_weights(w)
        h = _activations(g, rows * (case["k"] if case.get("per_slot") else 1), case["cols"])
        s["h"] = h.to(torch.bfloat16) if case["h"] == "bf16" else _pack_rows(h)
        if kind == "expert_gemv":
            s["routed"] = _routed(g, rows, case["k"], experts, case["empty"])
    return s


def _chain(s):
    """The chain of one kernel that a program keeps for this operator: weights inside, everything else fresh in each call."""
    import paper_2503_19779_amd as pg
    from pg_workloads import ChainSpec, EXT, INT, KernelSpec, Ref, TensorSpec, WEIGHT

    c = s["case"]
    kind, rows, e, w = c["kind"], c["rows"], lambda i: Ref(EXT, i), lambda i: Ref(WEIGHT, i)
    if kind == "route":
        flags = pg.ROUTE_SIGMOID * c["sigmoid"] | pg.ROUTE_RENORMALIZE * c["renorm"] | pg.ROUTE_GROUP_TOP2 * c["top2"]
        k = KernelSpec("route", c["dtype"], 0, (e(0), w(0)) if c["bias"] else (e(0),), c["k"], rows=rows, cols=c["experts"], m=c["groups"], inner=c["kept"],
                       eps=c["scale"], flags=flags)
        ext, ints = [TensorSpec(c["dtype"], rows * c["experts"])], [TensorSpec("routed", rows * c["k"])]
        weights, s["ext"] = [s["bias"]] if c["bias"] else [], [s["scores"]]
    elif kind == "quantize":
        k = KernelSpec("quantize", c["dtype"], 0, (e(0),), c["cols"], rows=rows, cols=c["cols"])
        ext, ints = [TensorSpec(c["dtype"], rows * c["cols"])], [TensorSpec("f8_rows", pg.scaled_rows_bytes(rows, c["cols"]))]
        weights, s["ext"] = [], [s["x"]]
    elif kind == "expert_sum":
        k = KernelSpec("expert_sum", c["dtype"], 0, (e(0), e(1), e(2)) if c["residual"] else (e(0), e(1)), c["n"], rows=rows, m=c["k"])
        ext = [TensorSpec(c["dtype"], rows * c["k"] * c["n"]), TensorSpec("routed", rows * c["k"])]
        s["ext"] = [s["z"], s["routed"]]
        if c["residual"]:
            ext.append(TensorSpec(c["dtype"], rows * c["n"]))
            s["ext"].append(s["x"])
        ints, weights = [TensorSpec(c["dtype"], rows * c["n"])], []
    else:
        slots = rows * c.get("k", 1)
        hrows = slots if c.get("per_slot") else rows
        ext = [TensorSpec("bf16", hrows * c["cols"]) if c["h"] == "bf16" else TensorSpec("f8_rows", pg.scaled_rows_bytes(hrows, c["cols"]))]
        ints, weights, s["ext"] = [TensorSpec(c["out"], slots * c["n"])], [s["w"]], [s["h"]]
        if kind == "gemv_f8":
            k = KernelSpec("gemv_f8", c["out"], 0, (w(0), e(0)), c["n"], rows=rows, cols=c["cols"])
        else:
            k = KernelSpec("expert_gemv", c["out"], 0, (w(0), e(0), e(1)), c["n"], rows=rows, cols=c["cols"], m=c["k"], inner=c["experts"],
                           flags=pg.EXPERT_PER_SLOT * c["per_slot"])
            ext.append(TensorSpec("routed", slots))
            s["ext"].append(s["routed"])
    names = {torch.float32: "f32", torch.bfloat16: "bf16", torch.uint8: "f8_weight"}
    spec = ChainSpec(kind, [k], ext, ints, [TensorSpec(names[t.dtype], t.numel()) for t in weights], [0])
    return pg.Chain(spec, weights, DEVICE)


def prepare(case, seed):
    s = _make(case, seed)
    if own:
        torch.cuda.synchronize()       # the draws ran on torch's current stream, the chain runs on its own
        c = s["case"]
        s["chain"] = chain = _chain(s)
        if c["kind"] == "route":
            s["out"] = chain.routed(0, c["rows"], c["k"])
        elif c["kind"] == "quantize":
            s["out"] = chain.scaled_rows(0, c["rows"], c["cols"])
        else:
            s["out"] = chain.int_buffer(0).view((c["rows"], c["k"], c["n"]) if c["kind"] == "expert_gemv" else (c["rows"], c["n"]))
    return s


# ---- one pass ----------------------------------------------------------------------------------------------
def _route(s):
    c = s["case"]
    x = s["scores"].double()            # the choice in 64 bits: scores next to each other
    rows, experts = x.shape
    valid = x > -math.inf
    if c["sigmoid"]:
        p = torch.sigmoid(x)
    else:
        top = torch.where(valid, x, -math.inf).amax(1, keepdim=True)
        p = torch.where(valid, torch.exp(x - top), 0.0)
        p = p / p.sum(1, keepdim=True)
    # without a bias the scores themselves are in the order of p
    key = torch.where(valid, p + s["bias"].double() if c["bias"] else x, -math.inf)
    if c["groups"] > 1:
        by = torch.where(valid, p, -math.inf) if c["top2"] and not c["bias"] else key
        by = by.view(rows, c["groups"], -1)
        if c["top2"]:
            two = by.topk(min(2, by.shape[2]), dim=2).values
            best = two[..., 0] + torch.where(two > -math.inf, two, 0.0)[..., 1:].sum(2)
        else:
            best = by.amax(2)
        first = torch.sort(best, dim=1, descending=True, stable=True).indices[:, :c["kept"]]
        keep = torch.zeros_like(best, dtype=torch.bool).scatter_(1, first, True)
        key = torch.where(keep.unsqueeze(2).expand(by.shape).reshape(rows, experts), key, -math.inf)
    key, ids = torch.sort(key, dim=1, descending=True, stable=True)
    key, ids = key[:, :c["k"]], ids[:, :c["k"]]
    chosen = key > -math.inf
    w = torch.where(chosen, p.gather(1, ids), 0.0)
    if c["renorm"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, 0.0)
    return [torch.where(chosen, ids, -1).to(torch.int32), (w * c["scale"]).float()]


def _rows_f32(h, rows, cols):
    if h.dtype == torch.bfloat16:
        return h.float().view(rows, cols)
    q, e = _rows_parts(h, rows, cols)
    return (q.float().view(rows, -1, BLOCK) * _two_to(e.to(torch.int32) - 127).unsqueeze(2)).view(rows, -1)[:, :cols]


def _weights_f32(w, experts, n, cols, of=None):
    """fp32 weights of all experts, or of the given ones."""
    if w.dtype == torch.bfloat16:
        w = w.view(experts, n, cols)
        return (w if of is None else w[of]).float()
    q, s = _weights_parts(w, experts, n, cols)
    if of is not None:
        q, s = q.view(torch.uint8)[of].view(torch.float8_e4m3fn), s[of]
    s = s.repeat_interleave(BLOCK, 1)[:, :n].repeat_interleave(BLOCK, 2)
    return (q.float() * s)[:, :, :cols]


def _expert_gemv(s):
    c = s["case"]
    rows, k, experts, n, cols = c["rows"], c["k"], c["experts"], c["n"], c["cols"]
    slots = rows * k
    ids = s["routed"][..., 0].reshape(-1).long()
    used = ids >= 0
    h = _rows_f32(s["h"], slots if c["per_slot"] else rows, cols)
    if not c["per_slot"]:
        h = h.repeat_interleave(k, 0)
    if slots <= experts:                # few slots: each with its expert's matrix
        y = torch.bmm(_weights_f32(s["w"], experts, n, cols, ids.clamp(min=0)), h.unsqueeze(2)).squeeze(2)
    else:                               # else every expert with its slots, as many as the fullest has
        order = torch.sort(torch.where(used, ids, experts), stable=True).indices
        count = torch.bincount(ids[used], minlength=experts)
        start = torch.cumsum(count, 0) - count
        at = torch.arange(max(1, int(count.max())), device=DEVICE)
        place = torch.where(at < count.unsqueeze(1), start.unsqueeze(1) + at, 0)
        slot = order[place]
        each = torch.bmm(h[slot], _weights_f32(s["w"], experts, n, cols).transpose(1, 2))
        y = torch.zeros(slots + 1, n, device=DEVICE)
        y[torch.where(at < count.unsqueeze(1), slot, slots).view(-1)] = each.view(-1, n)
        y = y[:slots]
    return torch.where(used.unsqueeze(1), y, 0.0).to(DTYPES[c["out"]]).view(rows, k, n)


def run(s):
    c = s["case"]
    if own:
        s["chain"].eager(s["ext"], _stream())
        return s["out"]
    kind, rows = c["kind"], c["rows"]
    if kind == "route":
        return _route(s)
    if kind == "quantize":
        return list(_quantized(s["x"]))
    if kind == "gemv_f8":
        w = _weights_f32(s["w"], 1, c["n"], c["cols"])[0]
        return (_rows_f32(s["h"], rows, c["cols"]) @ w.t()).to(DTYPES[c["out"]])
    if kind == "expert_gemv":
        return _expert_gemv(s)
    used = s["routed"][..., 0] >= 0
    w = torch.where(used, s["routed"][..., 1].contiguous().view(torch.float32), 0.0).unsqueeze(2)
    y = (w * torch.where(used.unsqueeze(2), s["z"].float(), 0.0)).sum(1)
    return (y + s["x"].float() if c["residual"] else y).to(s["z"].dtype)


def work(case):
    kind, rows = case["kind"], case["rows"]
    size = {"f32": 4, "bf16": 2, "f8": 1}
    if kind == "route":
        n = rows * case["experts"]
        return {"bytes": n * size[case["dtype"]] + 8 * rows * case["k"] + 4 * case["experts"] * case["bias"], "flops": 8 * n}
    if kind == "quantize":
        n = rows * case["cols"]
        return {"bytes": n * size[case["dtype"]] + n + n // BLOCK, "flops": 3 * n}
    if kind == "expert_sum":
        n = rows * case["n"]
        return {"bytes": n * (case["k"] + 1 + case["residual"]) * size[case["dtype"]] + 8 * rows * case["k"], "flops": 2 * n * case["k"]}
    n, cols, k = case["n"], case["cols"], case.get("k", 1)
    hit = 1 if kind == "gemv_f8" else case["experts"] * (1 - (1 - k / case["experts"]) ** rows)     # experts that some row chooses
    used = rows * k * (1 - case.get("empty", 0.0))
    h = rows * (k if case.get("per_slot") else 1) * cols * size[case["h"]]
    return {"bytes": hit * n * cols * size[case.get("w", "f8")] + h + rows * k * n * size[case["out"]] + (8 * rows * k if kind == "expert_gemv" else 0),
            "flops": 2 * used * n * cols}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------
def _pow2(e):
    """2^e in fp64, exactly."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _e4m3(b):
    """What the bytes stand for: sign, four bits of exponent (bias 7), three of mantissa; all ones: not a number."""
    b = b.to(torch.int64)
    e, m = (b >> 3) & 15, b & 7
    v = torch.where(e == 0, m.double() * 2.0 ** -9, (8 + m).double() * _pow2(e - 10))
    v = torch.where((e == 15) & (m == 7), math.nan, v)
    return torch.where(b >= 128, -v, v)


def _exact_rows(h, rows, cols):
    if h.dtype == torch.bfloat16:
        return h.double().view(rows, cols)
    kp = (cols + 127) // 128 * 128
    e = h[rows * kp:].view(rows, -1).to(torch.int64)
    at = torch.arange(cols, device=DEVICE)
    return _e4m3(h[:rows * kp].view(rows, kp)[:, :cols]) * _pow2(e[:, at // 128] - 127)


def _exact_weights(w, experts, n, cols, x):
    if w.dtype == torch.bfloat16:
        return w.view(experts, n, cols)[x].double()
    kp = (cols + 127) // 128 * 128
    nb = kp // 128
    s = w[experts * n * kp:].view(torch.float32).view(experts, -1, nb)[x].double()
    j, i = torch.arange(n, device=DEVICE) // 128, torch.arange(cols, device=DEVICE) // 128
    return _e4m3(w[:experts * n * kp].view(experts, n, kp)[x, :, :cols]) * s[j][:, i]


def exact(case, seed):
    s = _make(case, seed)
    kind, rows = case["kind"], case["rows"]
    if kind == "route":
        x = s["scores"].double().cpu()
        experts, n_groups = x.shape[1], case["groups"]
        ok = ~(torch.isnan(x) | (x == -math.inf))
        z = torch.where(ok, x, -math.inf)
        if case["sigmoid"]:
            p = torch.where(ok, 1.0 / (1.0 + torch.exp(-z)), 0.0)
        else:
            p = torch.where(ok, torch.exp(z - torch.logsumexp(z, 1, keepdim=True)), 0.0)
        c = torch.where(ok, (p + s["bias"].double().cpu()) if case["bias"] else (p if case["top2"] and n_groups > 1 else z), -math.inf)
        open_ = ok.clone()
        if n_groups > 1:
            per = experts // n_groups
            score = torch.full((rows, n_groups), -math.inf, dtype=torch.float64)
            for j in range(n_groups):
                part = torch.sort(c[:, j * per:(j + 1) * per], dim=1, descending=True).values
                score[:, j] = part[:, 0]
                if case["top2"] and per > 1:
                    score[:, j] += torch.where(part[:, 1] > -math.inf, part[:, 1], 0.0)
            kept = torch.zeros(rows, n_groups, dtype=torch.bool)
            for _ in range(case["kept"]):
                best = torch.where(kept, -math.inf, score).argmax(1)        # (of equals the first)
                kept[torch.arange(rows), best] = True
            open_ &= kept.repeat_interleave(per, 1)
        c = z if not case["bias"] else c
        ids, w = torch.full((rows, case["k"]), -1, dtype=torch.int32), torch.zeros(rows, case["k"], dtype=torch.float64)
        r = torch.arange(rows)
        for j in range(case["k"]):
            left = torch.where(open_, c, -math.inf)
            best = left.argmax(1)
            got = left[r, best] > -math.inf
            ids[:, j] = torch.where(got, best, -1).to(torch.int32)
            w[:, j] = torch.where(got, p[r, best], 0.0)
            open_[r, best] = False
        if case["renorm"]:
            t = w.sum(1, keepdim=True)
            w = torch.where(t > 0, w / t, 0.0)
        return [ids, w * case["scale"]]
    if kind == "quantize":
        x = s["x"].double()
        pad = (-case["cols"]) % 128
        b = torch.cat([x, torch.zeros(rows, pad, dtype=torch.float64, device=DEVICE)], 1).view(rows, -1, 128) if pad else x.view(rows, -1, 128)
        a = b.abs().amax(2)
        e = torch.frexp(a).exponent.to(torch.int64) - 9                    # 2^(e + 8) <= a < 2^(e + 9)
        e = torch.where(a > _pow2(e) * 448.0, e + 1, e).clamp(-126, 127)
        e = torch.where(a > 0, e, -126)
        v = b / _pow2(e).unsqueeze(2)
        step = _pow2(torch.frexp(v).exponent.clamp(min=-5) - 4)            # the spacing of e4m3 around v
        return [(torch.round(v / step) * step).view(rows, -1), (e + 127).to(torch.uint8)]
    if kind == "expert_sum":
        used = s["routed"][..., 0] >= 0
        w = s["routed"][..., 1].contiguous().view(torch.float32).double()
        y = s["x"].double() if case["residual"] else torch.zeros(rows, case["n"], dtype=torch.float64, device=DEVICE)
        for j in range(case["k"]):
            y = y + torch.where(used[:, j:j + 1], w[:, j:j + 1] * s["z"][:, j].double(), 0.0)
        return y
    n, cols = case["n"], case["cols"]
    if kind == "gemv_f8":
        return _exact_rows(s["h"], rows, cols) @ _exact_weights(s["w"], 1, n, cols, 0).t().contiguous()
    k = case["k"]
    ids = s["routed"][..., 0].reshape(-1)
    h = _exact_rows(s["h"], rows * (k if case["per_slot"] else 1), cols)
    y = torch.zeros(rows * k, n, dtype=torch.float64, device=DEVICE)
    for x in range(case["experts"]):
        at = torch.nonzero(ids == x).view(-1)
        if at.numel():
            y[at] = h[at if case["per_slot"] else at // k] @ _exact_weights(s["w"], case["experts"], n, cols, x).t().contiguous()
    return y.view(rows, k, n)
