"""Plain 64-bit forms of the kernels of experts and of 8-bit weights, on CPU tensors, and how far a kernel may be from them.  What is
held in 8 bits is decoded from its bits here."""
import math

import torch

BLOCK = 128


def up(x, to):
    return (x + to - 1) // to * to


def e4m3(b):
    """What bytes stand for: sign, exponent (bias 7), three bits of mantissa; all ones: not a number."""
    b = b.to(torch.int64)
    e, m = (b >> 3) & 15, b & 7
    v = torch.where(e == 0, m.double() * 2.0 ** -9, (8 + m).double() * torch.pow(2.0, (e - 10).double()))
    v = torch.where((e == 15) & (m == 7), math.nan, v)
    return torch.where(b >= 128, -v, v)


def pack_rows(x):
    """PG_F8_ROWS of x [rows, cols], by the definition: the least e with max |x| <= 448 * 2^e."""
    rows, cols = x.shape
    kb = up(cols, BLOCK) // BLOCK
    b = torch.zeros(rows, kb * BLOCK, dtype=torch.float64)
    b[:, :cols] = x.double()
    b = b.view(rows, kb, BLOCK)
    fine = torch.isfinite(b)
    top = torch.where(fine, b.abs(), 0.0).amax(2)
    e = torch.full(top.shape, -126, dtype=torch.int64)
    for _ in range(256):
        e = torch.where(top > 448.0 * torch.pow(2.0, e.double()), e + 1, e)
    v = torch.where(fine, b / torch.pow(2.0, e.double()).unsqueeze(2), 0.0)
    step = torch.pow(2.0, torch.frexp(v).exponent.clamp(min=-5).double() - 4)
    q = torch.round(v / step) * step                       # ties to even
    byte = _bytes(q)
    byte = torch.where(fine, byte, torch.full_like(byte, 0x7f))
    out = torch.full((rows * (kb * BLOCK + up(kb, 4)),), 127, dtype=torch.uint8)
    out[:rows * kb * BLOCK] = byte.reshape(-1)
    out[rows * kb * BLOCK:].view(rows, up(kb, 4))[:, :kb] = (e + 127).to(torch.uint8)
    return out


def _bytes(q):
    table = e4m3(torch.arange(256))
    order = torch.argsort(torch.where(torch.isnan(table), math.inf, table), stable=True)[:254]
    at = torch.searchsorted(table[order].contiguous(), q.contiguous())
    byte = order[at.clamp(max=253)]
    return torch.where(q == 0, torch.where(torch.signbit(q), 0x80, 0), byte).to(torch.uint8)


def rows_of(buf, rows, cols):
    kp = up(cols, BLOCK)
    s = buf[rows * kp:].view(rows, -1).to(torch.int64)
    return e4m3(buf[:rows * kp].view(rows, kp)[:, :cols]) * torch.pow(2.0, (s[:, torch.arange(cols) // BLOCK] - 127).double())


def pack_weight(w, g):
    """PG_F8_WEIGHT of random bytes around w's values, with random scales; returns (bytes, what they stand for in 64 bits)."""
    experts, n, cols = w.shape
    kp, nb = up(cols, BLOCK), up(n, BLOCK) // BLOCK
    s = torch.rand(experts, nb, kp // BLOCK, generator=g) * 2.0 + 0.25
    q = (w * 64).to(torch.float8_e4m3fn)
    v = torch.zeros(experts, n, kp, dtype=torch.uint8)
    v[..., :cols] = q.view(torch.uint8)
    each = s.double()[:, torch.arange(n) // BLOCK][:, :, torch.arange(cols) // BLOCK]
    return torch.cat([v.reshape(-1), s.contiguous().view(torch.uint8).reshape(-1)]), e4m3(q.view(torch.uint8)) * each


def route(s, bias, k, groups=1, kept=1, sigmoid=False, renorm=False, top2=False, factor=1.0):
    """One row after the other, in Python numbers."""
    rows, experts = s.shape
    ids, ws = torch.full((rows, k), -1, dtype=torch.int64), torch.zeros(rows, k, dtype=torch.float64)
    for r in range(rows):
        x = [min(float(v), 3.4028234663852886e38) if v == v else -math.inf for v in s[r].double().tolist()]
        b = [0.0] * experts if bias is None else [float(v) for v in bias.double().tolist()]
        ok = [v > -math.inf and c > -math.inf for v, c in zip(x, b)]
        scored = [v for v in x if v > -math.inf]
        if sigmoid:
            p = [0.0 if v == -math.inf else 1.0 / (1.0 + math.exp(-v)) if v > -700 else 0.0 for v in x]
        elif scored:
            top = max(scored)
            z = [math.exp(v - top) if v > -math.inf else 0.0 for v in x]
            p = [v / math.fsum(z) for v in z]
        else:
            p = [0.0] * experts
        c = [p[e] + b[e] if bias is not None else x[e] for e in range(experts)]
        open_ = [e for e in range(experts) if ok[e]]
        if groups > 1:
            per = experts // groups
            score = []
            for g in range(groups):
                mine = sorted((p[e] + b[e] if (top2 or bias is not None) else x[e] for e in open_ if e // per == g), reverse=True)
                score.append(-math.inf if not mine else sum(mine[:2]) if top2 else mine[0])
            best = sorted(range(groups), key=lambda g: (-score[g], g))[:kept]
            open_ = [e for e in open_ if e // per in best]
        chosen = sorted(open_, key=lambda e: (-c[e], e))[:k]
        w = [p[e] for e in chosen]
        if renorm:
            t = math.fsum(w)
            w = [v / t if t > 0 else 0.0 for v in w]
        for j, e in enumerate(chosen):
            ids[r, j], ws[r, j] = e, w[j] * factor
    return ids, ws


def product(w, h, ids=None, per_slot=False):
    """(y, sum |w h|): [rows, n], or [rows, k, n] for slots ids [rows, k]; w [experts, n, cols], h [rows (* k), cols], 64 bits."""
    if ids is None:
        return h @ w[0].t(), h.abs() @ w[0].abs().t()
    rows, k = ids.shape
    n = w.shape[1]
    y, a = torch.zeros(rows, k, n, dtype=torch.float64), torch.zeros(rows, k, n, dtype=torch.float64)
    for r in range(rows):
        for t in range(k):
            e = int(ids[r, t])
            if 0 <= e < w.shape[0]:
                v = h[r * k + t if per_slot else r]
                y[r, t], a[r, t] = w[e] @ v, w[e].abs() @ v.abs()
    return y, a


HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def sum_tolerance(y, absolute, terms, dtype, eight=False):
    """fp32 sums of `terms` products in any order, each addition off by at most a step 2^-23 (a matrix instruction may cut instead of rounding),
    and the scale's product; then half a step of the stored type, taken of the value with that error on it.  eight: products of the 8-bit
    matrix instruction, which drops below 2^-13 of the largest of eight products what the other seven have there: 7 * 2^-13 of the
    largest ones, whose sum `absolute` bounds."""
    e = ((terms + 2) * 2.0 ** -23 + (7 * 2.0 ** -13 if eight else 0.0)) * absolute
    return e + HALF_STEP[dtype] * (y.abs() + e) + 2.0 ** -133


def assert_within(got, want, tol, what):
    got = got.double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside; first at {bad.nonzero()[0].tolist()}: {got[bad][0]} for {want[bad][0]} +- {tol[bad][0]}"
