"""Routing, 8-bit rows and weights, experts' products and their sum, kernel by kernel against plain 64-bit forms, in every replay mode."""
import math

import pytest
import torch

import paper_2503_19779_amd as pg
import plain_experts as plain
from pg_workloads import ChainSpec, EXT, INT, KernelSpec, Ref, TensorSpec, WEIGHT

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NAMES = {torch.float32: "f32", torch.bfloat16: "bf16", torch.uint8: "f8_rows"}


def say(*a):
    print(*a, flush=True)


def spec_of(kernels, ext, ints, weights):
    return ChainSpec("experts", kernels, ext, ints, weights, [0])


class Run:
    """A chain in every mode, launched and as graphs; all leave the same bits in the internal buffers, whatever was there before."""

    def __init__(self, spec, weights, device="cuda:0"):
        self.weights = [w.to(device) for w in weights]
        self.chains = [pg.Chain(spec, self.weights, device) for _ in range(2)]
        self.stream = torch.cuda.Stream(device=device)
        torch.cuda.synchronize()
        self.chains[1].set_launched_dispatches(0)
        for c in self.chains:
            c.capture(self.stream)
        self.spec = spec

    def __call__(self, ext, written):
        """written: for each internal buffer the elements that the chain writes."""
        ext = [t.cuda() if not t.is_cuda else t for t in ext]
        first = None
        for c in self.chains:
            for mode in ("eager", "replay_copy", "replay_indirect", "replay_update"):
                for again in range(2):                 # graphs are replayed, with the same results
                    for i, t in enumerate(self.spec.ints):
                        c.int_buffer(i).fill_(-1 if t.dtype == "routed" else 255 if t.dtype == "f8_rows" else math.nan)
                    torch.cuda.synchronize()
                    getattr(c, mode)(ext, self.stream)
                    self.stream.synchronize()
                    got = [c.int_buffer(i)[:n].clone() for i, n in enumerate(written)]
                    for i, t in enumerate(self.spec.ints):      # nothing behind what the chain writes
                        rest = c.int_buffer(i)[written[i]:]
                        fill = rest.float()
                        assert bool(((fill == -1) | (fill == 255) | fill.isnan()).all()), (mode, i, "written behind the result")
                    if first is None:
                        first = got
                    for a, b in zip(first, got):
                        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), (mode, again)
        return first

    def close(self):
        for c in self.chains:
            c.close()


def run_one(kernel, ext, out, written, weights=(), wtypes=()):
    """Chain of one kernel; `out` (dtype, numel) with a few elements behind the result."""
    spec = spec_of([kernel], [TensorSpec(d, n) for d, n in ext["specs"]], [TensorSpec(out[0], out[1] + 64)], [TensorSpec(d, w.numel()) for d, w in zip(wtypes, weights)])
    r = Run(spec, list(weights))
    got = r(ext["tensors"], [written])[0]
    r.close()
    return got


def at_odd_element(t):
    """The same values one element further than an allocation starts."""
    big = torch.empty(t.numel() + 9, dtype=t.dtype, device="cuda")
    v = big[1:1 + t.numel()].view(t.shape)
    v.copy_(t)
    return v


# ------------------------------------------------------------------ quantize
def quantize(x, odd=False):
    rows, cols = x.shape
    n = pg.scaled_rows_bytes(rows, cols)
    x = at_odd_element(x) if odd else x.cuda()
    return run_one(KernelSpec("quantize", NAMES[x.dtype], 0, (Ref(EXT, 0),), cols, rows=rows, cols=cols), {"specs": [(NAMES[x.dtype], x.numel())], "tensors": [x]},
                   ("f8_rows", n), n).cpu()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,odd", [(1, 1, False), (1, 7, True), (3, 128, False), (2, 129, False), (5, 640, True), (17, 1000, False), (9, 515, False), (1, 2048, False),
                                           (300, 1031, True), (33, 8192, False)])
def test_quantize(rows, cols, odd, dtype):
    say("quantize", rows, cols, odd, dtype)
    g = torch.Generator().manual_seed(rows * 1000 + cols)
    x = torch.randn(rows, cols, generator=g) * torch.exp(3 * torch.randn(rows, 1, generator=g))
    x = x.to(DT[dtype])
    assert torch.equal(quantize(x, odd), plain.pack_rows(x))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_edges(dtype):
    """Blocks of zeros, of the smallest and largest numbers, at the border of a scale, of ties between 8-bit values, with what is not finite."""
    say("quantize edges", dtype)
    rows = [torch.zeros(128), torch.full((128,), 448.0), torch.full((128,), 450.0), torch.full((128,), 2.0 ** -133), torch.full((128,), 3e38), torch.arange(128) * 2.0 ** -9 * 0.5,
            torch.arange(128) + 0.5, torch.linspace(-448, 448, 128), torch.full((128,), math.inf), torch.full((128,), -math.inf), torch.full((128,), math.nan),
            torch.full((128,), 2.0 ** -126)]
    rows[5][0] = 448.0
    mixed = torch.randn(128, generator=torch.Generator().manual_seed(1))
    mixed[3], mixed[4], mixed[100] = math.inf, math.nan, -math.inf
    if dtype == "f32":
        rows.append(torch.full((128,), 2.0 ** -149))
        rows.append(torch.full((128,), 448.0 * (1 + 2.0 ** -23)))
    x = torch.stack(rows + [mixed, -mixed]).to(DT[dtype])
    got, want = quantize(x), plain.pack_rows(x)
    nan = (want & 0x7f) == 0x7f
    nan[x.numel():] = False
    assert torch.equal(got[~nan], want[~nan])
    assert bool(((got[nan] & 0x7f) == 0x7f).all())


# ------------------------------------------------------------------ route
def do_route(s, bias, k, odd=False, **o):
    rows, experts = s.shape
    flags = pg.ROUTE_SIGMOID * o.get("sigmoid", False) | pg.ROUTE_RENORMALIZE * o.get("renorm", False) | pg.ROUTE_GROUP_TOP2 * o.get("top2", False)
    dt = NAMES[s.dtype]
    dev = at_odd_element(s) if odd else s.cuda()
    got = run_one(KernelSpec("route", dt, 0, (Ref(EXT, 0), Ref(WEIGHT, 0)) if bias is not None else (Ref(EXT, 0),), k, rows=rows, cols=experts, m=o.get("groups", 0),
                             inner=o.get("kept", 0), eps=o.get("factor", 0.0), flags=flags),
                  {"specs": [(dt, s.numel())], "tensors": [dev]}, ("routed", rows * k), rows * k, [bias] if bias is not None else [], ["f32"]).cpu()
    ids, w = got[:, 0].view(rows, k), got.view(torch.float32)[:, 1].view(rows, k)
    if not o.get("groups"):
        o.pop("kept", None)
    want_ids, want_w = plain.route(s, bias, k, **{**o, "groups": o.get("groups") or 1, "factor": o.get("factor") or 1.0})
    assert torch.equal(ids.long(), want_ids)
    # weights: 64-bit p, or fp32 exponentials and sums of up to 1024 terms; a few roundings each: 16 half steps of the value
    plain.assert_within(w, want_w, 16 * 2.0 ** -24 * want_w.abs() + 2.0 ** -140, "weights")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("rows,experts,k,groups,kept,bias,top2", [
    (1, 1, 1, 0, 0, False, False), (1, 64, 8, 0, 0, False, False), (5, 3, 3, 0, 0, True, False), (7, 65, 6, 0, 0, True, False), (4, 128, 8, 4, 2, False, False),
    (6, 160, 6, 8, 3, False, True), (9, 256, 8, 8, 4, True, True), (3, 512, 10, 16, 5, True, False), (2, 1024, 64, 64, 20, True, True), (130, 100, 7, 5, 5, False, True),
    (3, 1000, 33, 0, 0, False, False), (11, 24, 6, 8, 2, True, True), (2, 64, 64, 0, 0, False, False), (4, 12, 2, 12, 3, False, True)])
def test_route(rows, experts, k, groups, kept, bias, top2, sigmoid, dtype):
    say("route", rows, experts, k, groups, kept, bias, top2, sigmoid, dtype)
    g = torch.Generator().manual_seed(experts * 7 + rows)
    s = (torch.randn(rows, experts, generator=g) * 2).to(DT[dtype])
    s[torch.rand(s.shape, generator=g) < 0.15] = -math.inf
    b = torch.randn(experts, generator=g) * 0.1 if bias else None
    do_route(s, b, k, odd=rows % 2 == 1, groups=groups, kept=kept, top2=top2, sigmoid=sigmoid, renorm=rows % 3 != 0, factor=2.5 if rows % 2 else 0.0)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("groups", [0, 4])
def test_route_edges(groups, bias, sigmoid):
    """Rows with nothing to choose, ties, the type's lowest value as a mask, infinities, scores that are no numbers, groups that are empty."""
    say("route edges", groups, bias, sigmoid)
    E = 96
    rows = [torch.full((E,), -math.inf), torch.full((E,), math.nan), torch.zeros(E), torch.full((E,), torch.finfo(torch.float32).min), torch.full((E,), 7.0)]
    one = torch.full((E,), -math.inf)
    one[70] = -3.0
    two = torch.randn(E, generator=torch.Generator().manual_seed(3))
    two[10], two[20], two[30], two[31] = math.inf, math.nan, math.inf, -math.inf
    low = torch.full((E,), torch.finfo(torch.float32).min)
    low[5], low[60] = 1.0, 2.0
    half = torch.randn(E, generator=torch.Generator().manual_seed(4))
    half[24:] = -math.inf
    far = torch.linspace(-300.0, 300.0, E)
    s = torch.stack(rows + [one, two, low, half, far, torch.where(torch.arange(E) % 2 == 0, 0.0, -0.0)])
    b = None
    if bias:
        b = torch.randn(E, generator=torch.Generator().manual_seed(5)) * 0.1
        b[2], b[40] = -math.inf, math.nan
        b[50:60] = 0.25
    for top2 in ([False, True] if groups else [False]):
        do_route(s, b, 9, groups=groups, kept=2 if groups else 0, top2=top2, sigmoid=sigmoid, renorm=True)


# ------------------------------------------------------------------ products
def product_case(seed, rows, n, cols, w, h, out, experts=1, k=0, per_slot=False, odd=False, ids=None):
    g = torch.Generator().manual_seed(seed)
    hrows = rows * (k if per_slot else 1)
    wv = torch.randn(experts, n, cols, generator=g) * 0.05
    if w == "bf16":
        wt = wv.to(torch.bfloat16)
        w64 = wt.double()
    else:
        wt, w64 = plain.pack_weight(wv, g)
    hv = torch.randn(hrows, cols, generator=g) * torch.exp(torch.randn(hrows, 1, generator=g))
    if h == "bf16":
        ht = hv.to(torch.bfloat16)
        h64 = ht.double()
    else:
        ht = plain.pack_rows(hv)
        h64 = plain.rows_of(ht, hrows, cols)
    ht = at_odd_element(ht) if odd and h == "bf16" else ht.cuda()
    specs, tensors = [("bf16" if h == "bf16" else "f8_rows", ht.numel())], [ht]
    if k:
        pairs = torch.stack([ids, torch.zeros_like(ids)], -1).to(torch.int32).contiguous()
        kern = KernelSpec("expert_gemv", out, 0, (Ref(WEIGHT, 0), Ref(EXT, 0), Ref(EXT, 1)), n, rows=rows, cols=cols, m=k, inner=experts, flags=pg.EXPERT_PER_SLOT * per_slot)
        specs.append(("routed", rows * k))
        tensors.append(pairs.cuda())
    else:
        kern = KernelSpec("gemv_f8", out, 0, (Ref(WEIGHT, 0), Ref(EXT, 0)), n, rows=rows, cols=cols)
    total = rows * max(1, k) * n
    got = run_one(kern, {"specs": specs, "tensors": tensors}, (out, total), total, [wt.contiguous()], ["bf16" if w == "bf16" else "f8_weight"])
    y, a = plain.product(w64, h64, ids, per_slot)
    plain.assert_within(got.view(y.shape), y, plain.sum_tolerance(y, a, cols, DT[out], eight=h == "f8" and out == "bf16"), "product")
    if y.any():        # as a whole: no element further off than half a step, and what the 8-bit instruction drops, of random sign, far below
        assert float((got.view(y.shape).double().cpu() - y).norm() / y.norm()) <= (1.25 * 2.0 ** -8 if out == "bf16" else 2.0 ** -20)
    return got


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("h", ["bf16", "f8"])
@pytest.mark.parametrize("rows,n,cols,odd", [(1, 1, 1, False), (1, 16, 128, False), (2, 130, 100, True), (3, 500, 257, False), (16, 128, 2048, False), (17, 129, 1000, True), (37, 1000, 520, False),
                                             (64, 256, 384, False), (65, 300, 640, False), (130, 260, 136, True), (257, 140, 129, False), (300, 520, 1100, False), (4, 3000, 2048, False),
                                             (5, 70, 7, False), (1, 2048, 2048, False), (2, 777, 4096, False), (513, 384, 512, False)])
def test_gemv_f8(rows, n, cols, odd, h, out):
    say("gemv_f8", rows, n, cols, odd, h, out)
    product_case(rows * 31 + n, rows, n, cols, "f8", h, out, odd=odd)


def draw_ids(g, rows, k, experts, kind):
    if kind == "distinct":
        ids = torch.stack([torch.randperm(experts, generator=g)[:k] for _ in range(rows)])
    elif kind == "one":                   # everything to one expert
        ids = torch.full((rows, k), experts - 1)
    else:                                 # the same one twice, empty slots, numbers beyond the experts
        ids = torch.randint(-2, experts + 2, (rows, k), generator=g)
        ids[torch.rand(rows, k, generator=g) < 0.2] = -1
    return ids


@pytest.mark.parametrize("w,h", [("bf16", "bf16"), ("f8", "bf16"), ("f8", "f8")])
@pytest.mark.parametrize("rows,k,experts,n,cols,per_slot,kind,out,odd", [
    (1, 1, 1, 1, 1, False, "distinct", "bf16", False), (1, 8, 64, 256, 512, False, "distinct", "bf16", False), (1, 4, 7, 130, 129, True, "any", "f32", False),
    (3, 2, 5, 33, 100, False, "any", "bf16", True), (16, 4, 4, 128, 256, True, "distinct", "bf16", False), (40, 2, 8, 200, 136, False, "any", "f32", False),
    (100, 3, 6, 65, 200, True, "any", "bf16", True), (64, 2, 3, 300, 128, False, "one", "bf16", False), (260, 1, 2, 128, 384, False, "distinct", "bf16", False),
    (700, 2, 3, 132, 140, True, "any", "bf16", False), (5, 64, 200, 16, 64, False, "any", "f32", False), (3, 3, 1024, 17, 33, False, "distinct", "bf16", False),
    (2, 2, 3, 40, 5, False, "any", "bf16", False), (900, 1, 1, 260, 300, False, "one", "bf16", False)])
def test_expert_gemv(rows, k, experts, n, cols, per_slot, kind, out, odd, w, h):
    say("expert_gemv", rows, k, experts, n, cols, per_slot, kind, out, odd, w, h)
    ids = draw_ids(torch.Generator().manual_seed(rows + n), rows, k, experts, kind)
    product_case(rows * 13 + n, rows, n, cols, w, h, out, experts, k, per_slot, odd, ids)


def test_expert_gemv_all_empty():
    say("expert_gemv, no slot in use")
    got = product_case(5, 20, 70, 130, "f8", "bf16", "bf16", 4, 3, False, False, torch.full((20, 3), -1))
    assert not got.any()


# ------------------------------------------------------------------ sum
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows,k,n,odd", [(1, 1, 1, False), (1, 8, 2048, False), (3, 2, 100, True), (5, 4, 777, False), (64, 6, 128, False), (300, 3, 65, True), (2, 64, 1030, False), (7, 8, 4096, False)])
def test_expert_sum(rows, k, n, odd, residual, dtype):
    say("expert_sum", rows, k, n, odd, residual, dtype)
    g = torch.Generator().manual_seed(rows + n)
    z = torch.randn(rows, k, n, generator=g).to(DT[dtype])
    ids = torch.randint(-1, 5, (rows, k), generator=g)
    if rows > 2:
        ids[1] = -1                        # a row without experts
    z[ids < 0] = math.nan                  # not read
    w = torch.rand(rows, k, generator=g)
    x = torch.randn(rows, n, generator=g).to(DT[dtype])
    pairs = torch.stack([ids.to(torch.int32), w.view(torch.int32)], -1).contiguous()
    place = at_odd_element if odd else lambda t: t.cuda()
    kern = KernelSpec("expert_sum", dtype, 0, (Ref(EXT, 0), Ref(EXT, 1)) + ((Ref(EXT, 2),) if residual else ()), n, rows=rows, m=k)
    specs, tensors = [(dtype, z.numel()), ("routed", rows * k)], [place(z), pairs.cuda()]
    if residual:
        specs.append((dtype, x.numel()))
        tensors.append(place(x))
    got = run_one(kern, {"specs": specs, "tensors": tensors}, (dtype, rows * n), rows * n).view(rows, n)
    used = (ids >= 0).unsqueeze(2)
    terms = torch.where(used, w.double().unsqueeze(2) * z.double(), 0.0)
    y, a = terms.sum(1), terms.abs().sum(1)
    if residual:
        y, a = y + x.double(), a + x.double().abs()
    plain.assert_within(got, y, plain.sum_tolerance(y, a, k + 1, DT[dtype]), "sum")


# ------------------------------------------------------------------ together
def expert_layer(rows, hidden, width, experts, k, eightbit, seed=11):
    """A layer of experts on a residual stream x: RMSNorm, scores, routing, gate and up products, GELU(gate) * up, the down product,
    their weighted sum onto the stream; twice, so that the second finds the stream where the first left it."""
    e, i, w = lambda j: Ref(EXT, j), lambda j: Ref(INT, j), lambda j: Ref(WEIGHT, j)
    X, T, S, R, Q, G, U, Q2, D = range(9)
    slots = rows * k
    ks = []
    for layer in range(2):
        x = e(0) if layer == 0 else i(X)
        ks.append(KernelSpec("rmsnorm", "bf16", T, (x, w(0)), hidden, rows=rows, cols=hidden, eps=1e-6))
        ks.append(KernelSpec("gemv", "bf16", S, (w(1), i(T)), experts, rows=rows, cols=hidden))
        ks.append(KernelSpec("route", "bf16", R, (i(S), w(2)), k, rows=rows, cols=experts, flags=pg.ROUTE_SIGMOID | pg.ROUTE_RENORMALIZE, eps=1.5))
        h, h2 = T, G
        if eightbit:
            ks.append(KernelSpec("quantize", "bf16", Q, (i(T),), hidden, rows=rows, cols=hidden))
            h, h2 = Q, Q2
        ks.append(KernelSpec("expert_gemv", "bf16", G, (w(3), i(h), i(R)), width, rows=rows, cols=hidden, m=k, inner=experts))
        ks.append(KernelSpec("expert_gemv", "bf16", U, (w(4), i(h), i(R)), width, rows=rows, cols=hidden, m=k, inner=experts))
        ks.append(KernelSpec("gelu", "bf16", G, (i(G),), slots * width))
        ks.append(KernelSpec("mul", "bf16", G, (i(G), i(U)), slots * width, m=slots * width))
        if eightbit:
            ks.append(KernelSpec("quantize", "bf16", Q2, (i(G),), width, rows=slots, cols=width))
        ks.append(KernelSpec("expert_gemv", "bf16", D, (w(5), i(h2), i(R)), hidden, rows=rows, cols=width, m=k, inner=experts, flags=pg.EXPERT_PER_SLOT))
        ks.append(KernelSpec("expert_sum", "bf16", X, (i(D), i(R), x), hidden, rows=rows, m=k))
    ints = [TensorSpec("bf16", rows * hidden), TensorSpec("bf16", rows * hidden), TensorSpec("bf16", rows * experts), TensorSpec("routed", slots),
            TensorSpec("f8_rows", pg.scaled_rows_bytes(rows, hidden)), TensorSpec("bf16", slots * width), TensorSpec("bf16", slots * width),
            TensorSpec("f8_rows", pg.scaled_rows_bytes(slots, width)), TensorSpec("bf16", slots * hidden)]
    g = torch.Generator().manual_seed(seed)
    wts = [(1 + 0.1 * torch.randn(hidden, generator=g)).to(torch.bfloat16), (torch.randn(experts, hidden, generator=g) * 0.05).to(torch.bfloat16),
           torch.randn(experts, generator=g) * 0.02]
    w64 = [t.double() for t in wts]
    for n, cols in ((width, hidden), (width, hidden), (hidden, width)):
        b, v = plain.pack_weight(torch.randn(experts, n, cols, generator=g) * 0.02, g)
        wts.append(b)
        w64.append(v)
    wtypes = ["bf16", "bf16", "f32", "f8_weight", "f8_weight", "f8_weight"]
    spec = ChainSpec("expert_layer", ks, [TensorSpec("bf16", rows * hidden)], ints, [TensorSpec(d, t.numel()) for d, t in zip(wtypes, wts)], [X])
    return spec, wts, w64


@pytest.mark.parametrize("eightbit", [False, True])
@pytest.mark.parametrize("rows,hidden,width,experts,k", [(1, 256, 128, 8, 2), (5, 200, 136, 6, 3), (33, 512, 260, 16, 4), (150, 264, 128, 5, 2)])
def test_layer_of_experts(rows, hidden, width, experts, k, eightbit):
    """The whole layer in every mode with the same bits, and each kernel against its plain form on what it actually read."""
    say("layer of experts", rows, hidden, width, experts, k, eightbit)
    spec, wts, w64 = expert_layer(rows, hidden, width, experts, k, eightbit)
    r = Run(spec, wts)
    x = [torch.randn(rows, hidden, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()]
    n8 = (pg.scaled_rows_bytes(rows, hidden), pg.scaled_rows_bytes(rows * k, width)) if eightbit else (0, 0)
    r(x, [rows * hidden, rows * hidden, rows * experts, rows * k, n8[0], rows * k * width, rows * k * width, n8[1], rows * k * hidden])
    c = r.chains[0]

    def value(ref):
        t = x[0] if ref.kind == EXT else c.int_buffer(ref.index) if ref.kind == INT else wts[ref.index]
        return t.cpu()

    for n, kk in enumerate(spec.kernels):
        torch.cuda.synchronize()
        ins = [value(q) for q in kk.ins]
        c.eager_range(x, n, n + 1, r.stream)
        r.stream.synchronize()
        got = c.int_buffer(kk.out).cpu()
        if kk.op == "route":
            ids, w = plain.route(ins[0][:rows * experts].view(rows, experts), ins[1], k, sigmoid=True, renorm=True, factor=1.5)
            assert torch.equal(got[:rows * k, 0].view(rows, k).long(), ids)
            plain.assert_within(got[:rows * k].view(torch.float32)[:, 1].view(rows, k), w, 16 * 2.0 ** -24 * w.abs(), "weights")
        elif kk.op == "quantize":
            assert torch.equal(got[:pg.scaled_rows_bytes(kk.rows, kk.cols)], plain.pack_rows(ins[0][:kk.rows * kk.cols].view(kk.rows, kk.cols)))
        elif kk.op == "expert_gemv":
            hrows = rows * k if kk.flags else rows
            h = plain.rows_of(ins[1][:pg.scaled_rows_bytes(hrows, kk.cols)], hrows, kk.cols) if ins[1].dtype == torch.uint8 else ins[1][:hrows * kk.cols].double().view(hrows, kk.cols)
            y, a = plain.product(w64[kk.ins[0].index], h, ins[2][:rows * k, 0].view(rows, k), bool(kk.flags))
            plain.assert_within(got[:y.numel()].view(y.shape), y, plain.sum_tolerance(y, a, kk.cols, torch.bfloat16, eight=ins[1].dtype == torch.uint8), f"kernel {n}")
        elif kk.op == "expert_sum":
            w = ins[1][:rows * k].view(torch.float32)[:, 1].double().view(rows, k, 1)
            terms, xr = w * ins[0][:rows * k * hidden].double().view(rows, k, hidden), ins[2][:rows * hidden].double().view(rows, hidden)
            y, a = terms.sum(1) + xr, terms.abs().sum(1) + xr.abs()
            plain.assert_within(got[:y.numel()].view(y.shape), y, plain.sum_tolerance(y, a, k + 1, torch.bfloat16), f"kernel {n}")
    r.close()


# ------------------------------------------------------------------ lengths, tiles and orders
@pytest.mark.parametrize("w,h", [("bf16", "bf16"), ("f8", "bf16"), ("f8", "f8")])
@pytest.mark.parametrize("rows,k,experts,n,cols,out", [(33, 2, 9, 40, 264, "bf16"), (30, 8, 300, 33, 136, "f32"), (9, 20, 3, 300, 520, "bf16"), (128, 4, 6, 50, 136, "bf16"), (171, 3, 1024, 40, 72, "f32"),
                                                       (64, 8, 1024, 33, 264, "f32"), (65, 1, 64, 600, 131, "bf16"), (500, 1, 3, 70, 72, "bf16"), (16, 32, 130, 18, 200, "f32"),
                                                       (1000, 1, 16, 30, 72, "bf16"), (256, 4, 5, 40, 40, "f32"), (205, 5, 5, 33, 136, "bf16"), (1000, 1, 60, 70, 264, "bf16"),
                                                       (300, 4, 60, 700, 72, "bf16"), (250, 8, 40, 600, 515, "f32"), (90, 8, 12, 1700, 520, "bf16"), (9000, 4, 5, 20, 40, "bf16"),
                                                       (700, 60, 1024, 9, 24, "f32"), (1300, 4, 3, 520, 129, "bf16"), (4000, 1, 2, 1030, 72, "f32"), (2500, 2, 40, 700, 65, "bf16")])
def test_expert_gemv_slots(rows, k, experts, n, cols, out, w, h):
    """Slots on both sides of every bound of the sorting, in small and large tiles."""
    say("expert_gemv slots", rows, k, experts, n, cols, out, w, h)
    g = torch.Generator().manual_seed(rows + k)
    ids = torch.randint(-1, experts, (rows, k), generator=g)
    ids[torch.rand(rows, k, generator=g) < 0.3] = experts // 2            # one has many more than the others
    product_case(rows + n, rows, n, cols, w, h, out, experts, k, False, False, ids)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("h", ["bf16", "f8"])
@pytest.mark.parametrize("rows", [9, 20, 50, 140, 333])
@pytest.mark.parametrize("n,cols", [(50, 200), (8230, 72), (16500, 33)])
def test_gemv_f8_outputs(n, cols, rows, h, out):
    """Tiles of every number of rows and outputs, with a tail in both and in the columns."""
    say("gemv_f8 outputs", rows, n, cols, h, out)
    product_case(rows + n, rows, n, cols, "f8", h, out, odd=cols == 33)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("h", ["bf16", "f8"])
@pytest.mark.parametrize("rows,n,cols", [(803, 3700, 129), (3900, 3001, 65), (1500, 2500, 640), (2, 40, 40000), (40, 70, 33100), (420, 6200, 8330)])
def test_gemv_f8_large(rows, n, cols, h, out):
    """Large tiles, and more than 64 steps of columns, whose scales are loaded 64 at a time."""
    say("gemv_f8 large", rows, n, cols, h, out)
    product_case(rows + n, rows, n, cols, "f8", h, out)


@pytest.mark.parametrize("rows", [37, 300, 1500])
@pytest.mark.parametrize("w,h", [("bf16", "bf16"), ("f8", "bf16"), ("f8", "f8")])
def test_a_row_stays_its_own(rows, w, h):
    """What is infinite or no number in one row of h, or in the weights of one expert, reaches that row's slots or that expert's and no others: the
    rest keep their bits."""
    say("a row stays its own", rows, w, h)
    k, experts, n, cols = 2, 4, 260, 136
    g = torch.Generator().manual_seed(rows)
    ids = torch.randint(0, experts, (rows, k), generator=g)
    pairs = torch.stack([ids, torch.zeros_like(ids)], -1).to(torch.int32).contiguous()
    hv = torch.randn(rows, cols, generator=g)
    bad = hv.clone()
    bad[rows // 2, 5], bad[rows - 1, 130] = math.inf, math.nan
    wv = torch.randn(experts, n, cols, generator=g)
    wt = wv.to(torch.bfloat16) if w == "bf16" else plain.pack_weight(wv * 0.05, g)[0]
    if w == "bf16":
        broken = wt.clone()
        broken[1] = math.nan
    else:
        broken = wt.clone()
        broken[n * 256:2 * n * 256] = 0x7f
    kern = KernelSpec("expert_gemv", "bf16", 0, (Ref(WEIGHT, 0), Ref(EXT, 0), Ref(EXT, 1)), n, rows=rows, cols=cols, m=k, inner=experts)

    def run(hx, wx):
        t = hx.to(torch.bfloat16) if h == "bf16" else plain.pack_rows(hx)
        return run_one(kern, {"specs": [("bf16" if h == "bf16" else "f8_rows", t.numel()), ("routed", rows * k)], "tensors": [t.cuda(), pairs.cuda()]}, ("bf16", rows * k * n), rows * k * n,
                       [wx.contiguous()], ["bf16" if w == "bf16" else "f8_weight"]).view(rows, k, n).cpu()
    clean = run(hv, wt)
    assert bool(torch.isfinite(clean).all())
    got = run(bad, wt)
    other = torch.ones(rows, dtype=torch.bool)
    other[rows // 2] = other[rows - 1] = False
    assert torch.equal(got[other].view(torch.int16), clean[other].view(torch.int16))
    assert not bool(torch.isfinite(got[~other]).any())
    got = run(hv, broken)
    assert torch.equal(got[ids != 1].view(torch.int16), clean[ids != 1].view(torch.int16))
    assert bool(torch.isnan(got[ids == 1]).all())


# ------------------------------------------------------------------ products that share their slots' order
def shared_chain(rows, k, experts, n, cols, external):
    """Two products by one list of slots, which is then written anew, and a third."""
    E, I, W = (lambda j: Ref(EXT, j)), (lambda j: Ref(INT, j)), (lambda j: Ref(WEIGHT, j))
    r = E(3) if external else I(0)
    ks = [KernelSpec("route", "f32", 0, (E(0),), k, rows=rows, cols=experts),
          KernelSpec("expert_gemv", "bf16", 1, (W(0), E(2), r), n, rows=rows, cols=cols, m=k, inner=experts),
          KernelSpec("expert_gemv", "f32", 2, (W(0), E(2), r), n, rows=rows, cols=cols, m=k, inner=experts),
          KernelSpec("route", "f32", 0, (E(1),), k, rows=rows, cols=experts),
          KernelSpec("expert_gemv", "bf16", 3, (W(0), E(2), r), n, rows=rows, cols=cols, m=k, inner=experts),
          KernelSpec("expert_gemv", "bf16", 4, (W(0), E(2), r), n, rows=rows, cols=cols, m=k, inner=experts)]
    ext = [TensorSpec("f32", rows * experts)] * 2 + [TensorSpec("bf16", rows * cols)] + ([TensorSpec("routed", rows * k)] if external else [])
    total = rows * k * n
    return ChainSpec("shared", ks, ext, [TensorSpec("routed", rows * k), TensorSpec("bf16", total), TensorSpec("f32", total), TensorSpec("bf16", total), TensorSpec("bf16", total)],
                     [TensorSpec("bf16", experts * n * cols)], [1])


@pytest.mark.parametrize("rows,k", [(20, 2), (50, 2), (400, 3)])
def test_products_by_the_same_slots(rows, k):
    """The list is written again between products, and again with other inputs in the next replay: each product goes by what is there then."""
    say("products by the same slots", rows, k)
    experts, n, cols = 7, 136, 72
    spec = shared_chain(rows, k, experts, n, cols, False)
    g = torch.Generator().manual_seed(rows)
    w = (torch.randn(experts, n, cols, generator=g) * 0.1).to(torch.bfloat16)
    run = Run(spec, [w])
    for again in range(2):
        s = [torch.randn(rows, experts, generator=g) for _ in range(2)]
        h = torch.randn(rows, cols, generator=g).to(torch.bfloat16)
        got = run(s + [h], [rows * k] + [rows * k * n] * 4)
        for at, scores, dtype in ((1, s[0], torch.bfloat16), (2, s[0], torch.float32), (3, s[1], torch.bfloat16), (4, s[1], torch.bfloat16)):
            ids, _ = plain.route(scores, None, k)
            y, a = plain.product(w.double(), h.double(), ids)
            plain.assert_within(got[at].view(y.shape), y, plain.sum_tolerance(y, a, cols, dtype), f"product {at}")
    run.close()


@pytest.mark.parametrize("rows", [50, 300])
def test_slots_in_a_buffer_of_the_chain(rows):
    """The external list of slots is the chain's own buffer, written between the products: read there when a product runs, except in copy form, which
    reads it when the replay begins."""
    k, experts, n, cols = 2, 7, 136, 72
    say("slots in a buffer of the chain", rows)
    spec = shared_chain(rows, k, experts, n, cols, True)
    g = torch.Generator().manual_seed(3)
    w = (torch.randn(experts, n, cols, generator=g) * 0.1).to(torch.bfloat16)
    s = [torch.randn(rows, experts, generator=g).cuda() for _ in range(2)]
    h = torch.randn(rows, cols, generator=g).to(torch.bfloat16).cuda()
    stream = torch.cuda.Stream()
    c = pg.Chain(spec, [w.cuda()], "cuda:0")
    torch.cuda.synchronize()
    want = [plain.product(w.double(), h.cpu().double(), plain.route(x.cpu(), None, k)[0]) for x in s]
    for most in (0, 6):
        c.set_launched_dispatches(most)
        c.capture(stream)
        ext = s + [h, c.int_buffer(0)]
        for mode in ("eager", "replay_indirect", "replay_update", "replay_copy", "replay_indirect"):
            for again in range(2):
                for i in range(1, 5):
                    c.int_buffer(i).fill_(math.nan)
                torch.cuda.synchronize()
                getattr(c, mode)(ext, stream)
                stream.synchronize()
                for at, by in ((1, 0), (2, 0), (3, 1), (4, 1)):
                    y, a = want[1 if mode == "replay_copy" else by]
                    dt = torch.float32 if at == 2 else torch.bfloat16
                    plain.assert_within(c.int_buffer(at)[:y.numel()].view(y.shape), y, plain.sum_tolerance(y, a, cols, dt), f"{mode}, product {at}")
    c.close()


# ------------------------------------------------------------------ other ways in
@pytest.mark.parametrize("rows", [40, 300])
def test_static_pass_and_other_streams(rows):
    """The layer in the library's own scratch, with lists of sorted slots in it; eagerly on the default device's other streams; two chains at once."""
    say("static pass, other streams", rows)
    hidden, width, experts, k = 256, 128, 6, 2
    spec, wts, _ = expert_layer(rows, hidden, width, experts, k, True)
    dev = [t.cuda() for t in wts]
    chains = [pg.Chain(spec, dev, "cuda:0") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    xs = [torch.randn(rows, hidden, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).cuda() for i in range(2)]
    torch.cuda.synchronize()
    alone = []
    for c, x, s in zip(chains, xs, streams):
        c.eager([x], s)
        s.synchronize()
        alone.append(c.int_buffer(0)[:rows * hidden].clone())
    assert bool(torch.isfinite(alone[0]).all()) and not torch.equal(alone[0], alone[1])
    for c, s in zip(chains, streams):
        c.capture(s)
    for again in range(3):
        for c in chains:
            c.int_buffer(0).fill_(math.nan)
        torch.cuda.synchronize()
        for i in range(2):                                  # both under way at once
            chains[i].replay_indirect([xs[i]], streams[i])
        for i in range(2):
            chains[i].eager([xs[i]], streams[i])
            chains[i].replay_copy([xs[i]], streams[i])
        torch.cuda.synchronize()
        for c, want in zip(chains, alone):
            assert torch.equal(c.int_buffer(0)[:rows * hidden], want), again
    out = torch.full((rows * hidden,), math.nan, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    for i in range(2):
        pg.eager_static(spec, dev, [xs[i]], 0, out, streams[i])
        streams[i].synchronize()
        assert torch.equal(out, alone[i])
    for c in chains:
        c.close()


@pytest.mark.parametrize("rows", [50, 270])
def test_a_segment_of_its_own(rows):
    """The layer in four segments, each in every mode that it has."""
    say("segments", rows)
    hidden, width, experts, k = 128, 72, 5, 2
    spec, wts, _ = expert_layer(rows, hidden, width, experts, k, True)
    n = len(spec.kernels)
    ks = [KernelSpec(**{**vars(q), "segment": i * 4 // n}) for i, q in enumerate(spec.kernels)]
    spec = ChainSpec("segments", ks, spec.ext, spec.ints, spec.weights, spec.outputs)
    c = pg.Chain(spec, [t.cuda() for t in wts], "cuda:0")
    stream = torch.cuda.Stream()
    x = [torch.randn(rows, hidden, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()]
    torch.cuda.synchronize()
    c.capture(stream)
    c.eager(x, stream)
    stream.synchronize()
    want = c.int_buffer(0).clone()
    for modes in ([0, 1, 0, 1], [2, 0, 1, 0], [1, 1, 1, 1], [2, 1, 0, 1]):
        for again in range(2):
            c.int_buffer(0).fill_(math.nan)
            torch.cuda.synchronize()
            c.run_selected(modes, x, stream)
            stream.synchronize()
            assert torch.equal(c.int_buffer(0), want), modes
    c.close()
