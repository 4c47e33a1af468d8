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
                    [c.int_buffer(i).fill_(-1 if t.dtype in ("routed",) else 255 if t.dtype.startswith("f8") else math.nan)
                                        for i, t in enumerate(self.spec.ints)]
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
