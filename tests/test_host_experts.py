"""Descriptors of the kernels of experts and of 8-bit weights: what is accepted and refused, sizes, workspaces (no GPU)."""
import dataclasses

import pytest

import paper_2503_19779_amd as pg
from pg_workloads import ChainSpec, EXT, INT, KernelSpec, Ref, TensorSpec, WEIGHT

E, I, W = (lambda i: Ref(EXT, i)), (lambda i: Ref(INT, i)), (lambda i: Ref(WEIGHT, i))


def up(x, to):
    return (x + to - 1) // to * to


def test_layout_sizes():
    for n, cols, experts in ((1, 1, 1), (128, 128, 1), (129, 127, 3), (2048, 2049, 64), (7, 1000, 5)):
        kp = up(cols, 128)
        assert pg.scaled_weight_bytes(experts, n, cols) == experts * (n * kp + 4 * (up(n, 128) // 128) * (kp // 128))
        assert pg.scaled_rows_bytes(n, cols) == n * (kp + up(kp // 128, 4))
    for bad in ((0, 1, 1), (1, -1, 1), (1, 1, 0), (1 << 30, 1 << 30, 1 << 30), (1 << 62, 1 << 62, 1 << 62)):
        with pytest.raises(ValueError):
            pg.scaled_weight_bytes(*bad)
    for bad in ((0, 1), (1, 0), (-5, 3), (1 << 40, 128), ((1 << 63) - 1, (1 << 63) - 1)):
        with pytest.raises(ValueError):
            pg.scaled_rows_bytes(*bad)


def test_weights_are_packed_as_the_layout_says():
    import torch
    g = torch.Generator().manual_seed(1)
    q, s = torch.randn(3, 130, 200, generator=g).to(torch.float8_e4m3fn), torch.rand(3, 2, 2, generator=g)
    b = pg.pack_scaled_weight(q, s)
    v = b[:3 * 130 * 256].view(3, 130, 256)
    assert torch.equal(v[..., :200], q.view(torch.uint8)) and not v[..., 200:].any()
    assert torch.equal(b[3 * 130 * 256:].view(torch.float32).view(3, 2, 2), s)
    assert torch.equal(pg.pack_scaled_weight(q[0], s[0])[:130 * 256], v[0].reshape(-1))
    for bad in ((q.float(), s), (q, s.double()), (q, s[:, :1]), (q[0], s)):
        with pytest.raises((ValueError, IndexError)):
            pg.pack_scaled_weight(*bad)


def chains():
    """One valid chain for each kernel, with all its operands."""
    rb, wb = pg.scaled_rows_bytes, pg.scaled_weight_bytes
    return {
        "quantize": ChainSpec("q", [KernelSpec("quantize", "bf16", 0, (E(0),), 200, rows=4, cols=200)], [TensorSpec("bf16", 800)], [TensorSpec("f8_rows", rb(4, 200))], [], [0]),
        "gemv_f8": ChainSpec("g", [KernelSpec("gemv_f8", "bf16", 0, (W(0), E(0)), 70, rows=4, cols=200)], [TensorSpec("bf16", 800)], [TensorSpec("bf16", 280)],
                             [TensorSpec("f8_weight", wb(1, 70, 200))], [0]),
        "gemv_f8 rows": ChainSpec("g", [KernelSpec("gemv_f8", "f32", 0, (W(0), E(0)), 70, rows=4, cols=200)], [TensorSpec("f8_rows", rb(4, 200))], [TensorSpec("f32", 280)],
                                  [TensorSpec("f8_weight", wb(1, 70, 200))], [0]),
        "route": ChainSpec("r", [KernelSpec("route", "f32", 0, (E(0), W(0)), 3, rows=4, cols=12, m=4, inner=2, flags=7, eps=2.0)], [TensorSpec("f32", 48)], [TensorSpec("routed", 12)],
                           [TensorSpec("f32", 12)], [0]),
        "expert_gemv": ChainSpec("e", [KernelSpec("expert_gemv", "bf16", 0, (W(0), E(0), E(1)), 70, rows=4, cols=200, m=3, inner=5)],
                                 [TensorSpec("bf16", 800), TensorSpec("routed", 12)], [TensorSpec("bf16", 840)], [TensorSpec("bf16", 5 * 70 * 200)], [0]),
        "expert_gemv slots": ChainSpec("e", [KernelSpec("expert_gemv", "f32", 0, (W(0), E(0), E(1)), 70, rows=4, cols=200, m=3, inner=5, flags=1)],
                                       [TensorSpec("f8_rows", rb(12, 200)), TensorSpec("routed", 12)], [TensorSpec("f32", 840)], [TensorSpec("f8_weight", wb(5, 70, 200))], [0]),
        "expert_sum": ChainSpec("s", [KernelSpec("expert_sum", "bf16", 0, (E(0), E(1), E(2)), 70, rows=4, m=3)],
                                [TensorSpec("bf16", 840), TensorSpec("routed", 12), TensorSpec("bf16", 280)], [TensorSpec("bf16", 280)], [], [0]),
        "expert_sum alone": ChainSpec("s", [KernelSpec("expert_sum", "f32", 0, (E(0), E(1)), 70, rows=4, m=3)], [TensorSpec("f32", 840), TensorSpec("routed", 12)], [TensorSpec("f32", 280)], [], [0]),
    }


def changed(spec, **fields):
    return dataclasses.replace(spec, kernels=[dataclasses.replace(spec.kernels[0], **fields)] + spec.kernels[1:])


def sized(spec, where, index, dtype=None, by=0):
    ts = list(getattr(spec, where))
    ts[index] = TensorSpec(dtype or ts[index].dtype, ts[index].numel + by)
    return dataclasses.replace(spec, **{where: ts})


def test_valid_chains_build():
    for name, spec in chains().items():
        c = pg.Chain.host_only(spec)
        assert c.stats()["n_kernels"] == 1, name
        assert c.launch_shape(0)[0] >= 1 and c.graph_dispatches() == (1, 1)


REFUSED = {
    "quantize": [("n", dict(n=100)), ("rows", dict(rows=0)), ("cols", dict(cols=0, n=0)), ("cols", dict(cols=1 << 31, n=1 << 31)), ("flags", dict(flags=1)), ("dtype", dict(dtype="f32")),
                 ("more operands", dict(ins=(E(0), E(0)))), ("too many rows", dict(rows=5)), ("output", dict(out=1))],
    "gemv_f8": [("n", dict(n=0)), ("n", dict(n=71)), ("rows", dict(rows=-1)), ("rows", dict(rows=5)), ("cols", dict(cols=300)), ("operands", dict(ins=(W(0),))), ("swapped", dict(ins=(E(0), W(0)))),
                ("flags", dict(flags=1)), ("dtype", dict(dtype="f32"))],
    "route": [("k", dict(n=0)), ("k beyond the experts", dict(n=13)), ("k", dict(n=65)), ("groups", dict(m=5)), ("groups", dict(m=-4)), ("kept", dict(inner=0)), ("kept", dict(inner=5)),
              ("flags", dict(flags=8)), ("factor", dict(eps=float("nan"))), ("factor", dict(eps=float("inf"))), ("experts", dict(cols=1025, m=0)), ("dtype", dict(dtype="bf16")), ("rows", dict(rows=5))],
    "expert_gemv": [("slots", dict(m=0)), ("slots", dict(m=65)), ("slots", dict(m=4)), ("experts", dict(inner=0)), ("experts", dict(inner=6)), ("experts", dict(inner=1025)), ("flags", dict(flags=2)),
                    ("a row of h for each slot", dict(flags=1)), ("rows", dict(rows=1 << 23)), ("operands", dict(ins=(W(0), E(0)))), ("not routed", dict(ins=(W(0), E(0), E(0)))), ("cols", dict(cols=201))],
    "expert_sum": [("slots", dict(m=0)), ("slots", dict(m=65)), ("n", dict(n=71)), ("rows", dict(rows=5)), ("operands", dict(ins=(E(0),))), ("not routed", dict(ins=(E(0), E(0)))), ("flags", dict(flags=1)),
                   ("in place on z", dict(ins=(I(0), E(1)))), ("dtype", dict(dtype="f32"))],
}


@pytest.mark.parametrize("op,what,fields", [(op, what, f) for op, fs in REFUSED.items() for what, f in fs])
def test_refused(op, what, fields):
    with pytest.raises(pg.PgError) as e:
        pg.Chain.host_only(changed(chains()[op], **fields))
    assert e.value.status == 1, what


def test_refused_tensors():
    c = chains()
    bad = [sized(c["quantize"], "ints", 0, by=-1), sized(c["quantize"], "ints", 0, "bf16"), sized(c["gemv_f8"], "weights", 0, by=1), sized(c["gemv_f8"], "weights", 0, "bf16"),
           sized(c["gemv_f8 rows"], "ext", 0, by=-4), sized(c["gemv_f8 rows"], "ext", 0, by=4), sized(c["gemv_f8"], "ext", 0, "f32"), sized(c["route"], "ints", 0, "f32"),
           sized(c["route"], "weights", 0, "bf16"), sized(c["route"], "weights", 0, by=-1), sized(c["expert_gemv"], "ext", 0, "f8_rows"), sized(c["expert_gemv"], "weights", 0, by=-1),
           sized(c["expert_gemv slots"], "weights", 0, by=-4), sized(c["expert_gemv"], "ext", 1, by=-1), sized(c["expert_sum"], "ext", 2, by=-1), sized(c["expert_sum"], "ints", 0, by=-1)]
    for i, spec in enumerate(bad):
        with pytest.raises(pg.PgError) as e:
            pg.Chain.host_only(spec)
        assert e.value.status == 1, i
    # the other kernels take none of these types
    for dtype in ("f8_weight", "f8_rows", "routed"):
        for k in (KernelSpec("add", "bf16", 0, (E(0), E(0)), 8, m=8), KernelSpec("gemv", "bf16", 0, (E(0), E(0)), 1, rows=1, cols=8)):
            with pytest.raises(pg.PgError):
                pg.Chain.host_only(ChainSpec("x", [k], [TensorSpec(dtype, 64)], [TensorSpec("bf16", 64)], [], [0]))


def test_rows_are_read_as_they_were_written():
    def chain(rows, cols, read_rows, read_cols, again=None):
        ks = [KernelSpec("quantize", "bf16", 0, (E(0),), cols, rows=rows, cols=cols)]
        if again:
            ks.append(KernelSpec("quantize", "bf16", 0, (E(0),), again[1], rows=again[0], cols=again[1]))
        ks.append(KernelSpec("gemv_f8", "bf16", 1, (W(0), I(0)), 8, rows=read_rows, cols=read_cols))
        return ChainSpec("c", ks, [TensorSpec("bf16", 4096)], [TensorSpec("f8_rows", 8192), TensorSpec("bf16", 4096)], [TensorSpec("f8_weight", pg.scaled_weight_bytes(1, 8, read_cols))], [1])
    pg.Chain.host_only(chain(4, 256, 4, 256))
    pg.Chain.host_only(chain(4, 256, 2, 130, again=(2, 130)))
    for bad in (chain(4, 256, 2, 256), chain(4, 256, 4, 128), chain(4, 256, 4, 256, again=(2, 130)), chain(4, 256, 4, 255)):
        with pytest.raises(pg.PgError):
            pg.Chain.host_only(bad)


def test_unwritten_and_misaligned_operands():
    spec = ChainSpec("c", [KernelSpec("expert_sum", "bf16", 0, (E(0), I(1)), 8, rows=2, m=2)], [TensorSpec("bf16", 32)], [TensorSpec("bf16", 16), TensorSpec("routed", 4)], [], [0])
    with pytest.raises(pg.PgError):
        pg.Chain.host_only(spec)
    for name, index, ok, off in (("gemv_f8 rows", 0, 16, 8), ("expert_gemv", 1, 8, 4), ("gemv_f8", 0, 2, 1)):
        s = chains()[name]
        c = pg.Chain.host_only(s)
        ptrs = [0x10000 * (i + 1) for i in range(len(s.ext))]
        ptrs[index] += off
        with pytest.raises(pg.PgError) as e:
            c.eager(ptrs, 1)
        assert "aligned" in str(e.value), name


def test_workspace_sizes_of_unvalidated_descriptors():
    """A size query answers or refuses; it does not overflow."""
    big = (1 << 31) - 1
    for rows, m, inner in ((big, 64, 1024), (1 << 40, 1 << 40, 1), (-1, 3, 3), (4, -3, 5), (0, 0, 0)):
        s = changed(chains()["expert_gemv"], rows=rows, m=m, inner=inner)
        try:
            pg.Chain.host_only(s)
        except pg.PgError:
            pass


def test_sizes_near_32_bits():
    """Row, output and column numbers reach up to 512 beyond the last one; a launch has fewer than 2^32 threads.  At the limit: built or refused, by the
    same rule in 64 bits."""
    most, over = (1 << 31) - 513, (1 << 31) - 512
    wb, rb = pg.scaled_weight_bytes, pg.scaled_rows_bytes

    def one(op, ins, n, ext, out, weights=(), dtype="bf16", **f):
        return ChainSpec("x", [KernelSpec(op, dtype, 0, ins, n, **f)], [TensorSpec(*t) for t in ext], [TensorSpec(*out)], [TensorSpec(*t) for t in weights], [0])

    def products(n, cols):
        return [one("gemv_f8", (W(0), E(0)), n, [("bf16", cols)], ("bf16", n), [("f8_weight", wb(1, n, cols))], rows=1, cols=cols),
                one("expert_gemv", (W(0), E(0), E(1)), n, [("bf16", cols), ("routed", 1)], ("bf16", n), [("bf16", n * cols)], rows=1, cols=cols, m=1, inner=1)]
    quantize = lambda cols: one("quantize", (E(0),), cols, [("bf16", cols)], ("f8_rows", rb(1, cols)), rows=1, cols=cols)
    total = lambda n: one("expert_sum", (E(0), E(1)), n, [("bf16", n), ("routed", 1)], ("bf16", n), rows=1, m=1)
    route = lambda rows: one("route", (E(0),), 1, [("bf16", rows)], ("routed", rows), rows=rows, cols=1)
    for spec in [quantize(most), total(most), route((1 << 26) - 4)] + products(1, most) + products((1 << 24) - 16, 1):
        pg.Chain.host_only(spec)
    for spec in [quantize(over), total(over), route(over), route(1 << 26)] + products(1, over) + products(over, 1):
        with pytest.raises(pg.PgError) as e:
            pg.Chain.host_only(spec)
        assert e.value.status == 1
