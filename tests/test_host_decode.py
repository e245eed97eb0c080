"""Operators of single-token inference, without a GPU: shapes, refusals, how their blocks are planned, and the oracle's definitions
against plain loops."""
import numpy as np
import pytest

import decode_graphs as dg
from oracle.interp import run_graph
from paper_2108_13342_amd import api


def plan(spec, **kw):
    g, _ = api.graph_from_spec(spec)
    g.rewrite()
    return api.Plan(g, [1] * len(spec.weights()), **kw)


def kernels(p):
    return [d["kernel_name"].split(":")[-1] for d in p.describe()]


# ------------------------------------------------------------------------------------------------ the oracle
def test_oracle_attention_against_loops():
    spec = dg.attend_graph("f32", "i8", [9, 0, 21], HQ=6, HK=2, DK=16, DV=32, S=4, M=6, attrs={"window": 7})
    t = {n: np.asarray(x.data, dtype=np.float64) for n, x in spec.tensors.items() if x.data is not None}
    got = run_graph(spec)["o"]
    for b, held in enumerate([9, 0, 21]):
        for h in range(6):
            num, den = np.zeros(32), 0.0
            for p in range(max(0, held - 7), held):
                at = (int(t["table"][b, p // 4]), h // 3, p % 4)
                e = np.exp(np.dot(t["q"][b, h], t["k_pool"][at] * t["k_scale"][at]) / 4.0)
                num, den = num + e * t["v_pool"][at] * t["v_scale"][at], den + e
            np.testing.assert_allclose(got[b, h], num / den if held else 0.0, rtol=1e-12, atol=1e-15)


def test_oracle_quantises_to_half_a_step():
    spec = dg.write_graph("f32", "i8", 5, [2, 7])
    out = run_graph(spec)
    for b, first in enumerate((2, 7)):
        for t in range(5):
            page, slot = spec.tensors["table"].data[b, (first + t) // 8], (first + t) % 8
            for n in "kv":
                n8, step, x = out[f"{n}_pool_new"][page, :, slot], out[f"{n}_scale_new"][page, :, slot, None], np.asarray(spec.tensors[n].data)[b, t]
                assert np.all(np.abs(n8) <= 127) and np.all(n8 == np.rint(n8)) and np.all(np.abs(n8).max(-1) == 127)
                assert np.all(np.abs(n8 * step - x) <= step * (0.5 + 127 * 2.0 ** -23))


def test_oracle_read_returns_what_was_written():
    w = dg.write_graph("f32", "f32", 13, [0, 0], [13, 4], DK=16, DV=48)
    pools = run_graph(w)
    r = dg.read_graph("f32", "f32", [13, 4], 15, DK=16, DV=48)
    out = run_graph(r, feeds={"k_pool": pools["k_pool_new"], "v_pool": pools["v_pool_new"]})
    for n in "kv":
        want = np.zeros((2, 15) + w.tensors[n].shape[2:])
        want[0, :13], want[1, :4] = w.tensors[n].data[0], w.tensors[n].data[1, :4]
        np.testing.assert_array_equal(out[n + "_out"], want)


def test_oracle_int4_against_loops():
    spec = dg.int4_graph("f32", (2,), 71, 3, 32, True)
    t = {n: np.asarray(x.data, dtype=np.float64) for n, x in spec.tensors.items() if x.data is not None}
    y = next(iter(run_graph(spec).values()))
    for m in range(2):
        for n in range(3):
            s = 0.0
            for k in range(71):
                byte = int(t["w"][n, k // 2])
                s += t["x"][m, k] * ((byte >> 4 if k % 2 else byte & 15) - t["z"][n, k // 32]) * t["s"][n, k // 32]
            assert abs(y[m, n] - s) <= 1e-12 * 71


# ------------------------------------------------------------------------------------------------ plans
def test_blocks_of_a_decode_step():
    from workloads import configs

    p = plan(configs.gpt2_decode_step(**configs.SMALL_EXTRA["gpt2_decode_step"]))
    ops = [d["ops"] for d in p.describe()]
    # what follows a product runs in its kernel: bias, heads, residual sums, the activation
    assert ["MatMulInt4", "Add", "Split", "Reshape", "Reshape", "Reshape"] in ops and ["MatMulInt4", "Add", "Add"] in ops
    assert any(o[0] == "MatMulInt4" and "Tanh" in o for o in ops)
    assert ops.count(["CacheWrite"]) == 2 and ops.count(["CacheAttention"]) == 2
    # every attention stands behind the write that fills its pools
    flat = [o[0] for o in ops]
    assert [o for o in flat if o.startswith("Cache")] == ["CacheWrite", "CacheAttention"] * 2


def test_short_capacity_takes_one_kernel_and_long_capacity_is_split():
    assert kernels(plan(dg.attend_graph("bf16", "bf16", [9], M=8))) == ["cache_attend_split1_16"]
    info = plan(dg.attend_graph("bf16", "bf16", [9], M=80)).describe()[0]
    assert info["n_kernel_launches"] == 2 and "split10_" in info["kernel_name"]
    # a window bounds what there is to split
    assert kernels(plan(dg.attend_graph("bf16", "bf16", [9], M=80, attrs={"window": 90}))) == ["cache_attend_split1_16"]


def test_mapping_types_and_families():
    assert api.op_kind_mapping_type("CacheRead") == api.MAPPING_NAMES.index("One-to-Many")
    for k in ("CacheWrite", "CacheAttention", "MatMulInt4"):
        assert api.op_kind_mapping_type(k) == api.MAPPING_NAMES.index("Many-to-Many")
    assert api.FAMILY_NAMES[plan(dg.attend_graph("bf16", "bf16", [9])).describe()[0]["family"]] == "cache"
    assert api.FAMILY_NAMES[plan(dg.int4_graph("f16", (1,), 64, 64, 32)).describe()[0]["family"]] == "int4-gemm"


def test_casts_next_to_typed_operands_stay():
    """A cast in front of or behind these operators is part of their types and is not merged away by the rewriting."""
    b = dg.GraphBuilder("cast", "f32")
    spec = dg.int4_graph("f32", (2,), 64, 48, 32)
    b.g = spec
    x16 = b.input("x16", (2, 64), dg.normal(1, 1, (2, 64), "f16"), dtype="f16")
    spec.ops[0].inputs[0] = b.op("Cast", [x16], (2, 64), {"to": 1})
    y = spec.ops[0].outputs[0]
    spec.tensors[y].kind = "intermediate"
    b.g.ops = [spec.ops[1], spec.ops[0]]
    y16 = b.op("Cast", [y], (2, 48), {"to": 10}, out_dtype="f16")
    b.mark_output(y16)
    del spec.tensors["x"]
    g, _ = api.graph_from_spec(spec)
    g.rewrite()
    assert [k for _, k, _ in g.live_ops()].count("Cast") == 2
    api.Plan(g, [1] * 2)


def test_data_format_selection_leaves_cache_rows_alone():
    """A convolution's result that goes into the cache keeps the declared order; the one in front of it need not."""
    b = dg.GraphBuilder("conv_cache", "f16")
    x = b.input("x", (2, 16, 8, 32), dg.normal(1, 1, (2, 16, 8, 32), "f16"))
    w = [b.weight(f"w{i}", (16, 16, 3, 3), dg.normal(2, i, (16, 16, 3, 3), "f16")) for i in range(2)]
    conv = {"strides": [1, 1], "pads": [1, 1, 1, 1], "group": 1}
    y = b.op("Relu", [b.op("Conv", [b.op("Relu", [b.op("Conv", [x, w[0]], (2, 16, 8, 32), conv)], (2, 16, 8, 32)), w[1]], (2, 16, 8, 32), conv)], (2, 16, 8, 32))
    table, P = dg.pages_of(5, 2, 2)
    pools = dg.pool_inputs(b, 5, "f16", P, 8, 16, 32, 32)
    ins = pools + [y, y, b.input("table", table.shape, table, dtype="i32"), b.input("first", (2,), np.array([0, 3]), dtype="i32")]
    b.g.ops.append(dg.OpSpec("CacheWrite", ins, [b._add(p + "_new", "f16", b.shape(p), "output") for p in pools]))
    p = plan(b.finish(), layout=1)
    assert [d["ops"] for d in p.describe() if not d["prepare_only"]][-1] == ["CacheWrite"]


# ------------------------------------------------------------------------------------------------ refusals
def refused(spec, match, code=None):
    with pytest.raises(api.DnnfError, match=match) as e:
        api.graph_from_spec(spec)
    assert code is None or e.value.code == code


def retyped(spec, name, dtype):
    spec.tensors[name].dtype = dtype
    return spec


def reshaped(spec, name, shape):
    spec.tensors[name].shape, spec.tensors[name].data = shape, None
    return spec


def with_attrs(spec, **kw):
    spec.ops[0].attrs.update(kw)
    return spec


INVALID, MISMATCH, UNSUPPORTED = -1, -2, -3


@pytest.mark.parametrize("spec,match,code", [
    (lambda: reshaped(dg.attend_graph("bf16", "bf16", [1, 1]), "q", (2, 3, 64)), "no multiple of the key heads", MISMATCH),
    (lambda: reshaped(dg.attend_graph("bf16", "bf16", [1, 1]), "q", (2, 4, 32)), "channels of a key", MISMATCH),
    (lambda: reshaped(dg.attend_graph("bf16", "bf16", [1, 1]), "held", (3,)), "one number per sequence", MISMATCH),
    (lambda: reshaped(dg.attend_graph("bf16", "bf16", [1, 1]), "table", (16,)), "table", MISMATCH),
    (lambda: reshaped(dg.attend_graph("bf16", "i8", [1, 1]), "v_scale", (5, 2, 16)), "scale tensor", MISMATCH),
    (lambda: reshaped(dg.attend_graph("bf16", "bf16", [1, 1]), "v_pool", (19, 2, 8, 64)), "pools differ", MISMATCH),
    (lambda: dg.attend_graph("bf16", "bf16", [1, 1], DK=40), "multiple of 16", UNSUPPORTED),
    (lambda: dg.attend_graph("bf16", "bf16", [1, 1], DV=272), "at most 256", UNSUPPORTED),
    (lambda: retyped(dg.attend_graph("bf16", "bf16", [1, 1]), "q", "f16"), "share one type", INVALID),
    (lambda: retyped(dg.attend_graph("bf16", "bf16", [1, 1]), "held", "i64"), "I32", INVALID),
    (lambda: retyped(dg.attend_graph("bf16", "bf16", [1, 1]), "v_pool", "f16"), "share one type", INVALID),
    (lambda: retyped(dg.attend_graph("bf16", "i8", [1, 1]), "k_scale", "bf16"), "F32", INVALID),
    (lambda: dg.attend_graph("bf16", "bf16", [1], attrs={"window": -1}), "window", INVALID),
    (lambda: dg.attend_graph("bf16", "bf16", [1], attrs={"window": 2.5}), "window", INVALID),
    (lambda: dg.attend_graph("bf16", "bf16", [1], attrs={"scale": float("nan")}), "scale", INVALID),
    (lambda: dg.attend_graph("bf16", "bf16", [1], attrs={"scale": 1e39}), "scale", INVALID),
    (lambda: dg.attend_graph("bf16", "bf16", [1], attrs={"window": 1e30}), "window", INVALID),
    (lambda: dg.attend_graph("bf16", "bf16", [1], attrs={"window": float("nan")}), "window", INVALID),
    (lambda: with_attrs(dg.read_graph("f16", "f16", [1], 4), length=4.5), "length", INVALID),
    (lambda: with_attrs(dg.read_graph("f16", "f16", [1], 4), length=-1e300), "length", INVALID),
    (lambda: with_attrs(dg.int4_graph("f16", (1,), 64, 8, 32), group_size=float("inf")), "group_size", INVALID),
    (lambda: with_attrs(dg.read_graph("f16", "f16", [1], 4), length=0), "length", INVALID),
    (lambda: with_attrs(dg.read_graph("f16", "f16", [1], 4), length=5), "declared", MISMATCH),
    (lambda: retyped(dg.read_graph("f16", "f16", [1], 4), "k_out", "f32"), "share one type", INVALID),
    (lambda: retyped(dg.write_graph("f16", "f16", 1, [1]), "k", "f32"), "share one type", INVALID),
    (lambda: retyped(dg.write_graph("f16", "f16", 1, [1]), "k_pool_new", "bf16"), "differs in type", INVALID),
    (lambda: dg.int4_graph("f16", (1,), 64, 8, 16), "group_size", INVALID),
    (lambda: dg.int4_graph("f16", (1,), 64, 8, 48), "group_size", INVALID),
    (lambda: reshaped(dg.int4_graph("f16", (1,), 64, 8, 32), "w", (8, 31)), "bytes", MISMATCH),
    (lambda: reshaped(dg.int4_graph("f16", (1,), 64, 8, 32), "s", (8, 3)), "groups of K", MISMATCH),
    (lambda: retyped(dg.int4_graph("f16", (1,), 64, 8, 32), "s", "f32"), "share a float type", INVALID),
    (lambda: retyped(dg.int4_graph("f16", (1,), 64, 8, 32), "w", "i8"), "U8", INVALID),
    (lambda: retyped(dg.int4_graph("f16", (1,), 64, 8, 32, True), "z", "i8"), "U8", INVALID),
])
def test_refusals(spec, match, code):
    refused(spec(), match, code)


def test_operand_counts():
    spec = dg.attend_graph("bf16", "bf16", [1])
    spec.ops[0].inputs.append("held")
    refused(spec, "too many operands", INVALID)
    spec = dg.attend_graph("bf16", "bf16", [1])
    spec.ops[0].inputs.pop()
    refused(spec, "no operand for held", INVALID)
    spec = dg.write_graph("bf16", "i8", 1, [1])
    spec.ops[0].outputs.pop()
    refused(spec, "has 4 results", INVALID)


def test_pools_are_inputs_updated_in_place():
    spec = dg.write_graph("bf16", "bf16", 1, [1])
    spec.tensors["k_pool"].kind = "weight"
    refused(spec, "must be an INPUT", INVALID)
    spec = dg.write_graph("bf16", "bf16", 1, [1])
    spec.tensors["v_pool_new"].kind = "intermediate"
    refused(spec, "must be an INPUT", INVALID)
    # nobody else reads the pool under the name it had before
    spec = dg.write_graph("bf16", "bf16", 1, [1])
    b = dg.GraphBuilder("reader", "bf16")
    b.g = spec
    held = b.input("held", (1,), np.array([1]), dtype="i32")
    b.g.ops.append(dg.OpSpec("CacheRead", ["k_pool", "v_pool_new", "table", held], [b._add(n, "bf16", (1, 4, 2, 32), "output") for n in ("ko", "vo")], {"length": 4}))
    refused(spec, "other operators read its result", INVALID)
    # one pool as keys and values at once
    spec = dg.write_graph("bf16", "bf16", 1, [1])
    spec.ops[0].inputs[1] = "k_pool"
    refused(spec, "other operators read its result", INVALID)


def test_other_operators_refuse_tensors_of_8_bits():
    b = dg.GraphBuilder("other", "f32")
    x = b.input("x", (4, 4), np.zeros((4, 4)), dtype="i8")
    b.mark_output(b.op("Relu", [x], (4, 4), out_dtype="i8"))
    refused(b.finish(), "8 bits", UNSUPPORTED)


def test_sizes_beyond_the_index_ranges():
    def declared(P, S, M, T=1):
        g = api.Graph()
        pools = [g.add_tensor(n, "bf16", (P, 8, S, 128), "input") for n in "kv"]
        rest = [g.add_tensor("q", "bf16", (1, 8, 128), "input"), g.add_tensor("t", "i32", (1, M), "input"), g.add_tensor("h", "i32", (1,), "input")]
        g.add_op("CacheAttention", [rest[0]] + pools + rest[1:], [g.add_tensor("o", "bf16", (1, 8, 128), "output")])
        g.finalize()

    declared(1 << 20, 128, 1 << 16)
    with pytest.raises(api.DnnfError, match="2\\^31 rows"):
        declared(1 << 24, 16, 4)
    with pytest.raises(api.DnnfError, match="2\\^30 positions"):
        declared(16, 1024, 1 << 20)


def test_host_code_under_sanitizers(tmp_path):
    """Checks, plans and generated sources of these operators, refusals among them, through the instrumented library."""
    from test_host_sanitizers import run, write_spec

    from paper_2108_13342_amd import build
    from workloads import configs

    fine = {"decode_step": configs.gpt2_decode_step(**configs.SMALL_EXTRA["gpt2_decode_step"]), "write": dg.write_graph("f32", "i8", 40, [0, 7]),
            "read": dg.read_graph("bf16", "bf16", [3], 20), "attend": dg.attend_graph("f32", "i8", [9], HQ=34, M=80, DV=112),
            "int4": dg.int4_graph("f32", (3, 2), 77, 40, 32, True, bias=True)}
    bad = {"window": (dg.attend_graph("bf16", "bf16", [1], attrs={"window": 1e30}), -1), "heads": (reshaped(dg.attend_graph("bf16", "bf16", [1, 1]), "q", (2, 3, 64)), -2),
           "channels": (dg.attend_graph("bf16", "bf16", [1], DK=40), -3), "group": (with_attrs(dg.int4_graph("f16", (1,), 64, 8, 32), group_size=1e30), -1)}
    files = []
    for name, (spec, code) in {**{n: (s, 0) for n, s in fine.items()}, **bad}.items():
        files.append(str(tmp_path / (name + ".txt")))
        write_spec(spec, files[-1], expect_finalize=code)
    r = run(build.build_sanitizer_driver(), files)
    assert r.returncode == 0, (r.stdout[-2000:], r.stderr[-6000:])
    assert "Sanitizer" not in r.stderr and "runtime error" not in r.stderr, r.stderr[-6000:]
    assert r.stdout.count("\nok ") + r.stdout.startswith("ok ") == len(files), r.stdout


# ------------------------------------------------------------------------------------------------ storage that is shared
@pytest.mark.parametrize("how", dg.CASTS)
@pytest.mark.parametrize("fusion", [0, 1])
def test_storage_is_shared_between_tensors_of_one_type_only(how, fusion):
    """A Cast behind or in front of a Reshape is merged into it by the rewriting: that Reshape converts, and shares nothing."""
    p = plan(dg.cast_graph(how), fusion=fusion)
    for b in p.dump_json()["blocks"]:
        if api.FAMILY_NAMES[b["family"]] == "alias":
            assert len({t["dtype"] for t in b["inputs"] + b["outputs"]}) == 1, b


@pytest.mark.parametrize("graphs", [0, 1])
def test_buffers_are_looked_at_before_anything_is_launched(graphs):
    """Two layers' caches.  Nothing is at these addresses, and there is no GPU: a refusal of the second layer's buffers comes before
    the first layer's kernel is so much as loaded."""
    spec = dg.two_caches_graph()
    p = plan(spec, graphs=graphs)
    names = [t.name for t in spec.inputs()]
    at = {n: (i + 1) << 20 for i, n in enumerate(names)}
    outs = [at[t.name.replace("_new", "")] for t in spec.outputs()]

    def call(match, ins=(), out=()):
        a = [dict(ins).get(n, at[n]) for n in names]
        o = [dict(out).get(t.name, x) for t, x in zip(spec.outputs(), outs)]
        for run in (lambda: p.run(a, o, 1 << 30), lambda: p.bind(a, o, 1 << 30).run()):
            with pytest.raises(api.DnnfError, match=match) as e:
                run()
            assert e.value.code == INVALID

    call("v_pool1_new is input v_pool1 updated in place", out=[("v_pool1_new", 12345 << 4)])
    call("v_pool1_new", out=[("v_pool1_new", 0)])
    call("missing input pointer for k1", ins=[("k1", 0)])
    for other in ("k_pool0", "v_pool0", "k_pool1"):      # two pools in one buffer, or in buffers that overlap
        for off in (0, 64, -64):
            call("share one buffer", ins=[("v_pool1", at[other] + off)], out=[("v_pool1_new", at[other] + off)])


def test_writing_many_pages_is_no_square_of_work():
    """Up to 4096 pages a call every workgroup looks through them all; above, three kernels settle who writes a slot."""
    few = plan(dg.write_graph("f16", "f16", 2048, [0, 0], S=1, M=2048)).describe()[0]
    assert few["n_kernel_launches"] == 1 and "cache_write_chunk1" in few["kernel_name"]
    p = plan(dg.write_graph("f16", "i8", 2049, [0, 0], S=1, M=2049))
    assert p.describe()[0]["n_kernel_launches"] == 3 and "cache_write_owned_i8" in p.describe()[0]["kernel_name"]
    pages = 2 * 2049 + 3
    assert p.workspace_bytes() >= 4 * pages      # a place for every slot of the pool
    p.precompile()


def test_writing_into_a_large_page_takes_workgroups_for_its_tokens_only():
    for T, S, most in ((1, 1 << 17, 2 * 1), (40, 1 << 17, 2 * 2 * 3), (40, 64, 2 * 2 * 3), (64, 64, 2 * 2 * 4), (1 << 10, 64, 2 * 17 * 4)):
        g = api.Graph()
        pools = [g.add_tensor(n, "f16", (2, 1, S, 16), "input") for n in "kv"]
        new = [g.add_tensor(n + "n", "f16", (2, T, 1, 16), "input") for n in "kv"]
        at = [g.add_tensor("table", "i32", (2, 16), "input"), g.add_tensor("first", "i32", (2,), "input")]
        g.add_op("CacheWrite", pools + new + at, [g.add_tensor(n + "o", "f16", (2, 1, S, 16), "output") for n in "kv"])
        g.finalize()
        grid = api.Plan(g, []).dump_json()["blocks"][0]["launches"][0]["grid"]
        assert grid[0] <= most and grid[1] == 1, (T, S, grid)


def test_bytes_and_operations_are_of_the_rows_that_are_reached():
    """A pool far larger than what its operators touch: counted is what the tables and attributes reach, rows once."""
    def block(spec):
        d = plan(spec).describe()[0]
        return d["bytes"], d["flops"]

    # 2 sequences, 3 tokens, 2 heads of 32 + 32 channels: rows in, rows out, tables and positions
    assert block(dg.write_graph("f16", "f16", 3, [0, 9], P=5000))[0] == 2 * (2 * 3 * 2 * 64 * 2) + 4 * (2 * 6 + 2)
    assert block(dg.write_graph("f32", "i8", 3, [0, 9], [1, 2], P=5000))[0] == 2 * 3 * 2 * (64 * 4 + 64 + 8) + 4 * (2 * 6 + 2 + 2)
    assert block(dg.read_graph("f16", "i8", [5, 9], 10))[0] == 2 * 10 * 2 * (64 + 8 + 64 * 2) + 4 * (2 * 6 + 2)
    assert block(dg.read_graph("f16", "f16", [5], 60, table=[[0, 1]]))[0] == 16 * 2 * 64 * 2 + 60 * 2 * 64 * 2 + 4 * (2 + 1)
    # 2 x 128 positions, 2 key heads and 4 query heads of 64 + 64 channels
    assert block(dg.attend_graph("bf16", "bf16", [9, 9], P=5000)) == (2 * 128 * 2 * 128 * 2 + 2 * 4 * 128 * 2 + 4 * (16 + 2), 2.0 * 2 * 4 * 128 * 128)
    assert block(dg.attend_graph("bf16", "i8", [9, 9], P=5000, attrs={"window": 10})) == (2 * 10 * 2 * (128 + 8) + 2 * 4 * 128 * 2 + 4 * (16 + 2), 2.0 * 2 * 4 * 10 * 128)
    # two sequences on one page
    assert block(dg.attend_graph("bf16", "bf16", [9, 9], M=1, table=[[0], [0]], P=1))[0] == 16 * 2 * 128 * 2 + 2 * 4 * 128 * 2 + 4 * (2 + 2)


def test_products_and_launches_beyond_the_index_ranges():
    def product(M, K, N, G=32):
        g = api.Graph()
        ins = [g.add_tensor("x", "f16", (M, K), "input"), g.add_tensor("w", "u8", (N, (K + 1) // 2), "weight"), g.add_tensor("s", "f16", (N, -(-K // G)), "weight")]
        g.add_op("MatMulInt4", ins, [g.add_tensor("y", "f16", (M, N), "output")], {"group_size": G})
        g.finalize()
        return api.Plan(g, [1, 1]).block_source(0)

    # a tile's last columns lie behind the last one: their numbers have to fit too
    for M, N in ((1, (1 << 31) - 300), (1, 1 << 31)):
        assert "typedef long long idx_t" in product(M, 2, N)
    assert "typedef int idx_t" in product(1, 2, 1 << 30)
    product(1, (1 << 31) - 257, 1)
    for K in ((1 << 31) - 256, 1 << 31, 1 << 33):
        with pytest.raises(api.DnnfError, match="contraction of 2\\^31") as e:
            product(1, K, 1)
        assert e.value.code == UNSUPPORTED
    # 2^32 threads and more in a launch
    with pytest.raises(api.DnnfError, match="more workgroups than one launch takes") as e:
        product(1 << 30, 32, 64)
    assert e.value.code == UNSUPPORTED
    g = api.Graph()
    pools = [g.add_tensor(n, "f16", (4, 16, 16, 16), "input") for n in "kv"]
    ins = [g.add_tensor("q", "f16", (1 << 19, 16 * 64, 16), "input")] + pools + [g.add_tensor("t", "i32", (1 << 19, 1), "input"), g.add_tensor("h", "i32", (1 << 19,), "input")]
    g.add_op("CacheAttention", ins, [g.add_tensor("o", "f16", (1 << 19, 16 * 64, 16), "output")])
    g.finalize()
    with pytest.raises(api.DnnfError, match="more workgroups than one launch takes"):
        api.Plan(g, [])


def test_later_host_code_under_sanitizers(tmp_path):
    """Plans with converting Reshapes, the write of many pages and two caches, through the instrumented library."""
    from test_host_sanitizers import run, write_spec

    from paper_2108_13342_amd import build

    specs = {how: dg.cast_graph(how) for how in dg.CASTS}
    specs.update(two=dg.two_caches_graph(), many=dg.write_graph("f32", "i8", 2049, [0, 7], [3, 2049], S=1, M=2100))
    files = []
    for name, spec in specs.items():
        files.append(str(tmp_path / (name + ".txt")))
        write_spec(spec, files[-1], expect_finalize=0)
    r = run(build.build_sanitizer_driver(), files)
    assert r.returncode == 0, (r.stdout[-2000:], r.stderr[-6000:])
    assert "Sanitizer" not in r.stderr and "runtime error" not in r.stderr, r.stderr[-6000:]
    assert r.stdout.count("\nok ") + r.stdout.startswith("ok ") == len(files), r.stdout
