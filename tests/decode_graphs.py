"""Small graphs of the operators of single-token inference, shared by the host and the GPU tests."""
import numpy as np

from workloads import rng
from workloads.graph import GraphBuilder, OpSpec

HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}      # half a unit in the last place, relative


def normal(seed, k, shape, dtype, std=1.0):
    return rng.round_to(rng.normal(seed, k, shape, 0.0, std), dtype)


def pages_of(seed, B, M, P=None):
    """A table [B, M] of distinct pages in a mixed order, and the pages of the pool (three more than the table names)."""
    P = P or B * M + 3
    return np.resize(np.argsort(rng.uniform(seed, 77, (P,)), kind="stable"), (B, M)).astype(np.int64), P


def pool_inputs(b, seed, cache, P, HK, S, DK, DV):
    names = []
    for i, (n, D) in enumerate((("k", DK), ("v", DV))):
        data = rng.integers(seed, 11 + i, (P, HK, S, D), -127, 128) if cache == "i8" else normal(seed, 11 + i, (P, HK, S, D), cache)
        names.append(b.input(f"{n}_pool", (P, HK, S, D), data, dtype=cache))
    if cache == "i8":
        names += [b.input(f"{n}_scale", (P, HK, S), rng.round_to(rng.uniform(seed, 21 + i, (P, HK, S), 0.005, 0.02), "f32"), dtype="f32")
                  for i, n in enumerate("kv")]
    return names


def write_graph(dtype, cache, T, first, count=None, HK=2, DK=32, DV=32, S=8, M=6, seed=5, table=None, P=None, k=None, v=None):
    B = len(first)
    b = GraphBuilder("cache_write", dtype)
    made, made_P = pages_of(seed, B, M, P)
    table, P = (made if table is None else np.asarray(table)), P or made_P
    pools = pool_inputs(b, seed, cache, P, HK, S, DK, DV)
    kn = b.input("k", (B, T, HK, DK), normal(seed, 1, (B, T, HK, DK), dtype) if k is None else k)
    vn = b.input("v", (B, T, HK, DV), normal(seed, 2, (B, T, HK, DV), dtype) if v is None else v)
    ins = pools + [kn, vn, b.input("table", table.shape, table, dtype="i32"), b.input("first", (B,), np.asarray(first), dtype="i32")]
    if count is not None:
        ins.append(b.input("count", (B,), np.asarray(count), dtype="i32"))
    outs = [b._add(p + "_new", b.g.tensors[p].dtype, b.shape(p), "output") for p in pools]
    b.g.ops.append(OpSpec("CacheWrite", ins, outs))
    return b.finish()


def read_graph(dtype, cache, held, L, HK=2, DK=32, DV=32, S=8, M=6, seed=5, table=None):
    B = len(held)
    b = GraphBuilder("cache_read", dtype)
    made, P = pages_of(seed, B, M)
    table = made if table is None else np.asarray(table)
    pools = pool_inputs(b, seed, cache, P, HK, S, DK, DV)
    ins = pools + [b.input("table", table.shape, table, dtype="i32"), b.input("held", (B,), np.asarray(held), dtype="i32")]
    outs = [b._add(n, dtype, (B, L, HK, D), "output") for n, D in (("k_out", DK), ("v_out", DV))]
    b.g.ops.append(OpSpec("CacheRead", ins, outs, {"length": L}))
    return b.finish()


def attend_graph(dtype, cache, held, HQ=4, HK=2, DK=64, DV=64, S=16, M=8, seed=5, table=None, attrs=None, P=None, q_std=1.0):
    B = len(held)
    b = GraphBuilder("cache_attend", dtype)
    made, made_P = pages_of(seed, B, M, P)
    table, P = (made if table is None else np.asarray(table)), P or made_P
    q = b.input("q", (B, HQ, DK), normal(seed, 1, (B, HQ, DK), dtype, q_std))
    pools = pool_inputs(b, seed, cache, P, HK, S, DK, DV)
    ins = [q] + pools + [b.input("table", table.shape, table, dtype="i32"), b.input("held", (B,), np.asarray(held), dtype="i32")]
    b.g.ops.append(OpSpec("CacheAttention", ins, [b._add("o", dtype, (B, HQ, DV), "output")], dict(attrs or {})))
    return b.finish()


def int4_graph(dtype, lead, K, N, G, zeros=False, bias=False, seed=5):
    b = GraphBuilder("matmul_int4", dtype)
    groups = -(-K // G)
    x = b.input("x", tuple(lead) + (K,), normal(seed, 1, tuple(lead) + (K,), dtype))
    ins = [x, b.weight("w", (N, (K + 1) // 2), rng.integers(seed, 2, (N, (K + 1) // 2), 0, 256), dtype="u8"),
           b.weight("s", (N, groups), rng.round_to(rng.uniform(seed, 3, (N, groups), 0.01, 0.05), dtype))]
    if zeros:
        ins.append(b.weight("z", (N, groups), rng.integers(seed, 4, (N, groups), 0, 16), dtype="u8"))
    y = b.op("MatMulInt4", ins, tuple(lead) + (N,), {"group_size": G})
    if bias:
        y = b.op("Relu", [b.op("Add", [y, b.weight("bias", (N,), normal(seed, 6, (N,), dtype))], tuple(lead) + (N,))], tuple(lead) + (N,))
    b.mark_output(y)
    return b.finish()


def cast_graph(how):
    """A Cast between float types with a Reshape between it and an operator that fixes its operands' types."""
    b = GraphBuilder("cast_" + how, "f32")
    f16 = dict(out_dtype="f16")
    if how == "attend_reshape_cast":           # fp32 results, reshaped, narrowed, multiplied in float16
        b.g = attend_graph("f32", "i8", [9, 40])
        y = b.op("Cast", [b.op("Reshape", ["o"], (2, 256), {"shape": [2, 256]})], (2, 256), {"to": 10}, **f16)
        b.g.tensors["o"].kind = "intermediate"
        y = b.op("MatMul", [y, b.weight("proj", (256, 32), normal(7, 7, (256, 32), "f16", 0.1), dtype="f16")], (2, 32), **f16)
    elif how == "cast_reshape_attend":         # float16 queries, widened, reshaped, attended with in fp32
        b.g = attend_graph("f32", "i8", [9, 40])
        x = b.input("x", (512,), normal(7, 7, (512,), "f16"), dtype="f16")
        b.g.ops[0].inputs[0] = b.op("Reshape", [b.op("Cast", [x], (512,), {"to": 1})], (2, 4, 64), {"shape": [2, 4, 64]})
        del b.g.tensors["q"]
        y = "o"
    elif how == "cast_reshape_int4":
        b.g = int4_graph("f32", (3,), 96, 40, 32, True)
        x = b.input("x16", (288,), normal(7, 7, (288,), "f16"), dtype="f16")
        b.g.ops[0].inputs[0] = b.op("Reshape", [b.op("Cast", [x], (288,), {"to": 1})], (3, 96), {"shape": [3, 96]})
        del b.g.tensors["x"]
        y = b.g.ops[0].outputs[0]
    elif how == "int4_reshape_cast":
        b.g = int4_graph("f32", (3,), 96, 40, 32, True)
        y = b.g.ops[0].outputs[0]
        b.g.tensors[y].kind = "intermediate"
        y = b.op("Cast", [b.op("Reshape", [y], (120,), {"shape": [120]})], (120,), {"to": 10}, **f16)
    elif how == "write_and_read":              # new rows widened and reshaped, the cache's contents reshaped and narrowed
        b.g = write_graph("f32", "f32", 5, [0, 6])
        for n in "kv":
            x = b.input(n + "16", (640,), normal(7, ord(n), (640,), "f16"), dtype="f16")
            b.g.ops[0].inputs[2 + "kv".index(n)] = b.op("Reshape", [b.op("Cast", [x], (640,), {"to": 1})], (2, 5, 2, 32), {"shape": [2, 5, 2, 32]})
            del b.g.tensors[n]
        kept, held = b.g.ops[0].outputs, b.input("held", (2,), np.array([5, 11]), dtype="i32")
        write = b.g.ops.pop(0)
        b.g.ops.append(write)
        rows = [b._add(n + "_all", "f32", (2, 12, 2, 32), "intermediate") for n in "kv"]
        b.g.ops.append(OpSpec("CacheRead", kept + ["table", held], rows, {"length": 12}))
        for r in rows:
            y = b.op("Relu", [b.op("Cast", [b.op("Reshape", [r], (24, 64), {"shape": [24, 64]})], (24, 64), {"to": 10}, **f16)], (24, 64), **f16)
            b.mark_output(y)
    else:                                      # ordinary operators: widened, reshaped, and a product in fp32
        x = b.input("x", (288,), normal(7, 7, (288,), "f16"), dtype="f16")
        y = b.op("Reshape", [b.op("Cast", [x], (288,), {"to": 1})], (3, 96), {"shape": [3, 96]})
        y = b.op("MatMul", [y, b.weight("proj", (96, 32), normal(7, 8, (96, 32), "f32", 0.1))], (3, 32))
    b.mark_output(y)
    order, done = [], {n for n, t in b.g.tensors.items() if t.kind in ("input", "weight")}
    while len(order) < len(b.g.ops):           # operators behind what they read
        for op in b.g.ops:
            if op not in order and all(i in done for i in op.inputs):
                order.append(op)
                done.update(op.outputs)
    b.g.ops = order
    return b.finish()


CASTS = ("attend_reshape_cast", "cast_reshape_attend", "cast_reshape_int4", "int4_reshape_cast", "write_and_read", "cast_reshape_matmul")


def two_caches_graph():
    """Two layers' caches, written one after the other in one graph."""
    b = GraphBuilder("two_caches", "f16")
    table, P = pages_of(5, 2, 4)
    t, first = b.input("table", table.shape, table, dtype="i32"), b.input("first", (2,), np.array([0, 3]), dtype="i32")
    for layer in range(2):
        pools = [b.input(f"{n}_pool{layer}", (P, 2, 8, 32), normal(6, 2 * layer + i, (P, 2, 8, 32), "f16")) for i, n in enumerate("kv")]
        new = [b.input(f"{n}{layer}", (2, 3, 2, 32), normal(7, 2 * layer + i, (2, 3, 2, 32), "f16")) for i, n in enumerate("kv")]
        b.g.ops.append(OpSpec("CacheWrite", pools + new + [t, first], [b._add(p + "_new", "f16", b.shape(p), "output") for p in pools]))
    return b.finish()
