"""The operators of single-token inference against their definitions in 64 bits: a paged key / value cache written in place,
read back and attended over, and products with weights of four bits."""
import numpy as np
import pytest

import decode_graphs as dg
from oracle.interp import run_graph

pytestmark = pytest.mark.gpu


def run(spec, **kw):
    from paper_2108_13342_amd import api

    s = api.Session(spec, guard_bytes=256, **kw)
    s.run()
    got = s.result()
    assert s.guards_intact(), f"{spec.name}: a kernel wrote outside an output buffer or the workspace"
    return s, got


def data(spec, name):
    return np.asarray(spec.tensors[name].data, dtype=np.float64)


# ------------------------------------------------------------------------------------------------ CacheWrite
def check_written(spec):
    _, got = run(spec)
    for n, want in run_graph(spec).items():
        np.testing.assert_array_equal(got[n], want, err_msg=n)      # rows are copied, or quantised by correctly rounded quotients


@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f32", "i8"), ("f16", "i8"), ("bf16", "i8")])
@pytest.mark.parametrize("T,first,count", [(1, [0, 7, 8, 47], None), (1, [47, 48, -1, 3], None), (11, [0, 5, 36, 40], [11, 0, 11, 3]),
                                           (29, [-4, 13, 2000000000, -2147483648], [29, 40, 7, 29])])
def test_write(dtype, cache, T, first, count):
    check_written(dg.write_graph(dtype, cache, T, first, count))


@pytest.mark.parametrize("DK,DV,HK,S", [(16, 16, 1, 1), (48, 80, 3, 5), (256, 16, 2, 64), (128, 128, 5, 40), (80, 256, 1, 100)])
@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f32", "i8"), ("f16", "i8"), ("f32", "f32")])
def test_write_shapes(dtype, cache, DK, DV, HK, S):
    check_written(dg.write_graph(dtype, cache, 2 * S + 3, [1, 0, S - 1], [2 * S + 3, 2 * S, 1], HK=HK, DK=DK, DV=DV, S=S, M=4))


@pytest.mark.parametrize("S", [1, 8, 100])
def test_write_at_the_ends_of_the_number_range(S):
    # positions around the largest and the smallest 32-bit number, behind the table, counts below zero and above the operand's tokens
    check_written(dg.write_graph("bf16", "i8", 5, [2147483647, 2147483643, -2147483648, 6 * S - 2, -3, 0], [5, 2147483647, -1, 5, 2147483647, -2147483648], S=S))


def test_write_leaves_out_pages_that_are_not_there():
    table = np.array([[0, -1, 3, 99, 2, 1], [4, 5, 6, 7, -2147483648, 2147483647]])
    check_written(dg.write_graph("bf16", "bf16", 40, [3, 1], table=table, P=8))
    check_written(dg.write_graph("bf16", "i8", 40, [3, 1], table=table, P=8))


@pytest.mark.parametrize("cache", ["f16", "i8"])
def test_a_slot_written_twice_keeps_the_last(cache):
    # two sequences on the same pages, one sequence with a page twice in its row, and one that meets neither
    table = np.array([[0, 1, 2, 0, 1, 1], [2, 1, 0, 3, 3, 3], [4, 5, 6, 7, 8, 9]])
    check_written(dg.write_graph("f16", cache, 44, [2, 0, 1], [44, 17, 30], table=table, P=10))
    check_written(dg.write_graph("f16", cache, 1, [3, 19, 3], table=table, P=10))


def test_rows_at_the_ends_of_the_range_of_a_step():
    k = dg.normal(3, 1, (6, 1, 2, 32), "f32").astype(np.float32)
    k[0] = 0.0
    k[1, 0, 0, 3], k[1, 0, 1, 5] = np.inf, np.nan
    k[2] *= np.float32(1e-37)
    k[3] *= np.float32(3e37)
    k[4, 0, 0] = np.float32(2.0 ** -120)
    k[4, 0, 1] = np.float32(2.0 ** -119)
    k[5, 0, 0, :] = np.arange(32) - 15.5           # values in the middle between two whole numbers of the step
    k[5, 0, 0, 0] = 127.0
    check_written(dg.write_graph("f32", "i8", 1, [0, 1, 2, 3, 4, 5], k=k, v=k))


# ------------------------------------------------------------------------------------------------ CacheRead
@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f32", "i8"), ("f16", "i8"), ("bf16", "i8")])
@pytest.mark.parametrize("L,held,HK,DK,DV,S", [(1, [0, 1, 5], 2, 32, 32, 8), (41, [41, 17, -3], 3, 48, 80, 5), (70, [100, 48, 9], 1, 256, 16, 16), (48, [8, 16, 2000000000], 4, 128, 128, 8)])
def test_read(dtype, cache, L, held, HK, DK, DV, S):
    spec = dg.read_graph(dtype, cache, held, L, HK=HK, DK=DK, DV=DV, S=S)
    _, got = run(spec)
    for n, want in run_graph(spec).items():
        if cache != "i8":
            np.testing.assert_array_equal(got[n], want, err_msg=n)
        else:      # one product in 32 bits, one rounding to the result's type
            assert np.all(np.abs(got[n] - want) <= np.abs(want) * (dg.HALF_STEP[dtype] + 2.0 ** -24 * 1.01)), n


def test_read_of_pages_that_are_not_there():
    table = np.array([[0, -1, 3, 99, 2, 1], [4, 5, 6, 7, -2147483648, 2147483647]])
    spec = dg.read_graph("bf16", "bf16", [48, 48], 48, table=table)
    _, got = run(spec)
    for n, want in run_graph(spec).items():
        np.testing.assert_array_equal(got[n], want)


# ------------------------------------------------------------------------------------------------ CacheAttention
def check_attention(spec, got=None):
    """|o - o64| <= u |o64| + c sum_j p_j |v_j|: u is the rounding of the result; c what each probability may be off by,
    relatively - its own rounding to the operand of the second product (16-bit pools; twice, for the sum's share), and the
    error of its score, (channels + 8) roundings of 2^-24 of sum |q k|, the exponential's 2 and the sums' one per key.  Pools of 8
    bits: rows are summed as whole numbers n + 128 <= 255 and 128 sum p is taken off, in fp32, 32 keys in two or three parts and
    the offset at a time: 98 roundings of 2^-24 of sums up to 255 sum_j p_j step_j, whatever the channel's own values are."""
    if got is None:
        _, got = run(spec)
    op = spec.ops[0]
    want = run_graph(spec)["o"]
    q, pools = data(spec, op.inputs[0]), [data(spec, n) for n in op.inputs[1:-2]]
    size = dg.GraphBuilder("size", spec.dtype)
    size.g.tensors, size.g.ops = dict(spec.tensors), [op]
    magnitude = run_graph(size.g, feeds={op.inputs[2]: np.abs(pools[1])})["o"]
    kmax = np.abs(pools[0] * (pools[2][..., None] if len(pools) == 4 else 1.0)).max()
    score = np.abs(q).sum(-1).max() * kmax * abs(op.attrs.get("scale", 1.0 / np.sqrt(q.shape[-1])))
    keys = spec.tensors[op.inputs[-2]].shape[1] * pools[0].shape[2]
    p16 = 2 * dg.HALF_STEP[spec.dtype] if len(pools) == 2 and spec.dtype != "f32" else 0.0
    c = p16 + 2.0 ** -24 * (2 * (q.shape[-1] + 8) * score + 16 + keys)
    flat = 2.0 ** -24 * 98 * 255 * pools[3][np.isfinite(pools[3])].max() if len(pools) == 4 else 0.0
    off = np.abs(got["o"] - want) - (dg.HALF_STEP[spec.dtype] * np.abs(want) * (1 + 2.0 ** -8) + c * magnitude + np.where(magnitude.max(-1, keepdims=True) > 0, flat, 0.0))
    assert np.all(off <= 0), f"{spec.name}: {off.max():.3e} over its bound"


@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f32", "i8"), ("f16", "i8"), ("bf16", "i8")])
@pytest.mark.parametrize("HQ,HK,DK,DV,S,M,held", [
    (4, 4, 64, 64, 16, 8, [1, 2, 31, 32, 33, 128, 0]),
    (8, 2, 128, 128, 16, 40, [640, 129, 300]),
    (7, 1, 48, 80, 5, 13, [65, 64, 1]),
    (34, 2, 96, 16, 20, 7, [140, 77]),          # more than sixteen query heads a key head
    (3, 3, 256, 256, 1, 150, [150, 5]),
    (32, 2, 32, 112, 64, 3, [192, 100]),
    (6, 6, 16, 32, 100, 2, [200, 101, 99]),
])
def test_attention(dtype, cache, HQ, HK, DK, DV, S, M, held):
    check_attention(dg.attend_graph(dtype, cache, held, HQ, HK, DK, DV, S, M))


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f16", "i8"), ("f32", "f32")])
@pytest.mark.parametrize("window", [1, 5, 32, 33, 200, 100000])
def test_attention_window(dtype, cache, window):
    check_attention(dg.attend_graph(dtype, cache, [1, 40, 257, 512, 300], S=16, M=32, attrs={"window": window}))


@pytest.mark.parametrize("scale", [0.5, -0.25, 0.0, 3.0])
def test_attention_scale(scale):
    check_attention(dg.attend_graph("f16", "f16", [100, 17], S=16, M=8, attrs={"scale": scale}))


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f32", "f32"), ("f16", "i8")])
def test_attention_split_over_long_sequences(dtype, cache):
    # one sequence of thousands of keys among short and empty ones: split, joined, and splits that nothing is left for
    check_attention(dg.attend_graph(dtype, cache, [5000, 3, 0, 1300], HQ=4, HK=1, DK=64, DV=64, S=16, M=313))


def test_attention_over_capacity_and_below_zero():
    check_attention(dg.attend_graph("bf16", "bf16", [2147483647, -5, -2147483648, 129], S=16, M=8))


@pytest.mark.parametrize("cache", ["bf16", "i8"])
@pytest.mark.parametrize("S", [16, 5])
def test_attention_sees_only_pages_that_are_there(cache, S):
    table, P = dg.pages_of(5, 3, 12)
    table[0, 3], table[0, 5], table[1, :], table[2, 11] = -1, P, -7, 2147483647
    spec = dg.attend_graph("bf16", cache, [12 * S, 12 * S, 12 * S], S=S, M=12, table=table, P=P)
    _, got = run(spec)
    assert np.all(got["o"][1] == 0.0)
    check_attention(spec, got)


@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("bf16", "i8")])
def test_what_masked_slots_hold_does_not_matter(dtype, cache):
    """Slots behind a sequence's keys, slots before its window and pages that no table names hold infinities and NaN."""
    held, S, M = [37, 100, 1, 0], 16, 8
    spec = dg.attend_graph(dtype, cache, held, S=S, M=M, attrs={"window": 50})
    want = run(spec)[1]["o"]
    table = spec.tensors["table"].data
    seen = np.zeros(spec.tensors["k_pool"].shape[0] * S, dtype=bool).reshape(-1, S)
    for b, n in enumerate(held):
        for p in range(max(0, n - 50), n):
            seen[table[b, p // S], p % S] = True
    names = ["k_scale", "v_scale"] if cache == "i8" else ["k_pool", "v_pool"]
    for i, n in enumerate(names):
        t = spec.tensors[n]
        t.data = np.array(t.data)
        bad = np.where(np.arange(t.data.size).reshape(t.data.shape) % 3 == 0, np.nan, np.inf if i else -np.inf)
        m = seen[:, None, :] if cache == "i8" else seen[:, None, :, None]
        t.data = np.where(m, t.data, bad)
    np.testing.assert_array_equal(run(spec)[1]["o"], want)


def test_scores_far_apart():
    # a later key far above all earlier ones (the reference moves), probabilities that vanish, and scores of tens of thousands
    for std in (10.0, 300.0):
        spec = dg.attend_graph("f32", "f32", [400, 33], HQ=2, HK=1, DK=64, DV=32, S=16, M=25, q_std=std)
        check_attention(spec)


def test_a_pool_beyond_32_bits():
    """Rows whose element offsets pass 2^31 and 2^32, through all three operators (as torch tensors: 8 GiB a pool)."""
    import torch

    from paper_2108_13342_amd import api

    HK, S, D = 4, 64, 128
    P = (1 << 32) // (HK * S * D) + 40
    dev = torch.device("cuda:0")
    k, v = (torch.zeros((P, HK, S, D), dtype=torch.float16, device=dev) for _ in range(2))
    table = torch.tensor([[P - 1, 7, P - 2, P // 2 + 3]], dtype=torch.int32, device=dev)
    T = 4 * S - 5
    gen = torch.Generator(device=dev).manual_seed(3)
    fresh = [torch.randn((1, T, HK, D), generator=gen, device=dev).half() for _ in range(2)]
    q = torch.randn((1, HK, D), generator=gen, device=dev).half()
    first, held = torch.zeros(1, dtype=torch.int32, device=dev), torch.full((1,), T, dtype=torch.int32, device=dev)
    out = [torch.empty((1, T, HK, D), dtype=torch.float16, device=dev) for _ in range(2)] + [torch.empty((1, HK, D), dtype=torch.float16, device=dev)]
    g = api.Graph()
    tin = [k, v, *fresh, table, first, held, q]
    ids = [g.add_tensor(f"i{n}", {torch.float16: "f16", torch.int32: "i32"}[t.dtype], t.shape, "input") for n, t in enumerate(tin)]
    outs = [g.add_tensor(f"o{n}", "f16", t.shape, "output") for n, t in enumerate([k, v] + out)]
    g.add_op("CacheWrite", ids[:6], outs[:2])
    g.add_op("CacheRead", outs[:2] + [ids[4], ids[6]], outs[2:4], {"length": T})
    g.add_op("CacheAttention", [ids[7]] + outs[:2] + [ids[4], ids[6]], outs[4:5])
    g.finalize()
    stream = torch.cuda.current_stream().cuda_stream
    plan = api.Plan(g, [], stream=stream)
    ws = torch.empty(max(plan.workspace_bytes(), 256), dtype=torch.uint8, device=dev)
    plan.prepare(ws.data_ptr(), stream)
    plan.run([t.data_ptr() for t in tin], [t.data_ptr() for t in [k, v] + out], ws.data_ptr(), stream)
    torch.cuda.synchronize()
    assert torch.equal(out[0], fresh[0]) and torch.equal(out[1], fresh[1])
    s = (fresh[0][0].double() * q.double()).sum(-1) / D ** 0.5
    want = (torch.softmax(s, 0)[..., None] * fresh[1][0].double()).sum(0)
    assert (out[2][0].double() - want).abs().max() <= 4e-3      # |v| <= 5: two roundings of 2^-11 of the probabilities, sums and result below that


# ------------------------------------------------------------------------------------------------ MatMulInt4
def check_int4(spec, **kw):
    """|y - y64| <= u |y64| + 2^-24 (K + 16) sum_k |x_k| 62 s: u the rounding of the result (and, where every operator is a kernel of
    its own, that of the product), and fp32 sums over K of terms up to |x| (16 + 15 and, for the zero point, 16 + 15) s."""
    _, got = run(spec, **kw)
    env = run_graph(spec, keep="all")
    x, s = data(spec, "x"), data(spec, "s")
    K = x.shape[-1]
    terms = np.abs(x) @ np.repeat(s, spec.ops[0].attrs["group_size"], axis=1)[:, :K].T
    for n, y in got.items():
        rounded = np.abs(env[n]) + (np.abs(env[spec.ops[0].outputs[0]]) if kw.get("fusion") == 0 and len(spec.ops) > 1 else 0.0)
        off = np.abs(y - env[n]) - (dg.HALF_STEP[spec.dtype] * rounded * (1 + 2.0 ** -7) + 2.0 ** -24 * (K + 16) * 62 * terms)
        assert np.all(off <= 0), f"{n}: {off.max():.3e} over its bound"


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,K,N,G,zeros", [(1, 1, 1, 32, False), (1, 31, 5, 32, True), (1, 128, 16, 128, False), (1, 129, 33, 64, True), (1, 768, 2304, 64, False),
                                           (3, 96, 40, 96, True), (16, 256, 64, 256, True), (17, 200, 100, 32, False), (33, 321, 47, 96, True),
                                           (64, 1024, 130, 128, True), (65, 130, 70, 64, True), (150, 64, 1100, 32, False), (2, 4000, 24, 4096, True),
                                           (5, 2049, 9000, 128, True)])
def test_int4(dtype, M, K, N, G, zeros):
    check_int4(dg.int4_graph(dtype, (M,), K, N, G, zeros))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,K,N,G", [(1, 160, 40, 32), (2, 320, 37, 64), (6, 480, 33, 96), (9, 1000, 70, 160), (5, 1344, 48, 192), (16, 224, 10300, 32), (16, 416, 10300, 96),
                                     (6, 192, 5200, 64)])
@pytest.mark.parametrize("zeros", [False, True])
def test_int4_groups_that_fill_no_chunk(dtype, M, K, N, G, zeros):
    check_int4(dg.int4_graph(dtype, (M,), K, N, G, zeros))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,K,N,G", [(1, 8320, 41, 128), (2, 8801, 24, 96), (20, 10947, 151, 128), (5, 16400, 17, 64), (1, 70000, 1, 32), (130, 8330, 100, 160)])
def test_int4_long_contractions_into_few_columns(dtype, M, K, N, G):
    check_int4(dg.int4_graph(dtype, (M,), K, N, G, True, bias=True))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lead", [(1, 1), (2, 3), (2, 2, 5)])
def test_int4_with_what_follows_it(dtype, lead):
    check_int4(dg.int4_graph(dtype, lead, 160, 72, 32, True, bias=True))
    check_int4(dg.int4_graph(dtype, lead, 160, 72, 32, True, bias=True), fusion=0)


def test_every_code_and_zero_point():
    """Each of the 16 codes against each of the 16 zero points, exactly: x of ones and twos, a scale of one half."""
    for dtype in ("f32", "f16", "bf16"):
        spec = dg.int4_graph(dtype, (2,), 32, 256, 32, True)
        n = np.arange(256)
        spec.tensors["w"].data = np.repeat(((n % 16) * 17)[:, None], 16, axis=1)
        spec.tensors["z"].data = (n // 16)[:, None]
        spec.tensors["s"].data = np.full((256, 1), 0.5)
        spec.tensors["x"].data = np.stack([np.eye(32)[3], 2 * np.eye(32)[30]])
        want = np.stack([(n % 16 - n // 16) * 0.5, (n % 16 - n // 16) * 1.0])
        _, got = run(spec)
        np.testing.assert_array_equal(next(iter(got.values())), want)


def test_int4_large_and_tiny_activations():
    spec = dg.int4_graph("f32", (2,), 96, 50, 32)
    for scale in (1e-30, 1e30):
        spec.tensors["x"].data = dg.normal(4, 1, (2, 96), "f32") * np.float32(scale)
        check_int4(spec)


# ------------------------------------------------------------------------------------------------ together
def rounded_graph(spec):
    """The oracle with every operator's result rounded to its storage type."""
    from oracle.interp import eval_op
    from workloads import rng

    env = {t.name: np.asarray(t.data).astype(np.int64 if t.dtype[0] in "iu" else np.float64) for t in spec.tensors.values() if t.data is not None}
    for op in spec.ops:
        res = eval_op(op.kind, [env[i] for i in op.inputs], op.attrs)
        for n, v in zip(op.outputs, res if isinstance(res, (list, tuple)) else [res]):
            d = spec.tensors[n].dtype
            env[n] = rng.round_to(np.asarray(v, dtype=np.float64), d).astype(np.float64) if d in dg.HALF_STEP else np.asarray(v, dtype=np.float64)
    return env


@pytest.mark.parametrize("cache", ["bf16", "i8"])
@pytest.mark.parametrize("fusion", [0, 1])
def test_decode_step_of_a_stack(cache, fusion):
    """One step of a two-layer decoder stack against the oracle.  The storage roundings of the operators' results alone (the oracle
    with them, against the oracle) move the logits by 1.9e-2 of their size and the new rows by up to 6e-3; the executor rounds at the
    same places, or at fewer, other values than these: twice that distance.  A row of 8 bits moves by whole steps."""
    from parity import rel_err
    from workloads import configs

    spec = configs.gpt2_decode_step(**configs.SMALL_EXTRA["gpt2_decode_step"], cache=cache)
    want, near = run_graph(spec), rounded_graph(spec)
    _, got = run(spec, fusion=fusion)
    for n, w in want.items():
        if cache == "i8" and n.endswith(("k_new", "v_new")):
            scale = n.replace("_new", "_scale_new")
            x, y, z = (e[n] * e[scale][..., None] for e in (got, want, near))
            assert np.all(np.abs(x - y) <= 2 * np.abs(z - y).max() + want[scale][..., None]), n
        else:
            assert rel_err(got[n], w) <= 2 * rel_err(near[n], w), n


@pytest.mark.parametrize("cache", ["f16", "i8"])
def test_tokens_generated_one_by_one(cache):
    """A cache filled token by token gives what one filled at once gives, bit for bit, and each step attends over what is there."""
    import torch

    from paper_2108_13342_amd import api

    T, HK, HQ, D, S, M, B = 37, 2, 4, 64, 8, 5, 2
    whole = dg.write_graph("f16", cache, T, [0, 0], HK=HK, DK=D, DV=D, S=S, M=M)
    _, once = run(whole)
    k, v = (np.asarray(whole.tensors[n].data) for n in "kv")

    # one graph for a step: write the token, attend over all up to it
    spec = dg.write_graph("f16", cache, 1, [0, 0], HK=HK, DK=D, DV=D, S=S, M=M, k=k[:, :1], v=v[:, :1])
    b = dg.GraphBuilder("step", "f16")
    b.g = spec
    q = b.input("q", (B, HQ, D), dg.normal(9, 1, (B, HQ, D), "f16"))
    kept = list(spec.ops[0].outputs)
    held = b.input("held", (B,), np.array([1, 1]), dtype="i32")
    b.g.ops.append(dg.OpSpec("CacheAttention", [q] + kept + ["table", held], [b._add("o", "f16", (B, HQ, D), "output")]))
    s = api.Session(spec, guard_bytes=256)
    at = {t.name: s.inputs[0][i] for i, t in enumerate(t for t in spec.tensors.values() if t.kind == "input")}
    for t in range(T):
        at["k"].copy_(torch.from_numpy(k[:, t:t + 1]))
        at["v"].copy_(torch.from_numpy(v[:, t:t + 1]))
        at["first"].fill_(t)
        at["held"].fill_(t + 1)
        s.run()
        if t in (0, 7, 8, T - 1):
            got = s.result()
            now = dg.attend_graph("f16", cache, [t + 1] * B, HQ, HK, D, D, S, M, attrs={}, P=spec.tensors["k_pool"].shape[0])
            for n in kept:
                now.tensors[n.replace("_new", "")].data = got[n]
            now.tensors["q"].data, now.tensors["table"].data = spec.tensors["q"].data, spec.tensors["table"].data
            check_attention(now, {"o": got["o"]})
    got = s.result()
    assert s.guards_intact()
    for n, w in once.items():
        np.testing.assert_array_equal(got[n], w, err_msg=n)


def test_on_another_stream_and_replayed():
    """A step recorded into a graph and replayed, with eager work between the replays, gives the eager results every time; the
    buffers' new contents count."""
    import torch

    from paper_2108_13342_amd import api

    spec = dg.attend_graph("bf16", "bf16", [3000, 40], HQ=4, HK=1, S=16, M=190)
    s = api.Session(spec)
    bound = s.plan.bind(s.in_ptrs(), s.out_ptrs(), s.workspace.data_ptr())
    at = {t.name: s.inputs[0][i] for i, t in enumerate(t for t in spec.tensors.values() if t.kind == "input")}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        bound.run(side.cuda_stream)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            bound.run(torch.cuda.current_stream().cuda_stream)
    for i, held in enumerate(([3000, 40], [1, 3040], [0, 2999], [777, 778])):
        at["held"].copy_(torch.tensor(held, dtype=torch.int32))
        at["q"].mul_(1.25)
        s.outputs[0][0].fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        replayed = s.outputs[0][0].clone()
        s.outputs[0][0].fill_(float("nan"))
        bound.run(torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(replayed, s.outputs[0][0]), f"replay {i}"
        assert torch.isfinite(replayed.float()).all()


def test_two_runs_are_alike_bit_for_bit():
    for spec in (dg.attend_graph("bf16", "i8", [2500, 900], HQ=8, HK=1, S=16, M=160), dg.int4_graph("f16", (3,), 1500, 200, 64, True)):
        s, got = run(spec)
        for _ in range(3):
            s.run()
            again = s.result()
            for n in got:
                np.testing.assert_array_equal(got[n], again[n])


def test_a_cached_prefix_continued_by_ordinary_products():
    """A chunk of new tokens written behind a cached prefix, everything read back, and attended over with MatMul - Softmax - MatMul
    (as one streaming block and as separate kernels)."""
    from parity import TOL, rel_err

    for attention in (0, 1):
        spec = dg.write_graph("f16", "i8", 16, [48, 48], HK=2, DK=64, DV=64, S=16, M=4)
        b = dg.GraphBuilder("prefix", "f16")
        b.g = spec
        kept = list(spec.ops[0].outputs)
        held = b.input("held", (2,), np.array([64, 64]), dtype="i32")
        k, v = (b._add(n, "f16", (2, 64, 2, 64), "intermediate") for n in ("k_all", "v_all"))
        b.g.ops.append(dg.OpSpec("CacheRead", kept + ["table", held], [k, v], {"length": 64}))
        q = b.input("q", (2, 2, 16, 64), dg.normal(9, 1, (2, 2, 16, 64), "f16"))
        kt = b.op("Transpose", [k], (2, 2, 64, 64), {"perm": [0, 2, 3, 1]})
        vt = b.op("Transpose", [v], (2, 2, 64, 64), {"perm": [0, 2, 1, 3]})
        s = b.op("Mul", [b.op("MatMul", [q, kt], (2, 2, 16, 64)), b.const("scale", 0.125)], (2, 2, 16, 64))
        mask = np.where(np.arange(64)[None, :] <= 48 + np.arange(16)[:, None], 0.0, -10000.0)
        s = b.op("Add", [s, b.input("mask", (16, 64), dg.rng.round_to(mask, "f16"))], (2, 2, 16, 64))
        b.mark_output(b.op("MatMul", [b.op("Softmax", [s], (2, 2, 16, 64), {"axis": -1}), vt], (2, 2, 16, 64), out_names=["o"]))
        spec.tensors["o"].kind = "output"
        session, got = run(spec, attention=attention)
        assert any(d["family"] == 6 for d in session.plan.describe()) == bool(attention)
        assert rel_err(got["o"], run_graph(spec)["o"]) <= TOL["f16"]


@pytest.mark.parametrize("how", ["slice", "transpose", "split", "reshape"])
def test_int4_of_a_view(how):
    """x as a part, another order or another shape of what is stored: folded into the addresses, or stored first."""
    b = dg.GraphBuilder("view", "bf16")
    K, N = 96, 40
    if how == "slice":
        x = b.op("Slice", [b.input("in", (7, 2 * K + 3), dg.normal(5, 1, (7, 2 * K + 3), "bf16"))], (5, K), {"starts": [1, 3], "ends": [6, 3 + K], "axes": [0, 1]})
    elif how == "transpose":
        x = b.op("Transpose", [b.input("in", (K, 5), dg.normal(5, 1, (K, 5), "bf16"))], (5, K), {"perm": [1, 0]})
    elif how == "split":
        x = b.op("Split", [b.input("in", (5, 3 * K), dg.normal(5, 1, (5, 3 * K), "bf16"))], [(5, K)] * 3, {"axis": 1, "split": [K] * 3})[1]
    else:
        x = b.op("Reshape", [b.input("in", (5, 4, K // 4), dg.normal(5, 1, (5, 4, K // 4), "bf16"))], (5, K), {"shape": [5, K]})
    w = b.weight("w", (N, K // 2), dg.rng.integers(5, 2, (N, K // 2), 0, 256), dtype="u8")
    s = b.weight("s", (N, K // 32), dg.rng.round_to(dg.rng.uniform(5, 3, (N, K // 32), 0.01, 0.05), "bf16"))
    b.mark_output(b.op("MatMulInt4", [x, w, s], (5, N), {"group_size": 32}))
    spec = b.finish()
    env = run_graph(spec, keep="all")
    terms = np.abs(env[x]) @ np.repeat(data(spec, "s"), 32, axis=1).T
    for kw in ({}, {"fusion": 0}, {"intra_block": 0}):
        _, got = run(spec, **kw)
        for n, y in got.items():
            assert np.all(np.abs(y - env[n]) <= 2.0 ** -8 * np.abs(env[n]) * 1.01 + 2.0 ** -24 * (K + 16) * 62 * terms), (how, kw)


def test_replayed_by_the_plan_itself():
    """The plan option `graphs`: the run loop with an in-place cache becomes a graph on the second run and follows its buffers."""
    import torch

    from paper_2108_13342_amd import api
    from workloads import configs

    spec = configs.gpt2_decode_step(**configs.SMALL_EXTRA["gpt2_decode_step"], cache="i8")
    one, two = api.Session(spec, graphs=0), api.Session(spec, graphs=1)
    ids = [i for i, t in enumerate(t for t in spec.tensors.values() if t.kind == "input") if t.name in ("input_ids", "position", "held")]
    for step in range(5):
        for s in (one, two):
            s.run()
        torch.cuda.synchronize()
        for x, y in zip(one.outputs[0], two.outputs[0]):
            assert torch.equal(x, y), f"step {step}"
        for s in (one, two):
            s.inputs[0][ids[0]].add_(7).remainder_(211)
            for i in ids[1:]:
                s.inputs[0][i].add_(1)


@pytest.mark.parametrize("cache", ["bf16", "i8"])
def test_nothing_held_at_all(cache):
    for M in (1, 60):
        _, got = run(dg.attend_graph("bf16", cache, [0, 0, -1], S=16, M=M))
        assert np.all(got["o"] == 0.0)


def test_steps_of_either_sign():
    """A cache of 8 bits that somebody else filled, with negative steps."""
    spec = dg.attend_graph("f16", "i8", [100, 31], S=16, M=8)
    for n in ("k_scale", "v_scale"):
        t = spec.tensors[n]
        t.data = np.where(np.arange(t.data.size).reshape(t.data.shape) % 3 == 0, -t.data, t.data)
    _, got = run(spec)
    want = run_graph(spec)["o"]
    # |o - o64|: the result's rounding, and fp32 sums (98 roundings a step of sums up to 255 steps, scores to (64 + 8) 2^-24 sum |q k|)
    q, ks, vs = data(spec, "q"), data(spec, "k_scale"), data(spec, "v_scale")
    score = np.abs(q).sum(-1).max() * 127 * np.abs(ks).max() / 8
    assert np.all(np.abs(got["o"] - want) <= 2.0 ** -11 * np.abs(want) * 1.01 + 2.0 ** -24 * (98 * 255 + 127 * (2 * 72 * score + 16 + 128)) * np.abs(vs).max())


def test_in_place_results_take_their_operand_s_buffer():
    from paper_2108_13342_amd import api

    s = api.Session(dg.write_graph("bf16", "bf16", 1, [0, 3]))
    ins, outs = s.in_ptrs(), s.out_ptrs()
    with pytest.raises(api.DnnfError, match="in place"):
        s.plan.run(ins, [outs[0], ins[2]], s.workspace.data_ptr(), s.stream)
    with pytest.raises(api.DnnfError, match="share one buffer"):
        s.plan.run([ins[0], ins[0]] + ins[2:], [ins[0], ins[0]], s.workspace.data_ptr(), s.stream)
    s.plan.run(ins, outs, s.workspace.data_ptr(), s.stream)
    s.result()


def test_static_workspace():
    from paper_2108_13342_amd import api

    spec = dg.attend_graph("bf16", "bf16", [1500, 700], HQ=4, HK=1, S=16, M=100)
    s, got = run(spec)
    s.outputs[0][0].zero_()
    s.plan.run_static(s.in_ptrs(), s.out_ptrs(), s.stream)
    np.testing.assert_array_equal(s.result()["o"], got["o"])


# ------------------------------------------------------------------------------------------------ types on the way
@pytest.mark.parametrize("how", dg.CASTS)
@pytest.mark.parametrize("fusion", [0, 1])
def test_casts_behind_reshapes(how, fusion):
    """Casts that the rewriting merges into a Reshape next to operators of another type: rows of the cache to half a step of
    float16 (the written pools exactly), the other results to parity's bound of 16 bits - bytes read as another type are off by
    the values' own size."""
    from parity import TOL, rel_err

    spec = dg.cast_graph(how)
    _, got = run(spec, fusion=fusion)
    for n, w in run_graph(spec).items():
        if n.endswith("_new"):
            np.testing.assert_array_equal(got[n], w, err_msg=n)
        elif how == "write_and_read":
            assert np.all(np.abs(got[n] - w) <= np.maximum(dg.HALF_STEP["f16"] * np.abs(w), 2.0 ** -25)), n
        else:
            assert rel_err(got[n], w) <= TOL["f16"], n


@pytest.mark.parametrize("graphs", [0, 1])
def test_a_refused_call_leaves_the_caches_alone(graphs):
    """The second layer's pointers are wrong: the first layer's pools are as they were.  The right call still works afterwards."""
    import torch

    from paper_2108_13342_amd import api

    spec = dg.two_caches_graph()
    s = api.Session(spec, graphs=graphs)
    ins, outs = s.in_ptrs(), s.out_ptrs()
    before = [t.clone() for t in s.outputs[0]]
    spare = torch.zeros_like(before[3])
    at = [t.name for t in spec.inputs()].index("v_pool1")
    for i, o in ((ins, outs[:3] + [spare.data_ptr()]), (ins[:at] + [outs[0]] + ins[at + 1:], outs[:3] + [outs[0]])):
        with pytest.raises(api.DnnfError):
            s.plan.run(i, o, s.workspace.data_ptr(), s.stream)
        with pytest.raises(api.DnnfError):
            s.plan.run_static(i, o, s.stream)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(before, s.outputs[0]))
    for _ in range(3):
        s.run()
    got = s.result()
    for n, w in run_graph(spec).items():
        np.testing.assert_array_equal(got[n], w, err_msg=n)


# ------------------------------------------------------------------------------------------------ many pages in one call
@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f32", "i8"), ("bf16", "i8")])
@pytest.mark.parametrize("T,S,M,first,count", [
    (1400, 1, 1500, [0, 150, -9], [1400, 1400, 1400]),                       # the second runs off its table, the third begins before its own
    (1400, 1, 1400, [0, 2147483647, -2147483648], None),
    (2801, 2, 1410, [1, 7, 0], [2801, 0, -3]),
    (2800, 2, 1401, [0, 0, 1], [2147483647, 1, 2800]),
])
def test_write_many_pages(dtype, cache, T, S, M, first, count):
    spec = dg.write_graph(dtype, cache, T, first, count, S=S, M=M, DK=48, DV=16, HK=3)
    s, _ = run(spec)
    assert "owned" in s.plan.describe()[0]["kernel_name"]
    check_written(spec)


@pytest.mark.parametrize("B,T,S,M", [(2, 2200, 1, 2200), (700, 4, 4, 2), (2100, 4, 4, 2), (1400, 1, 16, 1), (40, 30, 1, 30)])
@pytest.mark.parametrize("cache", ["f16", "i8"])
def test_a_slot_written_many_times_keeps_the_last(B, T, S, M, cache):
    """Tables of few pages, so that most slots are written over and over, some entries not there: on both sides of the number of
    pages up to which workgroups look through them, and replayed."""
    P = 60
    table = dg.rng.integers(9, 1, (B, M), -2, P + 2)
    first = dg.rng.integers(9, 2, (B,), -1, 2 * S)
    count = dg.rng.integers(9, 3, (B,), T // 2, T + 2)
    spec = dg.write_graph("f16", cache, T, first, count, S=S, M=M, table=table, P=P, DK=16, DV=32)
    s, got = run(spec)
    want = run_graph(spec)
    for _ in range(3):
        for n, w in want.items():
            np.testing.assert_array_equal(got[n], w, err_msg=n)
        s.run()
        got = s.result()


@pytest.mark.parametrize("T,S,M,first,count", [(1, 300, 1, [0, 299, 150, 300], None), (37, 300, 2, [290, 0, 263, 599], None), (37, 100, 3, [-9, 95, 64, 250], [37, 20, 36, 37]),
                                               (300, 128, 3, [1, 127, 100, 200], [300, 300, 17, 150])])
@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f32", "i8")])
def test_write_into_large_pages(dtype, cache, T, S, M, first, count):
    check_written(dg.write_graph(dtype, cache, T, first, count, S=S, M=M))
    table = np.array([[0] * M, [1] * M, [0] * M, [0] * M])      # and where three sequences share a page
    check_written(dg.write_graph(dtype, cache, T, first, count, S=S, M=M, table=table, P=2))


@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f32", "i8"), ("f16", "i8"), ("bf16", "i8")])
@pytest.mark.parametrize("DK", [64, 80])
def test_queries_with_infinities(dtype, cache, DK):
    """Scores of -infinity alone give zeros, +infinity and NaN among them NaN, and the other heads' results stay as they were."""
    spec = dg.attend_graph(dtype, cache, [150, 40], HQ=6, HK=1, DK=DK, DV=32, S=16, M=10)
    q, k = (np.array(spec.tensors[n].data, dtype=np.float64) for n in ("q", "k_pool"))
    k[..., 3] = np.where(k[..., 3] == 0, 1, np.abs(k[..., 3]))          # channel 3 above zero in all keys, 5 in all but one held one
    k[..., 5] = np.where(k[..., 5] == 0, 1, np.abs(k[..., 5]))
    table = spec.tensors["table"].data
    k[table[0, 4], :, 2, 5] = -1
    k[..., 70 % DK] = np.where(k[..., 70 % DK] == 0, 1, np.abs(k[..., 70 % DK]))
    k[table[0, 4], :, 2, 9] = 0
    spec.tensors["k_pool"].data = k
    spec.tensors["q"].data = q
    want = run(spec)[1]["o"]
    q = np.array(q)
    q[0, 0, 3] = -np.inf                 # -infinity everywhere
    q[0, 1, 5] = -np.inf                 # +infinity once
    q[0, 2, 9] = np.inf                  # infinity times zero once
    q[0, 3, [3, 70 % DK]] = -np.inf      # two channels, of one sign
    q[1, 4, 40] = np.nan
    spec.tensors["q"].data = q
    got = run(spec)[1]["o"]
    assert np.all(got[0, [0, 3]] == 0.0)
    assert np.all(np.isnan(got[0, 1])) and np.all(np.isnan(got[0, 2])) and np.all(np.isnan(got[1, 4]))
    np.testing.assert_array_equal(got[0, 4:], want[0, 4:])
    np.testing.assert_array_equal(got[1, [0, 1, 2, 3, 5]], want[1, [0, 1, 2, 3, 5]])


@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f32", "i8"), ("f16", "i8"), ("bf16", "i8")])
@pytest.mark.parametrize("HQ,HK,DK,DV,S,M,held", [
    (24, 1, 256, 256, 16, 40, [640, 129, 3]),        # more than 64 KiB of LDS to join in, a second half-filled tile of queries
    (28, 4, 256, 128, 20, 7, [140, 77]),
    (48, 3, 128, 256, 8, 20, [160, 0, 33]),
])
def test_attention_of_many_heads_over_wide_channels(dtype, cache, HQ, HK, DK, DV, S, M, held):
    check_attention(dg.attend_graph(dtype, cache, held, HQ, HK, DK, DV, S, M))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_probabilities_keep_their_second_part(dtype):
    """check_attention without the allowance for one rounding of the probabilities: given in two parts, each is off by the square of
    half a step u (float16: or by half of its smallest number, 2^-25, where the row's largest is 1 or more).  Small scores and few keys,
    so that this is what is left; the oracle with probabilities rounded once is outside the bound."""
    u = dg.HALF_STEP[dtype]
    spec = dg.attend_graph(dtype, dtype, [9, 16, 30], HQ=8, HK=2, DK=64, DV=256, S=16, M=2, q_std=0.1)
    q, k, v, table = (data(spec, n) for n in ("q", "k_pool", "v_pool", "table"))
    want, once, bound = (np.zeros((3, 8, 256)) for _ in range(3))
    for b, held in enumerate([9, 16, 30]):
        at = [(int(table[b, p // 16]), p % 16) for p in range(held)]
        for h in range(8):
            kk, vv = (np.stack([x[page, h // 4, slot] for page, slot in at]) for x in (k, v))
            s = kk @ q[b, h] / 8
            p = np.exp(s - s.max())
            rounded = dg.rng.round_to(p, dtype).astype(np.float64)
            want[b, h], once[b, h] = p @ vv / p.sum(), rounded @ vv / p.sum()
            score = np.abs(kk * q[b, h]).sum(-1).max() / 8
            c = u * u + 2.0 ** -24 * (2 * (64 + 8) * score + 16 + held)
            bound[b, h] = u * np.abs(want[b, h]) * (1 + 2.0 ** -8) + c * (p @ np.abs(vv)) / p.sum() + 2.0 ** -25 * np.abs(vv).sum(0)
    np.testing.assert_allclose(run_graph(spec)["o"], want, rtol=1e-9, atol=1e-12)
    assert np.mean(np.abs(once - want) > bound) > 0.05
    off = np.abs(run(spec)[1]["o"] - want) - bound
    assert np.all(off <= 0), f"{off.max():.3e} over its bound"


def test_many_pages_captured_and_replayed():
    """The write of many pages in a captured graph: what a replay leaves depends on the buffers' contents at that time alone, not
    on what earlier calls left in the workspace; eager work and other contents between the replays."""
    import torch

    from paper_2108_13342_amd import api

    B, T, S, M, P = 2100, 2, 4, 2, 50
    spec = dg.write_graph("f16", "i8", T, np.zeros(B, dtype=np.int64), S=S, M=M, table=np.zeros((B, M), dtype=np.int64), P=P, DK=16, DV=16, HK=1)
    s = api.Session(spec)
    bound = s.plan.bind(s.in_ptrs(), s.out_ptrs(), s.workspace.data_ptr())
    at = {t.name: s.inputs[0][i] for i, t in enumerate(spec.inputs())}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        bound.run(side.cuda_stream)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            bound.run(torch.cuda.current_stream().cuda_stream)
    for step in range(4):
        spec.tensors["table"].data = dg.rng.integers(step, 1, (B, M), -1, P)
        spec.tensors["first"].data = dg.rng.integers(step, 2, (B,), 0, 7)
        for n in ("table", "first"):
            at[n].copy_(torch.from_numpy(spec.tensors[n].data))
        s.workspace.random_(0, 256)
        for n in [t.name for t in spec.inputs() if "pool" in t.name or "scale" in t.name]:
            at[n].copy_(torch.from_numpy(np.asarray(spec.tensors[n].data)))
        graph.replay()
        torch.cuda.synchronize()
        for n, w in run_graph(spec).items():
            np.testing.assert_array_equal(s.result()[n], w, err_msg=f"{n}, replay {step}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_steps_below_the_normal_numbers(dtype):
    """A cache of 8 bits that somebody else filled, some values' steps zero or below 2^-126, alone among their neighbours or not: such
    rows are within 127 * 2^-126 of zero, and so is what they add."""
    spec = dg.attend_graph(dtype, "i8", [100, 31, 64], S=16, M=8)
    t, table = spec.tensors["v_scale"], spec.tensors["table"].data
    t.data = np.array(t.data)
    t.data[table[0, 2]] = 1e-40
    t.data[table[0, 4], :, 3] = 2.0 ** -149
    t.data[table[1, :]] = 1e-39
    t.data[table[2, :2]] = 0.0
    _, got = run(spec)
    assert np.all(np.abs(got["o"][1]) <= 127 * 2.0 ** -126)
    assert np.all(np.isfinite(got["o"]))
    check_attention(spec, got)


@pytest.mark.parametrize("how", ["held_computed", "table_gathered", "q_transposed", "all_weights", "residual", "weights_only", "weights_only_split"])
@pytest.mark.parametrize("fusion", [0, 1])
def test_operands_that_other_operators_make(how, fusion):
    """Positions, tables and queries that the graph computes, and products and attention over weights alone (computed at prepare)."""
    b = dg.GraphBuilder(how, "bf16")
    if how in ("residual", "weights_only", "weights_only_split"):
        K, N = (16384 if how == "weights_only_split" else 96), 96
        x = (b.input if how == "residual" else b.weight)("x", (5, K), dg.normal(5, 1, (5, K), "bf16"))
        w = b.weight("w", (N, K // 2), dg.rng.integers(5, 2, (N, K // 2), 0, 256), dtype="u8")
        s = b.weight("s", (N, K // 32), dg.rng.round_to(dg.rng.uniform(5, 3, (N, K // 32), 0.01, 0.05), "bf16"))
        y = b.op("MatMulInt4", [x, w, s], (5, N), {"group_size": 32})
        y = b.op("Add", [y, x if how == "residual" else b.input("r", (5, N), dg.normal(5, 4, (5, N), "bf16"))], (5, N))
    else:
        b.g = dg.attend_graph("bf16", "bf16", [9, 40, 77])
        op, y = b.g.ops.pop(), "o"
        if how == "held_computed":
            del b.g.tensors["held"]
            op.inputs[-1] = b.op("Add", [b.input("first", (3,), np.array([8, 39, 76]), dtype="i32"), b.const("one", 1, dtype="i32")], (3,), out_dtype="i32")
        elif how == "table_gathered":
            t = b.g.tensors.pop("table").data
            who = b.input("who", (3,), np.array([4, 1, 2]), dtype="i64")
            op.inputs[-2] = b.op("Gather", [b.input("tables", (5, 8), np.concatenate([t, t[:2]]), dtype="i32"), who], (3, 8), {"axis": 0}, out_dtype="i32")
        elif how == "q_transposed":
            del b.g.tensors["q"]
            op.inputs[0] = b.op("Transpose", [b.input("qt", (4, 3, 64), dg.normal(5, 1, (4, 3, 64), "bf16"))], (3, 4, 64), {"perm": [1, 0, 2]})
        else:
            for t in b.g.tensors.values():
                t.kind = "weight" if t.kind == "input" else t.kind
        b.g.ops.append(op)
        b.g.tensors["o"].kind = "intermediate"
        y = b.op("Add", ["o", b.input("r", (3, 4, 64), dg.normal(5, 4, (3, 4, 64), "bf16"))], (3, 4, 64))
    b.mark_output(y)
    spec = b.finish()
    from parity import TOL, rel_err

    _, got = run(spec, fusion=fusion)
    assert rel_err(got[y], run_graph(spec)[y]) <= TOL["bf16"]
