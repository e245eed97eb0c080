"""Cases of the operators of single-token inference: a paged key / value cache that is written, read back and attended
over (`CacheWrite`, `CacheRead`, `CacheAttention`), and products with weights of four bits (`MatMulInt4`).

`run` computes a case in elementary torch operations (`own = False`) or through the framework's plan (`own = True`).
Every size that says how much work a case is (lengths, counts) follows from the case alone; values and the order of the
pages follow from the seed.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "i32": torch.int32, "i8": torch.int8, "u8": torch.uint8}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "i8": 1}
TINY = 2.0 ** -119       # a row whose largest magnitude lies below is kept as zeros


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # one new token of four conversations written into the cache: all latency
        dict(name="write_bf16_token", op="write", dtype="bf16", cache="bf16", B=4, T=1, start=1000, HK=12, D=64, S=16),
        # the keys and values of four prompts of unequal length, written by the pass that reads the prompts
        dict(name="write_bf16_prompt", op="write", dtype="bf16", cache="bf16", B=4, T=1024, start=0, HK=12, D=64, S=16),
        # a cached prefix read back so that a prompt's continuation can attend over it with the ordinary products
        dict(name="read_f16_prefix", op="read", dtype="f16", cache="f16", B=8, L=2048, HK=8, D=128, S=64),
        # the same through a cache of 8 bits, stored and read back: one new chunk of a prompt, and long prompts
        dict(name="pack_i8_chunk", op="pack", dtype="bf16", cache="i8", B=2, T=37, start=75, HK=12, D=64, S=16),
        dict(name="pack_i8_prompt", op="pack", dtype="f16", cache="i8", B=8, T=2048, start=0, HK=8, D=128, S=64),
        # one new token against the cache: a single conversation, a batch of unequal ones with shared key heads, one very
        # long document, and a large batch over a cache of 8 bits
        dict(name="attend_bf16_one", op="attend", dtype="bf16", cache="bf16", B=1, L=1024, HQ=12, HK=12, D=64, S=16),
        dict(name="attend_f16_batch", op="attend", dtype="f16", cache="f16", B=16, L=4001, HQ=32, HK=8, D=128, S=16),
        dict(name="attend_bf16_long", op="attend", dtype="bf16", cache="bf16", B=1, L=131072, HQ=32, HK=8, D=128, S=64),
        dict(name="attend_i8_batch", op="attend", dtype="bf16", cache="i8", B=64, L=2048, HQ=32, HK=8, D=128, S=32),
        # products of single tokens with 4-bit weights: a small layer, a large one, and the vocabulary for a batch of 16
        dict(name="int4_f16_qkv", op="int4", dtype="f16", M=1, K=768, N=2304, G=64, zeros=False),
        dict(name="int4_bf16_wide", op="int4", dtype="bf16", M=1, K=4096, N=11008, G=128, zeros=True),
        dict(name="int4_bf16_vocabulary", op="int4", dtype="bf16", M=16, K=768, N=50257, G=128, zeros=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "read", "pack", "attend", "attend", "int4", "int4"])
    dtype = rng.choice(["f16", "bf16", "f16", "bf16", "f32"])
    if op == "int4":
        K, M = _log(rng, 64, 11008), _log(rng, 1, 64)
        if rng.random() < 0.6:
            K = (K + 63) // 64 * 64
        N = _log(rng, 64, min(50257, 45_000_000 // K))
        return dict(op=op, dtype=dtype, M=M, K=K, N=N, G=rng.choice([32, 64, 96, 128, 256]), zeros=rng.random() < 0.5)
    HK, share = rng.choice([(12, 1), (16, 1), (8, 4), (4, 7), (2, 8), (1, 24), (8, 1), (5, 2)])
    D, S = rng.choice([32, 48, 64, 80, 96, 128, 128, 256]), rng.choice([1, 8, 16, 16, 20, 32, 64, 100])
    c = dict(op=op, dtype=dtype, cache=dtype, HK=HK, D=D, S=S)
    if op == "attend":
        most = 250_000_000 // (2 * HK * D * BYTES[dtype])          # keys of all sequences together
        L = _log(rng, 1, min(131072, most))
        c.update(B=_log(rng, 1, max(1, min(128, most // L))), L=L, HQ=HK * share, cache=rng.choice([dtype, "i8"]))
        if rng.random() < 0.2:
            c["window"] = _log(rng, 1, 4096)
        return c
    most = 40_000_000 // (2 * HK * D * BYTES[dtype])
    T = _log(rng, 1, min(4096, most))
    B = _log(rng, 1, max(1, min(64, most // T)))
    if op == "read":
        c.update(B=B, L=T)
    else:
        c.update(B=B, T=T, start=rng.choice([0, rng.randint(1, 300)]))
        if op == "pack":
            c["cache"] = "i8"
    return c


def _spread(n, top, low):
    """n sequence lengths between low and top, unequal, the first one top."""
    return [low + int((top - low) * (1.0 - (k * 0.6180339887498949) % 1.0)) for k in range(n)]


def _sizes(c):
    """(first written position, tokens written, keys held) of every sequence, and the pages of a table row."""
    if c["op"] in ("write", "pack"):
        first, count = _spread(c["B"], c["start"], (c["start"] + 1) // 2), _spread(c["B"], c["T"], (c["T"] + 1) // 2)
        held = [f + n for f, n in zip(first, count)]
    else:
        first, count, held = [], [], _spread(c["B"], c["L"], (c["L"] + 3) // 4)
    return first, count, held, (max(held) + c["S"] - 1) // c["S"]


def work(case):
    c = case
    if c["op"] == "int4":
        M, K, N, e = c["M"], c["K"], c["N"], BYTES[c["dtype"]]
        groups = -(-K // c["G"])
        return {"bytes": M * K * e + N * ((K + 1) // 2) + N * groups * (e + int(c["zeros"])) + M * N * e, "flops": 2.0 * M * K * N}
    first, count, held, pages = _sizes(c)
    row, kept = 2 * c["HK"] * c["D"] * BYTES[c["dtype"]], 2 * c["HK"] * (c["D"] * BYTES[c["cache"]] + (4 if c["cache"] == "i8" else 0))
    if c["op"] == "write":
        return {"bytes": sum(count) * (row + kept) + c["B"] * 8, "flops": 0.0}
    if c["op"] == "pack":          # written, and everything held read back and laid out in full
        return {"bytes": sum(count) * (row + kept) + sum(held) * kept + c["B"] * (c["start"] + c["T"]) * row, "flops": 0.0}
    if c["op"] == "read":
        return {"bytes": sum(held) * kept + c["B"] * c["L"] * row, "flops": 0.0}
    seen = sum(min(n, c.get("window", n)) for n in held)
    return {"bytes": seen * kept + 2 * c["B"] * c["HQ"] * c["D"] * BYTES[c["dtype"]], "flops": 4.0 * seen * c["HQ"] * c["D"]}


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    c, dev = case, torch.device("cuda:0")
    gen = torch.Generator(device=dev).manual_seed(seed)
    t = TYPES[c["dtype"]]

    def normal(*shape, std=1.0, dtype=t):
        return (torch.randn(shape, generator=gen, device=dev, dtype=torch.float32) * std).to(dtype)

    s = {"case": c}
    if c["op"] == "int4":
        groups = -(-c["K"] // c["G"])
        s["x"] = normal(c["M"], c["K"])
        s["w"] = torch.randint(0, 256, (c["N"], (c["K"] + 1) // 2), generator=gen, device=dev, dtype=torch.uint8)
        # steps of a weight of standard deviation 0.02 that was cut into sixteen
        s["scale"] = (torch.rand((c["N"], groups), generator=gen, device=dev) * 0.006 + 0.004).to(t)
        if c["zeros"]:
            s["zero"] = torch.randint(5, 11, (c["N"], groups), generator=gen, device=dev, dtype=torch.uint8)
        s["y"] = torch.empty((c["M"], c["N"]), dtype=t, device=dev)
    else:
        first, count, held, pages = _sizes(c)
        B, HK, D, S = c["B"], c["HK"], c["D"], c["S"]
        P = B * pages + 3
        s["table"] = torch.randperm(P, generator=gen, device=dev)[:B * pages].reshape(B, pages).to(torch.int32)
        for n in ("k", "v"):
            if c["cache"] == "i8":
                s[n + "_pool"] = torch.randint(-127, 128, (P, HK, S, D), generator=gen, device=dev, dtype=torch.int8)
                s[n + "_scale"] = torch.rand((P, HK, S), generator=gen, device=dev) * 0.02 + 0.005
            else:
                s[n + "_pool"] = normal(P, HK, S, D)
        if first:
            s["first"], s["count"] = torch.tensor(first, dtype=torch.int32, device=dev), torch.tensor(count, dtype=torch.int32, device=dev)
            s["k"], s["v"] = normal(B, c["T"], HK, D), normal(B, c["T"], HK, D)
        if c["op"] != "write":
            s["held"] = torch.tensor(held, dtype=torch.int32, device=dev)
        if c["op"] == "attend":
            s["q"] = normal(B, c["HQ"], D)
            s["o"] = torch.empty((B, c["HQ"], D), dtype=t, device=dev)
        elif c["op"] != "write":
            L = c["L"] if c["op"] == "read" else c["start"] + c["T"]
            s["k_out"], s["v_out"] = (torch.empty((B, L, HK, D), dtype=t, device=dev) for _ in range(2))
    if own:
        s["plan"], s["bound"], s["workspace"] = _plan(s)
    return s


def _plan(s):
    """The case as an operator graph of the framework, planned, and bound to the state's buffers."""
    from paper_2108_13342_amd import api
    from paper_2108_13342_amd.build import CACHE

    c = s["case"]
    names = {torch.float32: "f32", torch.float16: "f16", torch.bfloat16: "bf16", torch.int32: "i32", torch.int8: "i8", torch.uint8: "u8"}
    g, ptrs = api.Graph(), {"input": [], "weight": [], "output": []}

    def tensor(name, kind, like=None):
        t = s[like or name]
        ptrs[kind].append(t.data_ptr())
        return g.add_tensor(name, names[t.dtype], t.shape, kind)

    if c["op"] == "int4":
        ins = [tensor("x", "input"), tensor("w", "weight"), tensor("scale", "weight")] + ([tensor("zero", "weight")] if c["zeros"] else [])
        g.add_op("MatMulInt4", ins, [tensor("y", "output")], {"group_size": c["G"]})
    else:
        pool_names = ["k_pool", "v_pool"] + (["k_scale", "v_scale"] if c["cache"] == "i8" else [])
        pools, table = [tensor(n, "input") for n in pool_names], tensor("table", "input")
        if c["op"] in ("write", "pack"):
            new = [tensor(n, "input") for n in ("k", "v")]
            at = [tensor(n, "input") for n in ("first", "count")]
            written = [tensor(n + "_new", "output", n) for n in pool_names]      # the pools are updated in place
            g.add_op("CacheWrite", pools + new + [table] + at, written)
            pools = written
        if c["op"] in ("read", "pack"):
            outs = [tensor("k_out", "output"), tensor("v_out", "output")]
            g.add_op("CacheRead", pools + [table, tensor("held", "input")], outs, {"length": s["k_out"].shape[1]})
        if c["op"] == "attend":
            attrs = {"window": c["window"]} if "window" in c else {}
            g.add_op("CacheAttention", [tensor("q", "input")] + pools + [table, tensor("held", "input")], [tensor("o", "output")], attrs)
    g.finalize()
    stream = torch.cuda.current_stream().cuda_stream
    plan = api.Plan(g, ptrs["weight"], stream=stream, cache_dir=CACHE)
    workspace = torch.empty(max(plan.workspace_bytes(), 256), dtype=torch.uint8, device="cuda:0")
    plan.prepare(workspace.data_ptr(), stream)
    return plan, plan.bind(ptrs["input"], ptrs["output"], workspace.data_ptr()), workspace


def _outputs(s):
    op = s["case"]["op"]
    if op == "int4":
        return s["y"]
    if op == "attend":
        return s["o"]
    if op == "write":
        return {"k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    if op == "read":
        return {"k": s["k_out"], "v": s["v_out"]}
    return {"k": s["k_out"], "v": s["v_out"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    s = state
    if own:
        s["bound"].run(torch.cuda.current_stream().cuda_stream)
        return _outputs(s)
    op = s["case"]["op"]
    if op == "int4":
        return _plain_int4(s)
    if op == "attend":
        return _plain_attend(s)
    if op in ("write", "pack"):
        _plain_write(s)
    if op in ("read", "pack"):
        s["k_out"], s["v_out"] = _plain_read(s, "k"), _plain_read(s, "v")
    return _outputs(s)


def _plain_int4(s):
    c = s["case"]
    codes = torch.stack((s["w"] & 15, s["w"] >> 4), dim=-1).reshape(c["N"], -1)[:, :c["K"]].float()
    spread = lambda t: t.float().repeat_interleave(c["G"], dim=1)[:, :c["K"]]  # noqa: E731
    w = (codes - (spread(s["zero"]) if c["zeros"] else 8.0)) * spread(s["scale"])
    return (s["x"].float() @ w.t()).to(s["x"].dtype)


def _plain_write(s):
    c = s["case"]
    t = torch.arange(c["T"], device="cuda:0")
    valid = t[None, :] < s["count"][:, None]
    at = torch.where(valid, s["first"][:, None] + t[None, :], s["first"][:, None]).long()      # a row behind the count repeats the first
    page, slot = s["table"].gather(1, at // c["S"]).long(), at % c["S"]
    for n in ("k", "v"):
        x = torch.where(valid[:, :, None, None], s[n], s[n][:, :1])
        if c["cache"] == "i8":
            x = x.float()
            top = x.abs().amax(-1)
            scale = torch.where(top < TINY, torch.zeros_like(top), top / 127.0)
            x = torch.where(scale[..., None] > 0, torch.round(x / scale[..., None]), torch.zeros_like(x)).clamp(-127, 127).to(torch.int8)
            s[n + "_scale"][page, :, slot] = scale
        s[n + "_pool"][page, :, slot] = x


def _plain_read(s, n):
    c, L = s["case"], s[n + "_out"].shape[1]
    x = s[n + "_pool"][s["table"].long()]                                                       # [B, pages, HK, S, D]
    if c["cache"] == "i8":
        x = x.float() * s[n + "_scale"][s["table"].long()][..., None]
    x = x.transpose(2, 3).reshape(c["B"], -1, c["HK"], c["D"])
    x = torch.cat((x, x.new_zeros((c["B"], max(0, L - x.shape[1]), c["HK"], c["D"]))), 1)[:, :L]
    t = torch.arange(L, device="cuda:0")
    return torch.where(t[None, :, None, None] < s["held"][:, None, None, None], x, torch.zeros_like(x)).to(s[n + "_out"].dtype)


def _plain_attend(s):
    c = s["case"]
    B, HK, D = c["B"], c["HK"], c["D"]

    def gathered(n):
        x = s[n + "_pool"][s["table"].long()].float()
        if c["cache"] == "i8":
            x = x * s[n + "_scale"][s["table"].long()][..., None]
        return x.transpose(1, 2).reshape(B, HK, -1, D)

    k, v = gathered("k"), gathered("v")
    q = s["q"].float().reshape(B, HK, -1, D)
    score = torch.matmul(k, q.transpose(2, 3).contiguous()) / math.sqrt(D)                      # [B, HK, keys, queries of a key head]
    t, held = torch.arange(k.shape[2], device="cuda:0"), s["held"][:, None]
    seen = (t[None, :] < held) & (t[None, :] >= held - c.get("window", 1 << 30))
    score = torch.where(seen[:, None, :, None], score, torch.full_like(score, -math.inf))
    p = torch.exp(score - score.amax(2, keepdim=True))
    p = p / p.sum(2, keepdim=True)
    return torch.matmul(p.transpose(2, 3).contiguous(), v).reshape(B, c["HQ"], D).to(s["q"].dtype)


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "int4":
        k = torch.arange(c["K"], device="cuda:0")
        code = (s["w"][:, k // 2].to(torch.int32) >> (4 * (k % 2)).to(torch.int32)) & 15
        zero = s["zero"][:, k // c["G"]].double() if c["zeros"] else torch.tensor(8.0, dtype=torch.float64, device="cuda:0")
        return torch.matmul(s["x"].double(), ((code.double() - zero) * s["scale"][:, k // c["G"]].double()).t().contiguous())
    first, count, held, pages = _sizes(c)
    table, S = s["table"].long(), c["S"]

    def rows(b, lo, hi):
        p = torch.arange(lo, hi, device="cuda:0")
        return table[b, p // S], p % S

    pool = {n: s[n + "_pool"].double() for n in ("k", "v")} if c["op"] != "attend" else None
    scale = {n: s[n + "_scale"].double() for n in ("k", "v")} if c["cache"] == "i8" else None
    if c["op"] in ("write", "pack"):
        for b in range(c["B"]):
            page, slot = rows(b, first[b], first[b] + count[b])
            for n in ("k", "v"):
                x = s[n][b, :count[b]].double()
                if scale is not None:          # the step is kept in 32 bits; the number of steps is that of the exact quotient
                    step = (x.abs().amax(-1) / 127.0).float().double()
                    scale[n][page, :, slot] = step
                    x = torch.round(x / step[..., None])
                pool[n][page, :, slot] = x
        if c["op"] == "write":
            return {"k_pool": pool["k"], "v_pool": pool["v"]}
    if c["op"] in ("read", "pack"):
        out = {}
        for n in ("k", "v"):
            out[n] = torch.zeros(s[n + "_out"].shape, dtype=torch.float64, device="cuda:0")
            for b in range(c["B"]):
                page, slot = rows(b, 0, held[b])
                out[n][b, :held[b]] = pool[n][page, :, slot] * (scale[n][page, :, slot][..., None] if scale is not None else 1.0)
            if c["op"] == "pack":
                out[n + "_scale"] = scale[n]
        return out
    o = torch.empty((c["B"], c["HQ"], c["D"]), dtype=torch.float64, device="cuda:0")
    share = c["HQ"] // c["HK"]
    for b in range(c["B"]):
        page, slot = rows(b, max(0, held[b] - c.get("window", held[b])), held[b])
        k, v = (s[n + "_pool"][page, :, slot].double() * (scale[n][page, :, slot][..., None] if scale is not None else 1.0) for n in ("k", "v"))
        q = s["q"][b].double().reshape(c["HK"], share, c["D"])
        w = torch.softmax(torch.matmul(q, k.permute(1, 2, 0).contiguous()) / math.sqrt(c["D"]), dim=-1)
        o[b] = torch.matmul(w, v.transpose(0, 1).contiguous()).reshape(c["HQ"], c["D"])
    return o
