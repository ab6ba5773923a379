"""The operators of an attention block trained through the coded step, and how they are measured.

Three operators of `paper_2605_15890_amd.api`: the rotation of queries and keys by their positions (`agc_rotary_apply`),
differential attention with its partial gradients (`agc_diff_attn_forward`, `agc_diff_attn_partial_gradients`) and
dropout with the residual that it is added to (`agc_dropout`).

`run` computes them in their plain form, elementary torch operations in binary32, or through the library.
"""
import math

import torch

own = False   # True: through the library

DEVICE = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
IDS = {"i32": torch.int32, "i64": torch.int64}
# bytes or flops of the largest listed case of each
LARGEST = {"rotary": 1.02e8, "dropout": 8.1e8, "forward": 2.8e11, "train": 4.9e11}
MOST_SCORES = 2.2e9   # values of the padded score tensor that the plain form holds


def listed():
    return [
        # serving: three sequences' new token, queries and keys of a layer side by side, far positions; latency
        dict(name="rotary_token", op="rotary", tokens=3, heads=10, dim=128, rot=128, layout="half", value="bf16",
             ids="i64", scaling="none", factor=1.0, reach=100000, gap=0, inverse=False),
        # a training batch: queries and keys of a buffer that holds the values behind them
        dict(name="rotary_batch", op="rotary", tokens=16384, heads=24, dim=64, rot=64, layout="half", value="bf16",
             ids="i32", scaling="none", factor=1.0, reach=4096, gap=512, inverse=False),
        # gradients of a long context: part of the head, neighbours paired, frequencies scaled by parts, odd sizes
        dict(name="rotary_long", op="rotary", tokens=8191, heads=5, dim=81, rot=56, layout="interleaved", value="f32",
             ids="i64", scaling="parts", factor=16.0, reach=1 << 20, gap=3, inverse=True),
        # a few tokens into their residual
        dict(name="dropout_token", op="dropout", rows=5, cols=1024, value="bf16", sum="bf16", p=0.1, residual=True),
        # a training batch into the residual stream
        dict(name="dropout_batch", op="dropout", rows=65536, cols=2048, value="bf16", sum="bf16", p=0.1, residual=True),
        # the gradient of an odd width
        dict(name="dropout_grad", op="dropout", rows=16383, cols=1501, value="f32", sum="f32", p=0.25, residual=False),
        # serving: one new token each of eight sequences, ragged caches, four query heads to a key head
        dict(name="attn_decode", op="forward", seqs=8, queries=8, keys=131072, ragged=True, heads=16, kv_heads=4, dim=64,
             vdim=128, causal=True, parts=1),
        # one short prompt: latency
        dict(name="attn_prompt", op="forward", seqs=1, queries=37, keys=37, ragged=False, heads=4, kv_heads=4, dim=64,
             vdim=128, causal=True, parts=1),
        # forward pass of a training batch
        dict(name="attn_batch", op="forward", seqs=4, queries=16384, keys=16384, ragged=False, heads=16, kv_heads=4,
             dim=64, vdim=128, causal=True, parts=1),
        # wide heads, ragged sequences, every key in sight
        dict(name="attn_wide", op="forward", seqs=5, queries=8111, keys=8111, ragged=True, heads=8, kv_heads=2, dim=128,
             vdim=256, causal=False, parts=1),
        # a training step: forward, then the partial gradients of eight workers' partitions
        dict(name="attn_train", op="train", seqs=8, queries=16384, keys=16384, ragged=False, heads=16, kv_heads=16, dim=64,
             vdim=128, causal=True, parts=8),
        # a small odd one: ragged, shared key heads, sequences with more queries than keys among them
        dict(name="attn_train_odd", op="train", seqs=6, queries=2999, keys=2501, ragged=True, heads=6, kv_heads=2, dim=40,
             vdim=72, causal=True, parts=5),
    ]


def _between(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm; every third or so a multiple of 64, and the
    lower quarter of the range, where few real sizes lie, half as often as the rest."""
    if rng.random() < 0.5:
        lo = max(lo, round(lo ** 0.75 * hi ** 0.25))
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, v // 64 * 64) if rng.random() < 0.35 and hi >= 128 else v


def draw(rng):
    op = rng.choice(["rotary", "dropout", "forward", "forward", "train"])
    if op == "rotary":
        dim = _between(rng, 2, 256)
        rot = dim // 2 * 2 if rng.random() < 0.6 else 2 * rng.randint(1, dim // 2)
        scaling = rng.choice(["none", "linear", "parts"])
        case = dict(op=op, tokens=_between(rng, 1, 50000), heads=_between(rng, 1, 64), dim=dim, rot=rot,
                    layout=rng.choice(["half", "interleaved"]), value=rng.choice(["bf16", "f32"]),
                    ids=rng.choice(["i32", "i64"]), scaling=scaling,
                    factor=1.0 if scaling == "none" else rng.choice([2.0, 8.0, 32.0]),
                    reach=_between(rng, 1, 1 << 21), gap=rng.choice([0, 0, 1, 8, 128]), inverse=rng.random() < 0.5)
        shrink = ("tokens", "heads")
    elif op == "dropout":
        case = dict(op=op, rows=_between(rng, 1, 200000), cols=_between(rng, 1, 12000), value=rng.choice(["bf16", "f32"]),
                    sum=rng.choice(["bf16", "f32"]), p=rng.choice([0.0, 0.05, 0.1, 0.5, 0.9]), residual=rng.random() < 0.5)
        shrink = ("rows", "cols")
    else:
        kv_heads, group = _between(rng, 1, 8), rng.choice([1, 1, 2, 4, 7])
        dim = rng.choice([16, 32, 64, 64, 80, 128, rng.randint(1, 128)])
        queries = _between(rng, 1, 20000)
        seqs = min(_between(rng, 1, 48), queries)
        way = rng.random()
        keys = queries if way < 0.6 else _between(rng, 1, 100000)
        if way > 0.8 and op == "forward":
            queries = seqs
        case = dict(op=op, seqs=seqs, queries=queries, keys=keys, ragged=rng.random() < 0.6, heads=kv_heads * group,
                    kv_heads=kv_heads, dim=dim, vdim=min(256, 2 * dim if rng.random() < 0.7 else rng.randint(1, 256)),
                    causal=rng.random() < 0.6, parts=_between(rng, 1, 16) if op == "train" else 1)
        shrink = ("queries", "keys")
    while _cost(case) > LARGEST[op] or _scores(case) > MOST_SCORES:
        most = max(shrink, key=lambda f: case[f])
        if case.get("keys") == case.get("queries", 0):
            case["keys"] = case["queries"] = case["queries"] * 2 // 3
        else:
            case[most] = max(1, case[most] * 2 // 3)
        if "seqs" in case:
            case["seqs"] = max(1, min(case["seqs"], case["queries"]))
    return case


def _cost(case):
    w = work(case)
    return w["bytes"] if case["op"] in ("rotary", "dropout") else w["flops"]


def _lengths(case):
    """Queries and keys of every sequence.  Ragged ones differ by a factor of about three, every fifth has neither."""
    def spread(total, shape):
        whole = [int(total * s / sum(shape)) for s in shape]
        whole[0] += total - sum(whole)
        return whole

    n = case["seqs"]
    level = [1.0] * n
    if case["ragged"]:
        level = [0.0 if i % 5 == 3 else 0.5 + (i * 0.6180339887 + 0.3) % 1.0 for i in range(n)]
    queries = [1] * n if case["queries"] == n else spread(case["queries"], level)
    return queries, spread(case["keys"], level)


def _scores(case):
    if case["op"] in ("rotary", "dropout"):
        return 0
    queries, keys = _lengths(case)
    return 2.0 * case["heads"] * case["seqs"] * max(queries) * max(keys)


def work(case):
    if case["op"] == "rotary":
        size = 4 if case["value"] == "f32" else 2
        whole = case["tokens"] * case["heads"] * case["dim"]
        return {"bytes": 2.0 * size * whole + case["tokens"] * (8 if case["ids"] == "i64" else 4),
                "flops": 3.0 * case["tokens"] * case["heads"] * case["rot"]}
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        summed = 4 if case["sum"] == "f32" else 2
        return {"bytes": float(n * ((4 if case["value"] == "f32" else 2) + summed * (2 if case["residual"] else 1))),
                "flops": 2.0 * n}
    pairs = 0
    for lq, lk in zip(*_lengths(case)):
        seen = min(lq, lk)
        # under the causal mask the last query sees all keys, the one before it all but one
        pairs += seen * (lk - seen) + seen * (seen + 1) // 2 if case["causal"] else lq * lk
    h, hk, d, e = case["heads"], case["kv_heads"], case["dim"], case["vdim"]
    read = 2.0 * (case["queries"] * 2 * h * d + case["keys"] * hk * (2 * d + e))
    out = 2.0 * case["queries"] * h * e
    # two maps of scores, one product of their difference with the values
    flops = pairs * h * (4.0 * d + 2.0 * e)
    if case["op"] == "forward":
        return {"bytes": read + out, "flops": flops}
    # scores again, the maps' gradients from the values, and three products for dq, dk and dv
    return {"bytes": 3.0 * read + 3.0 * out + 4.0 * h * case["parts"], "flops": flops + pairs * h * (12.0 * d + 4.0 * e)}


def frequencies(rot, scaling, factor, base=10000.0, original=4096.0):
    """Angles a position turns the pairs by, and the factor of the rotated values."""
    freq = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        return [f / factor for f in freq], 1.0
    if scaling == "parts":
        # pairs that turn less than once over the original length are stretched, those that turn more than 32 times stay
        def at(turns):
            return rot * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))
        low, high = max(0.0, math.floor(at(32.0))), min(rot - 1.0, math.ceil(at(1.0)))
        ramp = [min(1.0, max(0.0, (i - low) / max(high - low, 1e-3))) for i in range(rot // 2)]
        return [f / factor * r + f * (1.0 - r) for f, r in zip(freq, ramp)], 0.1 * math.log(factor) + 1.0
    return freq, 1.0


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    host = torch.Generator().manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device=DEVICE) * std + mean).to(dtype)

    s = dict(case)
    if case["op"] == "rotary":
        width = case["heads"] * case["dim"]
        rows = normal(case["tokens"], width + case["gap"], dtype=TYPES[case["value"]])
        s["x"], s["out"] = rows[:, :width], torch.empty_like(rows)[:, :width]
        start = int(torch.randint(0, max(1, case["reach"] - case["tokens"]), (1,), generator=host))
        s["positions"] = ((torch.arange(case["tokens"], device=DEVICE) + start) % case["reach"]).to(IDS[case["ids"]])
        s["freq"], s["amplitude"] = frequencies(case["rot"], case["scaling"], case["factor"])
        # a position's share of a whole turn in units of 2^-64
        s["turns"] = torch.tensor([_signed(round(f / (2 * math.pi) * 2 ** 64)) for f in s["freq"]], device=DEVICE)
    elif case["op"] == "dropout":
        shape = (case["rows"], case["cols"])
        s["x"] = normal(*shape, dtype=TYPES[case["value"]])
        s["res"] = normal(*shape, dtype=TYPES[case["sum"]]) if case["residual"] else None
        s["out"] = torch.empty(shape, dtype=TYPES[case["sum"]], device=DEVICE)
        s["seed"], s["step"], s["site"] = 0x9E3779B97F4A7C15 ^ seed, 5 + seed, 3
    else:
        bf16 = torch.bfloat16
        h, hk, d, e = case["heads"], case["kv_heads"], case["dim"], case["vdim"]
        # scores of a standard deviation of about 1.5, keys with a part that all of a head share
        s["q"] = normal(case["queries"], 2 * h * d, std=1.5, dtype=bf16)
        s["k"] = (normal(case["keys"], 2 * hk * d) + normal(1, 2 * hk * d, std=0.5)).to(bf16)
        s["v"] = (normal(case["keys"], hk * e) + normal(1, hk * e, std=0.3)).to(bf16)
        s["lam"] = torch.rand(h, generator=g, device=DEVICE) * 0.6 + 0.2
        s["scale"] = d ** -0.5
        s["lq"], s["lk"] = _lengths(case)
        s["q_end"], s["k_end"] = (torch.tensor(n, device=DEVICE).cumsum(0).to(torch.int32) for n in (s["lq"], s["lk"]))
        s["out"] = torch.zeros(case["queries"], h * e, dtype=bf16, device=DEVICE)
        if case["op"] == "train":
            s["dout"] = normal(case["queries"], h * e, std=1e-3, dtype=bf16)
            cuts = torch.randint(0, case["queries"] + 1, (case["parts"] - 1,), generator=host).sort().values.tolist()
            s["part_end"] = cuts + [case["queries"]]
            s["dq"], s["dk"], s["dv"] = (torch.zeros_like(s[n]) for n in ("q", "k", "v"))
            s["lse"] = torch.empty(2 * h, case["queries"], device=DEVICE)
            s["G"] = torch.empty(case["parts"], h, device=DEVICE)
    if own:
        from paper_2605_15890_amd import api
        s["api"] = api
        if case["op"] in ("forward", "train"):
            need = api.agc_diff_attn_workspace_bytes(case["queries"], case["keys"], case["seqs"], case["heads"],
                                                     case["kv_heads"], case["dim"], case["vdim"], case["op"] == "train")
            s["workspace"] = torch.empty(max(256, need), dtype=torch.uint8, device=DEVICE)
    return s


def _signed(word):
    """The 64-bit word as torch holds it."""
    return word - (1 << 64) if word >= 1 << 63 else word


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    api = s["api"]
    if s["op"] == "rotary":
        api.agc_rotary_apply(s["x"], s["heads"], s["positions"], s["turns"], s["layout"], s["out"], amplitude=s["amplitude"],
                             inverse=s["inverse"])
        return {"out": s["out"]}
    if s["op"] == "dropout":
        api.agc_dropout(s["x"], s["p"], s["seed"], s["step"], s["site"], s["out"], residual=s["res"])
        return {"out": s["out"]}
    masks = (s["heads"], s["kv_heads"], s["lam"], s["q_end"], s["k_end"], s["scale"], s["causal"])
    if s["op"] == "forward":
        api.agc_diff_attn_forward(s["q"], s["k"], s["v"], *masks, s["out"], s["workspace"])
        return {"out": s["out"]}
    api.agc_diff_attn_forward(s["q"], s["k"], s["v"], *masks, s["out"], s["workspace"], lse=s["lse"])
    api.agc_diff_attn_partial_gradients(s["q"], s["k"], s["v"], *masks, s["lse"], s["dout"], s["part_end"], s["dq"],
                                        s["dk"], s["dv"], s["G"], s["workspace"])
    return {n: s[n] for n in ("out", "dq", "dk", "dv", "G")}


def _run_plain(s):
    return {"rotary": _plain_rotary, "dropout": _plain_dropout, "forward": _plain_attention, "train": _plain_attention}[s["op"]](s)


def _plain_rotary(s):
    half = s["rot"] // 2
    # the product wraps at a whole turn; far positions keep their 64 bits
    angle = (s["positions"].long()[:, None] * s["turns"]).double() * (2 * math.pi / 2 ** 64)
    if s["inverse"]:
        angle = -angle
    cos, sin = (s["amplitude"] * f(angle).float()[:, None] for f in (torch.cos, torch.sin))
    x = s["x"].float().unflatten(1, (s["heads"], s["dim"]))
    turned, rest = x[..., :s["rot"]], x[..., s["rot"]:]
    pairs = turned.unflatten(2, (half, 2)) if s["layout"] == "interleaved" else turned.unflatten(2, (2, half)).transpose(2, 3)
    a, b = pairs[..., 0], pairs[..., 1]
    new = (a * cos - b * sin, a * sin + b * cos)
    turned = torch.stack(new, -1).flatten(2) if s["layout"] == "interleaved" else torch.cat(new, 2)
    return {"out": torch.cat((turned, rest), 2).flatten(1).to(s["x"].dtype)}


WORD = 0xFFFFFFFF


def _philox(c0, c1, step, seed):
    """Philox4x32-10 of the counters (c0, c1, step lo, step hi), broadcast: a tensor of four words behind them."""
    c0, c1 = torch.broadcast_tensors(c0, c1)
    c2, c3 = torch.full_like(c0, step & WORD), torch.full_like(c0, step >> 32 & WORD)
    k0, k1 = seed & WORD, seed >> 32 & WORD
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (b >> 32 & WORD) ^ c1 ^ k0, b & WORD, (a >> 32 & WORD) ^ c3 ^ k1, a & WORD
        k0, k1 = k0 + 0x9E3779B9 & WORD, k1 + 0xBB67AE85 & WORD
    return torch.stack((c0, c1, c2, c3), -1)


def _uniforms(s):
    """48 random bits of every place: sixteen from a block shared by eight columns, 32 from one shared by four."""
    rows = torch.arange(s["rows"], device=DEVICE)[:, None]
    cols = torch.arange((s["cols"] + 7) // 8, device=DEVICE)
    top = _philox(cols + (s["site"] << 16), rows + (1 << 30), s["step"], s["seed"])
    top = torch.stack((top & 0xFFFF, top >> 16), -1).flatten(1)
    cols = torch.arange((s["cols"] + 7) // 8 * 2, device=DEVICE)
    low = _philox(cols + (s["site"] << 16), rows + (3 << 30), s["step"], s["seed"]).flatten(1)
    return ((top << 32) + low)[:, :s["cols"]]


def _plain_dropout(s):
    keep = _uniforms(s) >= round(s["p"] * 2 ** 48)
    y = torch.where(keep, s["x"].float() * (1.0 / (1.0 - s["p"])), 0.0)
    if s["res"] is not None:
        y = y + s["res"].float()
    return {"out": y.to(s["out"].dtype)}


def _padded(ends, lens):
    """For every sequence the rows of its places, those behind its end pointing at row 0, and which are real; and for
    every row its sequence and place."""
    ends = ends.long()
    begin = torch.cat((ends.new_zeros(1), ends[:-1]))
    place = torch.arange(max(lens), device=DEVICE)
    real = place < (ends - begin)[:, None]
    row = torch.arange(sum(lens), device=DEVICE)
    seq = torch.searchsorted(ends, row, right=True)
    return torch.where(real, begin[:, None] + place, 0), real, seq, row - begin[seq]


def _plain_attention(s):
    h, hk, d, e = s["heads"], s["kv_heads"], s["dim"], s["vdim"]
    at_q, real_q, seq_q, place_q = _padded(s["q_end"], s["lq"])
    at_k, real_k, seq_k, place_k = _padded(s["k_end"], s["lk"])

    def heads(x, at, n, width):   # (sequence, kv head, query head of it, map, place, width)
        x = x.float().view(len(x), hk, n // hk, -1, width)[at]
        return x.permute(0, 2, 3, 4, 1, 5)

    q, k, v = heads(s["q"], at_q, h, d), heads(s["k"], at_k, hk, d), heads(s["v"], at_k, hk, e)
    seen = real_q[:, :, None] & real_k[:, None, :]
    if s["causal"]:
        last = (real_k.sum(1) - real_q.sum(1))[:, None, None]
        seen &= torch.arange(max(s["lk"]), device=DEVICE) <= torch.arange(max(s["lq"]), device=DEVICE)[:, None] + last
    seen = seen[:, None, None, None]
    p = torch.where(seen, torch.matmul(q, k.transpose(-1, -2)).mul_(s["scale"]), -math.inf)
    top = p.amax(-1, keepdim=True)
    p = torch.exp(p.sub_(torch.where(top == -math.inf, 0.0, top)))
    total = p.sum(-1, keepdim=True)
    p = p.div_(torch.where(total > 0, total, 1.0))
    lam = s["lam"].view(hk, h // hk, 1, 1)
    mixed = p[:, :, :, 0] - lam * p[:, :, :, 1]
    v = v[:, :, :, 0]
    out = torch.matmul(mixed, v)
    # back to rows: (row, kv head, query head, width)
    answer = {"out": out.permute(0, 3, 1, 2, 4)[seq_q, place_q].flatten(1).to(torch.bfloat16)}
    if s["op"] == "forward":
        return answer
    dout = torch.where(real_q[:, None, None, :, None], heads(s["dout"], at_q, h, e)[:, :, :, 0], 0.0)
    dp = torch.matmul(dout, v.transpose(-1, -2))[:, :, :, None]
    mean = (p * dp).sum(-1, keepdim=True)
    factor = torch.stack((torch.ones_like(lam), -lam), 2)
    dscore = p.mul_(dp - mean).mul_(factor * s["scale"])
    dq = torch.matmul(dscore, k)
    dk = torch.matmul(dscore.transpose(-1, -2), q).sum(2)
    dv = torch.matmul(mixed.transpose(-1, -2), dout).sum(2)
    answer["dq"] = dq.permute(0, 4, 1, 2, 3, 5)[seq_q, place_q].flatten(1).to(torch.bfloat16)
    answer["dk"] = dk.permute(0, 3, 1, 2, 4)[seq_k, place_k].flatten(1).to(torch.bfloat16)
    answer["dv"] = dv.permute(0, 2, 1, 3)[seq_k, place_k].flatten(1).to(torch.bfloat16)
    # a query's share of the gradient of its head's weight, added up over the partitions
    share = -mean[:, :, :, 1, :, 0].permute(0, 3, 1, 2)[seq_q, place_q].flatten(1)
    part = torch.searchsorted(torch.tensor(s["part_end"], device=DEVICE), torch.arange(s["queries"], device=DEVICE), right=True)
    inside = (part == torch.arange(s["parts"], device=DEVICE)[:, None]).float()
    answer["G"] = torch.matmul(inside, share)
    return answer


def exact(case, seed):
    """The definition in 64 bits: angles from the frequencies, attention one sequence and key head at a time with
    gradients by automatic differentiation."""
    was = globals()["own"]
    globals()["own"] = False
    try:
        s = prepare(case, seed)
    finally:
        globals()["own"] = was
    if case["op"] == "rotary":
        x = s["x"].double().clone().view(case["tokens"], case["heads"], case["dim"])
        out = x.clone()
        sign = -1.0 if case["inverse"] else 1.0
        for i, f in enumerate(s["freq"]):
            a, b = (2 * i, 2 * i + 1) if case["layout"] == "interleaved" else (i, i + case["rot"] // 2)
            turn = torch.polar(torch.full_like(s["positions"], 1, dtype=torch.float64) * s["amplitude"],
                               sign * s["positions"].double() * f)
            z = torch.complex(x[:, :, a], x[:, :, b]) * turn[:, None]
            out[:, :, a], out[:, :, b] = z.real, z.imag
        return {"out": out.view(case["tokens"], -1)}
    if case["op"] == "dropout":
        kept = (_uniforms(s).double() / 2.0 ** 48 >= case["p"]).double()
        y = s["x"].double() * kept / (1 - case["p"])
        return {"out": y if s["res"] is None else s["res"].double() + y}
    h, hk, d, e = case["heads"], case["kv_heads"], case["dim"], case["vdim"]
    group, train = h // hk, case["op"] == "train"
    q, k, v = (s[n].double().view(-1, hk, m, w) for n, m, w in (("q", 2 * group, d), ("k", 2, d), ("v", 1, e)))
    out = torch.zeros(case["queries"], hk, group, e, dtype=torch.float64, device=DEVICE)
    dq, dk, dv = (torch.zeros_like(t) for t in (q, k, v))
    share = torch.zeros(case["queries"], h, dtype=torch.float64, device=DEVICE)
    i = j = 0
    for lq, lk in zip(s["lq"], s["lk"]):
        hidden = torch.zeros(lq, lk, dtype=torch.bool, device=DEVICE)
        if case["causal"]:
            hidden = torch.ones_like(hidden).triu(lk - lq + 1)
        empty = hidden.all(1) if lk else hidden.new_ones(lq)
        for c in range(hk if lq and lk else 0):
            qs, ks, vs = (t[a:b, c].clone().requires_grad_(train) for t, a, b in ((q, i, i + lq), (k, j, j + lk), (v, j, j + lk)))
            for n in range(group):
                maps = []
                for m in range(2):
                    score = (qs[:, 2 * n + m] @ ks[:, m].t()) * s["scale"]
                    score = score.masked_fill(hidden & ~empty[:, None], -math.inf)
                    maps.append(torch.softmax(score, 1).masked_fill(empty[:, None], 0.0) @ vs[:, 0])
                o = maps[0] - s["lam"][c * group + n].double() * maps[1]
                out[i:i + lq, c, n] = o.detach()
                if train:
                    do = s["dout"][i:i + lq].double().view(lq, hk, group, e)[:, c, n]
                    share[i:i + lq, c * group + n] = -(do * maps[1].detach()).sum(1)
                    (o * do).sum().backward()
            if train:
                dq[i:i + lq, c], dk[j:j + lk, c], dv[j:j + lk, c] = qs.grad, ks.grad, vs.grad
        i, j = i + lq, j + lk
    answer = {"out": out.flatten(1)}
    if train:
        answer |= {"dq": dq.flatten(1), "dk": dk.flatten(1), "dv": dv.flatten(1)}
        ends = [0] + s["part_end"]
        answer["G"] = torch.stack([share[a:b].sum(0) for a, b in zip(ends, ends[1:])])
    return answer
