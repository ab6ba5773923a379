"""The operators round the coded step that a token model needs, and how they are measured.

Three operators of `paper_2605_15890_amd.api`: the embedding (`agc_embed_forward`,
`agc_embed_partial_gradients`), the gated feed-forward block (`agc_gated_forward`,
`agc_gated_partial_gradients`) and the orthogonalised update (`agc_muon_update`).  The first two produce
rows of G, one for each data partition; the third consumes the estimate that the coded step returns.

`run` computes them in their plain form, elementary torch operations in binary32, or through the library.
"""
import math

import torch

own = False   # True: through the library

DEVICE = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
IDS = {"i32": torch.int32, "i64": torch.int64}
NS_A, NS_B, NS_C = 3.4445, -4.7750, 2.0315   # coefficients of the odd quintic of the Newton-Schulz products
MUON_EPS = 1e-7
MOMENTUM, LR = 0.95, 0.02
LARGEST = {"embed": 0.8e9, "gated": 1.1e12, "muon": 2.7e12}   # bytes or flops of the largest listed case of each


def listed():
    return [
        # serving, one short prompt: latency of the lookup
        dict(name="embed_prompt", op="embed", way="forward", tokens=37, vocab=32000, dim=768, table="f32", value="bf16",
             ids="i64", parts=1, ragged=False, law="zipf", empty=0.0),
        # a training batch of 64 partitions of 2048 tokens, binary32 parameters to 16-bit activations
        dict(name="embed_batch", op="embed", way="forward", tokens=131072, vocab=50000, dim=1024, table="f32",
             value="bf16", ids="i32", parts=64, ragged=False, law="zipf", empty=0.0),
        # the same model's gradient, eight partitions: dense rows of G, most of them zero
        dict(name="embed_grad", op="embed", way="gradient", tokens=16384, vocab=32000, dim=768, table="f32",
             value="bf16", ids="i32", parts=8, ragged=False, law="zipf", empty=0.0),
        # bytes as tokens: few rows, each of them very often; ragged partitions with padding, odd width
        dict(name="embed_grad_bytes", op="embed", way="gradient", tokens=65537, vocab=257, dim=201, table="f32",
             value="f32", ids="i64", parts=5, ragged=True, law="zipf", empty=0.1),
        # single tokens of a few sequences in serving
        dict(name="gated_decode", op="gated", way="forward", tokens=5, d_in=1024, d_ff=4096, act="silu", parts=1,
             ragged=False),
        # forward pass of a training batch
        dict(name="gated_batch", op="gated", way="forward", tokens=8192, d_in=2048, d_ff=8192, act="silu", parts=1,
             ragged=False),
        # partial gradients, 16 workers' partitions
        dict(name="gated_grad", op="gated", way="gradient", tokens=8192, d_in=2048, d_ff=5632, act="silu", parts=16,
             ragged=False),
        # a small odd block, ragged partitions
        dict(name="gated_grad_odd", op="gated", way="gradient", tokens=1999, d_in=519, d_ff=1101, act="gelu", parts=5,
             ragged=True),
        # one small matrix: latency of the update
        dict(name="muon_small", op="muon", rows=96, cols=64, mats=1, nesterov=True, decay=0.0, copy=False, rank=0),
        # the matrices of a model of twelve blocks, one shape of them, with the 16-bit copy that the next step reads
        dict(name="muon_blocks", op="muon", rows=1024, cols=4096, mats=12, nesterov=True, decay=0.01, copy=True, rank=0),
        # odd and tall, gradients of low rank (few samples)
        dict(name="muon_odd", op="muon", rows=1501, cols=515, mats=3, nesterov=False, decay=0.01, copy=False, rank=40),
        # large square matrices
        dict(name="muon_large", op="muon", rows=4096, cols=4096, mats=2, nesterov=True, decay=0.01, copy=True, rank=0),
    ]


def _between(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm; every third or so a multiple of 64, and the
    lower quarter of the range, where few real sizes lie, half as often as the rest."""
    if rng.random() < 0.5:
        lo = max(lo, round(lo ** 0.75 * hi ** 0.25))
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.35 and hi >= 128:
        v = max(lo, v // 64 * 64)
    return 3071 if v == 3072 else v


def draw(rng):
    op = rng.choice(["embed", "gated", "muon"])
    if op == "embed":
        way = rng.choice(["forward", "gradient"])
        case = dict(op=op, way=way, tokens=_between(rng, 1, 200000), vocab=_between(rng, 2, 100000),
                    dim=_between(rng, 1, 4096), table=rng.choice(["f32", "bf16"]), value=rng.choice(["f32", "bf16"]),
                    ids=rng.choice(["i32", "i64"]), parts=_between(rng, 1, 64), ragged=rng.random() < 0.5,
                    law=rng.choice(["zipf", "uniform"]), empty=rng.choice([0.0, 0.1, 1.0 if rng.random() < 0.1 else 0.5]))
        shrink = ("tokens", "vocab", "dim", "parts")
    elif op == "gated":
        case = dict(op=op, way=rng.choice(["forward", "gradient"]), tokens=_between(rng, 1, 16384),
                    d_in=_between(rng, 8, 4096), d_ff=_between(rng, 8, 12288), act=rng.choice(["silu", "gelu"]),
                    parts=_between(rng, 1, 32), ragged=rng.random() < 0.5)
        shrink = ("tokens", "d_in", "d_ff", "parts")
    else:
        case = dict(op=op, rows=_between(rng, 1, 8192), cols=_between(rng, 1, 8192), mats=_between(rng, 1, 16),
                    nesterov=rng.random() < 0.5, decay=rng.choice([0.0, 0.01]), copy=rng.random() < 0.5,
                    rank=rng.choice([0, 0, 7]))
        shrink = ("rows", "cols", "mats")
    while _cost(case) > LARGEST[op] or _held(case) > 2.0e9:
        most = max(shrink, key=lambda f: case[f])
        if op != "muon" and case["parts"] > 8:
            most = "parts"
        if op == "muon" and case["mats"] > 4:
            most = "mats"
        case[most] = max(1, case[most] * 2 // 3)
    return case


def _cost(case):
    w = work(case)
    return w["bytes"] if case["op"] == "embed" else w["flops"]


def _held(case):
    """Bytes of the largest tensor that a pass returns."""
    if case["op"] == "embed":
        return 4.0 * case["dim"] * (case["tokens"] if case["way"] == "forward" else case["parts"] * case["vocab"])
    if case["op"] == "gated":
        return 8.0 * case["parts"] * case["d_in"] * case["d_ff"] if case["way"] == "gradient" else 0.0
    return 4.0 * case["mats"] * case["rows"] * case["cols"]


def work(case):
    if case["op"] == "embed":
        t, d = case["tokens"], case["dim"]
        value, index = 4 if case["value"] == "f32" else 2, 8 if case["ids"] == "i64" else 4
        held = t * (1 - case["empty"])
        if case["way"] == "forward":
            rows = min(held, case["vocab"])   # a row that several places name is read once
            return {"bytes": t * index + rows * d * (4 if case["table"] == "f32" else 2) + t * d * value, "flops": t * d}
        return {"bytes": t * index + held * d * value + 4.0 * case["parts"] * case["vocab"] * d, "flops": held * d}
    if case["op"] == "gated":
        t, d, f = case["tokens"], case["d_in"], case["d_ff"]
        if case["way"] == "forward":
            return {"bytes": 2.0 * (t * d + 2 * f * d + t * f), "flops": 4.0 * t * d * f}
        return {"bytes": 2.0 * (2 * t * d + 2 * f * d + t * f) + 8.0 * case["parts"] * f * d, "flops": 12.0 * t * d * f}
    m, n = sorted((case["rows"], case["cols"]))
    k = case["mats"]
    # symmetric products count half
    return {"bytes": k * m * n * (20.0 + (2.0 if case["copy"] else 0.0)), "flops": 5.0 * k * (m * m * n + m ** 3 + 2.0 * m * m * n)}


def _parts(case, g):
    """Ends of the partitions: equal ones, or random cuts (empty partitions among them)."""
    t, k = case["tokens"], case["parts"]
    if not case["ragged"]:
        return [t * (i + 1) // k for i in range(k)]
    cuts = torch.randint(0, t + 1, (k - 1,), generator=g).sort().values.tolist()
    return cuts + [t]


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    host = torch.Generator().manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device=DEVICE) * std).to(dtype)

    s = dict(case)
    if case["op"] == "embed":
        t, v, d = case["tokens"], case["vocab"], case["dim"]
        r = torch.rand(t, generator=g, device=DEVICE, dtype=torch.float64)
        ids = (torch.exp(r * math.log(v + 1.0)) - 1.0 if case["law"] == "zipf" else r * v).long().clamp_(0, v - 1)
        gone = torch.rand(t, generator=g, device=DEVICE) < case["empty"]
        s["tokens_dev"] = torch.where(gone, torch.full_like(ids, -1), ids).to(IDS[case["ids"]])
        s["scale"] = math.sqrt(d)
        value = TYPES[case["value"]]
        if case["way"] == "forward":
            s["table_dev"] = normal(v, d, std=0.02, dtype=TYPES[case["table"]])
            s["out"] = torch.empty(t, d, dtype=value, device=DEVICE)
        else:
            s["dout"] = normal(t, d, std=1e-3, dtype=value)
            s["part_end"] = _parts(case, host)
            s["G"] = torch.empty(case["parts"], (v * d + 3) // 4 * 4, device=DEVICE)[:, :v * d]
    elif case["op"] == "gated":
        t, d, f = case["tokens"], case["d_in"], case["d_ff"]
        bf16 = torch.bfloat16
        s["x"] = normal(t, d, dtype=bf16)
        s["wg"], s["wu"] = normal(f, d, std=d ** -0.5, dtype=bf16), normal(f, d, std=d ** -0.5, dtype=bf16)
        if case["way"] == "forward":
            s["h"] = torch.empty(t, f, dtype=bf16, device=DEVICE)
        else:
            s["dh"] = normal(t, f, std=1e-3, dtype=bf16)
            s["dx"] = torch.empty(t, d, dtype=bf16, device=DEVICE)
            s["part_end"] = _parts(case, host)
            s["G"] = torch.empty(case["parts"], (2 * f * d + 3) // 4 * 4, device=DEVICE)[:, :2 * f * d]
    else:
        rows, cols, k = case["rows"], case["cols"], case["mats"]
        gap = (rows * cols + 255) // 256 * 256 + 256   # other parameters lie between the matrices
        s["offsets"] = [i * gap for i in range(k)]
        s["gap"] = gap
        s["beta"] = normal(k * gap, std=0.02)
        if case["rank"]:
            r = min(case["rank"], rows, cols)
            s["ghat"], s["m1"] = (normal(k * gap, std=1e-9) for _ in range(2))
            for vec in (s["ghat"], s["m1"]):
                _matrices(vec, s).add_(torch.bmm(normal(k, rows, r, std=1e-3), normal(k, r, cols)))
        else:
            s["ghat"], s["m1"] = normal(k * gap, std=1e-3), normal(k * gap, std=1e-3)
        s["lr_scale"] = math.sqrt(max(1.0, rows / cols))
        s["copy_dev"] = s["beta"].to(torch.bfloat16) if case["copy"] else None
    if own:
        from paper_2605_15890_amd import api
        s["api"] = api
        need = 0
        if case["op"] == "embed" and case["way"] == "gradient":
            need = api.agc_embed_workspace_bytes(case["tokens"], case["vocab"], case["dim"], case["parts"])
        elif case["op"] == "gated":
            k = case["parts"] if case["way"] == "gradient" else 0
            need = api.agc_gated_workspace_bytes(case["tokens"], case["d_in"], case["d_ff"], k)
        elif case["op"] == "muon":
            need = api.agc_muon_workspace_bytes(case["rows"], case["cols"], case["mats"])
        s["workspace"] = torch.empty(max(16, need), dtype=torch.uint8, device=DEVICE)
    return s


def _matrices(vec, s):
    """The matrices inside a parameter vector, as one view."""
    return vec.as_strided((s["mats"], s["rows"], s["cols"]), (s["gap"], s["cols"], 1), vec.storage_offset())


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    api = s["api"]
    if s["op"] == "embed":
        if s["way"] == "forward":
            api.agc_embed_forward(s["table_dev"], s["tokens_dev"], s["scale"], s["out"])
            return {"out": s["out"]}
        api.agc_embed_partial_gradients(s["dout"], s["tokens_dev"], s["part_end"], s["vocab"], s["scale"], s["G"],
                                        s["workspace"])
        return {"G": s["G"]}
    if s["op"] == "gated":
        if s["way"] == "forward":
            api.agc_gated_forward(s["x"], s["wg"], s["wu"], s["act"], s["h"], s["workspace"])
            return {"h": s["h"]}
        half = s["d_in"] * s["d_ff"]
        api.agc_gated_partial_gradients(s["x"], s["wg"], s["wu"], s["act"], s["dh"], s["part_end"], s["dx"],
                                        s["G"][:, :half], s["G"][:, half:], s["workspace"])
        return {"dx": s["dx"], "G": s["G"]}
    api.agc_muon_update(s["beta"], s["m1"], s["ghat"], s["offsets"], s["rows"], s["cols"], LR, MOMENTUM, s["nesterov"],
                        s["decay"], s["lr_scale"], 5, s["workspace"], beta_bf16=s["copy_dev"])
    return _updated(s)


def _updated(s):
    out = {"beta": s["beta"], "m1": s["m1"]}
    if s["copy"]:
        out["copy"] = s["copy_dev"]
    return out


def _part_of(s):
    """The partition of every token."""
    ends = torch.tensor(s["part_end"], device=DEVICE)
    return torch.searchsorted(ends, torch.arange(s["tokens"], device=DEVICE), right=True)


def _act(a, kind):
    """The activation and its derivative."""
    if kind == "silu":
        sig = 1.0 / (1.0 + torch.exp(-a))
        return a * sig, sig * (1.0 + a * (1.0 - sig))
    cdf = 0.5 * (1.0 + torch.erf(a * math.sqrt(0.5)))
    return a * cdf, cdf + a * torch.exp(-0.5 * a * a) * (1.0 / math.sqrt(2.0 * math.pi))


def _run_plain(s):
    if s["op"] == "embed":
        ids = s["tokens_dev"].long()
        held = (ids >= 0) & (ids < s["vocab"])
        if s["way"] == "forward":
            rows = s["table_dev"][torch.where(held, ids, 0)].float() * s["scale"]
            return {"out": torch.where(held[:, None], rows, 0.0).to(s["out"].dtype)}
        v, d = s["vocab"], s["dim"]
        rows = torch.where(held[:, None], s["dout"].float() * s["scale"], 0.0)
        G = torch.zeros(s["parts"] * v, d, device=DEVICE)
        G.index_add_(0, _part_of(s) * v + torch.where(held, ids, 0), rows)
        return {"G": G.view(s["parts"], v * d)}
    if s["op"] == "gated":
        x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
        a, u = x @ wg.t(), x @ wu.t()
        act, slope = _act(a, s["act"])
        if s["way"] == "forward":
            return {"h": (act * u).to(torch.bfloat16)}
        dh = s["dh"].float()
        da, du = dh * u * slope, dh * act
        dx = (da @ wg + du @ wu).to(torch.bfloat16)
        # rows of each partition side by side, shorter partitions filled up with zeros
        ends = torch.tensor([0] + s["part_end"], device=DEVICE)
        longest = max(e - b for b, e in zip([0] + s["part_end"], s["part_end"]))
        at = ends[:-1, None] + torch.arange(longest, device=DEVICE)
        inside = at < ends[1:, None]
        at = torch.where(inside, at, 0)
        xp = torch.where(inside[:, :, None], x[at], 0.0)
        both = torch.cat([da, du], 1)[at]
        G = torch.bmm(both.transpose(1, 2), xp)
        return {"dx": dx, "G": G.view(s["parts"], -1)}
    m1, ghat, beta = (_matrices(s[k], s) for k in ("m1", "ghat", "beta"))
    m1.mul_(MOMENTUM).add_(ghat)
    x = ghat + MOMENTUM * m1 if s["nesterov"] else m1
    x = x / (torch.sqrt((x * x).sum((1, 2), keepdim=True)) + MUON_EPS)
    tall = s["rows"] > s["cols"]
    x = x.transpose(1, 2).contiguous() if tall else x
    for _ in range(5):
        gram = torch.bmm(x, x.transpose(1, 2))
        x = NS_A * x + torch.bmm(NS_B * gram + NS_C * torch.bmm(gram, gram), x)
    x = x.transpose(1, 2) if tall else x
    beta.mul_(1.0 - LR * s["decay"]).sub_(LR * s["lr_scale"] * x)
    if s["copy"]:
        _matrices(s["copy_dev"], s).copy_(beta)
    return _updated(s)


def exact(case, seed):
    """The definition in 64 bits, each operator one partition, token or matrix at a time."""
    was = globals()["own"]
    globals()["own"] = False
    try:
        s = prepare(case, seed)
    finally:
        globals()["own"] = was
    if case["op"] == "embed":
        ids = s["tokens_dev"].long()
        at = torch.nonzero((ids >= 0) & (ids < case["vocab"]))[:, 0]
        if case["way"] == "forward":
            out = torch.zeros(case["tokens"], case["dim"], dtype=torch.float64, device=DEVICE)
            out[at] = s["scale"] * s["table_dev"].double().index_select(0, ids[at])
            return {"out": out}
        G = torch.zeros(case["parts"], case["vocab"], case["dim"], dtype=torch.float64, device=DEVICE)
        start = 0
        for p, end in enumerate(s["part_end"]):
            mine = at[(at >= start) & (at < end)]
            G[p].index_put_((ids[mine],), s["scale"] * s["dout"][mine].double(), accumulate=True)
            start = end
        return {"G": G.view(case["parts"], -1)}
    if case["op"] == "gated":
        x, wg, wu = (s[k].double() for k in ("x", "wg", "wu"))
        a, u = torch.mm(x, wg.t()), torch.mm(x, wu.t())
        if case["act"] == "silu":
            p = torch.special.expit(a)
            act, slope = a * p, p + a * p * torch.special.expit(-a)
        else:
            p = torch.special.ndtr(a)
            act, slope = a * p, p + a * torch.exp(-a.square() / 2) / math.sqrt(2 * math.pi)
        if case["way"] == "forward":
            return {"h": act * u}
        dh = s["dh"].double()
        da, du = dh * u * slope, dh * act
        rows, start = [], 0
        for end in s["part_end"]:
            xp = x[start:end]
            rows.append(torch.cat([torch.mm(da[start:end].t(), xp).flatten(), torch.mm(du[start:end].t(), xp).flatten()]))
            start = end
        return {"dx": torch.mm(da, wg) + torch.mm(du, wu), "G": torch.stack(rows)}
    rows, cols = case["rows"], case["cols"]
    beta, m1 = s["beta"].double(), s["m1"].double()
    copy = s["copy_dev"].double() if case["copy"] else None
    for off in s["offsets"]:
        here = slice(off, off + rows * cols)
        g = s["ghat"][here].double()
        m1[here] = MOMENTUM * m1[here] + g
        u = (g + MOMENTUM * m1[here] if case["nesterov"] else m1[here]).view(rows, cols)
        u = u / (torch.linalg.matrix_norm(u) + MUON_EPS)
        # every factor is a polynomial of the first Gram matrix, on the short side: they commute
        gram = u @ u.t() if rows <= cols else u.t() @ u
        eye = torch.eye(len(gram), dtype=torch.float64, device=DEVICE)
        q = eye
        for _ in range(5):
            p = NS_A * eye + gram @ (NS_B * eye + NS_C * gram)
            q = p @ q
            gram = p @ gram @ p
        x = q @ u if rows <= cols else u @ q
        beta[here] = (1 - LR * case["decay"]) * beta[here] - LR * s["lr_scale"] * x.flatten()
        if copy is not None:
            copy[here] = beta[here]
    out = {"beta": beta, "m1": m1}
    if copy is not None:
        out["copy"] = copy
    return out
