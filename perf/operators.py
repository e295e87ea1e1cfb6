"""Cases of the operators that a step over drafted tokens consists of: projections with an adapter per row, rotary positions,
attention of token trees over the paged cache, and the draw with temperature, top-k, top-p and min-p.

Kinds of case
  lora     C = A W^T + scale (A La^T) Lb^T, each row with the adapter of its request
  rope     rotary positions on the heads of a packed projection output
  tree     attention of trees of drafted tokens over the paged cache and over the trees themselves
  sample   tokens drawn from rows of logits by given uniform numbers

`own` chooses between the plain form (elementary torch operations, in 32 bits, in 64 where angles, long sums and values next to
a border need them) and the framework's kernels.
"""
import math
import random

import torch

own = False

DEV = "cuda"
PAGE = 16
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp32": 4}


def listed():
    return [
        # one decode step of sixteen requests, each with the adapter of its task: the attention output projection of an 8B-class layer
        {"name": "lora_decode_16", "op": "lora", "dtype": "bf16", "m": 16, "n": 4096, "k": 4096, "r": 8, "adapters": 16, "runs": False},
        # drafted trees of eight requests through the gate projection
        {"name": "lora_verify_250", "op": "lora", "dtype": "bf16", "m": 250, "n": 14336, "k": 4096, "r": 16, "adapters": 8, "runs": True},
        # prompts of four tasks together through the down projection
        {"name": "lora_prompt_4096", "op": "lora", "dtype": "bf16", "m": 4096, "n": 4096, "k": 14336, "r": 8, "adapters": 4, "runs": True},
        # the small fp32 model
        {"name": "lora_fp32_33", "op": "lora", "dtype": "fp32", "m": 33, "n": 688, "k": 256, "r": 8, "adapters": 4, "runs": False},
        # queries and keys of 64 drafted tokens inside a packed Q/K/V output, 8B-class heads, positions scaled by bands
        {"name": "rope_verify_64", "op": "rope", "dtype": "bf16", "rows": 64, "heads": 40, "hd": 128, "rot": 128, "packed": 48,
         "layout": "half", "scaling": "bands", "inverse": False},
        # a long prompt
        {"name": "rope_prompt_16k", "op": "rope", "dtype": "bf16", "rows": 16384, "heads": 40, "hd": 128, "rot": 128, "packed": 48,
         "layout": "half", "scaling": "none", "inverse": False},
        # the gradient of interleaved pairs on half of each head, odd number of rows
        {"name": "rope_part_gradient", "op": "rope", "dtype": "fp32", "rows": 1297, "heads": 16, "hd": 64, "rot": 32, "packed": 16,
         "layout": "interleaved", "scaling": "linear", "inverse": True},
        # one token of one request: the ordinary decode step, where latency counts
        {"name": "tree_one_token", "op": "tree", "dtype": "bf16", "batch": 1, "lo": 1000, "hi": 1000, "nlo": 1, "nhi": 1,
         "hq": 32, "hkv": 8, "hd": 128, "shape_seed": 0},
        # trees of up to 16 tokens for sixteen requests of mixed lengths
        {"name": "tree_16_requests", "op": "tree", "dtype": "bf16", "batch": 16, "lo": 300, "hi": 2300, "nlo": 9, "nhi": 16,
         "hq": 32, "hkv": 8, "hd": 128, "shape_seed": 1},
        # large trees over long contexts
        {"name": "tree_long_context", "op": "tree", "dtype": "bf16", "batch": 4, "lo": 20000, "hi": 32768, "nlo": 33, "nhi": 61,
         "hq": 32, "hkv": 8, "hd": 128, "shape_seed": 2},
        # one request, small vocabulary
        {"name": "sample_one_row", "op": "sample", "rows": 1, "vocab": 32000, "rules": "all"},
        # every node of sixteen drafted trees, large vocabulary, nucleus sampling
        {"name": "sample_256_rows", "op": "sample", "rows": 256, "vocab": 128256, "rules": "nucleus"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["lora", "rope", "tree", "sample"])
    if op == "lora":
        fp32 = rng.random() < 0.25
        k, n = 8 * _log(rng, 8, 256 if fp32 else 1792), _log(rng, 64, 2048 if fp32 else 14336)
        m = _log(rng, 1, 512 if fp32 else min(4096, 4096 * 4096 * 14336 // (n * k)))
        return {"op": op, "dtype": "fp32" if fp32 else "bf16", "m": m, "n": n, "k": k, "r": _log(rng, 1, 64),
                "adapters": _log(rng, 1, 32), "runs": rng.random() < 0.5}
    if op == "rope":
        hd = rng.choice([64, 128])
        heads = rng.randint(1, 48)
        return {"op": op, "dtype": rng.choice(["bf16", "fp32"]), "rows": _log(rng, 1, 8192), "heads": heads, "hd": hd,
                "rot": rng.choice([hd, hd, hd // 2, hd // 4, 2 * rng.randint(1, hd // 2)]), "packed": heads + rng.choice([0, 0, 1, 8]),
                "layout": rng.choice(["half", "interleaved"]), "scaling": rng.choice(["none", "linear", "bands"]), "inverse": rng.random() < 0.3}
    if op == "tree":
        fp32 = rng.random() < 0.2
        hq, hkv, hd = rng.choice([(32, 8, 128), (24, 8, 128), (32, 8, 64), (4, 4, 64), (16, 2, 128), (5, 1, 64)])
        batch = _log(rng, 1, 16)
        hi = _log(rng, 16, 2048 if fp32 else 131072 // batch)
        nhi = _log(rng, 1, 64)
        return {"op": op, "dtype": "fp32" if fp32 else "bf16", "batch": batch, "lo": rng.choice([0, 1, hi // 2, hi]), "hi": hi,
                "nlo": max(1, nhi // 2), "nhi": nhi, "hq": hq, "hkv": hkv, "hd": hd, "shape_seed": rng.randrange(1 << 20)}
    rows = _log(rng, 1, 256)
    return {"op": op, "rows": rows, "vocab": _log(rng, 100, 128256), "rules": rng.choice(["all", "nucleus", "top_k", "min_p", "none"])}


def _shape(case):
    """Cached lengths and numbers of drafted tokens of a tree case's sequences: part of the case."""
    rng = random.Random(case["shape_seed"])
    lens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]
    nodes = [rng.randint(case["nlo"], case["nhi"]) for _ in range(case["batch"])]
    return lens, nodes


def _normal(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std).to(dtype)


# ---- inputs --------------------------------------------------------------------------------------------------------------


def _prepare_lora(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = random.Random(seed)
    t, m, n, k, r, ad = TYPES[case["dtype"]], case["m"], case["n"], case["k"], case["r"], case["adapters"]
    if case["runs"]:                     # packed requests: runs of rows with one adapter
        ids = []
        while len(ids) < m:
            ids += [rng.randrange(ad)] * rng.randint(1, max(1, 2 * m // (ad + 1)))
        ids = ids[:m]
    else:                                # a row a request; some have no adapter
        ids = [rng.randrange(ad) if rng.random() < 0.9 else -1 for _ in range(m)]
    return {"A": _normal(g, (m, k), t), "W": _normal(g, (n, k), t, 0.02), "La": _normal(g, (ad, r, k), t, 0.02), "Lb": _normal(g, (ad, n, r), t, 0.02),
            "adapter": torch.tensor(ids, dtype=torch.int32, device=DEV), "scale": torch.full((ad,), 32.0 / r, device=DEV) * torch.rand(ad, generator=g, device=DEV),
            "C": torch.empty((m, n), dtype=torch.float32, device=DEV)}


def _prepare_rope(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rows, heads, hd = case["rows"], case["heads"], case["hd"]
    x = _normal(g, (rows, case["packed"], hd), TYPES[case["dtype"]])[:, :heads]
    pos = torch.randint(0, 131072 if case["scaling"] != "none" else 32768, (rows,), generator=g, device=DEV, dtype=torch.int32)
    return {"x": x, "pos": pos, "y": torch.empty((rows, heads, hd), dtype=x.dtype, device=DEV)}


def _prepare_tree(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = random.Random(seed)
    t, hq, hkv, hd = TYPES[case["dtype"]], case["hq"], case["hkv"], case["hd"]
    lens, nodes = _shape(case)
    N, most = sum(nodes), max(nodes)
    max_pages = max(1, max(-(-x // PAGE) for x in lens))
    n_pages = sum(-(-x // PAGE) for x in lens) + 3
    pool = torch.randn((n_pages, 2, hkv, PAGE, hd), generator=g, device=DEV, dtype=t)
    order = list(range(n_pages))
    rng.shuffle(order)
    table, at = torch.zeros((len(lens), max_pages), dtype=torch.int32), 0
    for b, x in enumerate(lens):
        c = -(-x // PAGE)
        table[b, :c] = torch.tensor(order[at:at + c], dtype=torch.int32)
        at += c
    words = -(-most // 64)
    masks = []
    for c in nodes:                      # a random tree, earlier nodes first: a node sees its ancestors and itself
        seen = []
        for i in range(c):
            parent = rng.randint(max(-1, i - 4), i - 1)
            seen.append((seen[parent] if parent >= 0 else 0) | 1 << i)
        masks += [[(s >> 64 * w & (1 << 64) - 1) - ((s >> 64 * w + 63 & 1) << 64) for w in range(words)] for s in seen]
    offs = [0]
    for c in nodes:
        offs.append(offs[-1] + c)
    return {"q": _normal(g, (N, hq, hd), t, 1.5), "k": _normal(g, (N, hkv, hd), t), "v": _normal(g, (N, hkv, hd), t), "pool": pool, "table": table.to(DEV),
            "lens": torch.tensor(lens, dtype=torch.int32, device=DEV), "offs": torch.tensor(offs, dtype=torch.int32, device=DEV),
            "mask": torch.tensor(masks, dtype=torch.int64, device=DEV).reshape(N, words), "max_nodes": most, "max_len": max(lens), "scale": hd ** -0.5,
            "out": torch.empty((N, hq, hd), dtype=t, device=DEV), "lse": torch.empty((N, hq), dtype=torch.float32, device=DEV)}


def _prepare_sample(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rows, vocab, rules = case["rows"], case["vocab"], case["rules"]
    uniform = lambda lo, hi: lo + (hi - lo) * torch.rand(rows, generator=g, device=DEV)  # noqa: E731
    logits = torch.randn((rows, vocab), generator=g, device=DEV) * uniform(0.5, 3.0)[:, None]
    peaks = torch.randint(0, vocab, (rows, 24), generator=g, device=DEV)       # a few tokens that the model means, on top of the rest
    logits.scatter_add_(1, peaks, torch.rand((rows, 24), generator=g, device=DEV) * 12.0)
    logits[::3] = logits[::3].bfloat16().float()                               # rows from a 16-bit head have many equal logits
    s = {"logits": logits, "u": torch.rand(rows, generator=g, device=DEV), "temperature": uniform(0.3, 1.2), "top_k": None, "top_p": None, "min_p": None,
         "token": torch.empty(rows, dtype=torch.int32, device=DEV), "logprob": torch.empty(rows, device=DEV),
         "kept": torch.empty(rows, dtype=torch.int32, device=DEV)}
    if rules in ("all", "top_k"):
        s["top_k"] = torch.randint(1, 101, (rows,), generator=g, device=DEV, dtype=torch.int32)
    if rules in ("all", "nucleus"):
        s["top_p"] = uniform(0.7, 0.98)
    if rules in ("all", "min_p"):
        s["min_p"] = uniform(0.01, 0.1)
    return s


def prepare(case, seed):
    s = {"lora": _prepare_lora, "rope": _prepare_rope, "tree": _prepare_tree, "sample": _prepare_sample}[case["op"]](case, seed)
    s["case"] = dict(case)
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------------


def _plain_lora(s):
    A, ad = s["A"].float(), s["La"].shape[0]
    r = s["La"].shape[1]
    mine = s["adapter"][:, None] == torch.arange(ad, device=DEV, dtype=torch.int32)             # [m, adapters]
    T = (A @ s["La"].float().reshape(ad * r, -1).t()).reshape(-1, ad, r) * (mine * s["scale"])[:, :, None]
    return A @ s["W"].float().t() + T.reshape(-1, ad * r) @ s["Lb"].float().permute(0, 2, 1).reshape(ad * r, -1)


BASE, FACTOR, LOW, HIGH, ORIGINAL = 500000.0, 8.0, 1.0, 4.0, 8192


def _frequencies(case):
    f = BASE ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device=DEV) / case["rot"])
    if case["scaling"] == "linear":
        return f / FACTOR
    if case["scaling"] == "bands":
        keep = ((ORIGINAL * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
        return (1 - keep) * f / FACTOR + keep * f
    return f


def _plain_rope(s):
    case = s["case"]
    rot = case["rot"]
    angle = s["pos"].double()[:, None] * _frequencies(case)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if case["inverse"]:
        sin = -sin
    x = s["x"].float()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if case["layout"] == "interleaved" else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v = a * cos - b * sin, a * sin + b * cos
    pairs = torch.stack((u, v), -1).flatten(-2) if case["layout"] == "interleaved" else torch.cat((u, v), -1)
    return torch.cat((pairs, x[..., rot:]), -1).to(s["x"].dtype)


def _plain_tree(s):
    q, table, lens, offs, hd = s["q"], s["table"], s["lens"], s["offs"], s["q"].shape[2]
    B, hq, hkv, most = lens.shape[0], q.shape[1], s["k"].shape[1], s["max_nodes"]
    cached = s["pool"][table.long()].float().permute(2, 0, 3, 1, 4, 5).reshape(2, B, hkv, -1, hd)              # [K|V, B, Hkv, positions, hd]
    at = offs[:-1, None].long() + torch.arange(most, device=DEV)                                                # [B, nodes]
    real = at < offs[1:, None]
    at = at.clamp(max=q.shape[0] - 1)
    tree = torch.stack((s["k"], s["v"]))[:, at].float().permute(0, 1, 3, 2, 4)                                 # [K|V, B, Hkv, nodes, hd]
    K, V = torch.cat((cached, tree), 3)
    Q = q[at].float().reshape(B, most, hkv, hq // hkv, hd).permute(0, 2, 3, 1, 4).reshape(B, hkv, -1, hd)
    bits = torch.arange(most, device=DEV)
    seen = (s["mask"][at][:, :, bits // 64] >> (bits % 64) & 1).bool() & real[:, None]                          # [B, nodes, nodes]
    old = (torch.arange(cached.shape[3], device=DEV) < lens[:, None])[:, None].expand(-1, most, -1)
    see = torch.cat((old, seen), 2)[:, None, None]
    score = (Q @ K.transpose(2, 3).contiguous() * s["scale"]).reshape(B, hkv, hq // hkv, most, -1)
    score = score.masked_fill(~see, float("-inf"))
    top = score.amax(-1, keepdim=True)
    w = torch.exp(score - torch.where(top.isinf(), torch.zeros_like(top), top))
    total = w.sum(-1, keepdim=True)
    o = (w.reshape(B, hkv, -1, w.shape[-1]) @ V).reshape(*total.shape[:-1], hd) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + total.log())[..., 0]
    b, j = real.nonzero(as_tuple=True)
    return {"out": o.permute(0, 3, 1, 2, 4).reshape(B, most, hq, hd)[b, j].to(q.dtype), "lse": lse.permute(0, 3, 1, 2).reshape(B, most, hq)[b, j]}


def _plain_sample(s):
    logits = s["logits"]
    rows, vocab = logits.shape
    l, order = torch.sort(logits.double(), dim=1, descending=True, stable=True)
    w = torch.exp((l - l[:, :1]) / s["temperature"].double()[:, None])
    place = torch.arange(vocab, device=DEV)
    if s["top_k"] is not None:
        w = w * (place < s["top_k"][:, None])
    keep = w > 0
    if s["top_p"] is not None:
        cum = w.cumsum(1)
        keep &= cum - w < s["top_p"].double()[:, None] * cum[:, -1:]
    if s["min_p"] is not None:
        keep &= w >= s["min_p"].double()[:, None]
    cum = (w * keep).cumsum(1)
    kept = keep.sum(1)
    at = torch.minimum((cum <= s["u"].double()[:, None] * cum[:, -1:]).sum(1), kept - 1)[:, None]
    return {"token": order.gather(1, at)[:, 0].int(), "logprob": (w.gather(1, at) / cum[:, -1:]).log()[:, 0].float(), "kept": kept.int()}


# ---- the framework's calls -----------------------------------------------------------------------------------------------


def _own(s):
    import paper_2410_12513_amd as P
    op = s["case"]["op"]
    if op == "rope":
        c = s["case"]
        P.op_rope(s["x"], s["pos"], s["y"], rot_dim=c["rot"], layout=c["layout"], base=BASE, scaling=c["scaling"], factor=FACTOR, low=LOW, high=HIGH,
                  original_len=ORIGINAL, inverse=c["inverse"])
        return s["y"]
    if "workspace" not in s:             # kept by the program from call to call
        need = {"lora": lambda: P.op_gemm_nt_lora_workspace(s["A"], s["W"], s["La"]), "sample": lambda: P.sample_workspace(s["logits"]),
                "tree": lambda: P.op_tree_attn_workspace(s["q"], s["k"], s["max_nodes"], s["max_len"], s["lens"].shape[0])}[op]()
        s["workspace"] = torch.empty(max(need, 1), dtype=torch.uint8, device=DEV)
    if op == "lora":
        P.op_gemm_nt_lora(s["A"], s["W"], s["La"], s["Lb"], s["adapter"], s["scale"], s["C"], workspace=s["workspace"])
        return s["C"]
    if op == "tree":
        P.op_tree_attn(s["q"], s["k"], s["v"], s["pool"], s["table"], s["lens"], s["offs"], s["out"], s["max_nodes"], s["max_len"], mask=s["mask"],
                       scale=s["scale"], lse=s["lse"], workspace=s["workspace"])
        return {"out": s["out"], "lse": s["lse"]}
    P.sample(s["logits"], s["u"], s["token"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], logprob=s["logprob"],
             kept=s["kept"], workspace=s["workspace"])
    return {"token": s["token"], "logprob": s["logprob"], "kept": s["kept"]}


def run(state):
    if own:
        return _own(state)
    return {"lora": _plain_lora, "rope": _plain_rope, "tree": _plain_tree, "sample": _plain_sample}[state["case"]["op"]](state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------


def work(case):
    if case["op"] == "lora":
        m, n, k, r, z = case["m"], case["n"], case["k"], case["r"], SIZE[case["dtype"]]
        used = min(case["adapters"], m)
        return {"bytes": (m * k + n * k + used * r * (n + k)) * z + 4 * m * n, "flops": 2 * m * n * k + 2 * m * r * (n + k)}
    if case["op"] == "rope":
        values = case["rows"] * case["heads"] * case["hd"]
        return {"bytes": 2 * values * SIZE[case["dtype"]] + 4 * case["rows"], "flops": 3 * values}
    if case["op"] == "tree":
        lens, nodes = _shape(case)
        z, hd, N = SIZE[case["dtype"]], case["hd"], sum(nodes)
        return {"bytes": (2 * case["hkv"] * hd * (sum(lens) + N) + 2 * N * case["hq"] * hd) * z + 4 * N * case["hq"],
                "flops": 4 * case["hq"] * hd * sum(c * (x + c) for x, c in zip(lens, nodes))}
    return {"bytes": 4 * case["rows"] * case["vocab"], "flops": 4 * case["rows"] * case["vocab"]}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------


def _exact_lora(case, s):
    A = s["A"].double()
    C = torch.empty((case["m"], case["n"]), dtype=torch.float64, device=DEV)
    for i in range(0, case["m"], 512):
        C[i:i + 512] = A[i:i + 512] @ s["W"].double().t()
    for a in range(case["adapters"]):
        rows = (s["adapter"] == a).nonzero()[:, 0]
        C[rows] += (A[rows] @ s["La"][a].double().t()) @ s["Lb"][a].double().t() * s["scale"][a].double()
    return C


def _exact_rope(case, s):
    f = []
    for i in range(case["rot"] // 2):
        wavelength = 2 * math.pi * BASE ** (2 * i / case["rot"])
        stretched = wavelength * FACTOR
        if case["scaling"] == "none" or (case["scaling"] == "bands" and ORIGINAL >= HIGH * wavelength):
            f.append(2 * math.pi / wavelength)
        elif case["scaling"] == "linear" or ORIGINAL <= LOW * wavelength:
            f.append(2 * math.pi / stretched)
        else:                            # between the bands: a blend by how many turns the original context holds
            share = (ORIGINAL / wavelength - LOW) / (HIGH - LOW)
            f.append(share * 2 * math.pi / wavelength + (1 - share) * 2 * math.pi / stretched)
    f = torch.tensor(f, dtype=torch.float64, device=DEV)
    x = s["x"].double()
    half = case["rot"] // 2
    index = torch.arange(half, device=DEV)
    first, second = (2 * index, 2 * index + 1) if case["layout"] == "interleaved" else (index, index + half)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), s["pos"].double()[:, None, None] * f)
    z = torch.complex(x[..., first], x[..., second]) * (turn.conj() if case["inverse"] else turn)
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_tree(case, s):
    lens, nodes = _shape(case)
    group = case["hq"] // case["hkv"]
    out, lse, at = [], [], 0
    for b, (x, c) in enumerate(zip(lens, nodes)):
        pages = s["pool"][s["table"][b, :-(-x // PAGE)].long()].double()
        bits = torch.arange(c, device=DEV)
        seen = (s["mask"][at:at + c][:, bits // 64] >> (bits % 64) & 1).bool()
        o, e = [], []
        for h in range(case["hkv"]):
            K = torch.cat((pages[:, 0, h].reshape(-1, case["hd"])[:x], s["k"][at:at + c, h].double()))
            V = torch.cat((pages[:, 1, h].reshape(-1, case["hd"])[:x], s["v"][at:at + c, h].double()))
            for i in range(h * group, h * group + group):
                score = s["q"][at:at + c, i].double() @ K.t().contiguous() * s["scale"]
                score[:, x:].masked_fill_(~seen, float("-inf"))
                o.append(torch.softmax(score, 1) @ V)
                e.append(torch.logsumexp(score, 1))
        out.append(torch.stack(o, 1))
        lse.append(torch.stack(e, 1))
        at += c
    return {"out": torch.cat(out), "lse": torch.cat(lse)}


def _exact_sample(case, s):
    import numpy as np
    host = {key: v.cpu().numpy() for key, v in s.items() if isinstance(v, torch.Tensor)}
    token, logprob, kept = [], [], []
    for i in range(case["rows"]):
        l = host["logits"][i].astype(np.float64)
        order = np.argsort(-l, kind="stable")
        if s["top_k"] is not None:
            order = order[:host["top_k"][i]]
        w = np.exp((l[order] - l[order[0]]) / np.float64(host["temperature"][i]))
        n = len(w)
        if s["top_p"] is not None:
            n = min(n, 1 + int(np.searchsorted(np.cumsum(w), np.float64(host["top_p"][i]) * w.sum())))
        if s["min_p"] is not None:
            n = min(n, int((w >= np.float64(host["min_p"][i])).sum()))
        cum = np.cumsum(w[:n])
        j = min(int(np.searchsorted(cum, np.float64(host["u"][i]) * cum[-1], side="right")), n - 1)
        token.append(order[j])
        kept.append(n)
        logprob.append(math.log(w[j] / cum[-1]))
    return {"token": torch.tensor(token, dtype=torch.int32), "logprob": torch.tensor(logprob, dtype=torch.float64), "kept": torch.tensor(kept, dtype=torch.int32)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"lora": _exact_lora, "rope": _exact_rope, "tree": _exact_tree, "sample": _exact_sample}[case["op"]](case, s)
