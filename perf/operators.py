"""What is measured of the operators around the decode step: low-rank adapters of many requests beside a shared
projection (``first_lora``), rotary positions (``first_rope``) and per-request sampling (``first_sample``).

``run`` computes an operator in plain torch operations, or, with ``own``, through the library's calls.  ``exact`` gives
the same results in 64 bits, written apart from the plain form."""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------ cases
def _lora(name, rows, adapters, rank, k, n, segs, x, y, w, order):
    return {"name": name, "op": "lora", "rows": rows, "adapters": adapters, "rank": rank, "k": k, "n": n, "segs": segs,
            "x": x, "y": y, "w": w, "order": order}


def _rope(name, tokens, hq, hk, hd, rot, layout, scaling, dtype, fused, far):
    return {"name": name, "op": "rope", "tokens": tokens, "hq": hq, "hk": hk, "hd": hd, "rot": rot, "layout": layout,
            "scaling": scaling, "dtype": dtype, "fused": fused, "far": far}


def _sample(name, rows, vocab, pad, mix, spread):
    return {"name": name, "op": "sample", "rows": rows, "vocab": vocab, "pad": pad, "mix": mix, "spread": spread}


def listed():
    return [
        # one request's adapter beside the 8B shape's q|k|v projection, at the paper's rank: latency
        _lora("lora_qkv_1row", 1, 4, 8, 4096, 6144, 3, "bf16", "f32", "bf16", "mixed"),
        # a decode batch of 32 requests over 16 adapters, q|k|v
        _lora("lora_qkv_32rows", 32, 16, 16, 4096, 6144, 3, "bf16", "f32", "bf16", "mixed"),
        # a batch of 256 requests over 64 adapters at the down projection
        _lora("lora_down_256rows", 256, 64, 32, 14336, 4096, 1, "f32", "f32", "bf16", "mixed"),
        # odd sizes, float32 adapters (the float32 models)
        _lora("lora_odd_f32", 77, 5, 24, 2040, 1000, 1, "f32", "f32", "f32", "mixed"),
        # prompts of a few requests: long runs of one adapter, gate|up
        _lora("lora_gate_up_1024rows", 1024, 8, 16, 4096, 28672, 2, "bf16", "bf16", "bf16", "runs"),
        # one decode step of 32 sequences at the 3B shape's scaled frequencies
        _rope("rope_step_32", 32, 24, 8, 128, 128, "half", "llama3", "bf16", False, 131072),
        # part of the head, interleaved pairs, q and k inside a fused q|k|v buffer, float32
        _rope("rope_part_interleaved", 4097, 32, 8, 64, 32, "interleaved", "none", "f32", True, 8192),
        # a long prompt batch, far positions
        _rope("rope_prompt_32k", 32768, 32, 8, 128, 128, "half", "yarn", "bf16", True, 1000000),
        # one answer at the paper's settings
        _sample("sample_1row_paper", 1, 128256, 0, "paper", 2.5),
        # a decode batch, every request with settings of its own
        _sample("sample_32rows_mixed", 32, 128256, 0, "mixed", 2.5),
        # a vocabulary of odd size in padded rows, nucleus sampling
        _sample("sample_61rows_odd", 61, 50257, 47, "top_p", 3.0),
        # the largest batch
        _sample("sample_256rows_mixed", 256, 128256, 0, "mixed", 2.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["lora", "rope", "sample"])
    if op == "lora":
        segs = rng.choice([1, 1, 2, 3])
        rows, k = _log(rng, 1, 1024), 8 * _log(rng, 16, 1792)
        n = segs * 16 * _log(rng, 4, max(5, 1792 // (segs * (1 if rows <= 256 else 4))))
        n -= rng.choice([0, 0, 1, 7])  # the last segment may end inside a tile
        w = rng.choice(["bf16", "bf16", "f32"])
        return {key: v for key, v in _lora("", rows, _log(rng, 1, 64), 8 * _log(rng, 1, 8), k, n, segs,
                                           "f32" if w == "f32" else rng.choice(["bf16", "f32"]),
                                           "f32" if w == "f32" else rng.choice(["bf16", "f32"]), w,
                                           rng.choice(["mixed", "runs"])).items() if key != "name"}
    if op == "rope":
        hd = rng.choice([32, 64, 96, 128, 128, 256])
        rot = hd if rng.random() < 0.6 else 2 * rng.randint(4, hd // 2)
        hk = rng.choice([1, 2, 4, 8])
        tokens = _log(rng, 1, 32768 * 128 * 32 // (hd * hk * 8 * 2))
        return {key: v for key, v in _rope("", min(tokens, 32768), hk * rng.choice([1, 2, 3, 4]), hk, hd, rot,
                                           rng.choice(["half", "interleaved"]),
                                           rng.choice(["none", "linear", "llama3", "yarn"]), rng.choice(["bf16", "f32"]),
                                           rng.random() < 0.5, _log(rng, 64, 1000000)).items() if key != "name"}
    return {key: v for key, v in _sample("", _log(rng, 1, 256), _log(rng, 500, 128256), rng.choice([0, 0, 1, 47]),
                                         rng.choice(["paper", "mixed", "mixed", "top_p", "min_p", "plain"]),
                                         rng.uniform(1.0, 4.0)).items() if key != "name"}


# ------------------------------------------------------------------ inputs
def _segments(case):
    """Borders of the output segments: q|k|v as 4:1:1 parts, gate|up as halves, in whole 16s; the last ends at n."""
    n, s = case["n"], case["segs"]
    if s == 1:
        return (0, n)
    parts = [4, 1, 1] if s == 3 else [1, 1]
    up = (n + 15) // 16
    edges, total = [0], 0
    for p in parts[:-1]:
        total += p
        edges.append(16 * max(len(edges), up * total // sum(parts)))
    return tuple(edges) + (n,)


def _inv_freq(case):
    """Rotary frequencies of the case's scheme, radians per position (64 bits), and the factor on cos and sin."""
    rot, base = case["rot"], 500000.0
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if case["scaling"] == "linear":
        return [v / 4.0 for v in f], 1.0
    if case["scaling"] == "llama3":  # factor 32, low 1, high 4, trained length 8192
        out = []
        for v in f:
            turns = 8192.0 * v / (2.0 * math.pi)
            smooth = min(1.0, max(0.0, (turns - 1.0) / (4.0 - 1.0)))
            out.append((1.0 - smooth) * v / 32.0 + smooth * v)
        return out, 1.0
    if case["scaling"] == "yarn":  # factor 16, beta 32 and 1, trained length 8192
        def dim(turns):
            return rot * math.log(8192.0 / (turns * 2.0 * math.pi)) / (2.0 * math.log(base))
        lo, hi = max(math.floor(dim(32.0)), 0), min(math.ceil(dim(1.0)), rot - 1)
        out = []
        for i, v in enumerate(f):
            ramp = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            out.append(v / 16.0 * ramp + v * (1.0 - ramp))
        return out, 0.1 * math.log(16.0) + 1.0
    return f, 1.0


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def uniform(n):
        return torch.rand(n, generator=g, device="cuda")

    if case["op"] == "lora":
        rows, n, r, k = case["rows"], case["adapters"], case["rank"], case["k"]
        wt = DTYPES[case["w"]]
        ids = torch.arange(rows, device="cuda") % n
        ids = ids.sort().values if case["order"] == "runs" else ids[torch.randperm(rows, generator=g, device="cuda")]
        if rows >= 16:
            ids[5::16] = -1  # requests of the base model
        return {"case": case, "x": normal(rows, k).to(DTYPES[case["x"]]),
                "a": (normal(n, case["segs"] * r, k) / math.sqrt(k)).to(wt), "b": (normal(n, case["n"], r) / math.sqrt(r)).to(wt),
                "ids": ids.to(torch.int32), "scales": 0.5 + uniform(n), "y": normal(rows, case["n"]).to(DTYPES[case["y"]]),
                "segs": _segments(case)}
    if case["op"] == "rope":
        t, hq, hk, hd, dt = case["tokens"], case["hq"], case["hk"], case["hd"], DTYPES[case["dtype"]]
        if case["fused"]:  # q and k are views of a fused q|k|v buffer
            qkv = normal(t, hq + 2 * hk, hd).to(dt)
            q, k = qkv[:, :hq], qkv[:, hq:hq + hk]
        else:
            q, k = normal(t, hq, hd).to(dt), normal(t, hk, hd).to(dt)
        freq, factor = _inv_freq(case)
        pos = torch.randint(0, case["far"], (t,), generator=g, device="cuda", dtype=torch.int32)
        return {"case": case, "q": q, "k": k, "pos": pos, "factor": factor,
                "freq": torch.tensor(freq, dtype=torch.float64, device="cuda")}
    rows, v, mix = case["rows"], case["vocab"], case["mix"]
    logits = torch.full((rows, v + case["pad"]), 1e30, device="cuda")[:, :v]
    logits.copy_(case["spread"] * normal(rows, v))
    if mix == "mixed":  # every fourth request is held to a grammar: half of the tokens are closed
        logits[1::4].masked_fill_(torch.rand(v, generator=g, device="cuda") < 0.5, -math.inf)
    s = {"case": case, "logits": logits, "u": uniform(rows), "tokens": torch.empty(rows, dtype=torch.int32, device="cuda"),
         "temperature": None, "top_k": None, "top_p": None, "min_p": None}
    if mix == "paper":  # temperature 0.8, top-k over 10 tokens
        s["temperature"] = torch.full((rows,), 0.8, device="cuda")
        s["top_k"] = torch.full((rows,), 10, dtype=torch.int32, device="cuda")
    elif mix != "plain":
        s["temperature"] = 0.5 + uniform(rows)
    if mix in ("mixed", "top_p"):
        s["top_p"] = 0.8 + 0.2 * uniform(rows)
    if mix in ("mixed", "min_p"):
        s["min_p"] = 0.1 * uniform(rows)
    if mix == "mixed":  # a third of the requests each: no top-k, some tens, some thousands; some greedy
        kind = torch.randint(0, 3, (rows,), generator=g, device="cuda")
        k = torch.where(kind == 0, 0, torch.where(kind == 1, 5 + (95 * uniform(rows)).int(), 1000 + (4000 * uniform(rows)).int()))
        s["top_k"] = k.to(torch.int32)
        s["min_p"] = torch.where(uniform(rows) < 0.5, 0.0, s["min_p"])
        s["temperature"] = torch.where(uniform(rows) < 0.1, 0.0, s["temperature"])
    return s


# ------------------------------------------------------------------ the operators
def run(state):
    case = state["case"]
    if own:
        import paper_2410_12513_b200 as lib
        if case["op"] == "lora":
            lib.first_lora(state["x"], state["a"], state["b"], state["ids"], state["y"], scales=state["scales"], segments=state["segs"])
            return state["y"]
        if case["op"] == "rope":
            lib.first_rope(state["q"], state["k"], state["pos"], state["freq"], factor=state["factor"],
                           interleaved=case["layout"] == "interleaved")
            return {"q": state["q"], "k": state["k"]}
        lib.first_sample(state["logits"], state["u"], state["tokens"], temperature=state["temperature"], top_k=state["top_k"],
                         top_p=state["top_p"], min_p=state["min_p"])
        return state["tokens"]
    return {"lora": _plain_lora, "rope": _plain_rope, "sample": _plain_sample}[case["op"]](state)


def _plain_lora(s):
    """y[r] += scale * B (A x[r]) with the adapter of row r; each output feature takes its own segment's part of A x."""
    live = s["ids"] >= 0
    a = s["ids"].clamp(min=0).long()
    rank = s["b"].shape[2]
    h = torch.bmm(s["a"][a].float(), s["x"].float()[:, :, None])[:, :, 0]  # [rows][segments * rank]
    seg = torch.bucketize(torch.arange(s["y"].shape[1], device="cuda"), torch.tensor(s["segs"][1:-1], device="cuda"), right=True)
    h = h.view(h.shape[0], -1, rank) * (s["scales"][a] * live)[:, None, None]
    b = s["b"][a].float()
    per = torch.bmm(b, h.transpose(1, 2))  # [rows][n][segments]: every segment's part, of which each feature takes one
    delta = per.gather(2, seg[None, :, None].expand(per.shape[0], -1, 1))[:, :, 0]
    s["y"].copy_(s["y"].float() + delta)
    return s["y"]


def _plain_rope(s):
    case, rot = s["case"], s["case"]["rot"]
    angle = s["pos"].double()[:, None, None] * s["freq"]  # in 64 bits: positions reach a million
    c, sn = (s["factor"] * torch.cos(angle)).float(), (s["factor"] * torch.sin(angle)).float()
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if case["layout"] == "interleaved" else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = s["q"][:, :, first].float(), s["q"][:, :, second].float()
    s["q"][:, :, first], s["q"][:, :, second] = (a * c - b * sn).to(s["q"].dtype), (b * c + a * sn).to(s["q"].dtype)
    a, b = s["k"][:, :, first].float(), s["k"][:, :, second].float()
    s["k"][:, :, first], s["k"][:, :, second] = (a * c - b * sn).to(s["k"].dtype), (b * c + a * sn).to(s["k"].dtype)
    return {"q": s["q"], "k": s["k"]}


def _plain_sample(s):
    """Candidates in descending order, equal logits by index; every filter keeps a prefix of that order."""
    x = s["logits"].float() + 0.0
    rows, v = x.shape
    x, order = torch.sort(x, dim=1, descending=True, stable=True)
    x = x.double()  # cumulative weights decide which token a draw falls on: 64 bits
    t = s["temperature"].double() if s["temperature"] is not None else torch.ones(rows, dtype=torch.float64, device="cuda")
    greedy = t <= 0
    w = torch.exp((x - x[:, :1]) / torch.where(greedy, 1.0, t)[:, None])
    keep = x > -math.inf
    if s["top_k"] is not None:
        k = torch.where(s["top_k"] > 0, s["top_k"].long(), v)
        keep &= torch.arange(v, device="cuda") < k[:, None]
    if s["min_p"] is not None:
        keep &= w >= s["min_p"].double()[:, None]
    w = w * keep
    cum = torch.cumsum(w, 1)
    if s["top_p"] is not None:
        keep &= (cum - w < s["top_p"].double()[:, None] * cum[:, -1:]) | (s["top_p"] >= 1)[:, None]
        w = w * keep
        cum = torch.cumsum(w, 1)
    over = keep & (cum > s["u"].double()[:, None] * cum[:, -1:])
    at = torch.where(greedy, 0, over.to(torch.int8).argmax(1))
    s["tokens"].copy_(order.gather(1, at[:, None])[:, 0])
    return s["tokens"]


def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["op"] == "lora":
        rows, n, r, k = case["rows"], case["n"], case["rank"], case["k"]
        live = rows - (len(range(5, rows, 16)) if rows >= 16 else 0)
        used = min(case["adapters"], live)
        return {"bytes": live * k * size[case["x"]] + 2 * live * n * size[case["y"]] + 4 * rows
                + used * (case["segs"] * r * k + n * r) * size[case["w"]],
                "flops": 2 * live * r * (case["segs"] * k + n)}
    if case["op"] == "rope":
        values = case["tokens"] * (case["hq"] + case["hk"]) * case["rot"]
        return {"bytes": 2 * values * size[case["dtype"]] + 4 * case["tokens"], "flops": 3 * values}
    return {"bytes": 4 * case["rows"] * (case["vocab"] + 2), "flops": 4 * case["rows"] * case["vocab"]}


# ------------------------------------------------------------------ 64 bits, from the definitions
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "lora":
        y, rank, segs = s["y"].double(), case["rank"], s["segs"]
        for a in range(case["adapters"]):
            rows = (s["ids"] == a).nonzero()[:, 0]
            if rows.numel() == 0:
                continue
            x = s["x"][rows].double()
            for j in range(case["segs"]):
                h = x @ s["a"][a, j * rank:(j + 1) * rank].double().T
                y[rows, segs[j]:segs[j + 1]] += float(s["scales"][a]) * (h @ s["b"][a, segs[j]:segs[j + 1]].double().T)
        return y
    if case["op"] == "rope":
        rot, out = case["rot"], {}
        turn = torch.polar(torch.full((1, 1), float(s["factor"]), dtype=torch.float64, device="cuda"),
                           s["pos"].double()[:, None] * s["freq"][None, :])[:, None, :]  # factor * e^(i pos w)
        for name in ("q", "k"):
            x = s[name].double().clone()
            if case["layout"] == "interleaved":
                z = torch.view_as_complex(x[..., :rot].reshape(*x.shape[:2], rot // 2, 2).contiguous()) * turn
                x[..., :rot] = torch.view_as_real(z).reshape(*x.shape[:2], rot)
            else:
                z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * turn
                x[..., :rot // 2], x[..., rot // 2:rot] = z.real, z.imag
            out[name] = x
        return out
    logits, u = s["logits"].cpu().numpy().astype(np.float64), s["u"].cpu().numpy().astype(np.float64)
    get = {k: None if s[k] is None else s[k].cpu().numpy().astype(np.float64) for k in ("temperature", "top_k", "top_p", "min_p")}
    tokens = np.empty(case["rows"], dtype=np.int32)
    for r in range(case["rows"]):
        x = logits[r]
        order = np.lexsort((np.arange(x.size), -x))
        temp = 1.0 if get["temperature"] is None else get["temperature"][r]
        if temp <= 0:
            tokens[r] = order[0]
            continue
        order = order[x[order] > -np.inf]
        if get["top_k"] is not None and get["top_k"][r] > 0:
            order = order[:int(get["top_k"][r])]
        w = np.exp((x[order] - x[order[0]]) / temp)
        if get["min_p"] is not None:
            w = w[w >= get["min_p"][r]]
        if get["top_p"] is not None and get["top_p"][r] < 1:
            before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
            w = w[before < get["top_p"][r] * w.sum()]
        cum = np.cumsum(w)
        tokens[r] = order[min(int(np.searchsorted(cum, u[r] * cum[-1], side="right")), w.size - 1)]
    return torch.from_numpy(tokens)
