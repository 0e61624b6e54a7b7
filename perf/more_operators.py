"""What is measured of the paged 8-bit cache and of drafted tokens: writing keys and values into pages and reading them
back (``first_append8``, ``first_read8``), attention over the pages (``first_attn8``), moving pages
(``first_copy_pages``) and the verification of drafts (``first_verify``).

``run`` computes an operator in plain torch operations, or, with ``own``, through the library's calls.  ``exact`` gives
the same results in 64 bits, written apart from the plain form."""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
FORMATS = {"int8": (torch.int8, 127.0), "e4m3": (torch.float8_e4m3fn, 448.0)}


# ------------------------------------------------------------------ cases
def _attn(name, seqs, lo, hi, new, hkv, group, hd, page, fmt, dtype):
    return {"name": name, "op": "attn", "seqs": seqs, "lo": lo, "hi": hi, "new": new, "hkv": hkv, "group": group, "hd": hd,
            "page": page, "fmt": fmt, "dtype": dtype}


def _append(name, seqs, lo, hi, new, hkv, hd, page, fmt, dtype, out):
    return {"name": name, "op": "append", "seqs": seqs, "lo": lo, "hi": hi, "new": new, "hkv": hkv, "hd": hd, "page": page,
            "fmt": fmt, "dtype": dtype, "out": out}


def _copy(name, layers, pages, moves, hkv, hd, page, order):
    return {"name": name, "op": "copy", "layers": layers, "pages": pages, "moves": moves, "hkv": hkv, "hd": hd, "page": page,
            "order": order}


def _verify(name, seqs, drafts, vocab, pad, kind, draft, spread):
    return {"name": name, "op": "verify", "seqs": seqs, "drafts": drafts, "vocab": vocab, "pad": pad, "kind": kind,
            "draft": draft, "spread": spread}


def listed():
    return [
        # one answer in progress at the 8B shape's heads: latency
        _attn("attn_1x700", 1, 700, 700, 1, 8, 4, 128, 64, "int8", "f32"),
        # a decode batch of 32 sequences of all lengths
        _attn("attn_32_mixed", 32, 300, 8192, 1, 8, 4, 128, 64, "int8", "bf16"),
        # five drafted tokens and the one before them, 16 sequences, the 3B shape's heads, small pages
        _attn("attn_16x6_drafts", 16, 45, 6001, 6, 8, 3, 128, 16, "e4m3", "bf16"),
        # one very long sequence
        _attn("attn_1x131072", 1, 131072, 131072, 1, 8, 4, 128, 64, "e4m3", "bf16"),
        # the largest decode batch
        _attn("attn_128_mixed", 128, 1024, 8192, 1, 8, 4, 128, 32, "int8", "f32"),
        # the new token of 32 sequences, into pages that hold some already
        _append("append_32x1", 32, 40, 5000, 1, 8, 128, 64, "int8", "bf16", "f32"),
        # the prompts of four requests
        _append("append_prompts", 4, 0, 0, 8190, 8, 128, 64, "e4m3", "bf16", "bf16"),
        # forked sequences take copies of their last pages, in every layer
        _copy("copy_forks", 32, 64, 64, 8, 128, 64, "mixed"),
        # a pool with holes is closed up
        _copy("copy_compact", 32, 480, 5120, 8, 128, 64, "down"),
        # one answer, four drafts of a smaller model
        _verify("verify_1x4", 1, 4, 128256, 0, "logits", "model", 2.5),
        # drafts looked up in the prompt (no model's probabilities), a vocabulary of odd size in padded rows
        _verify("verify_24x5_lookup", 24, 5, 50257, 46, "logits", "none", 8.0),
        # a large batch with a draft model
        _verify("verify_64x7", 64, 7, 128256, 0, "logits", "model", 2.5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "append", "copy", "verify"])
    if op == "attn":
        hkv, hd, new = rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 128]), rng.choice([1, 1, 1, 2, 5, 8])
        seqs = _log(rng, 1, 128)
        hi = _log(rng, max(16, new), min(131072, max(64, 128 * 4600 * 8 * 128 // (seqs * hkv * hd * 2))))
        case = _attn("", seqs, max(new, rng.randint(1, hi)), hi, new, hkv, rng.choice([1, 2, 3, 4, 8]), hd,
                     rng.choice([16, 32, 64, 128]), rng.choice(["int8", "e4m3"]), rng.choice(["bf16", "f32"]))
    elif op == "append":
        hkv, hd, seqs = rng.choice([1, 2, 4, 8]), rng.choice([32, 64, 128, 128]), _log(rng, 1, 128)
        hi = rng.choice([0, _log(rng, 1, 8192)])
        case = _append("", seqs, rng.randint(0, hi), hi, rng.choice([1, 1, 3, 8, _log(rng, 9, max(10, 32768 // seqs))]), hkv,
                       hd, rng.choice([16, 32, 64, 128]), rng.choice(["int8", "e4m3"]), rng.choice(["bf16", "f32"]),
                       rng.choice(["bf16", "f32"]))
    elif op == "copy":
        layers, hkv, page = rng.choice([1, 8, 16, 32]), rng.choice([1, 2, 8]), rng.choice([16, 32, 64, 128])
        hd = rng.choice([32, 64, 128])
        pages = _log(rng, 24, min(4096, 32 * 480 * 8 * 64 * 128 // (layers * hkv * page * hd)))
        case = _copy("", layers, pages, _log(rng, 1, max(2, layers * pages // 3)), hkv, hd, page, rng.choice(["mixed", "down"]))
    else:
        vocab, seqs = _log(rng, 500, 128256), _log(rng, 1, 64)
        draft = rng.choice(["model", "model", "none"])
        case = _verify("", seqs, rng.randint(1, 7), vocab, rng.choice([0, 0, 1, 46]), rng.choice(["logits", "logits", "probs"]),
                       draft, 8.0 if draft == "none" else rng.uniform(1.0, 4.0))
    return {k: v for k, v in case.items() if k != "name"}


# ------------------------------------------------------------------ inputs
def _spread(n, lo, hi):
    """n whole numbers from lo to hi, spread evenly and out of order."""
    if n == 1:
        return [hi]
    return [lo + int((hi - lo) * math.modf(0.5 + i * 0.6180339887498949)[0] + 0.5) for i in range(n - 1)] + [hi]


def _counts(case):
    """(tokens before, new tokens) of every sequence: the last sequences bring fewer new ones."""
    n = [max(1, case["new"] - (b % 3 if case["new"] > 1 else 0)) for b in range(case["seqs"])]
    total = _spread(case["seqs"], case["lo"], case["hi"])
    if case["op"] == "attn":  # lo and hi are the lengths with the new ones
        n = [min(a, t) for a, t in zip(n, total)]
        return [t - a for a, t in zip(n, total)], n
    return total, n


def _edges(n):
    return [0] + np.cumsum(n).tolist()


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _cache(g, n_pages, case):
    """Pages full of values, as they are after some use: what lies behind a sequence's last token is old."""
    dt, _ = FORMATS[case["fmt"]]
    shape = (n_pages, case["hkv"], case["page"], case["hd"])
    out = []
    for _ in range(2):
        x = torch.empty(shape, dtype=dt, device="cuda")
        for p in range(0, n_pages, 1024):
            r = torch.randn((min(1024, n_pages - p),) + shape[1:], generator=g, device="cuda")
            x[p:p + 1024] = (r * 36).round().clamp(-127, 127).to(dt) if case["fmt"] == "int8" else (r * 100).clamp(-448, 448).to(dt)
        unit = 1 / 36 if case["fmt"] == "int8" else 1 / 100
        out += [x, (0.5 + torch.rand((n_pages, case["hkv"]), generator=g, device="cuda")) * unit]
    return {"k": out[0], "k_scale": out[1], "v": out[2], "v_scale": out[3]}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    if case["op"] in ("attn", "append"):
        page, hd, hkv = case["page"], case["hd"], case["hkv"]
        before, n = _counts(case)
        need = [(a + b + page - 1) // page for a, b in zip(before, n)]
        width, n_pages = max(need), sum(need) + 3
        ids = torch.randperm(n_pages, generator=g, device="cuda").int()
        pages = torch.full((case["seqs"], width), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, c in enumerate(need):
            pages[b, :c] = ids[at:at + c]
            at += c
        s = {"case": case, "pages": pages, "len": _i32(before), "cu": _i32(_edges(n)), "max_new": max(n)} | _cache(g, n_pages, case)
        dt = DTYPES[case["dtype"]]
        if case["op"] == "attn":
            s["q"] = normal(sum(n), hkv * case["group"], hd).to(dt)
            s["out"] = torch.empty_like(s["q"])
            s["scale"] = 1.0 / math.sqrt(hd)
        else:
            s["k_new"], s["v_new"] = normal(sum(n), hkv, hd).to(dt), normal(sum(n), hkv, hd).to(dt)
            s["k_new"][:, :, ::16] *= 4.0  # keys have a few large channels
            start = [a // page * page for a in before]  # the first page that is written
            rows = [a + b - c for a, b, c in zip(before, n, start)]
            s |= {"start": _i32(start), "cu_read": _i32(_edges(rows)), "max_rows": max(rows)}
            s["k_out"], s["v_out"] = (torch.empty((sum(rows), hkv, hd), dtype=DTYPES[case["out"]], device="cuda") for _ in "kv")
        if own:
            import paper_2410_12513_b200 as lib
            s["cache"] = lib.Cache8(s["k"], s["v"], s["k_scale"], s["v_scale"])
        return s
    if case["op"] == "copy":
        layers, n, hkv = case["layers"], case["pages"], case["hkv"]
        shape = (layers, n, hkv, case["page"], case["hd"])
        k, v = (torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int8) for _ in "kv")
        ks, vs = (torch.rand(shape[:3], generator=g, device="cuda") for _ in "kv")
        per = [case["moves"] // layers + (l < case["moves"] % layers) for l in range(layers)]
        moves = []
        for l, m in enumerate(per):
            if case["order"] == "down":  # the last pages in use go to holes further down
                holes = torch.randperm(n - m, generator=g, device="cuda")[:m]
                src = torch.arange(n - m, n, device="cuda")
            else:
                both = torch.randperm(n, generator=g, device="cuda")
                src, holes = both[:m], both[m:2 * m]
            moves.append(torch.stack([torch.full((m,), l, device="cuda"), src, holes], 1))
        s = {"case": case, "k": k, "v": v, "k_scale": ks, "v_scale": vs, "moves": torch.cat(moves).int().contiguous(), "per": per}
        if own:
            import paper_2410_12513_b200 as lib
            s["caches"] = [lib.Cache8(*t) for t in zip(k, v, ks, vs)]
        return s
    seqs, kk, v = case["seqs"], case["drafts"], case["vocab"]
    target = torch.full((seqs, kk + 1, v + case["pad"]), 1e30, device="cuda")[:, :, :v]
    target.copy_(case["spread"] * normal(seqs, kk + 1, v))
    temperature = 0.6 + 0.6 * torch.rand(seqs, generator=g, device="cuda")
    draft = None
    if case["draft"] == "model":
        draft = torch.empty((seqs, kk, v + case["pad"]), device="cuda")[:, :, :v]
        draft.copy_(target[:, :kk] + 0.5 * normal(seqs, kk, v))
        noise = -torch.log(-torch.log(torch.rand(seqs, kk, v, generator=g, device="cuda").clamp(1e-7, 1 - 1e-6)))
        tokens = (draft / temperature[:, None, None] + noise).argmax(-1)  # drawn from the draft's distribution
    else:
        tokens = target[:, :kk].argmax(-1)
        tokens = torch.where(torch.rand(seqs, kk, generator=g, device="cuda") < 0.2, (tokens + 7) % v, tokens)
    stop = torch.rand(seqs, generator=g, device="cuda")
    if kk > 1:  # some sequences have fewer drafts
        tokens = torch.where((torch.arange(kk, device="cuda") > 0) & (stop < 0.2)[:, None] & (torch.arange(kk, device="cuda") >= kk - 1), -1, tokens)
    if seqs > 4:
        temperature[4::5] = 0.0  # greedy requests
    if case["kind"] == "probs":
        t = torch.where(temperature > 0, temperature, 0.05)[:, None, None]
        target.copy_(torch.softmax(target / t, -1))
        if draft is not None:
            draft.copy_(torch.softmax(draft / t, -1))
        temperature = None
    return {"case": case, "target": target, "draft": draft, "drafted": tokens.int().contiguous(), "temperature": temperature,
            "u": torch.rand(seqs, kk, generator=g, device="cuda"), "draws": torch.rand(seqs, generator=g, device="cuda"),
            "tokens": torch.empty((seqs, kk + 1), dtype=torch.int32, device="cuda"),
            "accepted": torch.empty(seqs, dtype=torch.int32, device="cuda")}


# ------------------------------------------------------------------ the operators
def run(s):
    case = s["case"]
    if own:
        import paper_2410_12513_b200 as lib
        if case["op"] == "attn":
            lib.first_attn8(s["q"], s["cache"], s["pages"], s["len"], s["out"], scale=s["scale"], cu_new=s["cu"], max_new=s["max_new"])
            return s["out"]
        if case["op"] == "append":
            lib.first_append8(s["k_new"], s["v_new"], s["cache"], s["pages"], s["len"], cu_new=s["cu"], max_new=s["max_new"])
            lib.first_read8(s["cache"], s["pages"], s["start"], s["k_out"], s["v_out"], cu=s["cu_read"], max_rows=s["max_rows"])
            return {"k": s["k_out"], "v": s["v_out"]}
        if case["op"] == "copy":
            lib.first_copy_pages(s["caches"], s["moves"])
            return {n: s[n] for n in ("k", "v", "k_scale", "v_scale")}
        lib.first_verify(s["target"], s["drafted"], s["u"], s["draws"], s["tokens"], s["accepted"], draft=s["draft"],
                         temperature=s["temperature"], probs=case["kind"] == "probs")
        return {"tokens": s["tokens"], "accepted": s["accepted"]}
    return {"attn": _plain_attn, "append": _plain_append, "copy": _plain_copy, "verify": _plain_verify}[case["op"]](s)


def _pick(x, ids):
    """Pages of a cache (8-bit floats move as bytes)."""
    return x[ids] if x.dtype == torch.int8 else x.view(torch.int8)[ids].view(x.dtype)


def _plain_attn(s):
    case, page, hkv, hd, grp = s["case"], s["case"]["page"], s["case"]["hkv"], s["case"]["hd"], s["case"]["group"]
    seqs, new = case["seqs"], s["max_new"]
    n = s["cu"][1:] - s["cu"][:-1]
    slot = torch.arange(new, device="cuda")
    rows = (s["cu"][:-1, None] + torch.minimum(slot, n[:, None] - 1)).long()  # rows behind a sequence's last repeat it
    q = s["q"][rows].float().view(seqs, new, hkv, grp, hd)
    ids = s["pages"].clamp(min=0).long()
    out = torch.empty((seqs, new, hkv, grp, hd), device="cuda")
    at = torch.arange(ids.shape[1] * page, device="cuda")
    seen = at[None, None, :] <= (s["len"][:, None] + torch.minimum(slot, n[:, None] - 1))[:, :, None]  # [seqs][new][tokens]
    step = max(1, (1 << 26) // (ids.shape[1] * page * hkv * hd))
    for b in range(0, seqs, step):  # a few sequences at a time: the values in 32 bits take four times the room
        e = slice(b, b + step)
        k = (_pick(s["k"], ids[e]).float() * s["k_scale"][ids[e]][..., None, None]).transpose(1, 2).reshape(-1, hkv, at.numel(), hd)
        v = (_pick(s["v"], ids[e]).float() * s["v_scale"][ids[e]][..., None, None]).transpose(1, 2).reshape(-1, hkv, at.numel(), hd)
        z = q[e].permute(0, 2, 1, 3, 4).reshape(-1, hkv, new * grp, hd) @ k.transpose(2, 3) * s["scale"]
        z = z.view(-1, hkv, new, grp, at.numel()).masked_fill(~seen[e][:, None, :, None, :], -math.inf)
        z = torch.exp(z - z.amax(-1, keepdim=True))
        z = z / z.sum(-1, keepdim=True)
        o = z.view(-1, hkv, new * grp, at.numel()) @ v
        out[e] = o.view(-1, hkv, new, grp, hd).permute(0, 2, 1, 3, 4)
    s["out"][rows.view(-1)] = out.view(seqs * new, hkv * grp, hd).to(s["out"].dtype)
    return s["out"]


def _to_e4m3(y):
    """The nearest 8-bit float (3 bits of mantissa, smallest exponent -6, largest value 448), ties to even, of 64-bit values."""
    y = y.clamp(-448.0, 448.0)
    e = torch.frexp(y)[1].clamp(min=-5).double() - 4.0  # y in [2^(e+3), 2^(e+4))
    step = torch.exp2(e)
    return (torch.round(y / step) * step).float().to(torch.float8_e4m3fn)


def _plain_append(s):
    case, page, seqs = s["case"], s["case"]["page"], s["case"]["seqs"]
    dt, top = FORMATS[case["fmt"]]
    n = s["cu"][1:] - s["cu"][:-1]
    first, last = s["len"] // page, (s["len"] + n - 1) // page
    j = torch.arange((s["max_new"] + page - 2) // page + 1, device="cuda")
    idx = torch.minimum(first[:, None] + j, last[:, None]).long()  # [seqs][pages]; those behind the last repeat it
    ids = s["pages"].gather(1, idx).long()
    pos = idx[:, :, None] * page + torch.arange(page, device="cuda")  # [seqs][pages][page]
    old = pos < s["len"][:, None, None]
    new = ~old & (pos < (s["len"] + n)[:, None, None])
    row = torch.where(new, s["cu"][:-1, None, None] + pos - s["len"][:, None, None], 0)
    for name in "kv":
        x = s[name + "_new"][row].permute(0, 1, 3, 2, 4).float()  # [seqs][pages][heads][page][hd]
        held, before = _pick(s[name], ids), s[name + "_scale"][ids]
        here = new[:, :, None, :, None]
        amax = torch.where(here, x, 0.0).abs().amax((3, 4))
        kept = torch.where(old.any(2)[:, :, None], before, 0.0)
        scale = torch.maximum(kept, amax / top)
        unit = torch.where(scale > 0, scale, 1.0).double()[..., None, None]  # in 64 bits: quotients next to a half
        was = held.double() if dt == torch.int8 else held.float().double()
        y = torch.where(here, x.double() / unit, was * kept.double()[..., None, None] / unit)
        grown = torch.round(y).clamp(-127, 127).to(dt) if dt == torch.int8 else _to_e4m3(y)
        keep = ~(old | new)[:, :, None, :, None]
        byte = torch.where(keep, held.view(torch.int8), grown.view(torch.int8))
        s[name].view(torch.int8)[ids] = byte
        s[name + "_scale"][ids] = scale
    # read back, as values
    rows = s["cu_read"][1:] - s["cu_read"][:-1]
    at = torch.arange(s["k_out"].shape[0], device="cuda")
    b = torch.bucketize(at, s["cu_read"][1:].long(), right=True)
    t = s["start"][b].long() + at - s["cu_read"][b]
    p = s["pages"][b, t // page].long()
    for name in "kv":
        val = s[name].view(torch.int8)[p, :, t % page].view(dt).float() * s[name + "_scale"][p][..., None]
        s[name + "_out"].copy_(val.to(s[name + "_out"].dtype))
    return {"k": s["k_out"], "v": s["v_out"]}


def _plain_copy(s):
    at = 0
    for l, m in enumerate(s["per"]):
        src, dst = s["moves"][at:at + m, 1].long(), s["moves"][at:at + m, 2].long()
        at += m
        for name in ("k", "v", "k_scale", "v_scale"):
            s[name][l, dst] = s[name][l, src]
    return {n: s[n] for n in ("k", "v", "k_scale", "v_scale")}


def _plain_probs(x, s):
    """Probabilities in 64 bits: which token a draw falls on hangs on their sums."""
    if s["temperature"] is None:
        return x.double()
    t = s["temperature"].double()[:, None, None]
    z = (x.double() - x.amax(-1, keepdim=True).double()) / torch.where(t > 0, t, 1.0)
    w = torch.exp(z)
    w = w / w.sum(-1, keepdim=True)
    hot = torch.arange(x.shape[-1], device="cuda") == x.argmax(-1, keepdim=True)
    return torch.where(t > 0, w, hot.double())


def _plain_verify(s):
    seqs, kk, v = s["case"]["seqs"], s["case"]["drafts"], s["case"]["vocab"]
    d = s["drafted"].long()
    there = torch.cumprod(((d >= 0) & (d < v)).int(), 1).bool()
    d = d.clamp(0, v - 1)
    p = _plain_probs(s["target"], s)
    pd = p[:, :kk].gather(2, d[:, :, None])[:, :, 0]
    if s["draft"] is not None:
        q = _plain_probs(s["draft"], s)
        qd = q.gather(2, d[:, :, None])[:, :, 0]
    else:
        qd = torch.ones_like(pd)
    run_ = torch.cumprod((there & (s["u"].double() * qd < pd)).int(), 1)
    a = run_.sum(1)
    b = torch.arange(seqs, device="cuda")
    row, at = p[b, a], a.clamp(max=kk - 1)
    less = q[b, at] if s["draft"] is not None else (torch.arange(v, device="cuda") == d[b, at][:, None]).double()
    refused = (a < kk) & there[b, at]
    left = torch.clamp(row - torch.where(refused[:, None], less, 0.0), min=0.0)
    left = torch.where(left.sum(1, keepdim=True) > 0, left, row)
    cum = torch.cumsum(left, 1)
    new = (cum > s["draws"].double()[:, None] * cum[:, -1:]).to(torch.int8).argmax(1)
    slot = torch.arange(kk + 1, device="cuda")
    out = torch.where(slot < a[:, None], torch.cat([d, d[:, :1]], 1), torch.where(slot == a[:, None], new[:, None], -1))
    s["tokens"].copy_(out)
    s["accepted"].copy_(a)
    return {"tokens": s["tokens"], "accepted": s["accepted"]}


def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["op"] == "attn":
        before, n = _counts(case)
        total = sum(before) + sum(n)
        hq = case["hkv"] * case["group"]
        seen = sum(a * b + a * (a + 1) // 2 for a, b in zip(n, before))
        blocks = sum((a + b + case["page"] - 1) // case["page"] for a, b in zip(before, n))
        return {"bytes": 2 * total * case["hkv"] * case["hd"] + 2 * sum(n) * hq * case["hd"] * size[case["dtype"]]
                + blocks * (8 * case["hkv"] + 4), "flops": 4 * seen * hq * case["hd"]}
    if case["op"] == "append":
        before, n = _counts(case)
        row = 2 * case["hkv"] * case["hd"]
        read = sum(n) + sum(a % case["page"] for a in before)
        return {"bytes": row * (sum(n) * (size[case["dtype"]] + 1) + read * (1 + size[case["out"]])), "flops": 4 * row * sum(n)}
    if case["op"] == "copy":
        return {"bytes": case["moves"] * (4 * case["hkv"] * (case["page"] * case["hd"] + 4) + 12), "flops": 0}
    rows = case["seqs"] * (2 * case["drafts"] + 1 if case["draft"] == "model" else case["drafts"] + 1)
    if case["kind"] == "probs":  # one row of each side, and the drafted tokens' entries
        rows = case["seqs"] * (2 if case["draft"] == "model" else 1)
    return {"bytes": 4 * rows * case["vocab"], "flops": 4 * rows * case["vocab"]}


# ------------------------------------------------------------------ 64 bits, from the definitions
def _nearest_e4m3(y):
    """By search among the 127 values from 0 to 448: the nearest one, the even code of two that are as near."""
    codes = torch.arange(127, dtype=torch.uint8, device=y.device)
    values = codes.view(torch.float8_e4m3fn).double()
    mag = y.abs().clamp(max=448.0).contiguous()
    hi = torch.searchsorted(values, mag).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, down = values[hi] - mag, mag - values[lo]
    take = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return values[take] * torch.sign(y)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attn":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        cu, before, page, grp = s["cu"].tolist(), s["len"].tolist(), case["page"], case["group"]
        for b in range(case["seqs"]):
            total = before[b] + cu[b + 1] - cu[b]
            ids = s["pages"][b, :(total + page - 1) // page].long()
            for h in range(case["hkv"]):
                k = (s["k"][:, h].view(torch.int8)[ids].view(s["k"].dtype).to(torch.float32).double()
                     * s["k_scale"][ids, h].double()[:, None, None]).reshape(-1, case["hd"])[:total]
                v = (s["v"][:, h].view(torch.int8)[ids].view(s["v"].dtype).to(torch.float32).double()
                     * s["v_scale"][ids, h].double()[:, None, None]).reshape(-1, case["hd"])[:total]
                for i, r in enumerate(range(cu[b], cu[b + 1])):
                    m = before[b] + i + 1
                    z = s["q"][r, h * grp:(h + 1) * grp].double() @ k[:m].T * s["scale"]
                    out[r, h * grp:(h + 1) * grp] = torch.softmax(z, -1) @ v[:m]
        return out
    if case["op"] == "append":
        cu, before, page, top = s["cu"].tolist(), s["len"].tolist(), case["page"], FORMATS[case["fmt"]][1]
        out = {}
        for name in "kv":
            parts, fresh, held, sc = [], s[name + "_new"].double(), s[name], s[name + "_scale"]
            for b in range(case["seqs"]):
                end = before[b] + cu[b + 1] - cu[b]
                for first in range(before[b] // page * page, end, page):
                    p = int(s["pages"][b, first // page])
                    n_old = min(max(before[b] - first, 0), page)
                    lo = max(first, before[b])
                    x = fresh[cu[b] + lo - before[b]:cu[b] + min(first + page, end) - before[b]].transpose(0, 1)  # [heads][new][hd]
                    scale = (x.abs().amax((1, 2)).float() / top).double()
                    if n_old:
                        scale = torch.maximum(scale, sc[p].double())
                    old = held[p, :, :n_old].float().double() * sc[p].double()[:, None, None]
                    y = torch.cat([old, x], 1) / scale[:, None, None]
                    y = torch.round(y) if case["fmt"] == "int8" else _nearest_e4m3(y)
                    parts.append((y * scale[:, None, None]).transpose(0, 1))
            out[name] = torch.cat(parts)
        return out
    if case["op"] == "copy":
        out = {n: s[n].clone() for n in ("k", "v", "k_scale", "v_scale")}
        for l, src, dst in s["moves"].tolist():
            for n in out:
                out[n][l, dst].copy_(s[n][l, src])
        return out
    kk, v = case["drafts"], case["vocab"]
    tokens, accepted = np.full((case["seqs"], kk + 1), -1, dtype=np.int32), np.zeros(case["seqs"], dtype=np.int32)
    temp = None if s["temperature"] is None else s["temperature"].tolist()

    def probs(x, b):
        x = x.cpu().numpy().astype(np.float64)
        if temp is None:
            return x
        if temp[b] <= 0:
            return (np.arange(v) == np.argmax(x)).astype(np.float64)
        w = np.exp((x - x.max()) / np.float64(temp[b]))
        return w / w.sum()
    for b in range(case["seqs"]):
        drafted, u = s["drafted"][b].tolist(), s["u"][b].tolist()
        for i in range(kk + 1):
            left = probs(s["target"][b, i], b)
            if i < kk and 0 <= drafted[i] < v:
                q = probs(s["draft"][b, i], b) if s["draft"] is not None else (np.arange(v) == drafted[i]).astype(np.float64)
                if u[i] * q[drafted[i]] < left[drafted[i]]:
                    tokens[b, i] = drafted[i]
                    continue
                rest = np.maximum(left - q, 0.0)
                left = rest if rest.sum() > 0 else left
            cum = np.cumsum(left)
            tokens[b, i], accepted[b] = int(np.searchsorted(cum, float(s["draws"][b]) * cum[-1], side="right")), i
            break
    return {"tokens": torch.from_numpy(tokens), "accepted": torch.from_numpy(accepted)}
