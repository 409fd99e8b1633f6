"""Operators of a server that keeps its cache in pages, in plain form and through the library.

A server with projections of its own norms and rotates the queries and keys
of the step's rows (`rotate`), or does that while it puts keys and values into
the pages of its windows (`append`), attends from the rows to the pages
(`attend`), and applies penalties, biases and a grammar's mask to the logits
before tokens are accepted or sampled by them (`adjust`).

Rows of all windows lie after each other, any number of them a window.  A page
holds `page` positions of every KV head in blocks of 32: keys [hd/32][32
positions][32 dims], values [hd][32 positions].  `own` says whether `run` takes
the library or torch operations in 32 bits (angles in 64).
"""
import math

import torch

own = False
DEV = "cuda"
# query heads, KV heads, head dim, type of the cache: the repository's decoder shapes, and one with odd groups
SHAPES = {
    "tiny": (4, 4, 32, "f32"),
    "1b": (32, 8, 64, "bf16"),
    "8b": (32, 8, 128, "bf16"),
    "13b": (40, 40, 128, "bf16"),
    "odd": (12, 4, 96, "bf16"),
}


def listed():
    return [
        # the one row of a decoding step of the small target: the launch is all it costs
        dict(name="rotate 1b 1 row", do="rotate", shape="1b", dtype="f32", rows=1, pos=4000, style="half", part=64, scaling="plain", norm=False),
        # a prompt's rows in a model that norms its heads
        dict(name="rotate 8b 2048 rows bf16", do="rotate", shape="8b", dtype="bf16", rows=2048, pos=0, style="half", part=128, scaling="bands", norm=True),
        # five drafts a window of speculation parallelism 7, at the benchmark's prefix
        dict(name="append 8b 7x6", do="append", shape="8b", dtype="f32", rows="6 6 6 6 6 6 6", past="2048 2059 2070 2081 2092 2103 2114", page=64,
             style="half", part=128, scaling="plain", norm=False),
        # a long prompt's chunk among decoding windows, far positions, half of each head rotated
        dict(name="append 13b 1021+5 ragged", do="append", shape="13b", dtype="bf16", rows="1 1 1021 1 1 1", past="509 4000 30001 33 0 70000", page=32,
             style="pairs", part=64, scaling="ramp", norm=True),
        # one new token for each of four windows after short prompts: the smallest attention
        dict(name="attend 1b 4xL512 r1", do="attend", shape="1b", dtype="f32", rows="1 1 1 1", past="512 500 37 263", page=32, reach=0),
        # an fp32 model's pages, odd lengths, a window that starts, one without rows
        dict(name="attend tiny 5 ragged", do="attend", shape="tiny", dtype="f32", rows="5 33 0 1 7", past="701 0 90 1300 64", page=96, reach=0),
        # speculation parallelism 7 with five drafts a window
        dict(name="attend 8b 7xL2048 r6", do="attend", shape="8b", dtype="f32", rows="6 6 6 6 6 6 6", past="2048 2059 2070 2081 2092 2103 2114", page=64, reach=0),
        # many windows decoding, from short to long contexts
        dict(name="attend 8b 32 decoding bf16", do="attend", shape="8b", dtype="bf16", rows="1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1", past="100 1101 2102 3103 4104 5105 6106 7107 8108 9109 10110 11111 12112 13113 14114 15115 16116 17117 18118 19119 20120 21121 22122 23123 24124 25125 26126 27127 28128 29129 30130 31131", page=64, reach=0),
        # a prompt's chunk of 512 rows beside seven decoding windows, each row seeing 4096 positions at most
        dict(name="attend 13b 512+7 reach bf16", do="attend", shape="13b", dtype="bf16", rows="1 1 512 1 1 1 1 1", past="900 6000 4500 31 2222 77 5011 640", page=64,
             reach=4096),
        # the last chunk of a long prompt
        dict(name="attend 8b 2048 at 30000 bf16", do="attend", shape="8b", dtype="bf16", rows="2048", past="30000", page=128, reach=0),
        # one row of a decoding step with penalties
        dict(name="adjust 1xV32000", do="adjust", windows=1, rows=1, vocab=32000, dtype="f32", pad=0, seen=300, bias=4, allowed=0),
        # the rows of seven verified windows over the largest vocabulary, a grammar's mask on every row
        dict(name="adjust 7x6xV128256 masked", do="adjust", windows=7, rows=6, vocab=128256, dtype="f32", pad=0, seen=2048, bias=16, allowed=60),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _text(numbers):
    return " ".join(map(str, numbers))


def _ints(text):
    return [int(x) for x in text.split()]


def draw(rng):
    do = rng.choice(["rotate", "append", "attend", "attend", "attend", "adjust", "adjust"])
    if do == "adjust":
        windows = rng.randint(1, 16)
        return dict(do=do, windows=windows, rows=rng.randint(1, 64 // windows), vocab=_log(rng, 1000, 128256), dtype=rng.choice(["f32", "f32", "bf16"]),
                    pad=rng.choice([0, rng.randint(1, 128)]), seen=_log(rng, 1, 8192), bias=rng.choice([0, rng.randint(1, 64)]),
                    allowed=rng.choice([0, 0, rng.randint(1, 99)]))
    shape, dtype = rng.choice(list(SHAPES)), rng.choice(["f32", "bf16"])
    hd = SHAPES[shape][2]
    turn = dict(style=rng.choice(["half", "pairs"]), part=rng.choice([hd, hd, 2 * rng.randint(4, hd // 2)]),
                scaling=rng.choice(["plain", "linear", "base", "bands", "ramp"]), norm=rng.random() < 0.5)
    if do == "rotate":
        return dict(do=do, shape=shape, dtype=dtype, rows=_log(rng, 1, 2048), pos=_log(rng, 1, 100000), **turn)
    page = 32 * rng.randint(1, 8)
    if do == "append":
        windows = rng.randint(1, 8)
        return dict(do=do, shape=shape, dtype=dtype, rows=_text(_log(rng, 1, 256) for _ in range(windows)), past=_text(_log(rng, 1, 8192) for _ in range(windows)), page=page, **turn)
    kind = rng.choice(["steps", "steps", "chunk", "mixed"])
    if kind == "chunk":
        rows, past = [_log(rng, 17, 2048)], [_log(rng, 1, 8192 if shape == "13b" else 24000)]
    elif kind == "steps":
        windows, each = rng.randint(1, 24), rng.randint(1, 8)
        rows = [rng.choice([1, each]) for _ in range(windows)]
        past = [_log(rng, 1, 8192 if shape == "13b" else 32000) for _ in range(windows)]
    else:
        windows = rng.randint(2, 8)
        rows = [rng.choice([0, 1, rng.randint(2, 8)]) for _ in range(windows)]
        past = [_log(rng, 1, 6000) for _ in range(windows)]
        rows[rng.randrange(windows)] = _log(rng, 17, 512)
    return dict(do=do, shape=shape, dtype=dtype, rows=_text(rows), past=_text(past), page=page, reach=rng.choice([0, 0, _log(rng, 1, 4096)]))


# ------------------------------------------------------------------- inputs


def _gen(seed, stream):
    return torch.Generator(device=DEV).manual_seed(1000003 * int(seed) + stream)


def _dtype(kind):
    return torch.float32 if kind == "f32" else torch.bfloat16


def _frequencies(part, scaling):
    """Radians per position of each rotated pair, and the factor on rotated entries: what a program works out once."""
    base, factor, context = 10000.0, 8.0, 8192
    i = torch.arange(part // 2, dtype=torch.float64)
    f, by = base ** (-2 * i / part), 1.0
    if scaling == "linear":
        f = f / factor
    elif scaling == "base":
        f = (base * factor ** (part / (part - 2))) ** (-2 * i / part)
    elif scaling == "bands":  # long waves slowed down, short ones kept, those between mixed
        s = ((context * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        f = (1 - s) * f / factor + s * f
    elif scaling == "ramp":  # by the pair's index, between 32 turns and one over the context
        at = [part * math.log(context / (2 * math.pi * turns)) / (2 * math.log(base)) for turns in (32.0, 1.0)]
        lo, hi = max(0, math.floor(at[0])), min(part - 1, math.ceil(at[1]))
        s = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        f, by = s * f / factor + (1 - s) * f, 0.1 * math.log(factor) + 1
    return f, by


def _inputs(case, seed):
    do, s, g = case["do"], {"case": case}, _gen(seed, 1)
    if do == "adjust":
        B, R, V = case["windows"], case["rows"], case["vocab"]
        logits = torch.randn((B * R, V + case["pad"]), generator=g, device=DEV) * 3
        s["logits"] = logits.to(_dtype(case["dtype"]))[:, :V]
        # a text's tokens: a few of them often
        often = lambda *n: (V * torch.rand(n, generator=g, device=DEV) ** 4).int().clamp_(0, V - 1)  # noqa: E731
        s["seen"] = often(B, case["seen"])
        s["n_seen"] = torch.randint(case["seen"] // 2, case["seen"] + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        s["window"] = often(B, R)  # the rows' own tokens: row i has seen the first i + 1 of them
        s["repetition"] = 1 + 0.3 * torch.rand(B, generator=g, device=DEV)
        s["frequency"], s["presence"] = torch.rand((2, B), generator=g, device=DEV).unbind()
        n = case["bias"]
        # ids of a window differ
        s["bias_ids"] = (torch.rand((B, V), generator=g, device=DEV).argsort(1)[:, :n]).int().contiguous()
        s["bias"] = 4 * torch.randn((B, n), generator=g, device=DEV)
        if case["allowed"]:
            words = torch.zeros((B * R, (V + 31) // 32), dtype=torch.int64, device=DEV)
            for bit in range(32):
                words |= (torch.rand(words.shape, generator=g, device=DEV) * 100 < case["allowed"]).long() << bit
            s["allowed"] = torch.where(words >= 2 ** 31, words - 2 ** 32, words).int()
        return s
    hq, hkv, hd, kind = SHAPES[case["shape"]]
    dt = _dtype(case["dtype"])
    if do == "rotate":
        n = case["rows"]
        # queries, keys and values leave one projection: a row holds all three
        s["qkv"] = torch.randn((n, (hq + 2 * hkv) * hd), generator=g, device=DEV).to(dt)
        s["pos"] = torch.arange(case["pos"], case["pos"] + n, device=DEV, dtype=torch.int32)
    else:
        rows, past, page = _ints(case["rows"]), _ints(case["past"]), case["page"]
        B, n, need = len(rows), sum(rows), [-(-(p + r) // page) for p, r in zip(past, rows)]
        s["windows"], s["most"] = B, max(rows)
        s["row0"] = torch.tensor([sum(rows[:b]) for b in range(B + 1)], device=DEV, dtype=torch.int32)
        s["past"] = torch.tensor(past, device=DEV, dtype=torch.int32)
        # pages come from anywhere in the pool; entries behind a window's last page are empty
        pages = sum(need) + 3
        order, most = torch.randperm(pages, generator=g, device=DEV).int(), max(need)
        s["table"] = torch.full((B, most), -1, device=DEV, dtype=torch.int32)
        for b in range(B):
            s["table"][b, :need[b]] = order[sum(need[:b]):sum(need[:b + 1])]
        s["k"] = torch.randn((pages, hkv, page // 32, hd // 32, 32, 32), generator=g, device=DEV, dtype=_dtype(kind))
        s["v"] = torch.randn((pages, hkv, page // 32, hd, 32), generator=g, device=DEV, dtype=_dtype(kind))
        s["n"] = n
        if do == "append":
            s["qkv"] = torch.randn((n, (hq + 2 * hkv) * hd), generator=g, device=DEV).to(dt)
        else:  # queries as they leave the rotation: scores of standard deviation 2
            s["q"] = (torch.randn((n, hq * hd), generator=g, device=DEV) * 2).to(dt)
    if do != "attend":
        f, s["factor"] = _frequencies(case["part"], case["scaling"])
        s["freq"] = f.to(DEV)
        s["gain_q"], s["gain_k"] = (1 + 0.1 * torch.randn((2, hd), generator=g, device=DEV)).unbind()
    return s


def prepare(case, seed):
    return _inputs(case, seed)


# ------------------------------------------------------------------- plain forms


def _turned(s, x, pos, gain):
    """x [rows][heads][hd] in 32 bits, each head normed and its first dims rotated by its row's position."""
    case = s["case"]
    if case["norm"]:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-5) * gain
    part = case["part"]
    angle = pos.double()[:, None, None] * s["freq"]
    c, d = torch.cos(angle).float() * s["factor"], torch.sin(angle).float() * s["factor"]
    if case["style"] == "half":
        a, b = x[..., :part // 2], x[..., part // 2:part]
        return torch.cat([a * c - b * d, b * c + a * d, x[..., part:]], -1)
    a, b = x[..., 0:part:2], x[..., 1:part:2]
    return torch.cat([torch.stack([a * c - b * d, b * c + a * d], -1).flatten(-2), x[..., part:]], -1)


def _rotate(s):
    hq, hkv, hd, _ = SHAPES[s["case"]["shape"]]
    n, dt = s["qkv"].shape[0], s["qkv"].dtype
    x = s["qkv"].view(n, hq + 2 * hkv, hd)
    q = _turned(s, x[:, :hq].float(), s["pos"], s["gain_q"])
    k = _turned(s, x[:, hq:hq + hkv].float(), s["pos"], s["gain_k"])
    return {"q": q.to(dt).flatten(1), "k": k.to(dt).flatten(1)}


def _places(s):
    """Window and slot of each row."""
    rows = torch.arange(s["n"], device=DEV)
    b = torch.searchsorted(s["row0"], rows.int(), right=True) - 1
    return b, s["past"][b].long() + rows - s["row0"][b]


def _append(s):
    case = s["case"]
    hq, hkv, hd, _ = SHAPES[case["shape"]]
    n, dt = s["qkv"].shape[0], s["qkv"].dtype
    x = s["qkv"].view(n, hq + 2 * hkv, hd)
    b, at = _places(s)
    q = _turned(s, x[:, :hq].float(), at, s["gain_q"])
    k = _turned(s, x[:, hq:hq + hkv].float(), at, s["gain_k"])
    page, place = s["table"][b, at // case["page"]].long(), at % case["page"]
    s["k"][page, :, place // 32, :, place % 32] = k.view(n, hkv, hd // 32, 32).to(s["k"].dtype)
    s["v"][page, :, place // 32, :, place % 32] = x[:, hq + hkv:].to(s["v"].dtype)
    return {"q": q.to(dt).flatten(1), "k": s["k"], "v": s["v"]}


def _attend(s):
    """Windows padded to the most rows and the longest context."""
    case = s["case"]
    hq, hkv, hd, _ = SHAPES[case["shape"]]
    B, R, page = s["windows"], s["most"], case["page"]
    table = s["table"].clamp(min=0).long()
    K = table.shape[1] * page
    k = s["k"][table].permute(0, 2, 1, 3, 5, 4, 6).reshape(B, hkv, K, hd).float()
    v = s["v"][table].permute(0, 2, 1, 3, 5, 4).reshape(B, hkv, K, hd).float()
    i = torch.arange(R, device=DEV)
    row = (s["row0"][:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][row].float().view(B, R, hkv, hq // hkv, hd).permute(0, 2, 3, 1, 4).reshape(B, hkv, -1, hd)
    z = torch.matmul(q, k.transpose(-1, -2)).view(B, hkv, -1, R, K).mul_(1 / math.sqrt(hd))
    at, j = (s["past"][:, None] + i)[:, :, None], torch.arange(K, device=DEV)
    dead = j > at
    if case["reach"]:
        dead = dead | (j <= at - case["reach"])
    z = z.masked_fill_(dead[:, None, None], -math.inf)
    z = z.sub_(z.amax(-1, keepdim=True)).exp_()
    z = z.div_(z.sum(-1, keepdim=True))
    o = torch.matmul(z.view(B, hkv, -1, K), v).view(B, hkv, -1, R, hd).permute(0, 3, 1, 2, 4).reshape(B, R, hq * hd)
    b, slot = _places(s)
    return {"out": o[b, slot - s["past"][b]].to(s["q"].dtype)}


def _adjust(s):
    case = s["case"]
    B, R, V = case["windows"], case["rows"], case["vocab"]
    live = torch.arange(case["seen"], device=DEV) < s["n_seen"][:, None]
    count = torch.zeros((B, V), device=DEV).scatter_add_(1, s["seen"].long(), live.float())
    first = torch.ones((R, R), device=DEV).tril().expand(B, R, R)
    count = count[:, None].repeat(1, R, 1).scatter_add_(2, s["window"].long()[:, None].expand(B, R, R), first)
    z = s["logits"].float().view(B, R, V)
    r, f, p = (s[n][:, None, None] for n in ("repetition", "frequency", "presence"))
    hit = count > 0
    z = torch.where(hit, torch.where(z > 0, z / r, z * r), z) - f * count - p * hit
    if case["bias"]:
        z = z.scatter_add(2, s["bias_ids"].long()[:, None].expand(B, R, -1), s["bias"][:, None].expand(B, R, -1))
    z = z.view(B * R, V)
    if case["allowed"]:
        bit = s["allowed"][:, :, None] >> torch.arange(32, device=DEV) & 1
        z = z.masked_fill(bit.flatten(1)[:, :V] == 0, -math.inf)
    return {"logits": z.to(s["logits"].dtype)}


# ------------------------------------------------------------------- the library


def _kept(s):
    """What a program keeps between its calls: output buffers, the pages' description, a workspace."""
    from paper_2405_14105_amd import dsi

    case, kinds = s["case"], {"f32": dsi.DSI_F32, "bf16": dsi.DSI_BF16}
    s["kept"] = True
    if case["do"] == "adjust":
        s["out"] = torch.empty((s["logits"].shape[0], case["vocab"]), dtype=s["logits"].dtype, device=DEV)
        return
    hq, hkv, hd, kind = SHAPES[case["shape"]]
    if case["do"] != "attend":
        s["rope"] = dsi.make_rope(case["part"], s["freq"], s["factor"], dsi.DSI_ROPE_HALF if case["style"] == "half" else dsi.DSI_ROPE_PAIRS)
        s["out"] = torch.empty((s["qkv"].shape[0], hq * hd), dtype=s["qkv"].dtype, device=DEV)
    if case["do"] == "rotate":
        s["out_k"] = torch.empty((s["qkv"].shape[0], hkv * hd), dtype=s["qkv"].dtype, device=DEV)
        return
    s["pages"] = dsi.make_pages(hkv, hd, kinds[kind], s["k"].shape[0], case["page"], s["k"], s["v"], s["windows"], s["table"].shape[1],
                                s["table"], s["past"], s["row0"])
    if case["do"] == "attend":
        s["out"] = torch.empty_like(s["q"])
        s["ws"] = torch.empty(dsi.dsi_page_attend_workspace(s["pages"], s["q"].shape[0], hq), dtype=torch.uint8, device=DEV)


def _own(s):
    from paper_2405_14105_amd import dsi

    case, stream = s["case"], torch.cuda.current_stream().cuda_stream
    if "kept" not in s:
        _kept(s)
    if case["do"] == "adjust":
        z, out = s["logits"], s["out"]
        dsi.dsi_adjust(stream, case["windows"], case["rows"], case["vocab"], z, out, dtype=dsi.DSI_F32 if case["dtype"] == "f32" else dsi.DSI_BF16,
                       ld=z.stride(0), ld_out=out.stride(0), d_seen=s["seen"], d_n_seen=s["n_seen"], ld_seen=case["seen"], d_tokens=s["window"],
                       d_repetition=s["repetition"], d_frequency=s["frequency"], d_presence=s["presence"], n_bias=case["bias"],
                       d_bias_ids=s["bias_ids"], d_bias=s["bias"], d_allowed=s.get("allowed"))
        return {"logits": out}
    hq, hkv, hd, _ = SHAPES[case["shape"]]
    kind = dsi.DSI_F32 if case["dtype"] == "f32" else dsi.DSI_BF16
    if case["do"] == "attend":
        dsi.dsi_page_attend(stream, s["pages"], s["q"].shape[0], hq, s["q"], s["out"], s["ws"], s["ws"].numel(), dtype=kind, reach=case["reach"])
        return {"out": s["out"]}
    x, gains = s["qkv"], (s["gain_q"], s["gain_k"]) if case["norm"] else (None, None)
    q, k, v = x, x[:, hq * hd:], x[:, (hq + hkv) * hd:]
    if case["do"] == "rotate":
        dsi.dsi_rotate(stream, x.shape[0], hq, hkv, hd, q, k, s["pos"], s["out"], s["out_k"], s["rope"], dtype=kind, ld_q=x.stride(0), ld_k=x.stride(0),
                       d_gain_q=gains[0], d_gain_k=gains[1], eps=1e-5)
        return {"q": s["out"], "k": s["out_k"]}
    dsi.dsi_page_append(stream, s["pages"], x.shape[0], hq, q, k, v, s["out"], s["rope"], dtype=kind, ld_q=x.stride(0), ld_k=x.stride(0), ld_v=x.stride(0),
                        d_gain_q=gains[0], d_gain_k=gains[1], eps=1e-5)
    return {"q": s["out"], "k": s["k"], "v": s["v"]}


def run(s):
    if own:
        return _own(s)
    return {"rotate": _rotate, "append": _append, "attend": _attend, "adjust": _adjust}[s["case"]["do"]](s)


def work(case):
    """Each input once, each output once; of pages the positions that a row sees."""
    if case["do"] == "adjust":
        size = 4 if case["dtype"] == "f32" else 2
        rows, V = case["windows"] * case["rows"], case["vocab"]
        return {"bytes": 2 * rows * V * size + 4 * case["windows"] * (case["seen"] + 2 * case["bias"]) + (rows * V // 8 if case["allowed"] else 0), "flops": 4 * rows * V}
    hq, hkv, hd, kind = SHAPES[case["shape"]]
    size, cache = (4 if case["dtype"] == "f32" else 2), (4 if kind == "f32" else 2)
    if case["do"] == "rotate":
        return {"bytes": 2 * case["rows"] * (hq + hkv) * hd * size, "flops": 8 * case["rows"] * (hq + hkv) * hd}
    rows, past = _ints(case["rows"]), _ints(case["past"])
    n = sum(rows)
    if case["do"] == "append":
        return {"bytes": n * hd * (2 * hq * size + 2 * hkv * (size + cache)), "flops": 8 * n * (hq + hkv) * hd}
    reach, seen, read = case["reach"] or 1 << 40, 0, 0
    for r, p in zip(rows, past):
        seen += sum(min(p + i + 1, reach) for i in range(r))
        read += min(p + r, reach + r - 1) if r else 0
    return {"bytes": 2 * read * hkv * hd * cache + 2 * n * hq * hd * size, "flops": 4 * seen * hq * hd}


# ------------------------------------------------------------------- in 64 bits


def _turn64(case, x, pos, gain):
    """Heads of x [rows][heads][hd] normed, then rotated as complex numbers."""
    x = x.double()
    if case["norm"]:
        x = x / ((x ** 2).sum(-1, keepdim=True) / x.shape[-1] + 1e-5).sqrt() * gain.double()
    f, by = _frequencies(case["part"], case["scaling"])
    w = torch.polar(torch.full((1,), by, dtype=torch.float64, device=DEV), torch.outer(pos.double(), f.to(DEV)))[:, None]
    part, y = case["part"], x.clone()
    if case["style"] == "half":
        t = torch.complex(x[..., :part // 2].contiguous(), x[..., part // 2:part].contiguous()) * w
        y[..., :part // 2], y[..., part // 2:part] = t.real, t.imag
    else:
        t = torch.complex(x[..., 0:part:2].contiguous(), x[..., 1:part:2].contiguous()) * w
        y[..., 0:part:2], y[..., 1:part:2] = t.real, t.imag
    return y


def exact(case, seed):
    s = _inputs(case, seed)
    if case["do"] == "adjust":
        R, V, outs = case["rows"], case["vocab"], []
        for b in range(case["windows"]):
            held = torch.bincount(s["seen"][b, :int(s["n_seen"][b])].long(), minlength=V)
            for i in range(R):
                n = (held + torch.bincount(s["window"][b, :i + 1].long(), minlength=V)).double()
                z = s["logits"][b * R + i].double()
                r = s["repetition"][b].double()
                z = torch.where(n > 0, torch.where(z > 0, z / r, z * r), z)
                z = z - s["frequency"][b].double() * n - torch.where(n > 0, s["presence"][b].double(), 0)
                z[s["bias_ids"][b].long()] += s["bias"][b].double()
                if case["allowed"]:
                    v = torch.arange(V, device=DEV)
                    z[(s["allowed"][b * R + i][v // 32] >> (v % 32)) % 2 == 0] = -math.inf
                outs.append(z)
        return {"logits": torch.stack(outs)}
    hq, hkv, hd, _ = SHAPES[case["shape"]]
    if case["do"] == "rotate":
        x = s["qkv"].view(-1, hq + 2 * hkv, hd)
        return {"q": _turn64(case, x[:, :hq], s["pos"], s["gain_q"]).flatten(1), "k": _turn64(case, x[:, hq:hq + hkv], s["pos"], s["gain_k"]).flatten(1)}
    if case["do"] == "append":
        x = s["qkv"].view(-1, hq + 2 * hkv, hd)
        k, v, q, r0, ps = s["k"].double(), s["v"].double(), [], 0, case["page"]
        for b, (n, past) in enumerate(zip(_ints(case["rows"]), _ints(case["past"]))):
            at = torch.arange(past, past + n, device=DEV)
            rows = x[r0:r0 + n]
            q.append(_turn64(case, rows[:, :hq], at, s["gain_q"]))
            kb = _turn64(case, rows[:, hq:hq + hkv], at, s["gain_k"])
            pages = s["table"][b].long()[at // ps]
            for h in range(hkv):
                for d in range(0, hd, 32):
                    k[pages, h, at % ps // 32, d // 32, at % 32] = kb[:, h, d:d + 32]
                v[pages, h, at % ps // 32, :, at % 32] = rows[:, hq + hkv + h].double()
            r0 += n
        return {"q": torch.cat(q).flatten(1), "k": k, "v": v}
    outs, r0, ps = [], 0, case["page"]
    for b, (n, past) in enumerate(zip(_ints(case["rows"]), _ints(case["past"]))):
        if not n:
            continue
        low = max(0, past - case["reach"] + 1) if case["reach"] else 0
        at = torch.arange(low, past + n, device=DEV)
        pages = s["table"][b].long()[at // ps]
        for h in range(hkv):
            k = s["k"][pages, h, at % ps // 32, :, at % 32].reshape(-1, hd).double()
            v = s["v"][pages, h, at % ps // 32, :, at % 32].double()
            q = s["q"][r0:r0 + n].view(n, hq, hd)[:, h * (hq // hkv):(h + 1) * (hq // hkv)].double()
            z = torch.tensordot(q, k, dims=([2], [1])) / math.sqrt(hd)
            own_at = torch.arange(past, past + n, device=DEV)[:, None]
            ok = at <= own_at
            if case["reach"]:
                ok &= at > own_at - case["reach"]
            p = torch.softmax(torch.where(ok[:, None], z, -math.inf), -1)
            outs.append((r0, h, torch.tensordot(p, v, dims=([2], [0]))))
        r0 += n
    out = torch.zeros((r0, hkv, hq // hkv, hd), dtype=torch.float64, device=DEV)
    for first, h, o in outs:
        out[first:first + o.shape[0], h] = o
    return {"out": out.view(r0, hq * hd)}
