"""Operators for several continuations of one prompt, in plain form and through the library.

A program that follows one prompt with several windows (speculation
parallelism on one GPU, best-of-n sampling, reranking of drafts) forks the
prompt's cached keys and values into the windows (`fork`), attends from all of
them at once to a prefix that they share and to what each has of its own
(`attend`), and scores tokens by the logits that come out (`logprobs`).

Shapes are those of the repository's own workloads.  Caches lie in the
library's block layout (32 positions a block: keys [hd/32][32 positions][32
dims], values [hd][32 positions]); `own` says whether `run` takes the library
or torch operations in 32 bits.
"""
import math

import torch

own = False
DEV = "cuda"
# query heads, KV heads, head dim, type of the cache: the attention of the repository's decoder shapes
SHAPES = {
    "tiny": (4, 4, 32, "f32"),
    "1b": (32, 8, 64, "bf16"),
    "8b": (32, 8, 128, "bf16"),
    "13b": (40, 40, 128, "bf16"),
}


def listed():
    return [
        # one new token for each of four continuations of a short prompt: launches are all it costs
        dict(name="attend 1b 4xL512 r1", do="attend", shape="1b", windows=4, rows=1, prefix=512, tail=24),
        # an fp32 model's cache, odd lengths
        dict(name="attend tiny 3xL701 r5", do="attend", shape="tiny", windows=3, rows=5, prefix=701, tail=40),
        # speculation parallelism 7 with five drafts a window, at the benchmark's prefix
        dict(name="attend 8b 7xL2048 r6", do="attend", shape="8b", windows=7, rows=6, prefix=2048, tail=77),
        # as many key heads as query heads, a prefix that ends inside a block
        dict(name="attend 13b 6xL8191 r7", do="attend", shape="13b", windows=6, rows=7, prefix=8191, tail=130),
        # a long context followed by as many rows as one verification carries
        dict(name="attend 8b 8xL32768 r8", do="attend", shape="8b", windows=8, rows=8, prefix=32768, tail=200),
        # a short prompt of the small target into three more windows
        dict(name="fork 1b L509 to 3", do="fork", shape="1b", layers=16, windows=4, prefix=509),
        # the benchmark's prompt into the windows of seven servers
        dict(name="fork 8b L2048 to 6", do="fork", shape="8b", layers=32, windows=7, prefix=2048),
        # one row of a decoding step with five alternatives, as an API answers with: the smallest call
        dict(name="logprobs 1xV32000 top5", do="logprobs", rows=1, vocab=32000, top=5, dtype="f32", pad=0, mask=0),
        # the rows of seven verified windows over the largest vocabulary
        dict(name="logprobs 42xV128256 top5", do="logprobs", rows=42, vocab=128256, top=5, dtype="f32", pad=0, mask=0),
        # a server's own bf16 logits, padded rows, tokens that its grammar forbids masked
        dict(name="logprobs 300xV32003 top20 bf16", do="logprobs", rows=300, vocab=32003, top=20, dtype="bf16", pad=61, mask=25),
        # a whole prompt's tokens scored, with their entropy
        dict(name="logprobs 2048xV128256 top1", do="logprobs", rows=2048, vocab=128256, top=1, dtype="f32", pad=0, mask=0),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    do = rng.choice(["attend", "attend", "attend", "fork", "logprobs", "logprobs"])
    if do == "logprobs":
        vocab = _log(rng, 1000, 128256)
        return dict(do=do, rows=_log(rng, 1, 2048), vocab=vocab, top=rng.choice([0, 1, 5, 20, rng.randint(1, 32)]),
                    dtype=rng.choice(["f32", "f32", "bf16"]), pad=rng.choice([0, rng.randint(1, 128)]),
                    mask=rng.choice([0, 0, rng.randint(1, 95)]))
    shape = rng.choice(list(SHAPES))
    hq, hkv, hd, _ = SHAPES[shape]
    if do == "fork":
        layers = {"tiny": 2, "1b": 16, "8b": rng.randint(8, 32), "13b": rng.randint(4, 10)}[shape]
        return dict(do=do, shape=shape, layers=layers, windows=rng.randint(2, 7), prefix=_log(rng, 16, 2048))
    windows = rng.randint(2, 16)
    rows = rng.choice([1, rng.randint(1, 64 // windows)])
    return dict(do=do, shape=shape, windows=windows, rows=rows, prefix=_log(rng, 16, 8192 if shape == "13b" else 32768 // (2 if rows * windows > 32 else 1)),
                tail=rng.randint(0, 200))


# ------------------------------------------------------------------- inputs


def _gen(seed, stream):
    return torch.Generator(device=DEV).manual_seed(1000003 * int(seed) + stream)


def _dtype(kind):
    return torch.float32 if kind == "f32" else torch.bfloat16


def _blocks(case):
    """Blocks of 32 positions of a window: the positions of its capacity in whole pairs of blocks."""
    return -(-_capacity(case) // 64) * 2


def _capacity(case):
    return case["prefix"] + case.get("tail", 0) + case.get("rows", 0) + 1


def _lengths(case):
    """Cached positions of each window: the shared prefix, and ragged tails; the last window has none."""
    B, t = case["windows"], case.get("tail", 0)
    return [case["prefix"] + t * (B - 1 - b) // max(1, B - 1) for b in range(B)]


def _caches(case, seed):
    """Keys and values of all windows, unit scale; window 0's prefix is what the others continue."""
    hq, hkv, hd, kind = SHAPES[case["shape"]]
    L, W, nb = case.get("layers", 1), case["windows"], _blocks(case)
    g, dt = _gen(seed, 1), _dtype(kind)
    k = torch.zeros((L, W, hkv, nb, hd // 32, 32, 32), device=DEV, dtype=dt)
    v = torch.zeros((L, W, hkv, nb, hd, 32), device=DEV, dtype=dt)
    k[:, 0].normal_(generator=g)
    v[:, 0].normal_(generator=g)
    return k, v


def _inputs(case, seed):
    do, s = case["do"], {"case": case}
    if do == "logprobs":
        rows, V, n = case["rows"], case["vocab"], case["top"]
        g = _gen(seed, 2)
        wide = torch.randn((rows, V + case["pad"]), generator=g, device=DEV) * 3
        # a model is sure of a few tokens in most places
        wide[:, :V].scatter_add_(1, torch.randint(0, V, (rows, 2), generator=g, device=DEV), 12 * torch.rand((rows, 2), generator=g, device=DEV))
        if case["mask"]:
            wide.masked_fill_(torch.rand(wide.shape, generator=g, device=DEV) * 100 < case["mask"], -math.inf)
        s["logits"] = wide.to(_dtype(case["dtype"]))[:, :V]
        # the tokens scored: seen ones, never masked ones
        s["tokens"] = torch.multinomial(torch.softmax(s["logits"][:, :V].float(), -1), 1, generator=g).view(-1).int()
        s["temperature"] = 0.8
        return s
    hq, hkv, hd, kind = SHAPES[case["shape"]]
    s["k"], s["v"] = _caches(case, seed)
    s["lens"] = torch.tensor(_lengths(case), device=DEV)
    if do == "attend":
        B, R, g = case["windows"], case["rows"], _gen(seed, 3)
        s["k"][:, 1:] = s["k"][:, :1]
        s["v"][:, 1:] = s["v"][:, :1]
        first = case["prefix"] // 32 * 32  # the windows differ from the prefix on; its last block in part
        at = torch.arange(first, _blocks(case) * 32, device=DEV).view(-1, 32)
        new = torch.randn((2, B, hkv, at.shape[0], hd, 32), generator=g, device=DEV).to(s["k"].dtype)
        tail = (at >= case["prefix"])[:, None, :]
        for b in range(B):
            kb, vb = s["k"][0, b, :, first // 32:], s["v"][0, b, :, first // 32:]
            kb.copy_(torch.where(tail[:, None].transpose(-1, -2), new[0, b].view(kb.shape), kb))
            vb.copy_(torch.where(tail, new[1, b], vb))
        # queries and keys as they leave RoPE: scores of standard deviation 2
        s["q"] = torch.randn((B * R, hq * hd), generator=g, device=DEV) * 2
        s["new_k"] = torch.randn((B * R, hkv * hd), generator=g, device=DEV)
        s["new_v"] = torch.randn((B * R, hkv * hd), generator=g, device=DEV)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _keep(s)
    return s


# ------------------------------------------------------------------- plain forms


def _attend(s):
    """Caches the rows' keys and values and attends from each row to its window up to itself."""
    case = s["case"]
    hq, hkv, hd, _ = SHAPES[case["shape"]]
    B, R, n = case["windows"], case["rows"], _blocks(case) * 32
    at = s["lens"][:, None] + torch.arange(R, device=DEV)  # slots of the new rows
    b = torch.arange(B, device=DEV)[:, None]
    s["k"][0][b, :, at // 32, :, at % 32] = s["new_k"].view(B, R, hkv, hd // 32, 32).to(s["k"].dtype)
    s["v"][0][b, :, at // 32, :, at % 32] = s["new_v"].view(B, R, hkv, hd).to(s["v"].dtype)
    k = s["k"][0].permute(0, 1, 2, 4, 3, 5).reshape(B, hkv, n, hd).float()
    v = s["v"][0].transpose(-1, -2).reshape(B, hkv, n, hd).float()
    q = s["q"].view(B, R, hkv, hq // hkv, hd).permute(0, 2, 3, 1, 4).reshape(B, hkv, -1, hd)
    z = torch.matmul(q, k.transpose(-1, -2)).view(B, hkv, -1, R, n) / math.sqrt(hd)
    dead = torch.arange(n, device=DEV) > at[:, None, None, :, None]
    z = z.masked_fill_(dead, -math.inf)
    z = torch.exp(z - z.amax(-1, keepdim=True))
    z = z / z.sum(-1, keepdim=True)
    o = torch.matmul(z.view(B, hkv, -1, n), v)
    return o.view(B, hkv, -1, R, hd).permute(0, 3, 1, 2, 4).reshape(B * R, hq * hd)


def _fork(s):
    """Window 0's prefix into the other windows; what lies behind it stays."""
    n = s["case"]["prefix"]
    full, rest = n // 32, n % 32
    s["k"][:, 1:, :, :full] = s["k"][:, :1, :, :full]
    s["v"][:, 1:, :, :full] = s["v"][:, :1, :, :full]
    if rest:
        s["k"][:, 1:, :, full, :, :rest] = s["k"][:, :1, :, full, :, :rest]
        s["v"][:, 1:, :, full, :, :rest] = s["v"][:, :1, :, full, :, :rest]


def _logprobs(s):
    """Log probability of each row's token, the row's entropy, and its `top` most probable tokens."""
    z = s["logits"].float() / s["temperature"]
    z = z - z.amax(-1, keepdim=True)
    e = torch.exp(z)
    total = e.sum(-1, keepdim=True)
    lp = z - torch.log(total)
    p = e / total
    entropy = -(p * torch.where(p > 0, lp, 0)).sum(-1)
    out = {"logprob": lp.gather(1, s["tokens"].long()[:, None])[:, 0], "entropy": entropy}
    if s["case"]["top"]:
        # in the logits' order: a division may make neighbours equal
        order = torch.sort(s["logits"].float(), dim=-1, descending=True, stable=True).indices[:, :s["case"]["top"]]
        out["top"], out["top_logprob"] = order.int(), lp.gather(1, order)
    return out


# ------------------------------------------------------------------- the library


def _outputs(s):
    """Output buffers and workspace of a scoring call, which a program keeps."""
    from paper_2405_14105_amd import dsi

    rows, V, n = s["case"]["rows"], s["case"]["vocab"], s["case"]["top"]
    s["out"] = {"logprob": torch.empty(rows, device=DEV), "entropy": torch.empty(rows, device=DEV)}
    if n:
        s["out"]["top"] = torch.empty((rows, n), dtype=torch.int32, device=DEV)
        s["out"]["top_logprob"] = torch.empty((rows, n), device=DEV)
    s["ws"] = torch.empty(dsi.dsi_logprobs_workspace(rows, V, n), dtype=torch.uint8, device=DEV)


class _Handle:
    """A model's shape and a cache in the program's own memory; destroyed with the state."""

    def __init__(self, s):
        from paper_2405_14105_amd import dsi

        case = s["case"]
        hq, hkv, hd, kind = SHAPES[case["shape"]]
        self.dsi, self.model, self.kv = dsi, None, None
        cfg = dsi.make_config(case.get("layers", 1), 32, hq, hkv, hd, 32, 32, kvdtype=dsi.DSI_F32 if kind == "f32" else dsi.DSI_BF16)
        self.model = dsi.dsi_model_create(cfg, torch.cuda.current_stream().cuda_stream)
        nbytes = s["k"].numel() * s["k"].element_size()
        self.kv = dsi.dsi_kv_wrap(self.model, case["windows"], _capacity(case), s["k"], s["v"], nbytes)
        dsi.dsi_kv_set_length(self.kv, 0, case["prefix"])
        if case["do"] == "attend":
            dsi.dsi_kv_fork(self.kv, 0, 1, case["windows"] - 1, case["prefix"])
            for b, n in enumerate(_lengths(case)):
                dsi.dsi_kv_set_length(self.kv, b, n)

    def __del__(self):
        if self.model is None:
            return
        torch.cuda.synchronize()
        if self.kv is not None:
            self.dsi.dsi_kv_destroy(self.kv)
        self.dsi.dsi_model_destroy(self.model)


def _keep(s):
    """What a program keeps between calls."""
    if s["case"]["do"] == "logprobs":
        _outputs(s)
        return
    s["handle"] = _Handle(s)
    if s["case"]["do"] == "attend":
        s["out"] = torch.empty_like(s["q"])


def _own(s):
    from paper_2405_14105_amd import dsi

    case = s["case"]
    if case["do"] == "logprobs":
        o, z = s["out"], s["logits"]
        dsi.dsi_logprobs(torch.cuda.current_stream().cuda_stream, case["rows"], case["vocab"], z, s["tokens"], case["top"], o["logprob"], o["entropy"],
                         o.get("top"), o.get("top_logprob"), s["ws"], s["ws"].numel(), s["temperature"],
                         dsi.DSI_F32 if case["dtype"] == "f32" else dsi.DSI_BF16, z.stride(0))
        return o
    h = s["handle"]
    if case["do"] == "fork":
        dsi.dsi_kv_fork(h.kv, 0, 1, case["windows"] - 1, case["prefix"])
        return {"k": s["k"], "v": s["v"]}
    dsi.dsi_attend(h.model, h.kv, 0, 0, case["windows"], case["rows"], s["q"], s["new_k"], s["new_v"], s["out"])
    return {"out": s["out"], "k": s["k"], "v": s["v"]}


def run(s):
    if own:
        return _own(s)
    do = s["case"]["do"]
    if do == "logprobs":
        return _logprobs(s)
    if do == "fork":
        _fork(s)
        return {"k": s["k"], "v": s["v"]}
    return {"out": _attend(s), "k": s["k"], "v": s["v"]}


def work(case):
    """A shared prefix counts once, a fork's source once and each copy once, a row of logits once."""
    if case["do"] == "logprobs":
        rows, V, n = case["rows"], case["vocab"], case["top"]
        size = 4 if case["dtype"] == "f32" else 2
        return {"bytes": rows * (V * size + 12 + 8 * n), "flops": 5 * rows * V}
    hq, hkv, hd, kind = SHAPES[case["shape"]]
    each = 2 * hkv * hd * (4 if kind == "f32" else 2)  # a position's keys and values in one layer
    if case["do"] == "fork":
        return {"bytes": case["layers"] * case["prefix"] * each * case["windows"], "flops": 0}
    M, R = case["windows"] * case["rows"], case["rows"]
    tails = sum(n - case["prefix"] for n in _lengths(case))
    seen = sum(R * n + R * (R + 1) // 2 for n in _lengths(case))
    return {"bytes": (case["prefix"] + tails + M) * each + 4 * M * (2 * hq + 2 * hkv) * hd, "flops": 4 * seen * hq * hd}


# ------------------------------------------------------------------- in 64 bits


def exact(case, seed):
    s = _inputs(case, seed)
    if case["do"] == "fork":
        # position by position: keys [..., block, hd/32, position, dim], values [..., block, dim, position]
        live = (torch.arange(_blocks(case) * 32, device=DEV) < case["prefix"]).view(-1, 1, 32)
        return {"k": torch.where(live[:, :, :, None], s["k"][:, :1], s["k"]).double(),
                "v": torch.where(live, s["v"][:, :1], s["v"]).double()}
    if case["do"] == "logprobs":
        parts = []
        for r0 in range(0, case["rows"], 256):
            z = s["logits"][r0:r0 + 256].double()
            lp = torch.log_softmax(z / s["temperature"], -1)
            part = [lp.gather(1, s["tokens"][r0:r0 + 256].long()[:, None])[:, 0], -torch.xlogy(lp.exp(), lp.exp()).sum(-1)]
            if case["top"]:
                part.append(lp.sort(-1, descending=True).values[:, :case["top"]])
            parts.append(part)
        out = [torch.cat(x) for x in zip(*parts)]
        d = {"logprob": out[0], "entropy": out[1]}
        if case["top"]:
            d["top"], d["top_logprob"] = None, out[2]
        return d
    hq, hkv, hd, _ = SHAPES[case["shape"]]
    R, outs = case["rows"], []
    cast = s["k"].dtype
    for b, n in enumerate(_lengths(case)):
        # keys [hkv][positions][hd] of the window: the cached ones and the rows of the call
        rows = slice(b * R, b * R + R)
        k = s["k"][0, b].movedim(3, 2).flatten(1, 2).flatten(2)[:, :n]
        v = s["v"][0, b].movedim(3, 2).flatten(1, 2)[:, :n]
        k = torch.cat([k, s["new_k"][rows].to(cast).view(R, hkv, hd).transpose(0, 1)], 1).double()
        v = torch.cat([v, s["new_v"][rows].to(cast).view(R, hkv, hd).transpose(0, 1)], 1).double()
        q = s["q"][rows].double().view(R, hkv, hq // hkv, hd)
        row = []
        for i in range(R):
            p = torch.softmax(torch.einsum("hgd,hnd->hgn", q[i], k[:, :n + i + 1]) / math.sqrt(hd), -1)
            row.append(torch.einsum("hgn,hnd->hgd", p, v[:, :n + i + 1]).reshape(-1))
        outs.append(torch.stack(row))
        for i in range(R):  # the caches after the call
            block, place = divmod(n + i, 32)
            s["k"][0, b, :, block, :, place] = k[:, n + i].view(hkv, -1, 32)
            s["v"][0, b, :, block, :, place] = v[:, n + i]
    return {"out": torch.cat(outs), "k": s["k"].double(), "v": s["v"].double()}
