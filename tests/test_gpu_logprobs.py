"""dsi_logprobs on the GPU against log_softmax, entropy and a stable sort in 64
bits: sizes, types, strides, masks, ties, and values that are not numbers."""
import math

import pytest
import torch

from paper_2405_14105_amd import dsi

pytestmark = pytest.mark.gpu

F = math.inf


def call(z, tokens, n, T=1.0, vocab=None, stream=None):
    rows, V = z.shape[0], vocab or z.shape[1]
    kind = dsi.DSI_F32 if z.dtype == torch.float32 else dsi.DSI_BF16
    o = {"logprob": torch.full((rows,), 7.0, device="cuda"), "entropy": torch.full((rows,), 7.0, device="cuda"),
         "ids": torch.full((rows, n), -7, dtype=torch.int32, device="cuda"), "top": torch.full((rows, n), 7.0, device="cuda")}
    nbytes = dsi.dsi_logprobs_workspace(rows, V, n)
    ws = torch.empty(nbytes + 64, dtype=torch.uint8, device="cuda").fill_(0xA5)
    s = stream if stream is not None else torch.cuda.current_stream()
    dsi.dsi_logprobs(s.cuda_stream, rows, V, z, tokens, n, o["logprob"], o["entropy"], o["ids"] if n else None,
                     o["top"] if n else None, ws, nbytes, T, kind, z.stride(0))
    torch.cuda.synchronize()
    assert (ws[nbytes:] == 0xA5).all()
    return o


def check(z, tokens, n, T, o):
    rows, V = z.shape
    x = z.double() / float(torch.tensor(T, dtype=torch.float32))
    lp = torch.log_softmax(x, -1)
    H = -torch.xlogy(lp.exp(), lp.exp()).sum(-1)
    # The exponents' factor log2(e)/T is rounded (2^-24 of the exponent), each e^x has
    # exp2's ulp (2^-23) and the sums of 16 terms theirs (16 2^-24): log S is off by
    # the mean exponent times 2^-24 and those, at most (|x| 2^-24 + 2^-19); the
    # entropy by as much for log S and for the mean, and each result by its rounding.
    span = (lp.exp() * (x.amax(-1, keepdim=True) - x).nan_to_num(0, 0, 0)).sum(-1)
    ds = (span + 1) * 2.0 ** -23 + 2.0 ** -19
    t = tokens.long().clamp(0, V - 1)[:, None]
    ref = torch.where((tokens >= 0) & (tokens < V), lp.gather(1, t)[:, 0], math.nan)
    close(o["logprob"], ref, ds + ref.abs().nan_to_num(0, 0, 0) * 2.0 ** -23)
    close(o["entropy"], H, (2 + span) * ds + H * 2.0 ** -23)
    if n:
        key = torch.where(z.isnan(), -F, z.float())
        order = torch.sort(key, dim=-1, descending=True, stable=True).indices[:, :n]
        ok = ~z.isnan().any(-1)
        assert torch.equal(o["ids"].long()[ok], order[ok])
        rt = lp.gather(1, order)
        close(o["top"], rt, ds[:, None] + rt.abs().nan_to_num(0, 0, 0) * 2.0 ** -23)


def close(got, ref, tol):
    got = got.double()
    assert torch.equal(got.isnan(), ref.isnan())
    inf = ref.isinf()
    assert torch.equal(got[inf], ref[inf])
    fin = torch.isfinite(ref)
    d = (got - ref).abs()[fin]
    assert (d <= tol.expand_as(ref)[fin]).all(), f"{(d / tol.expand_as(ref)[fin]).max().item():.2f} of the bound"


def logits(rows, V, seed, std=3.0, dt=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn((rows, V), generator=g, device="cuda") * std
    return z.to(dt), torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 7, 63, 64, 65, 1000, 1023, 1024, 1025, 4099, 32003, 128256])
@pytest.mark.parametrize("rows,n", [(1, 5), (3, 0), (42, 20), (64, 1)])
def test_sizes(dev, dt, V, rows, n):
    z, t = logits(rows, V, V + rows, dt=dt)
    n = min(n, V)
    check(z, t, n, 1.0, call(z, t, n))


@pytest.mark.parametrize("rows,V,n", [(5000, 777, 3), (2100, 5001, 64), (1, 300000, 64), (300, 20000, 33)])
def test_many_rows_and_long_ones(dev, rows, V, n):
    z, t = logits(rows, V, rows)
    check(z, t, n, 0.7, call(z, t, n, 0.7))


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("start", [0, 1, 2, 3, 5, 7])
@pytest.mark.parametrize("pad", [0, 1, 6])
def test_strides_and_alignment(dev, dt, start, pad):
    """Rows that begin and end anywhere; what lies between them is never read into a result."""
    rows, V = 9, 2051
    flat = torch.full((start + rows * (V + pad) + 8,), math.nan, device="cuda", dtype=dt)
    z = flat[start:start + rows * (V + pad)].view(rows, V + pad)[:, :V]
    x, t = logits(rows, V, 3, dt=dt)
    z.copy_(x)
    check(z, t, 7, 1.3, call(z, t, 7, 1.3))


@pytest.mark.parametrize("T", [1e-30, 0.01, 0.5, 1.0, 7.0, 1e6])
def test_temperatures(dev, T):
    z, t = logits(6, 3001, 9)
    check(z, t, 4, T, call(z, t, 4, T))


def test_ties_go_to_the_lowest_id(dev):
    for V in (50, 1500, 40000):
        z = torch.zeros((4, V), device="cuda")
        z[1] = torch.arange(V, device="cuda") % 3
        z[2] = -0.0
        z[2, ::2] = 0.0
        z[3, V - 5:] = 1.0
        t = torch.tensor([0, 1, 2, V - 1], device="cuda", dtype=torch.int32)
        check(z, t, 40, 1.0, call(z, t, 40))
        zb = logits(3, V, 1, dt=torch.bfloat16)[0].div(4).round()
        check(zb, t[:3], 40, 1.0, call(zb, t[:3].contiguous(), 40))


def test_orders_that_insert_most(dev):
    """Ascending and descending rows: every step of an ascending row beats all before it."""
    V = 30000
    up = torch.arange(V, device="cuda").float() / 500
    z = torch.stack([up, up.flip(0)])
    t = torch.tensor([5, V - 3], device="cuda", dtype=torch.int32)
    check(z, t, 64, 1.0, call(z, t, 64))


def test_masks_and_infinities(dev):
    V = 5000
    z, t = logits(9, V, 4)
    z[0, 100:] = -F                 # fewer live entries than the runs
    z[1, 1:] = -F                   # one token is certain
    z[2, :] = -F                    # nothing is
    z[3, 17] = F
    z[4, 17] = math.nan
    z[5, :] = math.nan
    z[6, :4990] = torch.finfo(torch.float32).min
    z[7, :] = torch.finfo(torch.float32).min
    z[8, :3000] = -F
    t[0], t[1], t[8] = 4000, 0, 0
    o = call(z, t, 12)
    keep = [0, 1, 6, 7, 8]
    check(z[keep], t[keep], 12, 1.0, {k: v[keep] for k, v in o.items()})
    for r in (2, 3, 4, 5):
        assert o["logprob"][r].isnan() and o["entropy"][r].isnan() and o["top"][r].isnan().all()
    assert o["ids"][2].tolist() == list(range(12))
    assert o["ids"][3][0] == 17 and o["ids"][5].tolist() == [-1] * 12
    rest = z[4].nan_to_num(-F).sort(descending=True, stable=True).indices[:12]
    assert torch.equal(o["ids"][4].long(), rest)
    assert o["logprob"][1] == 0 and o["entropy"][1] == 0 and o["ids"][1].tolist() == list(range(12))


def test_a_sure_row_keeps_its_digits(dev):
    """log p and entropy far below a float's step from 0 (relative to themselves)."""
    z = torch.zeros((3, 1000), device="cuda")
    for r, top in enumerate((25.0, 40.0, 80.0)):
        z[r, 123] = top
    t = torch.full((3,), 123, device="cuda", dtype=torch.int32)
    o = call(z, t, 2)
    x = z.double()
    rest = 999 * torch.exp(-x[:, 123])
    lp = -torch.log1p(rest)
    H = torch.log1p(rest) + rest / (1 + rest) * x[:, 123]
    # exponents up to 80 with 2^-24 of them, exp2's ulp; log1p of S - 1 keeps 2^-52 of 1
    assert ((o["logprob"].double() - lp).abs() <= lp.abs() * 2.0 ** -16 + 2.0 ** -51).all()
    assert ((o["entropy"].double() - H).abs() <= H * 2.0 ** -16 + 2.0 ** -45).all()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [2, 1000, 40000])
@pytest.mark.parametrize("margin", [17.0, 25.0, 40.0, 60.0, 80.0])
def test_a_sure_row_is_exact_relative_to_itself(dev, dt, V, margin):
    """1 - p far below the step of 1 in any type: log p, the entropy and the
    alternatives keep their digits, whichever run holds the token."""
    at = sorted({0, V // 3, V - 1})
    z = torch.full((len(at), V), 3.0, device="cuda", dtype=dt)
    for r, i in enumerate(at):
        z[r, i] = 3.0 + margin
    t = torch.tensor(at, device="cuda", dtype=torch.int32)
    o = call(z, t, 2)
    rest = (V - 1) * math.exp(-margin)
    lp, H = -math.log1p(rest), math.log1p(rest) + rest / (1 + rest) * margin
    # each e^-margin: its exponent's factor and product, 2^-24 of the exponent each,
    # exp2's ulp, and the sums of 16 terms (16 2^-24); the mean of the exponents has
    # those once more, the result its rounding
    tol = margin * 2.0 ** -23 + 2.0 ** -19
    assert ((o["logprob"].double() - lp).abs() <= -lp * tol).all()
    assert ((o["top"][:, 0].double() - lp).abs() <= -lp * tol).all()
    assert ((o["entropy"].double() - H).abs() <= H * 2 * tol).all()
    assert o["ids"][:, 0].tolist() == at and o["ids"][:, 1].tolist() == [1 if i == 0 else 0 for i in at]


def test_targets_outside_the_vocabulary(dev):
    z, _ = logits(4, 900, 5)
    t = torch.tensor([-1, 900, 2 ** 30, 899], device="cuda", dtype=torch.int32)
    check(z, t, 3, 1.0, call(z, t, 3))


def test_nullable_outputs(dev):
    z, t = logits(5, 2000, 6)
    full = call(z, t, 4)
    ws = torch.empty(dsi.dsi_logprobs_workspace(5, 2000, 4), dtype=torch.uint8, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    a, b = torch.zeros(5, device="cuda"), torch.zeros(5, device="cuda")
    dsi.dsi_logprobs(s, 5, 2000, z, t, 0, a, None, None, None, ws, ws.numel())
    dsi.dsi_logprobs(s, 5, 2000, z, None, 0, None, b, None, None, ws, ws.numel())
    ids, lp = torch.zeros((5, 4), dtype=torch.int32, device="cuda"), torch.zeros((5, 4), device="cuda")
    dsi.dsi_logprobs(s, 5, 2000, z, None, 4, None, None, ids, lp, ws, ws.numel())
    dsi.dsi_logprobs(s, 0, 2000, None, None, 4, None, b, ids, lp, None, 0)
    torch.cuda.synchronize()
    assert torch.equal(a, full["logprob"]) and torch.equal(b, full["entropy"])
    assert torch.equal(ids, full["ids"]) and torch.equal(lp, full["top"])


def test_two_streams_and_a_replayed_graph(dev):
    """Calls with workspaces of their own overlap; a captured call gives the eager results on new inputs."""
    z, t = logits(40, 32000, 7)
    z2, t2 = logits(40, 32000, 8)
    want, want2 = call(z, t, 5), call(z2, t2, 5)
    side = torch.cuda.Stream()
    buf, tb = z.clone(), t.clone()
    o = {"logprob": torch.zeros(40, device="cuda"), "entropy": torch.zeros(40, device="cuda"),
         "ids": torch.zeros((40, 5), dtype=torch.int32, device="cuda"), "top": torch.zeros((40, 5), device="cuda")}
    ws = torch.empty(dsi.dsi_logprobs_workspace(40, 32000, 5), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        dsi.dsi_logprobs(side.cuda_stream, 40, 32000, buf, tb, 5, o["logprob"], o["entropy"], o["ids"], o["top"], ws, ws.numel())
    for x, y, w in ((z2, t2, want2), (z, t, want), (z2, t2, want2)):
        buf.copy_(x)
        tb.copy_(y)
        for v in o.values():
            v.zero_()
        torch.cuda.synchronize()
        g.replay()
        other = call(z, t, 5, stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(o[k], w[k]) for k in o) and all(torch.equal(other[k], want[k]) for k in o)
