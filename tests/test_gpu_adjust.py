"""dsi_adjust on the GPU against the formula in 64 bits: sizes, types, strides,
what rows have seen, repeated ids, masks, in place, and verification by it."""
import math

import pytest
import torch

from paper_2405_14105_amd import dsi

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
KIND = {F32: dsi.DSI_F32, BF16: dsi.DSI_BF16}
HALF_STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def make(B, R, V, act, seen=50, n_bias=5, allowed=50, pad=0, seed=0):
    g = torch.Generator().manual_seed(seed)
    s = {"B": B, "R": R, "V": V, "act": act}
    s["z"] = (torch.randn((B * R, V + pad), generator=g) * 5).to(act)[:, :V]
    s["seen"] = torch.randint(-2, V + 2, (B, max(1, seen)), generator=g, dtype=torch.int32)
    s["seen"][:, :seen // 2] = s["seen"][:, :1]          # one token many times
    s["n_seen"] = torch.randint(0, seen + 1, (B,), generator=g, dtype=torch.int32)
    s["n_seen"][0] = seen + 7                             # more than there are: all of them
    s["tokens"] = torch.randint(-1, V + 1, (B, R), generator=g, dtype=torch.int32)
    s["rep"], s["freq"], s["pres"] = 0.5 + torch.rand(B, generator=g), torch.rand(B, generator=g), torch.rand(B, generator=g) - 0.3
    s["ids"] = torch.randint(-1, V + 1, (B, n_bias), generator=g, dtype=torch.int32)
    if n_bias > 2:
        s["ids"][:, -1] = s["ids"][:, 0]                  # an id twice: the last entry counts
    s["bias"] = torch.randn((B, n_bias), generator=g)
    words = (V + 31) // 32
    s["mask"] = None
    if allowed is not None:
        bits = torch.rand((B * R, words * 32), generator=g) * 100 < allowed
        w = (bits.view(B * R, words, 32).long() << torch.arange(32)).sum(-1)
        s["mask"], s["bits"] = torch.where(w >= 2 ** 31, w - 2 ** 32, w).int(), bits[:, :V]
    return s


def formula(s):
    """Result and a bound of the kernel's error: four roundings in fp32 of magnitudes up to the sum of the terms', and the type's."""
    B, R, V = s["B"], s["R"], s["V"]
    out, tol = torch.empty((B * R, V), dtype=torch.float64), torch.empty((B * R, V), dtype=torch.float64)
    for b in range(B):
        held = s["seen"][b, :min(max(int(s["n_seen"][b]), 0), s["seen"].shape[1])].tolist() if s["seen"] is not None else []
        bias = torch.zeros(V, dtype=torch.float64)
        for i, v in zip(s["ids"][b].tolist(), s["bias"][b].double().tolist()):
            if 0 <= i < V:
                bias[i] = v
        for r in range(R):
            c = torch.zeros(V, dtype=torch.float64)
            for t in held + (s["tokens"][b, :r + 1].tolist() if s["tokens"] is not None else []):
                if 0 <= t < V:
                    c[t] += 1
            z = s["z"][b * R + r].double()
            one = lambda n, d: float(s[n][b]) if s[n] is not None else d  # noqa: E731
            rep, f, p = one("rep", 1.0), one("freq", 0.0), one("pres", 0.0)
            y = torch.where(c > 0, torch.where(z > 0, z / rep, z * rep), z)
            big = y.abs() + abs(f) * c + abs(p) * (c > 0) + bias.abs()
            y = y - f * c - p * (c > 0) + bias
            if s["mask"] is not None:
                y = torch.where(s["bits"][b * R + r], y, -math.inf)
            out[b * R + r], tol[b * R + r] = y, 4 * 2.0 ** -24 * big
    return out, tol + out.abs().nan_to_num(0, 0, 0) * HALF_STEP[s["act"]]


def call(s, place=False, stream=None):
    d = {k: v.cuda() if torch.is_tensor(v) and k != "z" else v for k, v in s.items()}
    whole = s["z"].as_strided((s["z"].shape[0], s["z"].stride(0)), (s["z"].stride(0), 1)).cuda()
    z = whole[:, :s["V"]]
    out = z if place else torch.full_like(whole, 7.0)[:, :s["V"]]
    dsi.dsi_adjust((stream or torch.cuda.current_stream()).cuda_stream, s["B"], s["R"], s["V"], z, out, KIND[s["act"]], z.stride(0), out.stride(0),
                   d["seen"], d["n_seen"] if s["seen"] is not None else None, s["seen"].shape[1] if s["seen"] is not None else 0, d["tokens"],
                   d["rep"], d["freq"], d["pres"], s["ids"].shape[1], d["ids"], d["bias"], d["mask"])
    torch.cuda.synchronize()
    if s["z"].stride(0) > s["V"] and not place:
        assert (out.as_strided((out.shape[0], out.stride(0) - s["V"]), (out.stride(0), 1), s["V"]) == 7).all()
    return out.cpu()


def check(s, got):
    ref, tol = formula(s)
    inf = ref.isinf()
    assert torch.equal(got.double()[inf], ref[inf])
    err = (got.double() - ref).abs()[~inf]
    assert (err <= tol[~inf]).all(), (err - tol[~inf]).max()


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("V", [1, 3, 8, 31, 33, 1000, 4095, 4096, 4097, 8200, 32003])
@pytest.mark.parametrize("place", [False, True])
def test_vocabularies(act, V, place):
    s = make(2, 3, V, act, seed=V)
    check(s, call(s, place))


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("B,R", [(1, 1), (1, 64), (64, 1), (7, 6), (3, 0), (0, 3)])
@pytest.mark.parametrize("pad", [0, 1, 5])
def test_rows_and_strides(act, B, R, pad):
    if B * R == 0:
        dsi.dsi_adjust(0, B, R, 10, None, None)
        return
    s = make(B, R, 5003, act, pad=pad, seed=B)
    check(s, call(s))
    check(s, call(s, True))


@pytest.mark.parametrize("place", [False, True])
@pytest.mark.parametrize("drop", [["mask"], ["seen"], ["tokens"], ["rep"], ["freq", "pres"], ["seen", "tokens", "mask"], ["rep", "freq", "pres", "mask"]])
def test_arguments_left_out(drop, place):
    s = make(3, 4, 4500, F32)
    for name in drop:
        s[name] = None
    check(s, call(s, place))


@pytest.mark.parametrize("seen", [0, 1, 5000, 40000])
@pytest.mark.parametrize("n_bias", [0, 1, 1024])
def test_lengths_of_lists(seen, n_bias):
    s = make(2, 2, 9001, F32, seen=seen, n_bias=n_bias)
    check(s, call(s))


@pytest.mark.parametrize("allowed", [0, 1, 99, 100])
@pytest.mark.parametrize("place", [False, True])
def test_masks(allowed, place):
    """A row of which the mask leaves nothing is -inf throughout."""
    s = make(2, 3, 6001, BF16, allowed=allowed)
    check(s, call(s, place))


def test_values_that_are_not_finite():
    s = make(1, 2, 5000, F32, allowed=50)
    s["z"][:, 0:4000:7] = -math.inf
    s["z"][:, 1:4000:7] = math.nan
    s["z"][:, 2:4000:7] = math.inf
    s["z"][:, 3:4000:7] = torch.finfo(F32).min
    s["rep"] = torch.tensor([1.3])
    ref, _ = formula(s)
    for place in (False, True):
        got = call(s, place).double()
        # the lowest number of the type times a repetition, or less a penalty, is below every fp32
        low = ref < torch.finfo(F32).min * (1 + 2.0 ** -25)
        assert torch.equal(got.isnan(), ref.isnan())
        assert (got[low] == -math.inf).all()
        rest = ~low & ~ref.isnan()
        assert torch.equal(got[rest].isinf(), ref[rest].isinf())
        fin = rest & ~ref.isinf()
        assert ((got - ref).abs()[fin] <= 2.0 ** -21 * ref.abs()[fin].clamp(min=64)).all()


def test_nothing_else_of_a_row_is_touched_in_place():
    """Runs of 16 bytes that nothing changes are not written: what another stream writes there meanwhile stays (here: their bits)."""
    s = make(1, 1, 6000, F32, n_bias=0, allowed=None, seen=3)
    s["z"][:] = torch.tensor(float("nan"))   # a pattern that arithmetic would change
    s["z"].view(torch.int32)[:] = 0x7FA12345
    s["seen"][:], s["n_seen"][:], s["tokens"][:] = 17, 3, 4100
    got = call(s, True).view(torch.int32)
    rest = torch.ones(6000, dtype=torch.bool)
    rest[16:20] = rest[4100:4104] = False
    assert (got[0, rest] == 0x7FA12345).all()


def test_verification_by_adjusted_logits():
    """A verified window whose rows are judged by the text they continue: dsi_adjust, then dsi_accept, equal the
    argmax walk over the formula; captured and replayed with other tokens."""
    B, R, V = 3, 5, 2003
    s = make(B, R, V, F32, allowed=80, seed=4)
    s["tokens"] = torch.randint(0, V, (B, R), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    d = {k: v.cuda() if torch.is_tensor(v) else v for k, v in s.items()}
    out, n, tok = torch.empty((B * R, V), device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")

    def step():
        st = torch.cuda.current_stream().cuda_stream
        dsi.dsi_adjust(st, B, R, V, d["z"], out, dsi.DSI_F32, d_seen=d["seen"], d_n_seen=d["n_seen"], ld_seen=s["seen"].shape[1], d_tokens=d["tokens"],
                       d_repetition=d["rep"], d_frequency=d["freq"], d_presence=d["pres"], n_bias=s["ids"].shape[1], d_bias_ids=d["ids"], d_bias=d["bias"],
                       d_allowed=d["mask"])
        dsi.dsi_accept_noalloc(st, B, R - 1, V, out, d["tokens"], None, None, n, tok, mode=dsi.DSI_GREEDY)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    for turn in range(4):
        want = formula(s)[0].view(B, R, V).argmax(-1)
        for b in range(B):   # drafts that agree for a while
            s["tokens"][b, 1:1 + (turn + b) % R] = -1
            for i in range(1, 1 + (turn + b) % R):
                if i < R:
                    s["tokens"][b, i] = int(formula(s)[0].view(B, R, V)[b, i - 1].argmax())
        d["tokens"].copy_(s["tokens"].clamp(min=0))
        s["tokens"] = s["tokens"].clamp(min=0)
        graph.replay()
        torch.cuda.synchronize()
        best = formula(s)[0].view(B, R, V).argmax(-1)
        for b in range(B):
            k = 0
            while k < R - 1 and int(best[b, k]) == int(s["tokens"][b, k + 1]):
                k += 1
            assert int(n[b]) == k and int(tok[b]) == int(best[b, k])
        s["tokens"] = torch.randint(0, V, (B, R), generator=torch.Generator().manual_seed(turn + 2), dtype=torch.int32)


@pytest.mark.parametrize("act", [F32, BF16])
def test_entries_that_nothing_changes_are_not_written_in_place(act):
    """bf16: a NaN whose quiet bit is clear would come back with it set from a run that is read, rounded and written."""
    s = make(2, 3, 9001, act, n_bias=0, allowed=None, seen=2)
    bits, pattern = (torch.int32, 0x7FA12345) if act == F32 else (torch.int16, 0x7FA1)
    s["z"].view(bits)[:] = pattern
    s["seen"][:], s["n_seen"][:], s["tokens"][:] = torch.tensor([17, 8999]), 2, 4100
    got = call(s, True).view(bits)
    run = 16 // s["z"].element_size()   # entries of 16 bytes
    rest = torch.ones(9001, dtype=torch.bool)
    for token in (17, 8999, 4100):
        rest[token // run * run:token // run * run + run] = False
    assert (got[:, rest] == pattern).all()
    assert act == F32 or (got[:, 4101] != pattern).all()   # what the pattern shows where a run was written


def test_repetition_over_a_text_and_penalties_over_its_output_alone():
    """Two calls, the second in place: one count serves the three penalties of a call."""
    B, R, V = 3, 4, 5003
    s = make(B, R, V, F32, n_bias=5, allowed=70, seed=2)
    text, output = dict(s), dict(s)
    text.update(freq=None, pres=None, mask=None, ids=torch.zeros((B, 0), dtype=torch.int32), bias=torch.zeros((B, 0)))
    output.update(rep=None, seen=s["seen"][:, -9:].contiguous(), n_seen=torch.tensor([9, 0, 5], dtype=torch.int32))
    first, tol = formula(text)
    output["z"] = call(text)
    got = call(output, True)
    output["z"] = first
    ref, more = formula(output)
    inf = ref.isinf()
    assert torch.equal(got.double()[inf], ref[inf])
    assert ((got.double() - ref).abs() <= tol + more)[~inf].all()
