"""dsi_rotate and dsi_page_append on the GPU against norms and rotations in 64
bits: layouts, dims, types, strides, far positions, and where rows go in pages."""
import math

import pytest
import torch

from page_cases import HALF_STEP, KIND, Step, attend64
from paper_2405_14105_amd import dsi

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
STYLES = [dsi.DSI_ROPE_HALF, dsi.DSI_ROPE_PAIRS]


def turned64(x, pos, freq, gain, style, norm=None, eps=1e-5):
    """x [rows][heads][hd] in 64 bits: result, and what bounds its error."""
    x = x.double()
    hd, dim = x.shape[-1], 2 * len(freq)
    if norm is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * norm.double()
    y, mag = x.clone(), x.abs()
    a, b = (x[..., :dim // 2], x[..., dim // 2:dim]) if style == dsi.DSI_ROPE_HALF else (x[..., 0:dim:2], x[..., 1:dim:2])
    t = torch.outer(pos.double(), torch.tensor(freq, dtype=torch.float64))[:, None]
    turned = gain * (a * t.cos() - b * t.sin()), gain * (b * t.cos() + a * t.sin())
    both = abs(gain) * (a.abs() + b.abs())
    if style == dsi.DSI_ROPE_HALF:
        y[..., :dim // 2], y[..., dim // 2:dim] = turned
        mag[..., :dim // 2], mag[..., dim // 2:dim] = both, both
    else:
        y[..., 0:dim:2], y[..., 1:dim:2] = turned
        mag[..., 0:dim:2], mag[..., 1:dim:2] = both, both
    return y, mag


def close(got, ref, mag, hd, norm, kind):
    """Angles are reduced in fp64 and rounded to 2^-25 of a turn (2 pi 2^-25 < 2^-22), sines are good to 2^-22, the
    products round four times; a norm adds half the rounding of a sum of hd squares, and five operations."""
    tol = mag * (2.0 ** -21 + 4 * 2.0 ** -24 + ((hd / 2 + 8) * 2.0 ** -24 if norm else 0))
    tol = tol + ref.abs() * HALF_STEP[kind] + (0 if kind == F32 else tol * HALF_STEP[kind])
    err = (got.double() - ref).abs()
    assert (err <= tol).all(), (err / tol).nan_to_num(0).max()


def rows_of(n, heads, hd, act, seed, ld=0, device="cuda"):
    x = torch.randn((n, ld or heads * hd), generator=torch.Generator().manual_seed(seed)).to(act)
    return x.to(device)[:, :heads * hd]


def rotate(q, k, hq, hkv, hd, pos, freq, gain=1.0, style=0, gq=None, gk=None, place=False, dim=None):
    act = q.dtype
    f = torch.tensor(freq, dtype=torch.float64, device="cuda") if len(freq) else None
    qo = q if place else torch.full_like(q, 7.0)
    ko = k if place else torch.full_like(k, 7.0)
    dsi.dsi_rotate(torch.cuda.current_stream().cuda_stream, q.shape[0], hq, hkv, hd, q, k, pos.cuda() if pos is not None else None, qo, ko,
                   dsi.make_rope(2 * len(freq), f, gain, style), KIND[act], q.stride(0), k.stride(0), qo.stride(0), ko.stride(0), gq, gk)
    torch.cuda.synchronize()
    return qo, ko


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("style", STYLES)
@pytest.mark.parametrize("hd,dim", [(32, 32), (64, 64), (96, 96), (128, 128), (128, 64), (64, 34), (96, 2), (128, 126), (32, 0)])
@pytest.mark.parametrize("norm", [False, True])
def test_layouts_dims_and_norms(act, style, hd, dim, norm):
    hq, hkv, n = 5, 2, 7
    q, k = rows_of(n, hq, hd, act, 1), rows_of(n, hkv, hd, act, 2)
    pos = torch.tensor([0, 1, 2, 777, 100000, 1 << 20, -3], dtype=torch.int32)
    freq = dsi.dsi_rope_table(dim)[0] if dim else []
    g = [(1 + 0.1 * torch.randn(hd, generator=torch.Generator().manual_seed(i))) if norm else None for i in (3, 4)]
    qo, ko = rotate(q, k, hq, hkv, hd, pos, freq, 1.25, style, *[x.cuda() if x is not None else None for x in g])
    for x, o, heads, w in ((q, qo, hq, g[0]), (k, ko, hkv, g[1])):
        ref, mag = turned64(x.cpu().view(n, heads, hd), pos, freq, 1.25, style, w)
        got = o.cpu().view(n, heads, hd)
        close(got, ref, mag, hd, norm, act)
        if not norm:   # what is not rotated is kept to the bit
            assert torch.equal(got[..., dim:], x.cpu().view(n, heads, hd)[..., dim:])


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("rows,hq,hkv", [(1, 1, 1), (1, 32, 8), (3, 40, 40), (700, 4, 1), (9000, 12, 4)])
def test_rows_and_heads(act, rows, hq, hkv):
    hd = 64
    q, k = rows_of(rows, hq, hd, act, 1), rows_of(rows, hkv, hd, act, 2)
    pos = torch.arange(rows, dtype=torch.int32) + 5
    freq = dsi.dsi_rope_table(hd)[0]
    qo, ko = rotate(q, k, hq, hkv, hd, pos, freq)
    for x, o, heads in ((q, qo, hq), (k, ko, hkv)):
        ref, mag = turned64(x.cpu().view(rows, heads, hd), pos, freq, 1.0, 0)
        close(o.cpu().view(rows, heads, hd), ref, mag, hd, False, act)


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("style", STYLES)
@pytest.mark.parametrize("shift,pad", [(0, 64), (1, 0), (0, 3), (2, 1)])
def test_strides_alignment_and_in_place(act, style, shift, pad):
    """Parts of a fused projection's rows; the values between them stay."""
    hq, hkv, hd, n = 4, 2, 64, 9
    ld = shift + (hq + 2 * hkv) * hd + pad
    buf = torch.randn((n, ld), generator=torch.Generator().manual_seed(3)).to(act).cuda()
    was = buf.clone()
    q, k = buf[:, shift:shift + hq * hd], buf[:, shift + hq * hd:shift + (hq + hkv) * hd]
    pos = torch.arange(n, dtype=torch.int32) * 1000
    freq = dsi.dsi_rope_table(64)[0]
    qo, ko = rotate(q, k, hq, hkv, hd, pos, freq, 1.0, style)
    assert torch.equal(buf, was)
    rotate(q, k, hq, hkv, hd, pos, freq, 1.0, style, place=True)
    assert torch.equal(q, qo) and torch.equal(k, ko)
    rest = torch.ones(ld, dtype=torch.bool)
    rest[shift:shift + (hq + hkv) * hd] = False
    assert torch.equal(buf[:, rest.cuda()], was[:, rest.cuda()])
    ref, mag = turned64(was[:, shift:shift + hq * hd].cpu().reshape(n, hq, hd), pos, freq, 1.0, style)
    close(qo.cpu().reshape(n, hq, hd), ref, mag, hd, False, act)


def test_queries_or_keys_alone_and_no_rows():
    hd, n = 64, 3
    x = rows_of(n, 4, hd, F32, 1)
    pos, freq = torch.arange(n, dtype=torch.int32, device="cuda"), torch.tensor(dsi.dsi_rope_table(hd)[0], dtype=torch.float64, device="cuda")
    rope, s = dsi.make_rope(hd, freq), torch.cuda.current_stream().cuda_stream
    a, b = torch.zeros_like(x), torch.zeros_like(x)
    dsi.dsi_rotate(s, n, 4, 0, hd, x, None, pos, a, None, rope)
    dsi.dsi_rotate(s, n, 0, 4, hd, None, x, pos, None, b, rope)
    dsi.dsi_rotate(s, 0, 4, 4, hd, None, None, None, None, None, rope)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and a.abs().sum() > 0


# ------------------------------------------------------------------- append


def append(step, q, k, v, hq, freq, gain=1.0, style=0, gq=None, gk=None, pos=None, pages=None):
    out = torch.full_like(q, 7.0)
    f = torch.tensor(freq, dtype=torch.float64, device="cuda") if len(freq) else None
    dsi.dsi_page_append(torch.cuda.current_stream().cuda_stream, pages or step.pages(), step.n, hq, q, k, v, out, dsi.make_rope(2 * len(freq), f, gain, style),
                        KIND[q.dtype], q.stride(0), k.stride(0), v.stride(0), out.stride(0), pos, gq, gk)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("kv", [F32, BF16])
@pytest.mark.parametrize("style,hd,dim", [(0, 128, 128), (1, 64, 34), (0, 32, 30), (0, 96, 64), (1, 32, 0)])
@pytest.mark.parametrize("norm", [False, True])
def test_append(act, kv, style, hd, dim, norm):
    """Rows of ragged windows enter their pages; everything else of the pool, and rows of no window, stay."""
    hq, hkv = 6, 3
    step = Step([1, 0, 40, 7, 33, 8, 9], [95, 64, 20, 0, 31, 28, 24], hkv, hd, kv, 32, seed=hd, before=2, behind=3)
    step.k.zero_()
    step.v.zero_()
    was_k, was_v = step.k.clone(), step.v.clone()
    step.to("cuda")
    ld = (hq + 2 * hkv) * hd
    x = rows_of(step.n, hq + 2 * hkv, hd, act, 7, ld)
    q, k, v = x[:, :hq * hd], x[:, hq * hd:(hq + hkv) * hd], x[:, (hq + hkv) * hd:]
    freq = dsi.dsi_rope_table(dim)[0] if dim else []
    g = [(1 + 0.1 * torch.randn(hd, generator=torch.Generator().manual_seed(i))) if norm else None for i in (3, 4)]
    out = append(step, q, k, v, hq, freq, 0.75, style, *[w.cuda() if w is not None else None for w in g]).cpu()
    pos = torch.full((step.n,), -1, dtype=torch.int32)
    held_k, held_v = step.k.cpu(), step.v.cpu()
    r0 = step.before
    for b, (n, past) in enumerate(zip(step.rows, step.past)):
        rows, at = slice(r0, r0 + n), torch.arange(past, past + n)
        K, V = step.keys(b)
        ref, mag = turned64(k[rows].cpu().reshape(n, hkv, hd), at, freq, 0.75, style, g[1])
        close(K[past:], ref, mag, hd, norm, kv)
        assert torch.equal(V[past:], v[rows].cpu().reshape(n, hkv, hd).to(kv))
        ref, mag = turned64(q[rows].cpu().reshape(n, hq, hd), at, freq, 0.75, style, g[0])
        close(out[rows].view(n, hq, hd), ref, mag, hd, norm, act)
        pages, place = step.table[b].cpu().long()[at // 32], at % 32
        was_k[pages, :, 0, :, place] = held_k[pages, :, 0, :, place]
        was_v[pages, :, 0, :, place] = held_v[pages, :, 0, :, place]
        r0 += n
    assert torch.equal(held_k, was_k) and torch.equal(held_v, was_v)
    assert (out[:step.before] == 7).all() and (out[r0:] == 7).all()


@pytest.mark.parametrize("B", [64, 65, 130, 257, 1000, 4096])
def test_append_to_many_windows(B):
    hd = 32
    g = torch.Generator().manual_seed(B)
    rows = torch.randint(0, 3, (B,), generator=g).tolist()
    rows[B // 3] = 70
    past = torch.randint(0, 70, (B,), generator=g).tolist()
    step = Step(rows, past, 1, hd, BF16, 32, before=1, behind=2).to("cuda")
    x = rows_of(step.n, 1, hd, BF16, 5)
    out = append(step, x, x, x, 1, []).cpu()
    x, r0 = x.cpu(), step.before
    assert torch.equal(out[1:-2], x[1:-2]) and (out[:1] == 7).all() and (out[-2:] == 7).all()
    k, v, table = step.k.cpu(), step.v.cpu(), step.table.cpu().long()
    for b, n in enumerate(rows):
        at = torch.arange(past[b], past[b] + n)
        page, place = table[b][at // 32], at % 32
        assert torch.equal(k[page, 0, 0, 0, place], x[r0:r0 + n]) and torch.equal(v[page, 0, 0, :, place], x[r0:r0 + n])
        r0 += n


def test_append_without_queries_and_by_positions_of_its_own():
    """A token tree's rows: slots after each other, rotated by their depths."""
    hd, hkv = 64, 2
    step = Step([5, 3], [60, 7], hkv, hd, F32, 64).to("cuda")
    k, v = rows_of(8, hkv, hd, F32, 1), rows_of(8, hkv, hd, F32, 2)
    depth = torch.tensor([60, 61, 61, 62, 62, 7, 8, 8], dtype=torch.int32)
    f = torch.tensor(dsi.dsi_rope_table(hd)[0], dtype=torch.float64, device="cuda")
    dsi.dsi_page_append(torch.cuda.current_stream().cuda_stream, step.pages(), 8, 0, None, k, v, None, dsi.make_rope(hd, f), d_pos=depth.cuda())
    torch.cuda.synchronize()
    ref, mag = turned64(k.cpu().view(8, hkv, hd), depth, f.tolist(), 1.0, 0)
    close(torch.cat([step.keys(0)[0][60:], step.keys(1)[0][7:]]), ref, mag, hd, False, F32)


def test_rows_without_a_place_change_nothing():
    hd, hkv, hq = 64, 2, 2
    step = Step([4, 4, 4, 4], [30, 30, 30, 30], hkv, hd, BF16, 32).to("cuda")
    step.len = torch.tensor([-1, step.most * 32, 2 ** 31 - 1, 30], dtype=torch.int32, device="cuda")
    step.table[3] = torch.tensor([step.k.shape[0], -1] + [0] * (step.most - 2))
    was = step.k.clone(), step.v.clone()
    x = rows_of(step.n, 2, hd, BF16, 1)
    append(step, x, x, x, hq, dsi.dsi_rope_table(hd)[0])
    assert torch.equal(step.k.view(torch.int16), was[0].view(torch.int16)) and torch.equal(step.v.view(torch.int16), was[1].view(torch.int16))
    for row0 in ([-5, 20, 3, 9, 2], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 0, 5]):
        step.row0 = torch.tensor(row0, dtype=torch.int32, device="cuda")
        append(step, x, x, x, hq, dsi.dsi_rope_table(hd)[0])


@pytest.mark.parametrize("act,kv", [(F32, F32), (F32, BF16), (BF16, BF16)])
def test_a_server_step_by_step(act, kv):
    """A prompt in chunks, then single tokens and drafts that are taken back, on pages against the whole text at
    once: what append and attend do together, captured and replayed from the second chunk on."""
    hq, hkv, hd, page, B = 4, 2, 64, 32, 2
    lengths, g = [150, 90], torch.Generator().manual_seed(9)
    texts = [torch.randn((n, (hq + 2 * hkv) * hd), generator=g).to(act) for n in lengths]
    freq = dsi.dsi_rope_table(hd)[0]
    step = Step([75, 45], [75, 45], hkv, hd, kv, page).to("cuda")   # pages for 150 and 90 positions
    step.k.fill_(math.nan), step.v.fill_(math.nan)
    f = torch.tensor(freq, dtype=torch.float64, device="cuda")
    rope, pages = dsi.make_rope(hd, f), step.pages()
    most = 128
    x = torch.zeros((most, (hq + 2 * hkv) * hd), dtype=act, device="cuda")
    q, out = torch.zeros((most, hq * hd), dtype=act, device="cuda"), torch.zeros((most, hq * hd), dtype=act, device="cuda")
    nbytes = dsi.dsi_page_attend_workspace(pages, most, hq)
    ws = torch.zeros(nbytes, dtype=torch.uint8, device="cuda")

    def call():
        s = torch.cuda.current_stream().cuda_stream
        dsi.dsi_page_append(s, pages, most, hq, x, x[:, hq * hd:], x[:, (hq + hkv) * hd:], q, rope, KIND[act], x.stride(0), x.stride(0), x.stride(0))
        dsi.dsi_page_attend(s, pages, most, hq, q, out, ws, nbytes, KIND[act])

    got = [torch.zeros((n, hq * hd), dtype=act) for n in lengths]
    graph = None
    held = [0, 0]
    # rows of each window, and how many of them stay
    for rows, keep in (([70, 1], [70, 1]), ([1, 60], [1, 60]), ([6, 5], [2, 5]), ([4, 0], [4, 0]), ([70, 8], [60, 1]), ([13, 23], [13, 23])):
        step.len.copy_(torch.tensor(held))
        step.row0.copy_(torch.tensor([0, rows[0], sum(rows)]))
        x[:sum(rows)] = torch.cat([texts[b][held[b]:held[b] + rows[b]] for b in range(B)]).cuda()
        if graph is None:
            call()
            torch.cuda.synchronize()
            first = out.clone(), sum(rows)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                call()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out[:first[1]], first[0][:first[1]])
        else:
            graph.replay()
        torch.cuda.synchronize()
        o, r0 = out.cpu(), 0
        for b in range(B):
            got[b][held[b]:held[b] + rows[b]] = o[r0:r0 + rows[b]]
            r0 += rows[b]
            held[b] += keep[b]
    assert held == lengths
    for b, n in enumerate(lengths):
        t = texts[b].view(n, hq + 2 * hkv, hd)
        at = torch.arange(n)
        whole = Step([n], [0], hkv, hd, kv, page)
        whole.K, whole.V = [turned64(t[:, hq:hq + hkv], at, freq, 1.0, 0)[0].to(kv)], [t[:, hq + hkv:].to(kv)]
        qr = turned64(t[:, :hq], at, freq, 1.0, 0)[0].to(act)
        ref, mass, big = attend64(whole, qr, hq)
        # queries and keys carry a rotation's error (2^-20 in fp32, half a step of their type where they are rounded,
        # which may fall the other way): a score is off by those times the sum of magnitudes
        off = 2 * max(2.0 ** -20, 2 * HALF_STEP[act] if act == BF16 else 0, 2 * HALF_STEP[kv] if kv == BF16 else 0)
        tol = mass * (2 * big * off + 2.0 ** -17) + (ref.abs() + mass) * HALF_STEP[act]
        err = (got[b].double().view(n, hq, hd) - ref).abs()
        assert (err <= tol).all(), (err / tol).max()


@pytest.mark.parametrize("style", STYLES)
def test_sines_near_zero_keep_their_digits(style):
    """Pairs (1, 0) become (cos, sin): to 2^-21 of the value each (two steps of 2^-23 of the sine, half a step of the sum), and
    what fp64 leaves of the angle, three half steps of 2^-53.  An angle rounded to fp32 would be off by 2^-24 whatever the value."""
    hd, n = 128, 4096
    x = torch.zeros((n, hd))
    x[:, :hd // 2] = 1.0
    if style == dsi.DSI_ROPE_PAIRS:
        x = x.view(n, 2, hd // 2).transpose(1, 2).reshape(n, hd).contiguous()
    pos = torch.arange(n, dtype=torch.int32) * 37
    freq = dsi.dsi_rope_table(hd)[0]
    q, _ = rotate(x.cuda(), x.cuda().clone(), 1, 1, hd, pos, freq, 1.0, style)
    got = q.cpu().double()
    c, s = (got[:, :hd // 2], got[:, hd // 2:]) if style == dsi.DSI_ROPE_HALF else (got[:, 0::2], got[:, 1::2])
    angle = torch.outer(pos.double(), torch.tensor(freq, dtype=torch.float64))
    for y, ref in ((c, angle.cos()), (s, angle.sin())):
        tol = ref.abs() * 2.0 ** -21 + angle.abs() * 2.0 ** -51 + 2.0 ** -46
        err = (y - ref).abs()
        assert (err <= tol).all(), (err / tol).max()


@pytest.mark.parametrize("B,hkv,hd,page,kv", [(65, 2, 64, 64, BF16), (130, 8, 128, 96, BF16), (300, 3, 96, 64, F32)])
def test_append_to_many_windows_of_several_kv_heads(B, hkv, hd, page, kv):
    g = torch.Generator().manual_seed(B)
    rows, past = torch.randint(0, 3, (B,), generator=g).tolist(), torch.randint(0, 200, (B,), generator=g).tolist()
    rows[B // 3], rows[B - 1] = 100, 40
    step = Step(rows, past, hkv, hd, kv, page, before=1, behind=2).to("cuda")
    step.k.zero_(), step.v.zero_()
    k, v = rows_of(step.n, hkv, hd, BF16, 5), rows_of(step.n, hkv, hd, BF16, 6)
    freq = dsi.dsi_rope_table(hd)[0]
    out = append(step, k, k, v, hkv, freq).cpu().view(step.n, hkv, hd)
    step.to("cpu")
    k, v, r0 = k.cpu().view(step.n, hkv, hd), v.cpu().view(step.n, hkv, hd), step.before
    new_k = new_v = 0
    for b, n in enumerate(rows):
        at = torch.arange(past[b], past[b] + n)
        K, V = step.keys(b)
        ref, mag = turned64(k[r0:r0 + n], at, freq, 1.0, 0)
        close(K[past[b]:], ref, mag, hd, False, kv)
        close(out[r0:r0 + n], ref, mag, hd, False, BF16)
        assert torch.equal(V[past[b]:], v[r0:r0 + n].to(kv))
        new_k, new_v = new_k + (K[past[b]:] != 0).sum(), new_v + (V[past[b]:] != 0).sum()
        r0 += n
    assert (out[:1] == 7).all() and (out[-2:] == 7).all()
    assert (step.k != 0).sum() == new_k and (step.v != 0).sum() == new_v   # and nothing else
