"""Forked windows on the GPU: dsi_kv_fork against copies, dsi_attend against
attention in 64 bits over the same cache, dsi_verify and dsi_verify_tree of
forked windows against the same windows by themselves."""
import math

import numpy as np
import pytest
import torch

import dsi_synth as S
from gpu_rig import Rig
from share_cases import CASES
from paper_2405_14105_amd import dsi

pytestmark = pytest.mark.gpu

POISON = float("nan")


class Cache:
    """A cache in torch memory (dsi_kv_wrap) of a model that is a shape only."""

    def __init__(self, hq, hkv, hd, kind, windows, max_len, layers=1, seed=0):
        self.hq, self.hkv, self.hd, self.W, self.L, self.max_len = hq, hkv, hd, windows, layers, max_len
        self.dt = torch.float32 if kind == "f32" else torch.bfloat16
        cfg = dsi.make_config(layers, 32, hq, hkv, hd, 32, 32, kvdtype=dsi.DSI_F32 if kind == "f32" else dsi.DSI_BF16)
        self.model = dsi.dsi_model_create(cfg, torch.cuda.current_stream().cuda_stream)
        self.nb = -(-max_len // 64) * 2
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.k = torch.full((layers, windows, hkv, self.nb, hd // 32, 32, 32), POISON, device="cuda", dtype=self.dt)
        self.v = torch.full((layers, windows, hkv, self.nb, hd, 32), POISON, device="cuda", dtype=self.dt)
        nbytes = self.k.numel() * self.k.element_size()
        assert dsi.dsi_kv_bytes(self.model, windows, max_len) == nbytes
        self.kv = dsi.dsi_kv_wrap(self.model, windows, max_len, self.k, self.v, nbytes)

    def __enter__(self):
        return self

    def __exit__(self, *a):
        torch.cuda.synchronize()
        dsi.dsi_kv_destroy(self.kv)
        dsi.dsi_model_destroy(self.model)

    def rand(self, *shape, std=1.0):
        return torch.randn(shape, generator=self.gen, device="cuda") * std

    def keys(self, window, layer=0):       # [hkv][positions][hd]
        return _keys(self.k[layer, window])

    def values(self, window, layer=0):
        return _values(self.v[layer, window])

    def fill(self, window, a, b):
        """Random keys and values at positions [a, b) of a window, all layers."""
        for l in range(self.L):
            for p0 in range(a // 32, -(-b // 32)):
                lo, hi = max(a, 32 * p0) - 32 * p0, min(b, 32 * p0 + 32) - 32 * p0
                self.k[l, window, :, p0, :, lo:hi] = self.rand(self.hkv, self.hd // 32, hi - lo, 32).to(self.dt)
                self.v[l, window, :, p0, :, lo:hi] = self.rand(self.hkv, self.hd, hi - lo).to(self.dt)

    def attend(self, window0, windows, rows, q, k, v, layer=0, commit=False):
        out = torch.full((windows * rows, self.hq * self.hd), 7.0, device="cuda")
        dsi.dsi_attend(self.model, self.kv, layer, window0, windows, rows, q, k, v, out, commit)
        return out

    def rows(self, n, qstd=2.0):
        return self.rand(n, self.hq * self.hd, std=qstd), self.rand(n, self.hkv * self.hd), self.rand(n, self.hkv * self.hd)


def _keys(x):      # [hkv][nb][hd/32][32 pos][32] -> [hkv][positions][hd]
    h, nb, s, p, d = x.shape
    return x.permute(0, 1, 3, 2, 4).reshape(h, nb * p, s * d)


def _values(x):    # [hkv][nb][hd][32 pos]
    h, nb, d, p = x.shape
    return x.permute(0, 1, 3, 2).reshape(h, nb * p, d)


def attention64(c, window, n, q, k, v, layer=0):
    """out [rows][hq*hd] of rows behind n cached positions, and the bound on
    its error, in 64 bits."""
    R, G = q.shape[0], c.hq // c.hkv
    K = torch.cat([c.keys(window, layer)[:, :n], k.view(R, c.hkv, c.hd).transpose(0, 1).to(c.dt)], 1).double()
    V = torch.cat([c.values(window, layer)[:, :n], v.view(R, c.hkv, c.hd).transpose(0, 1).to(c.dt)], 1).double()
    Q = q.double().view(R, c.hkv, G, c.hd).permute(1, 2, 0, 3).reshape(c.hkv, G * R, c.hd)
    s = torch.matmul(Q, K.transpose(1, 2).contiguous()) / math.sqrt(c.hd)
    size = torch.matmul(Q.abs(), K.abs().transpose(1, 2).contiguous()) / math.sqrt(c.hd)
    see = torch.arange(n + R, device="cuda")[None, :] <= n + torch.arange(R, device="cuda")[:, None]
    see = see.repeat(G, 1)[None]
    p = torch.softmax(s.masked_fill(~see, -math.inf), -1)
    o = torch.matmul(p, V)
    # A score is off by at most its rounded queries' share (bf16 cache: hi + lo leave
    # half a step of a half step, 2^-18) and its fp32 sum's (hd terms); a weight by twice
    # that, by its own rounding (2^-18) and exp's; the sum over keys by its depth.
    split = 2.0 ** -18 if c.dt == torch.bfloat16 else 0.0
    ds = size.masked_fill(~see, 0).amax(-1, keepdim=True) * (split + (c.hd + 4) * 2.0 ** -24)
    rel = 2 * ds + split + 2.0 ** -20 + (n / 8 + 96) * 2.0 ** -24
    tol = rel * torch.matmul(p, V.abs())
    back = lambda x: x.view(c.hkv, G, R, c.hd).permute(2, 0, 1, 3).reshape(R, -1)
    return back(o), back(tol)


def check(c, out, window0, rows, lens, q, k, v, layer=0):
    for b, n in enumerate(lens):
        sl = slice(b * rows, b * rows + rows)
        ref, tol = attention64(c, window0 + b, n, q[sl], k[sl], v[sl], layer)
        d = (out[sl].double() - ref).abs()
        assert torch.isfinite(out[sl]).all(), f"window {window0 + b}"
        assert (d <= tol).all(), f"window {window0 + b}: {(d / tol).max().item():.2f} of the bound"


def forked(c, root, windows, prefix, tails):
    """Window `root` holds `prefix` positions, the others continue it by tails[w]."""
    c.fill(root, 0, prefix)
    dsi.dsi_kv_set_length(c.kv, root, prefix)
    for w in windows:
        if w != root:
            dsi.dsi_kv_fork(c.kv, root, w, 1, prefix)
    for w, t in zip(windows, tails):
        c.fill(w, prefix, prefix + t)
        dsi.dsi_kv_set_length(c.kv, w, prefix + t)
    return [prefix + t for t in tails]


SHAPES = [(4, 4, 32), (6, 2, 64), (8, 1, 64), (3, 3, 96), (8, 2, 96), (32, 8, 128), (5, 5, 128)]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd", SHAPES)
@pytest.mark.parametrize("windows,rows,prefix", [(2, 1, 128), (3, 5, 701), (7, 6, 1000)])
def test_shared_prefix(dev, kind, hq, hkv, hd, windows, rows, prefix):
    with Cache(hq, hkv, hd, kind, windows, prefix + 80 + rows) as c:
        lens = forked(c, 0, range(windows), prefix, [(37 * b + 5) % 71 for b in range(windows)])
        q, k, v = c.rows(windows * rows)
        check(c, c.attend(0, windows, rows, q, k, v), 0, rows, lens, q, k, v)


@pytest.mark.parametrize("prefix", [0, 1, 31, 32, 127, 129, 255, 256, 257, 511, 513, 2049])
@pytest.mark.parametrize("rows", [1, 3])
def test_prefix_lengths(dev, prefix, rows):
    with Cache(8, 2, 64, "bf16", 4, prefix + 40) as c:
        lens = forked(c, 0, range(4), prefix, [0, 1, 31, 33])
        q, k, v = c.rows(4 * rows)
        check(c, c.attend(0, 4, rows, q, k, v), 0, rows, lens, q, k, v)


@pytest.mark.parametrize("windows,rows", [(1, 1), (2, 2), (3, 11), (16, 4), (64, 1), (1, 64), (130, 1), (4, 150), (1, 1000)])
@pytest.mark.parametrize("hq,hkv,kind", [(8, 2, "bf16"), (4, 4, "f32")])
def test_row_counts(dev, windows, rows, hq, hkv, kind):
    with Cache(hq, hkv, 32, kind, windows, 400 + rows) as c:
        lens = forked(c, 0, range(windows), 333, [(7 * b) % 29 for b in range(windows)])
        q, k, v = c.rows(windows * rows)
        check(c, c.attend(0, windows, rows, q, k, v), 0, rows, lens, q, k, v)


@pytest.mark.parametrize("hq,hkv,hd,windows,rows,prefix,max_len,tiles,chunk", CASES)
def test_variants_of_the_shared_prefix(dev, hq, hkv, hd, windows, rows, prefix, max_len, tiles, chunk):
    with Cache(hq, hkv, hd, "bf16", windows, max_len) as c:
        lens = forked(c, 0, range(windows), prefix, [(37 * b + 5) % 71 for b in range(windows)])
        q, k, v = c.rows(windows * rows)
        check(c, c.attend(0, windows, rows, q, k, v), 0, rows, lens, q, k, v)


def test_three_groups_of_long_chunks(dev):
    with Cache(32, 8, 128, "bf16", 8, 6200) as c:
        lens = [0] * 8
        for wins, n in (((0, 1, 2), 6001), ((3, 4), 3000), ((5, 6, 7), 4500)):
            for w, x in zip(wins, forked(c, wins[0], wins, n, [11 * w % 37 for w in wins])):
                lens[w] = x
        q, k, v = c.rows(8 * 6)
        check(c, c.attend(0, 8, 6, q, k, v), 0, 6, lens, q, k, v)


def test_windows_of_their_own(dev):
    """No window was forked: long caches of each, and one that is empty."""
    with Cache(8, 2, 128, "bf16", 3, 3000) as c:
        lens = [2900, 0, 1031]
        for w, n in enumerate(lens):
            c.fill(w, 0, n)
            dsi.dsi_kv_set_length(c.kv, w, n)
        q, k, v = c.rows(3 * 4)
        check(c, c.attend(0, 3, 4, q, k, v), 0, 4, lens, q, k, v)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd,windows,rows", [(8, 2, 64, 4, 3), (8, 8, 32, 8, 1), (16, 2, 128, 3, 5)])
def test_long_continuations_and_a_window_beside_them(dev, kind, hq, hkv, hd, windows, rows):
    """Keys of the windows' own in several chunks: some, all, and one window that shares nothing."""
    prefix = 517
    for tails, lone in (([0, 0, 2900, 0, 700], 0), ([257, 1025, 3001], 1800), ([3], 5000), ([300], 33)):
        tails = [tails[i % len(tails)] for i in range(windows)]
        n = max([prefix + t for t in tails] + [lone])
        with Cache(hq, hkv, hd, kind, windows + 1, n + rows) as c:
            lens = forked(c, 0, range(windows), prefix, tails) + [lone]
            c.fill(windows, 0, lone)
            dsi.dsi_kv_set_length(c.kv, windows, lone)
            q, k, v = c.rows((windows + 1) * rows)
            check(c, c.attend(0, windows + 1, rows, q, k, v), 0, rows, lens, q, k, v)


def test_several_groups_and_a_root_outside_the_call(dev):
    with Cache(8, 2, 64, "bf16", 9, 1000) as c:
        lens = [0] * 9
        for root, wins, n in ((0, (1, 2, 3), 600), (8, (5, 6), 300)):
            for w, x in zip((root,) + wins, forked(c, root, (root,) + wins, n, [9 * w for w in (root,) + wins])):
                lens[w] = x
        c.fill(4, 0, 77)
        dsi.dsi_kv_set_length(c.kv, 4, 77)
        lens[4] = 77
        q, k, v = c.rows(6 * 2)
        check(c, c.attend(1, 6, 2, q, k, v), 1, 2, lens[1:7], q, k, v)
        check(c, c.attend(3, 3, 4, q, k, v), 3, 4, lens[3:6], q, k, v)


def test_sharing_ends_with_rollback_import_and_fork(dev):
    """After each the caches differ where they were shared; attention reads each window's own."""
    with Cache(4, 2, 64, "bf16", 4, 900, layers=2) as c:
        lens = forked(c, 0, range(4), 640, [0, 3, 40, 64])
        q, k, v = c.rows(4 * 2)

        def again(layer=1):
            check(c, c.attend(0, 4, 2, q, k, v, layer), 0, 2, lens, q, k, v, layer)

        def refill(w, a, b):
            c.fill(w, a, b)
            dsi.dsi_kv_set_length(c.kv, w, b)
            lens[w] = b
        again()
        dsi.dsi_kv_rollback(c.kv, 2, 400)
        refill(2, 400, 500)
        again()
        dsi.dsi_kv_rollback(c.kv, 0, 200)       # the window that the others continue
        refill(0, 200, 650)
        again()
        x = [c.rand(2, 300, 64).bfloat16() for _ in range(2)]
        dsi.dsi_kv_import(c.kv, 1, 1, 300, *x)
        again()
        dsi.dsi_kv_fork(c.kv, 3, 0, 1, 640)     # another prompt into the first root
        lens[0] = 640
        again()
        dsi.dsi_kv_set_length(c.kv, 3, 0)
        refill(3, 0, 130)
        again()


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_any_order_of_forks_and_cuts(dev, kind, seed):
    """Random forks (of forks, over roots), rollbacks, imports and commits: every window's own cache is what it attends to."""
    rng = np.random.default_rng(seed)
    W, most, rows = 6, 1500, 2
    with Cache(8, 2, 64, kind, W, most) as c:
        lens = [0] * W
        for step in range(40):
            w = int(rng.integers(W))
            op = rng.choice(["grow", "fork", "fork", "rollback", "import", "commit"])
            if op == "grow":                     # positions behind the length are the window's alone
                n = min(most - 64, lens[w] + int(rng.integers(1, 500)))
                if n > lens[w]:
                    c.fill(w, lens[w], n)
                    dsi.dsi_kv_set_length(c.kv, w, n)
                    lens[w] = n
            elif op == "fork":
                w0 = int(rng.integers(W))
                n = int(rng.integers(1, W - w0 + 1))
                if w < w0 or w >= w0 + n:
                    length = int(rng.integers(0, lens[w] + 1)) if rng.random() < 0.5 else -1
                    dsi.dsi_kv_fork(c.kv, w, w0, n, length)
                    lens[w0:w0 + n] = [lens[w] if length < 0 else length] * n
            elif op == "rollback":
                lens[w] = int(rng.integers(0, lens[w] + 1))
                dsi.dsi_kv_rollback(c.kv, w, lens[w])
            elif op == "import" and lens[w]:
                x = [c.rand(2, lens[w], 64).to(c.dt) for _ in range(2)]
                dsi.dsi_kv_import(c.kv, w, 0, lens[w], *x)
            w0 = int(rng.integers(W))
            n = int(rng.integers(1, W - w0 + 1))
            if max(lens[w0:w0 + n]) + rows > most:
                continue
            q, k, v = c.rows(n * rows)
            check(c, c.attend(w0, n, rows, q, k, v, commit=op == "commit"), w0, rows, lens[w0:w0 + n], q, k, v)
            if op == "commit":
                lens[w0:w0 + n] = [x + rows for x in lens[w0:w0 + n]]
        assert [dsi.dsi_kv_length(c.kv, w) for w in range(W)] == lens


def test_rows_that_are_not_finite_reach_only_those_that_see_them(dev):
    for kind in ("bf16", "f32"):
        with Cache(8, 2, 64, kind, 2, 300) as c:
            lens = forked(c, 0, range(2), 160, [5, 0])
            q, k, v = c.rows(2 * 6)
            for bad in (math.inf, -math.inf, math.nan):
                for t in (k, v):
                    t2 = t.clone()
                    t2[3], t2[6 + 5] = bad, bad    # row 3 of window 0, row 5 of window 1
                    out = c.attend(0, 2, 6, q, t2 if t is k else k, t2 if t is v else v)
                    clean = c.attend(0, 2, 6, q, k, v)
                    for r in (0, 1, 2, 6, 7, 8, 9, 10):
                        assert torch.equal(out[r], clean[r]), (kind, bad, r)
                    if t is v and bad == math.inf:
                        assert (out[3] == math.inf).all() and (out[5] == math.inf).all() and (out[11] == math.inf).all()
                    elif t is v:
                        assert not torch.isfinite(out[3:6]).any() and not torch.isfinite(out[11]).any()


def test_append_commit_and_what_stays(dev):
    """Rows are cached rounded to nearest even, lengths advance with commit, all other slots stay."""
    with Cache(4, 2, 96, "bf16", 3, 200, layers=2) as c:
        lens = forked(c, 0, range(3), 130, [0, 29, 30])
        q, k, v = c.rows(3 * 3)
        before = c.k.clone(), c.v.clone()
        c.attend(1, 2, 3, q, k, v, layer=1)
        assert [dsi.dsi_kv_length(c.kv, w) for w in range(3)] == lens
        c.attend(1, 2, 3, q, k, v, layer=1, commit=True)
        assert [dsi.dsi_kv_length(c.kv, w) for w in range(3)] == [lens[0], lens[1] + 3, lens[2] + 3]
        for b, w in enumerate((1, 2)):
            for i in range(3):
                blk, at = divmod(lens[w] + i, 32)
                before[0][1, w, :, blk, :, at] = k[b * 3 + i].view(2, 3, 32).bfloat16()
                before[1][1, w, :, blk, :, at] = v[b * 3 + i].view(2, 96).bfloat16()
        assert torch.equal(c.k.view(torch.int16), before[0].view(torch.int16))
        assert torch.equal(c.v.view(torch.int16), before[1].view(torch.int16))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("hkv,hd", [(1, 32), (3, 64), (2, 96), (8, 128)])
@pytest.mark.parametrize("length", [0, 1, 31, 32, 33, 95, 300, -1])
def test_fork_copies(dev, kind, hkv, hd, length):
    with Cache(hkv, hkv, hd, kind, 6, 333, layers=3) as c:
        for w in range(6):
            c.fill(w, 0, 300 if w == 2 else 40 * w)
            dsi.dsi_kv_set_length(c.kv, w, 300 if w == 2 else 40 * w)
        n = 300 if length < 0 else length
        want = c.k.clone(), c.v.clone()
        for dst in (3, 4, 5):
            for blk in range(c.nb):
                live = max(0, min(32, n - 32 * blk))
                want[0][:, dst, :, blk, :, :live] = want[0][:, 2, :, blk, :, :live]
                want[1][:, dst, :, blk, :, :live] = want[1][:, 2, :, blk, :, :live]
        dsi.dsi_kv_fork(c.kv, 2, 3, 3, length)
        assert [dsi.dsi_kv_length(c.kv, w) for w in range(6)] == [0, 40, 300, n, n, n]
        word = torch.int16 if kind == "bf16" else torch.int32
        assert torch.equal(c.k.view(word), want[0].view(word)) and torch.equal(c.v.view(word), want[1].view(word))


def test_fork_beyond_the_source_is_reported(dev):
    """The host knows a bound on a length; a fork past the length itself leaves the windows empty."""
    shape = S.SHAPES["tiny"]
    with Rig(shape, 0, 3, 200) as rig:
        rig.prefill(1, np.arange(50))
        bad = np.arange(60)
        bad[30] = shape.vocab                    # an invalid id: the prompt is not cached
        rig.prefill(0, bad)
        dsi.dsi_kv_fork(rig.kv, 0, 1, 2, 40)
        with pytest.raises(dsi.DsiError, match="fork beyond"):
            dsi.dsi_sync(rig.model)
        assert [rig.length(w) for w in range(3)] == [0, 0, 0]
        rig.prefill(0, np.arange(60))
        dsi.dsi_kv_fork(rig.kv, 0, 1, 2, 40)
        assert [rig.length(w) for w in range(3)] == [60, 40, 40]


def test_fork_of_a_window_past_the_caches_end(dev):
    """Replayed commits carry a length past max_len (still within the cache's last
    block of positions); a fork takes no positions from there and is reported."""
    shape, side = S.SHAPES["tiny"], torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side), Rig(shape, 0, 3, 100) as rig:
        rig.prefill(0, np.arange(90))
        rig.prefill(1, np.arange(9))
        rig.prefill(2, np.arange(7))
        t = rig.dev_i32([1])
        step = lambda: dsi.dsi_prefill(rig.model, rig.kv, 0, t, 1, None)
        step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step()
        for _ in range(14):                      # 91 + 14 positions; the cache's memory holds 128
            g.replay()
        torch.cuda.synchronize()
        dsi.dsi_kv_fork(rig.kv, 0, 1, 1)
        with pytest.raises(dsi.DsiError, match="fork beyond"):
            dsi.dsi_sync(rig.model)
        assert [rig.length(w) for w in range(3)] == [105, 0, 7]
        dsi.dsi_kv_rollback(rig.kv, 0, 100)
        dsi.dsi_kv_fork(rig.kv, 0, 1, 2)
        assert [rig.length(w) for w in range(3)] == [100, 100, 100]
        for w in (1, 2):
            for x, y in zip(rig.export_kv(0, 0, 100), rig.export_kv(w, 0, 100)):
                assert np.array_equal(x, y)


# ------------------------------------------------------------------- verification


@pytest.mark.parametrize("name", ["tiny", "gqa_hd64", "mha_hd128"])
@pytest.mark.parametrize("prefix", [100, 200, 517])
def test_verify_of_forked_windows(dev, name, prefix, monkeypatch):
    """Logits and decisions of forked windows against each window run by itself."""
    monkeypatch.setenv("DSI_SHARE", "1")
    shape, k, B = S.SHAPES[name], 4, 3
    rng = np.random.default_rng(prefix)
    prompt = rng.integers(0, shape.vocab, prefix)
    extra = [rng.integers(0, shape.vocab, n) for n in (0, 9, 40)]
    toks = rng.integers(0, shape.vocab, (B, k + 1))
    with Rig(shape, 0, B, prefix + 80) as rig:
        rig.prefill(0, prompt)
        dsi.dsi_kv_fork(rig.kv, 0, 1, B - 1)
        for w in range(B):
            if len(extra[w]):
                rig.prefill(w, extra[w])
        assert [rig.length(w) for w in range(B)] == [prefix + len(e) for e in extra]
        alone = [rig.verify(w, toks[w:w + 1], mode=dsi.DSI_GREEDY, commit=False) for w in range(B)]
        both = rig.verify(0, toks, mode=dsi.DSI_GREEDY, commit=False)
        la = np.concatenate([x["logits"] for x in alone])
        # two evaluations of one decoder, each within the project's bound on its
        # logits (1e-4 for fp32 weights, 2e-2 for bf16 ones) of the formula's
        bound = 2e-4 if shape.wdtype == "f32" else 4e-2
        assert np.abs(la - both["logits"]).max() <= bound
        tree = rig.verify_tree(0, toks, [[-1] + list(range(k))] * B, commit=False)
        assert np.abs(la - tree["logits"]).max() <= bound
        gap = np.sort(la, -1)
        if (gap[:, -1] - gap[:, -2]).min() > 2 * bound:
            assert [int(x["n"][0]) for x in alone] == list(both["n"])
            assert [int(x["token"][0]) for x in alone] == list(both["token"])
        # branches: two chains in one tree, and the committed path
        par = [[-1, 0, 1, 0, 3]] * B
        t1 = [rig.verify_tree(w, toks[w:w + 1], par[:1], commit=False)["logits"] for w in range(B)]
        t2 = rig.verify_tree(0, toks, par, commit=False)["logits"]
        assert np.abs(np.concatenate(t1) - t2).max() <= bound


def test_verify_of_a_long_shared_prefix(dev):
    """Long enough to be read once without being told."""
    shape, B = S.SHAPES["tiny"], 8
    rng = np.random.default_rng(1)
    n = (64 << 20) // (7 * 2 * shape.n_kv_heads * shape.head_dim * 4) + 40
    toks = rng.integers(0, shape.vocab, (B, 2))
    with Rig(shape, 0, B, n + 10) as rig:
        rig.prefill(0, rng.integers(0, shape.vocab, n))
        dsi.dsi_kv_fork(rig.kv, 0, 1, B - 1)
        alone = np.concatenate([rig.verify(w, toks[w:w + 1], mode=dsi.DSI_GREEDY, commit=False)["logits"] for w in range(B)])
        both = rig.verify(0, toks, mode=dsi.DSI_GREEDY, commit=False)["logits"]
        assert not np.array_equal(alone, both) and np.abs(alone - both).max() <= 2e-4


def test_verify_replays_of_forked_windows(dev, monkeypatch):
    """The recorded step is not replayed for another fork, and reads lengths and sharing as they are then."""
    monkeypatch.setenv("DSI_SHARE", "1")
    shape = S.SHAPES["tiny"]
    stream = torch.cuda.Stream()
    rng = np.random.default_rng(5)
    with torch.cuda.stream(stream), Rig(shape, 0, 3, 700) as rig:
        a, b = rng.integers(0, shape.vocab, 300), rng.integers(0, shape.vocab, 260)
        toks = rng.integers(0, shape.vocab, (3, 3)).astype(np.int32)
        t = rig.dev_i32(toks)
        n, tok = (torch.zeros(3, dtype=torch.int32, device="cuda") for _ in range(2))
        lg = torch.empty((9, shape.vocab), device="cuda")
        ref = torch.empty((9, shape.vocab), device="cuda")
        torch.cuda.synchronize()

        def step():
            dsi.dsi_verify(rig.model, rig.kv, 0, 3, 2, t, None, None, n, tok, 1.0, dsi.DSI_GREEDY, False, lg)
            for w in range(3):
                dsi.dsi_verify(rig.model, rig.kv, w, 1, 2, t[w], None, None, n[w:], tok[w:], 1.0, dsi.DSI_GREEDY, False, ref[3 * w:])
            torch.cuda.synchronize()
            assert (lg - ref).abs().max().item() <= 2e-4
        rig.prefill(0, a)
        dsi.dsi_kv_fork(rig.kv, 0, 1, 2)
        for _ in range(3):
            step()
        dsi.dsi_kv_rollback(rig.kv, 0, 140)      # what is shared shrinks to 140, then the root goes another way
        rig.prefill(0, b)
        for _ in range(2):
            step()
        dsi.dsi_kv_rollback(rig.kv, 1, 64)
        rig.prefill(1, b[:100])
        step()
        dsi.dsi_kv_fork(rig.kv, 2, 0, 2)         # another root for the same windows
        for _ in range(2):
            step()


# ------------------------------------------------------------------- together


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_decoding_from_a_fork(dev, kind):
    """A prompt forked into four windows that then go their own ways, several rows and one at a time."""
    with Cache(8, 2, 64, kind, 4, 700, layers=2) as c:
        lens = forked(c, 0, range(4), 517, [0, 0, 0, 0])
        for rows in (1, 5, 1, 1, 90, 1):
            for layer in range(2):
                q, k, v = c.rows(4 * rows)
                out = c.attend(0, 4, rows, q, k, v, layer, commit=layer == 1)
                check(c, out, 0, rows, lens, q, k, v, layer)
            lens = [n + rows for n in lens]
            assert [dsi.dsi_kv_length(c.kv, w) for w in range(4)] == lens


def test_replayed_attention(dev):
    """A captured step follows the lengths, what is still shared, and new inputs on every replay."""
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side), Cache(8, 2, 128, "bf16", 3, 900) as c:
        lens = forked(c, 0, range(3), 400, [0, 7, 20])
        buf = c.rows(3 * 2)
        out = c.attend(0, 3, 2, *buf)           # allocates
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            dsi.dsi_attend(c.model, c.kv, 0, 0, 3, 2, *buf, out, True)
        for i in range(5):
            if i == 2:
                dsi.dsi_kv_rollback(c.kv, 1, 256)
                c.fill(1, 256, 300)
                dsi.dsi_kv_set_length(c.kv, 1, 300)
                lens[1] = 300
            if i == 4:                           # another root: what the graph was captured for is no longer shared
                dsi.dsi_kv_set_length(c.kv, 2, lens[2])
                dsi.dsi_kv_fork(c.kv, 2, 0, 2, 390)
                lens[0] = lens[1] = 390
            new = c.rows(3 * 2)
            for x, y in zip(buf, new):
                x.copy_(y)
            out.fill_(7.0)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            check(c, out, 0, 2, lens, *new)
            lens = [n + 2 for n in lens]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_replays_until_the_cache_is_full(dev, kind):
    """A captured step replayed past max_len is reported: the full window gets no
    result and keeps its cache, the others go on."""
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side), Cache(4, 2, 64, kind, 4, 200) as c:
        lens = forked(c, 0, range(4), 130, [0, 62, 5, 63])
        buf = c.rows(3 * 3)
        out = c.attend(0, 3, 3, *buf)            # allocates
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            dsi.dsi_attend(c.model, c.kv, 0, 0, 3, 3, *buf, out, True)
        for i in range(5):
            new = c.rows(3 * 3)
            for x, y in zip(buf, new):
                x.copy_(y)
            out.fill_(7.0)
            before = c.k.clone(), c.v.clone()
            g.replay()
            torch.cuda.synchronize()
            full = lens[1] + 3 > 200
            assert full == (i >= 2)
            for b in range(3):
                sl = slice(3 * b, 3 * b + 3)
                if b == 1 and full:
                    assert out[sl].isnan().all()
                else:
                    ref, tol = attention64(c, b, lens[b], *(x[sl] for x in new))
                    assert ((out[sl].double() - ref).abs() <= tol).all(), (i, b)
                    lens[b] += 3
            word = torch.int16 if kind == "bf16" else torch.int32
            for now, was in zip((c.k, c.v), before):   # the full window, and the one behind the call
                assert torch.equal(now[:, 3].view(word), was[:, 3].view(word))
                assert not full or torch.equal(now[:, 1].view(word), was[:, 1].view(word))
            if full:
                with pytest.raises(dsi.DsiError, match="beyond the cache's end"):
                    dsi.dsi_sync(c.model)
            else:
                dsi.dsi_sync(c.model)
        assert [dsi.dsi_kv_length(c.kv, w) for w in range(4)] == lens == [145, 198, 150, 193]
        dsi.dsi_kv_fork(c.kv, 1, 0, 1)
        q, k, v = c.rows(2)
        assert dsi.dsi_kv_length(c.kv, 0) == 198
        check(c, c.attend(0, 1, 2, q, k, v), 0, 2, [198], q, k, v)


@pytest.mark.parametrize("name", ["tiny", "gqa_hd64"])
def test_scored_continuations(dev, name, monkeypatch):
    """Fork, verification and log probabilities together, against the oracle's decoder."""
    from oracle import forward64
    from paper_2405_14105_amd.executor import score_continuations

    monkeypatch.setenv("DSI_SHARE", "1")
    shape, T = S.SHAPES[name], 0.7
    rng = np.random.default_rng(3)
    prompt = rng.integers(0, shape.vocab, 200)
    conts = [list(map(int, rng.integers(0, shape.vocab, n))) for n in (5, 3, 0, 4)]
    get = lambda l, n: S.weight(shape, 0, l, n).astype(np.float64)
    with Rig(shape, 0, 6, 240) as rig:
        rig.prefill(5, prompt[:-1])
        got = [score_continuations(rig.model, rig.kv, 5, 1, int(prompt[-1]), conts, shape.vocab, T, 3) for _ in range(2)]
        assert [rig.length(w) for w in range(6)] == [0, 199, 199, 199, 199, 199]
    assert got[0] == got[1]
    # the project's bound on logits, for the token's and for log sum exp, over T; and fp32's rounding
    tol = 2 * (1e-4 if shape.wdtype == "f32" else 2e-2) / T + 1e-5
    for c, lp, H, ids, top in zip(conts, got[0].logprob, got[0].entropy, got[0].top_ids, got[0].top_logprobs):
        assert len(lp) == len(H) == len(ids) == len(top) == len(c)
        if not c:
            continue
        z = forward64(shape, get, np.concatenate([prompt, c[:-1]]))[0][len(prompt) - 1:] / T
        ref = z - z.max(-1, keepdims=True)
        ref -= np.log(np.exp(ref).sum(-1, keepdims=True))
        for i, tok in enumerate(c):
            assert abs(lp[i] - ref[i, tok]) <= tol
            for j in range(3):
                assert abs(top[i][j] - ref[i, ids[i][j]]) <= tol
            assert abs(top[i][0] - ref[i].max()) <= tol
            # entropy moves by at most tol (1 + |log p| spread) of the weights' change
            assert abs(H[i] + (np.exp(ref[i]) * ref[i]).sum()) <= tol * (2 + np.abs(ref[i] * np.exp(ref[i])).sum())
    with pytest.raises(ValueError):
        score_continuations(0, 0, 0, 1, 0, [[1] * 40] * 2, shape.vocab)
