"""Host code of the calls on pages, of dsi_rotate, dsi_rope_table and dsi_adjust,
without a GPU: frequencies, refusals, workspaces, and what is launched."""
import ctypes
import math

import pytest

from paper_2405_14105_amd import dsi
from test_host_runtime import pytestmark, run, stub  # noqa: F401

P = 4096
BIG = 2 ** 31 - 1


def refused(f, ok, *changes, status=dsi.DSI_EINVAL):
    for change in changes:
        with pytest.raises(dsi.DsiError) as e:
            f(**{**ok, **change})
        assert e.value.status == status, change


def test_frequencies():
    dim, base = 64, 10000.0
    plain = [base ** (-2 * j / dim) for j in range(dim // 2)]
    f, gain = dsi.dsi_rope_table(dim, base)
    assert gain == 1 and f == pytest.approx(plain, rel=1e-14)
    f, gain = dsi.dsi_rope_table(dim, base, dsi.DSI_ROPE_LINEAR, 8)
    assert gain == 1 and f == pytest.approx([x / 8 for x in plain], rel=1e-14)
    f, gain = dsi.dsi_rope_table(dim, base, dsi.DSI_ROPE_BASE, 8)
    assert gain == 1 and f[0] == 1 and f[-1] == pytest.approx(plain[-1] / 8, rel=1e-13)   # the slowest wave as with LINEAR
    f, gain = dsi.dsi_rope_table(dim, base, dsi.DSI_ROPE_BANDS, 8, low=1, high=4, context=8192)
    turns = [8192 * x / (2 * math.pi) for x in plain]
    assert gain == 1 and any(1 < c < 4 for c in turns)
    for got, x, c in zip(f, plain, turns):
        s = min(max((c - 1) / 3, 0), 1)
        assert got == pytest.approx((1 - s) * x / 8 + s * x, rel=1e-14)
    assert f[0] == 1 and f[-1] == pytest.approx(plain[-1] / 8, rel=1e-14)
    f, gain = dsi.dsi_rope_table(dim, base, dsi.DSI_ROPE_RAMP, 8, low=1, high=32, context=8192)
    assert gain == pytest.approx(0.1 * math.log(8) + 1, rel=1e-7)
    at = lambda c: dim * math.log(8192 / (2 * math.pi * c)) / (2 * math.log(base))  # noqa: E731
    lo, hi = math.floor(at(32)), math.ceil(at(1))
    for j, (got, x) in enumerate(zip(f, plain)):
        s = min(max((j - lo) / (hi - lo), 0), 1)
        assert got == pytest.approx(s * x / 8 + (1 - s) * x, rel=1e-14)
    assert dsi.dsi_rope_table(2)[0] == [1.0]


def test_frequency_refusals():
    lib = dsi.load()
    ok = dict(dim=64, base=1e4, scaling=dsi.DSI_ROPE_RAMP, factor=4.0, low=1.0, high=32.0, context=4096.0)
    dsi.dsi_rope_table(**ok)
    nan, inf = math.nan, math.inf
    refused(dsi.dsi_rope_table, ok, dict(dim=0), dict(dim=3), dict(dim=-2), dict(dim=258), dict(scaling=5), dict(scaling=-1), dict(base=1.0),
            dict(base=nan), dict(base=inf), dict(factor=0.5), dict(factor=nan), dict(factor=inf), dict(low=0.0), dict(low=32.0), dict(high=inf),
            dict(low=nan), dict(context=0.0), dict(context=nan), dict(context=inf), dict(scaling=dsi.DSI_ROPE_BASE, dim=2))
    assert lib.dsi_rope_table(None, None, None) == dsi.DSI_EINVAL


def test_rotate_refusals(stub):
    rope = lambda **k: dsi.make_rope(**{**dict(dim=64, d_freq=P), **k})  # noqa: E731
    ok = dict(stream=0, rows=5, n_heads=4, n_kv_heads=2, head_dim=64, d_q=1 << 20, d_k=2 << 20, d_pos=P, d_q_out=3 << 20, d_k_out=4 << 20, rope=rope())
    refused(dsi.dsi_rotate, ok, dict(rows=-1), dict(rows=(1 << 22) + 1), dict(n_heads=-1), dict(n_kv_heads=1025), dict(head_dim=48), dict(head_dim=160),
            dict(head_dim=0), dict(dtype=2), dict(d_q=None), dict(d_k=None), dict(d_q_out=None), dict(d_k_out=None), dict(d_pos=None), dict(d_pos=P + 2),
            dict(ld_q=255), dict(ld_k=127), dict(ld_q_out=-1), dict(ld_q=(1 << 40) + 1), dict(d_q=(1 << 20) + 2), dict(dtype=1, d_q=(1 << 20) + 1),
            dict(rope=rope(dim=63)), dict(rope=rope(dim=66)), dict(rope=rope(dim=-2)), dict(rope=rope(style=2)), dict(rope=rope(d_freq=None)),
            dict(rope=rope(d_freq=P + 4)), dict(rope=rope(gain=math.nan)), dict(d_gain_q=P, eps=-1.0), dict(d_gain_k=P, eps=math.nan), dict(d_gain_k=P + 1),
            dict(d_q_out=(1 << 20) + 64), dict(d_q_out=1 << 20, ld_q_out=512), dict(d_k_out=(2 << 20) - 64))
    assert dsi.load().dsi_rotate(None, None) == dsi.DSI_EINVAL
    dsi.dsi_rotate(**{**ok, "rows": 0, "d_q": None, "d_k": None, "d_pos": None})
    dsi.dsi_rotate(**{**ok, "n_heads": 0, "n_kv_heads": 0, "d_q": None, "d_k": None})
    run(stub, '''
    rope = dsi.make_rope(64, P)
    def grid(rows=5, hq=4, hkv=2, hd=64, dtype=0, **k):
        hip.stub_clear()
        dsi.dsi_rotate(0, rows, hq, hkv, hd, 1 << 30, 2 << 30, P, 3 << 30, 4 << 30, k.pop("rope", rope), dtype, **k)
        (name, args, g), = launches()
        return g[0]
    assert grid(1, 32, 8) > 0
    dsi.dsi_rotate(0, 5, 4, 2, 64, 1 << 20, 2 << 20, P, 1 << 20, 2 << 20, rope)          # in place
    dsi.dsi_rotate(0, 5, 4, 2, 64, 1 << 20, 2 << 20, None, 3 << 20, 4 << 20, dsi.make_rope(0, None))   # norms alone
    # groups of heads that a wave takes at a time: 64 lanes of 16 bytes a half
    groups = lambda heads, per: -(-heads // per)
    assert grid(1, 32, 8, 64) == -(-groups(40, 8) // 4) and grid(1, 40, 40, 128) == -(-groups(80, 4) // 4)
    assert grid(1, 32, 8, 64, 1) == -(-groups(40, 16) // 4)
    # 15 pairs in four lanes, 34 entries that are not turned in five: 16 lanes a head
    assert grid(1, 32, 8, 64, rope=dsi.make_rope(30, P)) == -(-groups(40, 4) // 4)
    assert grid(5000, 40, 40, 128) == 1250
    assert not hip.stub_mallocs()
    ''')


PAGES = dict(n_kv_heads=2, head_dim=64, kvdtype=dsi.DSI_BF16, n_pages=100, page_size=64, d_k=1 << 20, d_v=2 << 20, n_windows=3, max_pages=8, d_table=P,
             d_len=P, d_row0=P)
BAD_PAGES = [dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(head_dim=80), dict(head_dim=160), dict(kvdtype=2), dict(n_pages=0), dict(n_pages=-3),
             dict(page_size=0), dict(page_size=16), dict(page_size=48), dict(page_size=-32), dict(max_pages=0), dict(max_pages=1 << 25), dict(n_windows=0),
             dict(n_windows=4097), dict(n_pages=BIG), dict(page_size=1 << 30, max_pages=2)]
NULL_PAGES = [dict(d_k=None), dict(d_v=None), dict(d_k=P + 8), dict(d_v=P + 2), dict(d_table=None), dict(d_len=None), dict(d_row0=None), dict(d_table=P + 1),
              dict(d_len=P + 2), dict(d_row0=P + 3)]


def test_append_refusals():
    rope = dsi.make_rope(64, P)
    ok = dict(stream=0, pages=dsi.make_pages(**PAGES), rows=5, n_heads=4, d_q=1 << 20, d_k=2 << 20, d_v=3 << 20, d_q_out=4 << 20, rope=rope)
    refused(dsi.dsi_page_append, ok, *[dict(pages=dsi.make_pages(**{**PAGES, **c})) for c in BAD_PAGES + NULL_PAGES])
    refused(dsi.dsi_page_append, ok, dict(rows=-1), dict(n_heads=-1), dict(dtype=7), dict(d_q=None), dict(d_k=None), dict(d_v=None), dict(d_q_out=None),
            dict(ld_v=127), dict(ld_k=1), dict(d_v=P + 1), dict(d_pos=P + 1), dict(rope=dsi.make_rope(66, P)), dict(d_q_out=(1 << 20) + 16),
            dict(d_gain_q=P, eps=math.inf))
    lib = dsi.load()
    assert lib.dsi_page_append(None, None, None) == dsi.DSI_EINVAL
    assert lib.dsi_page_append(None, None, ctypes.byref(dsi.dsi_page_append_args())) == dsi.DSI_EINVAL
    dsi.dsi_page_append(**{**ok, "rows": 0, "d_q": None, "d_k": None, "d_v": None})


def test_attend_refusals_and_workspace():
    lib = dsi.load()
    pages = dsi.make_pages(**PAGES)
    need = dsi.dsi_page_attend_workspace(pages, 5, 4)
    ok = dict(stream=0, pages=pages, rows=5, n_heads=4, d_q=1 << 20, d_out=2 << 20, d_ws=3 << 20, ws_bytes=need)
    refused(dsi.dsi_page_attend, ok, *[dict(pages=dsi.make_pages(**{**PAGES, **c})) for c in BAD_PAGES + NULL_PAGES])
    refused(dsi.dsi_page_attend, ok, dict(rows=-1), dict(rows=(1 << 22) + 1), dict(n_heads=0), dict(n_heads=3), dict(n_heads=1026), dict(dtype=2),
            dict(reach=-1), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(d_q=None), dict(d_out=None), dict(d_q=(1 << 20) + 8),
            dict(d_out=(2 << 20) + 4), dict(ld_q=255), dict(ld_q=257), dict(ld_out=258), dict(dtype=1, ld_q=260), dict(d_out=1 << 20),
            dict(d_out=(1 << 20) + 256), dict(d_ws=None), dict(d_ws=(3 << 20) + 8), dict(ws_bytes=need - 1))
    dsi.dsi_page_attend(**{**ok, "rows": 0, "d_q": None, "d_out": None, "d_ws": None, "ws_bytes": 0})
    assert dsi.dsi_page_attend_workspace(pages, 0, 4) == 0
    n = ctypes.c_size_t()
    assert lib.dsi_page_attend_workspace(None, 5, 4, ctypes.byref(n)) == dsi.DSI_EINVAL
    assert lib.dsi_page_attend_workspace(ctypes.byref(pages), 5, 4, None) == dsi.DSI_EINVAL
    assert lib.dsi_page_attend(None, None, None) == dsi.DSI_EINVAL
    wide = dsi.make_pages(**{**PAGES, "n_kv_heads": 1})
    refused(dsi.dsi_page_attend_workspace, dict(pages=wide, rows=1 << 22, n_heads=64), dict(n_heads=65))
    # a workspace holds the parts of tiles that are cut, however many rows there are, and of no more chunks than
    # the pages have units of 128 keys
    slot = 32 * (64 * 4 + 8)
    assert dsi.dsi_page_attend_workspace(pages, 1 << 22, 4) == 2 * 2 * 2048 * slot
    assert dsi.dsi_page_attend_workspace(pages, 1, 4) == (1 + 1) * 2 * 4 * slot
    crowd = dsi.make_pages(**{**PAGES, "n_windows": 65})   # whose cut is written down: 4 + 3 * 65 numbers a kind of windows
    assert dsi.dsi_page_attend_workspace(crowd, 1 << 22, 4) == 2 * 2 * 2048 * slot + 2 * 800
    long = dsi.make_pages(**{**PAGES, "max_pages": 1 << 20})
    assert dsi.dsi_page_attend_workspace(long, 1, 4) == 2 * 2048 * slot
    # rows of the output may lie among those of the queries
    dsi_rows = dict(ok, d_q=1 << 20, d_out=(1 << 20) + 256 * 4, ld_q=600, ld_out=600)
    refused(dsi.dsi_page_attend, dsi_rows, dict(d_out=(1 << 20) + 255 * 4), dict(d_out=(1 << 20) + 348 * 4), dict(ld_out=604))


def test_adjust_refusals(stub):
    ok = dict(stream=0, n_windows=2, rows=3, vocab=1000, d_logits=1 << 20, d_out=2 << 20, d_seen=P, d_n_seen=P, ld_seen=10, d_tokens=P, d_repetition=P,
              d_frequency=P, d_presence=P, n_bias=4, d_bias_ids=P, d_bias=P, d_allowed=P)
    refused(dsi.dsi_adjust, ok, dict(n_windows=-1), dict(rows=-1), dict(n_windows=BIG, rows=BIG), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(dtype=2),
            dict(n_bias=-1), dict(n_bias=1025), dict(d_n_seen=None), dict(d_seen=None), dict(ld_seen=0), dict(ld_seen=(1 << 21) - 3), dict(ld_seen=-1),
            dict(n_windows=1, rows=1 << 21, d_seen=None, d_n_seen=None), dict(d_logits=None), dict(d_out=None), dict(d_logits=P + 2), dict(ld=999), dict(ld_out=1),
            dict(d_bias_ids=None), dict(d_bias=None), dict(ld_allowed=31), dict(d_allowed=P + 2), dict(d_tokens=P + 1), dict(d_bias=P + 2),
            dict(d_out=(1 << 20) + 16), dict(d_out=1 << 20, ld_out=1004), dict(rows=1 << 20, n_windows=4, vocab=1 << 30))
    assert dsi.load().dsi_adjust(None, None) == dsi.DSI_EINVAL
    for none in (dict(rows=0), dict(n_windows=0)):
        dsi.dsi_adjust(**{**ok, **none, "d_logits": None, "d_out": None})
    run(stub, '''
    def grid(B, R, V, place=False, dtype=0):
        hip.stub_clear()
        dsi.dsi_adjust(0, B, R, V, 1 << 20, 1 << 20 if place else 1 << 30, dtype)
        (name, args, g), = launches()
        assert name == "k_adjust"
        return g[0]
    # workgroups: vocabulary chunks, windows, and groups of rows while there are fewer than the card takes
    assert grid(1, 1, 4096) == 1 and grid(1, 1, 4097) == 2 and grid(1, 1, 4097, True, 1) == 2
    assert grid(1, 64, 4096) == 64
    assert grid(64, 1, 128256) == 64 * 32
    assert grid(7, 6, 128256) == 7 * 32 * 3
    assert not hip.stub_mallocs()
    ''')


def test_outputs_apart_from_the_other_rows(stub):
    """The parts of one fused row (queries, keys, values), and what overlaps them."""
    at = 1 << 20
    ok = dict(stream=0, rows=5, n_heads=4, n_kv_heads=2, head_dim=64, d_q=at, d_k=at + 1024, d_pos=P, d_q_out=at, d_k_out=at + 1024,
              rope=dsi.make_rope(64, P), ld_q=512, ld_k=512, ld_q_out=512, ld_k_out=512)
    refused(dsi.dsi_rotate, ok, dict(d_q_out=at + 1024), dict(d_q_out=2 << 20, d_k_out=at), dict(d_q_out=2 << 20, d_k_out=2 << 20),
            dict(d_q_out=at + 1536 + 1024), dict(d_q_out=2 << 20, d_k_out=(2 << 20) + 1020),
            dict(d_q_out=2 << 20, ld_q_out=256, d_k_out=(2 << 20) + 1024))
    pages = dsi.make_pages(2, 64, dsi.DSI_BF16, 8, 32, P, 2 * P, 1, 4, 3 * P, 4 * P, 5 * P)
    ok = dict(stream=0, pages=pages, rows=5, n_heads=4, d_q=at, d_k=at + 1024, d_v=at + 1536, d_q_out=at, rope=dsi.make_rope(64, P),
              ld_q=512, ld_k=512, ld_v=512, ld_q_out=512)
    refused(dsi.dsi_page_append, ok, dict(d_q_out=at + 1024), dict(d_q=2 << 20, d_q_out=at + 512), dict(d_q=2 << 20, d_q_out=at + 1536, ld_q_out=640))
    run(stub, '''
    rope = dsi.make_rope(64, 4096)
    at = 1 << 20
    hip.stub_clear()
    dsi.dsi_rotate(0, 5, 4, 2, 64, at, at + 1024, 4096, at, at + 1024, rope, ld_q=512, ld_k=512, ld_q_out=512, ld_k_out=512)
    dsi.dsi_rotate(0, 1, 4, 2, 64, at, at + 1024, 4096, at + 4096, at + 8192, rope)
    ''')


def test_adjust_refuses_lists_of_any_size_too_long():
    """Lengths whose sum with the rows would pass 64 bits, and those just too long."""
    ok = dict(stream=0, n_windows=2, rows=3, vocab=1000, d_logits=1 << 20, d_out=2 << 20, d_seen=P, d_n_seen=P, ld_seen=10)
    refused(dsi.dsi_adjust, ok, dict(ld_seen=(1 << 63) - 1), dict(ld_seen=(1 << 63) - 3), dict(ld_seen=1 << 31), dict(ld_seen=(1 << 21) - 3),
            dict(ld_seen=-(1 << 63)), dict(n_windows=1, rows=(1 << 22), ld_seen=1))


def test_attend_refuses_scales_that_are_infinite_to_the_base_2(stub):
    """Scores are kept to the base 2: a scale times log2(e) has to be a number."""
    ok = dict(stream=0, pages=dsi.make_pages(**PAGES), rows=5, n_heads=4, d_q=1 << 20, d_out=2 << 20, d_ws=3 << 20, ws_bytes=1 << 30)
    refused(dsi.dsi_page_attend, ok, dict(scale=2.36e38), dict(scale=3.4e38), dict(scale=math.inf), dict(scale=-math.inf))
    run(stub, '''
    pages = dsi.make_pages(2, 64, dsi.DSI_BF16, 100, 64, 1 << 20, 2 << 20, 3, 8, P, P, P)
    for scale in (0.0, 1e-45, 1.0, 2.35e38):
        dsi.dsi_page_attend(0, pages, 5, 4, 1 << 20, 2 << 20, 3 << 20, 1 << 30, scale=scale)
    ''')


def test_sizes_that_no_launch_holds_are_refused(stub):
    """A launch has fewer than 2^24 workgroups of 256 (one of 2^24 + 5 runs five of them without an error): the largest sizes
    that are taken, and those behind them, of which nothing is launched."""
    run(stub, '''
    def blocks(call):
        hip.stub_clear()
        call()
        return max(g[0] for _, _, g in launches())
    def none(call):
        hip.stub_clear()
        try:
            call()
        except dsi.DsiError as e:
            assert e.status == dsi.DSI_EINVAL and not launches(), (e, launches())
        else:
            raise AssertionError("taken")
    far = [x << 40 for x in range(1, 6)]
    pages = lambda n_kv, windows: dsi.make_pages(n_kv, 32, dsi.DSI_BF16, 100, 64, 1 << 20, 2 << 20, windows, 8, P, P, P)
    append = lambda n_kv, windows, rows: lambda: dsi.dsi_page_append(0, pages(n_kv, windows), rows, 1, *far[:4], dsi.make_rope(0, None))
    assert blocks(append(119, 1, 1 << 22)) == 119 * (2 + (1 << 22) // 32 - 1) + (1 << 20)
    none(append(120, 1, 1 << 22))
    none(append(1024, 4096, 1 << 19))
    def attend(n_kv, hq, windows, rows):
        p = pages(n_kv, windows)
        n = dsi.dsi_page_attend_workspace(p, rows, hq)
        return lambda: dsi.dsi_page_attend(0, p, rows, hq, far[0], far[1], far[2], n, dsi.DSI_BF16)
    assert 511 << 15 < blocks(attend(511, 511, 1, 1 << 22)) < 1 << 24
    assert 440 << 15 < blocks(attend(440, 440, 4096, 1 << 22)) < 1 << 24
    none(attend(512, 512, 1, 1 << 22))
    none(attend(456, 456, 4096, 1 << 22))
    adjust = lambda B, R, V: lambda: dsi.dsi_adjust(0, B, R, V, far[0], far[0], dsi.DSI_BF16)
    assert blocks(adjust(1 << 22, 1, 3 * 4096)) == 3 << 22
    assert blocks(adjust(1 << 17, 8, 127 * 4096)) == 127 << 17
    none(adjust(1 << 22, 1, 4 * 4096))
    none(adjust(1 << 17, 8, 127 * 4096 + 1))
    ''')
