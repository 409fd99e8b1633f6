"""Host code of forking, dsi_attend and dsi_logprobs, without a GPU: refusals,
what is launched and what is allocated, against a HIP runtime that runs
nothing (see test_host_runtime.py)."""
import ctypes

import pytest

from paper_2405_14105_amd import dsi
from test_host_runtime import pytestmark, run, stub  # noqa: F401


def test_fork_refusals(stub):
    run(stub, '''
    m = model(S.SHAPES["gqa_hd64"])
    kv = dsi.dsi_kv_create(m, 5, 300)
    dsi.dsi_prefill(m, kv, 1, P, 100, P)
    def refused(*a):
        hip.stub_clear()
        try:
            dsi.dsi_kv_fork(kv, *a)
        except dsi.DsiError as e:
            assert e.status == dsi.DSI_EINVAL
            assert not launches()
            return True
        return False
    for a in ((-1, 0, 1), (5, 0, 1), (1, -1, 2), (1, 2, 0), (1, 2, 4), (1, 0, 2), (1, 1, 1), (1, 2, 3, 101), (1, 2, 3, -2),
              (1, 2, 2 ** 31 - 1), (1, 2 ** 31 - 1, 1)):
        assert refused(*a), a
    for a in ((1, 2, 3), (1, 0, 1, 0), (1, 2, 3, 100), (1, 4, 1, 33)):
        assert not refused(*a), a
        assert [k for k, _, _ in launches()] == ["k_kv_fork"]
    # the host's bounds are the source's: what fits follows
    dsi.dsi_kv_fork(kv, 1, 2, 1)
    dsi.dsi_prefill(m, kv, 2, P, 200, P)
    try:
        dsi.dsi_prefill(m, kv, 2, P, 1, P)
        assert False
    except dsi.DsiError as e:
        assert e.status == dsi.DSI_ECAPACITY
    ''')


def test_wrap_refusals_and_ownership(stub):
    run(stub, '''
    m = model(S.SHAPES["gqa_hd64"])
    n = dsi.dsi_kv_bytes(m, 3, 100)
    s = S.SHAPES["gqa_hd64"]
    assert n == s.n_layers * 3 * s.n_kv_heads * 128 * s.head_dim * 2
    for a in ((0, 100, P, P, n), (3, 0, P, P, n), (3, 100, None, P, n), (3, 100, P, None, n), (3, 100, P + 8, P, n),
              (3, 100, P, P + 2, n), (3, 100, P, P, n - 1), (3, 100, P, P, n + 1)):
        try:
            dsi.dsi_kv_wrap(m, *a)
            assert False, a
        except dsi.DsiError as e:
            assert e.status == dsi.DSI_EINVAL, a
    # sizes that no memory holds are refused, not thrown or wrapped round
    big = 2 ** 31 - 1
    for f in (lambda w, l: dsi.dsi_kv_bytes(m, w, l), lambda w, l: dsi.dsi_kv_wrap(m, w, l, P, P, n), lambda w, l: dsi.dsi_kv_create(m, w, l)):
        for w, l in ((big, big), (big, big - 63), (1, big), (big, 1 << 30)):
            try:
                f(w, l)
                assert False
            except dsi.DsiError as e:
                assert e.status in (dsi.DSI_EINVAL, dsi.DSI_ENOMEM), e
    used = hip.stub_in_use()
    kv = dsi.dsi_kv_wrap(m, 3, 100, P, P, n)
    try:
        dsi.dsi_model_destroy(m)
        assert False
    except dsi.DsiError as e:
        assert e.status == dsi.DSI_ESTATE
    dsi.dsi_kv_destroy(kv)              # frees nothing of the caller's (the runtime aborts on an address it did not give)
    assert hip.stub_in_use() == used
    dsi.dsi_model_destroy(m)
    assert hip.stub_in_use() == 0
    ''')


def test_attend_refusals(stub):
    run(stub, '''
    m = model(S.SHAPES["gqa_hd64"])
    other = model(S.SHAPES["gqa_hd64"])
    kv = dsi.dsi_kv_create(m, 4, 100)
    ok = dict(layer=1, window0=0, n_windows=4, rows=3, d_q=P, d_k=P, d_v=P, d_out=P)
    def status(mm=m, **change):
        hip.stub_clear()
        try:
            dsi.dsi_attend(mm, kv, **{**ok, **change})
        except dsi.DsiError as e:
            assert not launches() and not hip.stub_mallocs()
            return e.status
        return 0
    assert status(other) == dsi.DSI_EINVAL
    for change in (dict(layer=-1), dict(layer=3), dict(n_windows=0), dict(rows=0), dict(rows=257), dict(n_windows=5), dict(window0=1),
                   dict(window0=-1), dict(d_q=None), dict(d_k=None), dict(d_v=None), dict(d_out=None), dict(d_q=P + 4), dict(d_out=P + 8), dict(d_k=P + 4), dict(d_v=P + 8),
                   dict(window0=2 ** 31 - 1), dict(n_windows=2 ** 31 - 1, rows=2 ** 31 - 1)):
        assert status(**change) == dsi.DSI_EINVAL, change
    assert status(rows=101, n_windows=1) == dsi.DSI_ECAPACITY
    assert status() == 0 and status(rows=100) == 0
    assert status(rows=60, commit=True) == 0
    assert status(rows=41) == dsi.DSI_ECAPACITY and status(rows=40) == 0
    # no weights are needed
    bare = dsi.dsi_model_create(dsi.make_config(1, 32, 4, 2, 64, 32, 32), STREAM)
    bkv = dsi.dsi_kv_create(bare, 1, 50)
    dsi.dsi_attend(bare, bkv, 0, 0, 1, 2, P, P, P, P)
    ''')


def test_what_runs_and_what_is_allocated(stub):
    """Windows that were not forked run as before; a step's buffers are allocated by its first call."""
    run(stub, '''
    import os
    os.environ["DSI_SHARE"] = "1"
    m = model(S.SHAPES["tiny"])
    kv = dsi.dsi_kv_create(m, 8, 2000)
    for w in range(8):
        dsi.dsi_prefill(m, kv, w, P, 300, P)
    def names(f):
        hip.stub_clear()
        f()
        return {k for k, _, _ in launches()}
    dsi.dsi_profile_begin(m, dsi.DSI_K_ATTN)      # launches one by one, no recorded step
    def verify(w0, n, k=3):
        return names(lambda: dsi.dsi_verify(m, kv, w0, n, k, P, P, P, P, P, commit=False))
    def tree(w0, n):
        return names(lambda: dsi.dsi_verify_tree(m, kv, w0, n, 4, P, P, P, P, P, commit=False))
    assert "k_attn" in verify(0, 8) and "k_share" not in verify(0, 8)
    dsi.dsi_kv_fork(kv, 2, 3, 2)
    for f in (verify, tree):
        for w0, n in ((2, 3), (3, 2), (0, 8), (2, 2)):
            assert "k_share" in f(w0, n) and "k_attn" not in f(w0, n), (w0, n)
        for w0, n in ((0, 3), (4, 4), (2, 1), (4, 1)):
            assert "k_attn" in f(w0, n) and "k_share" not in f(w0, n), (w0, n)
    # a chain of forks: the later root goes with its own
    dsi.dsi_kv_fork(kv, 4, 5, 1)
    assert "k_share" in verify(4, 2)
    # what is known to share nothing worth it runs as before
    dsi.dsi_kv_rollback(kv, 3, 127)
    assert "k_attn" in verify(2, 2) and "k_share" in verify(4, 2)
    dsi.dsi_kv_set_length(kv, 2, 100)
    for w0, n in ((2, 3), (3, 2), (2, 2)):
        assert "k_attn" in verify(w0, n) and "k_share" not in verify(w0, n)
    dsi.dsi_kv_import(kv, 4, 0, 10, P, P)
    assert "k_attn" in verify(0, 8) and "k_share" not in verify(0, 8)
    dsi.dsi_kv_fork(kv, 6, 2, 4, 128)
    assert "k_share" in verify(0, 8)
    attend = lambda rows, n=8: names(lambda: dsi.dsi_attend(m, kv, 0, 0, n, rows, P, P, P, P))
    assert attend(20) == {"k_share", "k_share_last"}
    for rows in (20, 1, 7):
        attend(rows)
        assert hip.stub_mallocs() == 0, rows
    hip.stub_clear()
    hip.stub_capture(1)
    dsi.dsi_attend(m, kv, 0, 0, 8, 20, P, P, P, P)
    dsi.dsi_kv_fork(kv, 0, 1, 2, 64)
    hip.stub_capture(0)
    assert hip.stub_refused() == 0 and hip.stub_mallocs() == 0
    ''')


def test_the_first_call_of_a_size_allocates_for_any_forks(stub):
    """A step captured after windows were forked or rolled back finds its buffers, whatever was forked at its first call."""
    run(stub, '''
    import random
    rng = random.Random(1)
    for hq, hkv, hd, kind, W, max_len in ((32, 8, 128, dsi.DSI_BF16, 4, 32768), (8, 8, 64, dsi.DSI_BF16, 6, 3000), (32, 8, 64, dsi.DSI_F32, 5, 9000),
                                          (40, 40, 128, dsi.DSI_BF16, 8, 8192), (4, 1, 32, dsi.DSI_F32, 12, 700), (64, 8, 128, dsi.DSI_BF16, 16, 4096)):
        for rows in (1, 6, 17, 64):
            m = dsi.dsi_model_create(dsi.make_config(1, 32, hq, hkv, hd, 32, 32, kvdtype=kind), STREAM)
            kv = dsi.dsi_kv_create(m, W, max_len)
            attend = lambda w0, n: dsi.dsi_attend(m, kv, 0, w0, n, rows, P, P, P, P)
            for w in range(W):
                dsi.dsi_kv_set_length(kv, w, max_len - rows)
            for n in range(1, W + 1):
                attend(0, n)
            for turn in range(30):
                for _ in range(rng.randint(1, 4)):
                    src, w0 = rng.randrange(W), rng.randrange(W)
                    n = rng.randint(1, W - w0)
                    if src < w0 or src >= w0 + n:
                        dsi.dsi_kv_fork(kv, src, w0, n)
                    if rng.random() < 0.3:
                        dsi.dsi_kv_set_length(kv, rng.randrange(W), rng.choice((0, 100, 500, max_len - rows)))
                hip.stub_clear()
                hip.stub_capture(1)
                w0 = rng.randrange(W)
                attend(w0, rng.randint(1, W - w0))
                attend(0, W)
                hip.stub_capture(0)
                assert hip.stub_refused() == 0 and hip.stub_mallocs() == 0, (hq, hkv, hd, rows, turn)
            dsi.dsi_kv_destroy(kv)
            dsi.dsi_model_destroy(m)
    # where there is no room for all that, a call takes what it needs itself
    m = dsi.dsi_model_create(dsi.make_config(1, 32, 32, 8, 128, 32, 32, kvdtype=dsi.DSI_BF16), STREAM)
    kv = dsi.dsi_kv_create(m, 4, 32768)
    hip.stub_budget(17 * 4 * 32 * (128 * 4 + 8) + 8192)
    for _ in range(3):
        dsi.dsi_attend(m, kv, 0, 0, 4, 1, P, P, P, P)
    hip.stub_clear()
    dsi.dsi_attend(m, kv, 0, 0, 4, 1, P, P, P, P)
    assert hip.stub_refused() == 0                       # not asked for again and again
    ''')


def test_forwards_without_room_for_a_shared_prefix_run_as_before(stub):
    """Captured after windows were forked, or short of memory: the window kernels, no refusal."""
    run(stub, '''
    import os
    os.environ["DSI_SHARE"], os.environ["DSI_GRAPHS"] = "1", "0"
    def names(f):
        hip.stub_clear()
        f()
        return {k for k, _, _ in launches()}
    for how in ("capture", "memory"):
        m = model(S.SHAPES["gqa_hd64"])
        kv = dsi.dsi_kv_create(m, 4, 900)
        verify = lambda: dsi.dsi_verify(m, kv, 0, 4, 5, P, P, P, P, P, commit=False)
        tree = lambda: dsi.dsi_verify_tree(m, kv, 0, 4, 6, P, P, P, P, P, commit=False)
        for w in range(4):
            dsi.dsi_prefill(m, kv, w, P, 600, P)
        for f in (verify, tree):
            assert "k_attn" in names(f)
        dsi.dsi_kv_fork(kv, 0, 1, 3)
        for f in (verify, tree):
            if how == "capture":
                hip.stub_capture(1)
            else:
                hip.stub_budget(0)
            got = names(f)
            assert "k_attn" in got and "k_share" not in got
            hip.stub_capture(0)
            hip.stub_budget(1 << 40)
        for f in (verify, tree):                         # with room, and captured once there is some
            assert "k_share" in names(f)
            hip.stub_capture(1)
            assert "k_share" in names(f) and hip.stub_refused() == 0
            hip.stub_capture(0)
        dsi.dsi_kv_destroy(kv)
        dsi.dsi_model_destroy(m)
    ''')


def test_a_prefix_is_read_once_where_that_saves_enough(stub):
    run(stub, '''
    import os
    def kernels(m, kv, n):
        dsi.dsi_profile_begin(m, dsi.DSI_K_ATTN)
        hip.stub_clear()
        dsi.dsi_verify(m, kv, 0, n, 1, P, P, P, P, P, commit=False)
        return {k for k, _, _ in launches()}
    each = 2 * 4 * 32 * 4                              # bytes of a position of a layer
    for env in (None, "0", "1"):
        os.environ.pop("DSI_SHARE", None)
        if env:
            os.environ["DSI_SHARE"] = env
        m = model(S.SHAPES["tiny"])
        kv = dsi.dsi_kv_create(m, 6, 20000)
        for length in (100, 128, 13106, 13108, 19000):
            dsi.dsi_kv_set_length(kv, 0, length)
            dsi.dsi_kv_fork(kv, 0, 1, 5)
            want = length >= 128 and env != "0" and (env == "1" or 5 * length * each >= 64 << 20)
            assert ("k_share" in kernels(m, kv, 6)) == want, (env, length)
            assert "k_share" not in kernels(m, kv, 1)
    ''')


def test_keys_of_a_windows_own_are_cut_into_chunks(stub):
    """One group in a call does not leave a long window, or a long continuation, to one workgroup a head."""
    run(stub, '''
    import os
    os.environ["DSI_SHARE"] = "1"
    def chunks(hq, hkv, rows, lens, shared, max_len=33000, grouped=True):
        """workgroups per window, KV head and query tile in the first launch, besides the prefix's"""
        m = dsi.dsi_model_create(dsi.make_config(1, 32, hq, hkv, 128, 32, 32, kvdtype=dsi.DSI_BF16), STREAM)
        kv = dsi.dsi_kv_create(m, len(lens), max_len)
        dsi.dsi_kv_set_length(kv, 0, max(shared))
        for w in range(1, len(lens)):
            if shared[w]:
                dsi.dsi_kv_fork(kv, 0, w, 1, shared[w])
        for w, n in enumerate(lens):
            dsi.dsi_kv_set_length(kv, w, n)
        hip.stub_clear()
        dsi.dsi_attend(m, kv, 0, 0, len(lens), rows, P, P, P, P)
        grid = [g[0] for k, _, g in launches() if k == "k_share"][0]
        n = hq // hkv * rows * sum(s > 0 for s in shared)
        tile = 256 if n > 128 else 128 if n > 64 else 64
        prefix = hkv * -(-n // tile) * (256 // (hkv * -(-n // tile)))
        t, rest = divmod(grid - prefix, len(lens) * hkv * -(-hq // hkv * rows // 16))
        assert rest == 0
        dsi.dsi_kv_destroy(kv)
        dsi.dsi_model_destroy(m)
        return t
    # little of their own: few workgroups, most of which only cache rows
    assert chunks(32, 8, 6, [8192] * 7, [8192] * 7) == 1
    assert chunks(32, 8, 1, [8192] + [8400] * 3, [8192] * 4) == 4
    # a window that shares nothing beside forked ones: 8 chunks and more of its 16384 keys
    assert chunks(32, 8, 6, [8192] * 7 + [16384], [8192] * 7 + [0]) == 8
    assert chunks(32, 8, 1, [8192] * 4 + [16384], [8192] * 4 + [0]) == 25
    assert chunks(40, 40, 7, [2048] * 6 + [16384], [2048] * 6 + [0]) == 3
    # continuations: one round of workgroups
    assert chunks(32, 8, 6, [8192 + 4096] * 7, [8192] * 7) == 2
    assert chunks(32, 8, 1, [8192 + 4096] * 8, [8192] * 8) == 4
    assert chunks(32, 8, 6, [8192, 8192, 8192, 14000, 8192, 8192, 8192], [8192] * 7) == 9
    assert chunks(40, 40, 1, [2048 + 4096] * 8, [2048] * 8) == 3          # 960 workgroups instead of 320, on 256 CUs
    # no more than their keys fill
    assert chunks(32, 8, 1, [8192 + 700] * 2, [8192] * 2) == 8 and chunks(32, 8, 6, [8192 + 700] * 2, [8192] * 2) == 4
    ''')


def test_windows_with_much_of_their_own_run_as_before(stub):
    run(stub, '''
    m = model(S.SHAPES["tiny"])
    kv = dsi.dsi_kv_create(m, 6, 60000)
    each = 2 * 4 * 32 * 4
    dsi.dsi_profile_begin(m, dsi.DSI_K_ATTN)
    for prefix in (14000, 20000):
        spare = 5 * prefix - (64 << 20) // each            # positions
        for own, want in ((0, True), (200, True), (4 * spare // 6 - 100, True), (4 * spare // 6 + 100, False), (30000, False)):
            dsi.dsi_kv_set_length(kv, 0, prefix)
            dsi.dsi_kv_fork(kv, 0, 1, 5)
            for w in range(6):
                dsi.dsi_kv_set_length(kv, w, prefix + own)
            hip.stub_clear()
            dsi.dsi_verify(m, kv, 0, 6, 1, P, P, P, P, P, commit=False)
            assert ("k_share" in {k for k, _, _ in launches()}) == want, (prefix, own)
    ''')


def test_an_fp32_prefix_is_shared_where_its_query_tiles_leave_something(stub):
    """fp32 caches read a prefix once per 16 queries, one workgroup a CU: what is saved is counted from that."""
    run(stub, '''
    import dataclasses
    def kernels(hq, hkv, hd, windows, rows, prefix, kind="f32"):
        shape = dataclasses.replace(S.SHAPES["tiny"], n_layers=1, n_heads=hq, n_kv_heads=hkv, head_dim=hd, kvdtype=kind)
        m = model(shape)
        kv = dsi.dsi_kv_create(m, windows, prefix + 100)
        dsi.dsi_kv_set_length(kv, 0, prefix)
        dsi.dsi_kv_fork(kv, 0, 1, windows - 1)
        dsi.dsi_profile_begin(m, dsi.DSI_K_ATTN)
        hip.stub_clear()
        dsi.dsi_verify(m, kv, 0, windows, rows - 1, P, P, P, P, P, commit=False)
        k = {k for k, _, _ in launches()}
        assert ("k_share" in k) != ("k_attn" in k)
        dsi.dsi_kv_destroy(kv)
        dsi.dsi_model_destroy(m)
        return "k_share" in k
    # 11 tiles of 16 queries make two rounds of the keys, as 16 would: nothing is gained
    for prefix in (6553, 13107, 40000):
        assert not kernels(32, 8, 64, 6, 7, prefix)
        assert not kernels(32, 8, 128, 6, 7, prefix)
        assert not kernels(32, 8, 64, 2, 11, prefix)
        assert kernels(32, 8, 128, 6, 7, prefix, "bf16")
    # one or two tiles for eight windows, and four rows each of sixteen
    assert kernels(32, 8, 64, 8, 1, 4681) and kernels(32, 8, 128, 8, 1, 4681) and kernels(32, 8, 128, 16, 4, 2184)
    assert kernels(32, 8, 128, 8, 8, 9362) and kernels(32, 8, 128, 3, 4, 16384)
    # many KV heads: from 512 positions on
    assert kernels(40, 40, 128, 6, 7, 655) and not kernels(40, 40, 128, 6, 7, 458) and not kernels(40, 40, 128, 16, 4, 218)
    ''')


def test_every_variant_of_the_shared_prefix_is_in_the_gpu_tests(stub):
    """What the cases of share_cases.py launch, and that they leave out no variant that is built."""
    run(stub, '''
    sys.path.insert(0, "tests")
    from share_cases import CASES
    seen = set()
    for hq, hkv, hd, windows, rows, prefix, max_len, tiles, chunk in CASES:
        m = dsi.dsi_model_create(dsi.make_config(1, 32, hq, hkv, hd, 32, 32, kvdtype=dsi.DSI_BF16), STREAM)
        kv = dsi.dsi_kv_create(m, windows, max_len)
        dsi.dsi_kv_set_length(kv, 0, prefix)
        dsi.dsi_kv_fork(kv, 0, 1, windows - 1)
        hip.stub_clear()
        dsi.dsi_attend(m, kv, 0, 0, windows, rows, P, P, P, P)
        (name, args, grid), = [x for x in launches() if x[0] == "k_share"]
        case = (hq, hkv, hd, windows, rows, prefix)
        assert args == (1, hd, tiles), (case, args)
        seen.add(args)
        # the grid: chunks of the prefix as the kernel cuts them, and each window's first chunk
        shared = prefix // 32 * 32
        p_tiles = -(-hq // hkv * rows * windows // (32 * tiles))
        p_chunks = min(256 // (hkv * p_tiles), -(-max_len // 128))
        units = hkv * -(-hq // hkv * rows // 16)
        assert grid[0] == hkv * p_tiles * p_chunks + windows * units * min(max(1, 128 // (windows * units)), -(-max_len // 256)), (case, grid)
        least = 192 if tiles == 8 and shared > 2048 else 128
        assert chunk == max(least, -(-(-(-shared // p_chunks)) // 64) * 64), case
        dsi.dsi_kv_destroy(kv)
        dsi.dsi_model_destroy(m)
    assert seen == {a for k, a in built() if k == "k_share" and a[0] == 1}
    ''')


def test_logprobs_refusals():
    lib = dsi.load()
    P = 4096
    n = ctypes.c_size_t()
    for a in ((-1, 100, 1), ((1 << 24) + 1, 100, 1), (1, 0, 0), (1, (1 << 30) + 1, 1), (1, 100, -1), (1, 100, 65), (1, 3, 4)):
        assert lib.dsi_logprobs_workspace(*a, ctypes.byref(n)) == dsi.DSI_EINVAL, a
    assert lib.dsi_logprobs_workspace(1, 10, 1, None) == dsi.DSI_EINVAL
    assert dsi.dsi_logprobs_workspace(0, 10, 1) == 0
    need = dsi.dsi_logprobs_workspace(5, 32000, 4)
    # what a row needs does not grow as the call gets larger, beyond four waves a SIMD in all
    assert dsi.dsi_logprobs_workspace(100000, 128256, 4) == 100000 * (24 + 32)
    ok = dict(rows=5, vocab=32000, d_logits=P, d_targets=P, n_top=4, d_logprob=P, d_entropy=P, d_top_ids=P, d_top_logprobs=P,
              d_ws=P, ws_bytes=need)
    for change in (dict(rows=-1), dict(vocab=0), dict(n_top=65), dict(n_top=-1), dict(dtype=2), dict(ld=31999), dict(ld=-5),
                   dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")),
                   dict(temperature=1e-39), dict(d_logits=None), dict(d_targets=None), dict(d_top_ids=None),
                   dict(d_top_logprobs=None), dict(d_ws=None), dict(d_ws=P + 4), dict(ws_bytes=need - 1), dict(d_logits=P + 2),
                   dict(dtype=dsi.DSI_BF16, d_logits=P + 1), dict(d_logprob=None, d_entropy=None, n_top=0)):
        with pytest.raises(dsi.DsiError) as e:
            dsi.dsi_logprobs(0, **{**ok, **change})
        assert e.value.status == dsi.DSI_EINVAL, change
    dsi.dsi_logprobs(0, **{**ok, "rows": 0, "d_logits": None, "d_ws": None, "ws_bytes": 0})
