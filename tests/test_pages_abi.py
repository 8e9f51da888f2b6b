"""The paged cache's and the rotary call's argument checks, which need no GPU: every refusal is made on the host, before any HIP
call."""
import ctypes

import pytest
import torch

from paper_2509_21354_amd import binding as kb

FAKE, ODD = 0x1000, 0x1004               # addresses that are never followed: validation fails first, or there is nothing to do


def _shape(**kw):
    return kb.make_shape(**dict(dict(L=2, B=3, H=8, H_kv=4, d=128, T=0, T_cap=1, C=1, N_cap=0, W=0, d_sum=1, d_g=1, dtype=kb.BF16), **kw))


def _far(i):
    return 0x10000000 * (i + 1)          # apart by more than the buffers are long


def _call(name, sh=None, pg=None, **kw):
    """A call that is right but for what `kw` says."""
    sh, pg, to = sh or _shape(), pg or kb.make_pages(32, 10, 7), kb.make_pages(32, 8, 7)
    r, p = ctypes.byref(sh), ctypes.byref(pg)
    axes = kb.make_rotary_axes((16, 24, 24))
    base = dict(
        append=[("shape", r), ("pages", p), ("K", _far(0)), ("V", _far(1)), ("Tn", 0), ("start", FAKE), ("n_new", None), ("table", FAKE), ("pool", FAKE), ("stream", None)],
        read=[("shape", r), ("pages", p), ("pool", FAKE), ("table", FAKE), ("first", FAKE), ("n", None), ("Tn", 0), ("K", _far(0)), ("V", _far(1)), ("stream", None)],
        attention=[("shape", r), ("pages", p), ("Q", _far(0)), ("Tq", 0), ("pool", FAKE), ("table", FAKE), ("length", FAKE), ("first", None), ("q_start", None),
                   ("Kc", None), ("Vc", None), ("count", None), ("k_cap", 0), ("O", _far(1)), ("ws", FAKE), ("ws_bytes", 1 << 40), ("stream", None)],
        reserve=[("shape", r), ("pages", p), ("n_new", FAKE), ("table", FAKE), ("length", _far(0)), ("refs", FAKE), ("pool", FAKE), ("start", _far(1)),
                 ("status", FAKE), ("ws", FAKE), ("ws_bytes", 1 << 20), ("stream", None)],
        fork=[("shape", r), ("pages", p), ("src", FAKE), ("dst", FAKE), ("n", 0), ("table", FAKE), ("length", FAKE), ("refs", FAKE), ("status", FAKE), ("stream", None)],
        trim=[("shape", r), ("pages", p), ("rows", None), ("n", 0), ("first", None), ("keep", None), ("table", FAKE), ("length", FAKE), ("refs", FAKE), ("stream", None)],
        copy=[("shape", r), ("pages", p), ("pool", FAKE), ("src", FAKE), ("dst", FAKE), ("n", 0), ("status", FAKE), ("stream", None)],
        compact=[("shape", r), ("pages", p), ("pool", _far(0)), ("table", _far(1)), ("refs", _far(2)), ("to", ctypes.byref(to)), ("to_pool", _far(3)), ("to_table", _far(4)),
                 ("to_refs", _far(5)), ("status", FAKE), ("ws", FAKE), ("ws_bytes", 1 << 20), ("stream", None)],
        rotary=[("shape", r), ("axes", ctypes.byref(axes)), ("freq", FAKE), ("pos", FAKE), ("Tq", 0), ("Q", _far(0)), ("K", _far(1)), ("Q_out", _far(2)),
                ("K_out", _far(3)), ("inverse", 0), ("stream", None)])[name]
    assert set(kw) <= {k for k, _ in base}
    f = {"append": "kvev_page_append", "read": "kvev_page_read", "attention": "kvev_page_attention", "rotary": "kvev_rotary"}.get(name, "kvev_pages_" + name)
    return getattr(kb.lib(), f)(*[kw.get(k, v) for k, v in base])


NOTHING_TO_DO = ("append", "read", "attention", "fork", "trim", "copy", "rotary")
ALL = NOTHING_TO_DO + ("reserve", "compact")


@pytest.mark.parametrize("name", NOTHING_TO_DO)
def test_nothing_to_do_is_ok(name):
    assert _call(name) == kb.OK


@pytest.mark.parametrize("name", [n for n in ALL if n != "rotary"])
def test_page_geometry(name):
    P = kb.make_pages
    for bad in (P(32, 0, 7), P(32, 10, 0), P(32, 10, -1), P(256, 10, 1 << 23), P(16, 1 << 30, 7)):
        assert _call(name, pg=bad) == kb.ERR_INVALID_ARG
    for bad in (P(0, 10, 7), P(8, 10, 7), P(48, 10, 7), P(512, 10, 7), P(-32, 10, 7)):
        assert _call(name, pg=bad) == kb.ERR_UNSUPPORTED
    assert _call(name, sh=_shape(B=1 << 20, L=1, H=4), pg=P(32, 10, 1 << 12)) == kb.ERR_INVALID_ARG       # table entries past 31 bits
    assert _call(name, pages=None) == kb.ERR_INVALID_ARG


@pytest.mark.parametrize("name", ALL)
def test_shape_and_stream_of_refusals(name):
    assert _call(name, shape=None) == kb.ERR_INVALID_ARG
    assert _call(name, sh=_shape(d=96)) == kb.ERR_UNSUPPORTED
    assert _call(name, sh=_shape(dtype=2)) == kb.ERR_UNSUPPORTED
    assert _call(name, sh=_shape(H_kv=3)) == kb.ERR_INVALID_ARG


# arrays that have to be there; what has to be 16-byte aligned
NEEDED = {"append": "K V start table pool", "read": "K V first table pool", "attention": "Q O pool table length", "reserve": "n_new table length refs pool start status",
          "fork": "src dst table length refs status", "trim": "table length refs", "copy": "pool src dst status",
          "compact": "pool table refs to to_pool to_table to_refs status", "rotary": "axes freq pos"}
WIDE = {"append": "K V pool", "read": "K V pool", "attention": "Q O pool", "reserve": "pool", "copy": "pool", "compact": "pool to_pool", "rotary": "Q K Q_out K_out"}


@pytest.mark.parametrize("name", ALL)
def test_missing_and_misaligned_arrays(name):
    for k in NEEDED[name].split():
        assert _call(name, **{k: None}) == kb.ERR_INVALID_ARG, k
        if k not in ("axes", "to"):
            assert _call(name, **{k: 0x1002}) == kb.ERR_INVALID_ARG, k
    for k in WIDE.get(name, "").split():
        assert _call(name, **{k: ODD}) == kb.ERR_INVALID_ARG, k


def test_counts():
    for name, k in (("append", "Tn"), ("read", "Tn"), ("attention", "Tq"), ("attention", "k_cap"), ("fork", "n"), ("trim", "n"), ("copy", "n"), ("rotary", "Tq")):
        assert _call(name, **{k: -1}) == kb.ERR_INVALID_ARG, (name, k)
    assert _call("fork", n=4) == kb.ERR_INVALID_ARG and _call("trim", n=4) == kb.ERR_INVALID_ARG and _call("copy", n=11) == kb.ERR_INVALID_ARG
    assert _call("append", Tn=1 << 28) == kb.ERR_INVALID_ARG and _call("read", Tn=1 << 28) == kb.ERR_INVALID_ARG      # 2^31 rows and more
    assert _call("attention", Tq=1 << 22) == kb.ERR_INVALID_ARG
    assert _call("attention", k_cap=4) == kb.ERR_INVALID_ARG                                                      # a store without its arrays
    assert _call("attention", k_cap=4, Kc=ODD, Vc=FAKE, count=FAKE) == kb.ERR_INVALID_ARG
    assert _call("attention", k_cap=1 << 28, Kc=FAKE, Vc=FAKE, count=FAKE) == kb.ERR_INVALID_ARG


def test_overlaps():
    assert _call("attention", Tq=1, Q=_far(0), O=_far(0) + 256) == kb.ERR_INVALID_ARG
    assert _call("read", Tn=4, K=_far(0), V=_far(0) + 256) == kb.ERR_INVALID_ARG
    assert _call("reserve", n_new=FAKE, start=FAKE) == kb.ERR_INVALID_ARG and _call("reserve", start=_far(0)) == kb.ERR_INVALID_ARG
    assert _call("reserve", n_new=_far(0)) == kb.ERR_INVALID_ARG and _call("reserve", start=_far(0) + 8) == kb.ERR_INVALID_ARG
    assert _call("reserve", n_new=_far(1) - 4) == kb.ERR_INVALID_ARG
    assert _call("compact", to_pool=_far(0) + 64) == kb.ERR_INVALID_ARG and _call("compact", to_refs=_far(2) + 4) == kb.ERR_INVALID_ARG
    assert _call("compact", to_table=_far(1) + 4) == kb.ERR_INVALID_ARG
    for kw in (dict(Q_out=_far(0) + 16), dict(K_out=_far(1) + 16), dict(K_out=_far(2)), dict(K_out=_far(0)), dict(Q_out=_far(1))):
        assert _call("rotary", Tq=1, **kw) == kb.ERR_INVALID_ARG, kw


def test_workspaces():
    for name, op in (("reserve", kb.OP_PAGES_RESERVE), ("compact", kb.OP_PAGES_COMPACT)):
        need = kb.page_workspace_bytes(op, _shape(), kb.make_pages(32, 10, 7), 0)
        assert need > 0
        assert _call(name, ws=None) == kb.ERR_WORKSPACE and _call(name, ws=ODD) == kb.ERR_WORKSPACE and _call(name, ws_bytes=need - 1) == kb.ERR_WORKSPACE
    sh, pg = _shape(B=1, L=1, T=4000, T_cap=4000), kb.make_pages(64, 100, 100)
    need = kb.page_workspace_bytes(kb.OP_PAGE_ATTENTION, sh, pg, 1)
    assert need > 0
    for kw in (dict(ws=None), dict(ws=ODD), dict(ws_bytes=64)):
        assert _call("attention", sh=sh, pg=pg, Tq=1, **kw) == kb.ERR_WORKSPACE
    # one query of the size serves every length that the launch may be planned for
    for T in (1, 64, 1000, 6400):
        sh.T = sh.T_cap = T
        assert kb.page_workspace_bytes(kb.OP_PAGE_ATTENTION, sh, pg, 1) == need
    assert kb.page_workspace_bytes(kb.OP_PAGE_ATTENTION, sh, pg, 1 << 30) == 0
    assert kb.page_workspace_bytes(99, sh, pg, 1) == 0 and kb.page_workspace_bytes(kb.OP_PAGE_ATTENTION, sh, pg, -1) == 0
    assert kb.page_workspace_bytes(kb.OP_PAGE_ATTENTION, sh, kb.make_pages(17, 1, 1), 1) == 0


@pytest.mark.parametrize("L,B,H,H_kv", [(1, 1, 1, 0), (1, 2, 32, 8), (2, 64, 32, 8), (32, 8, 8, 8)])
def test_attention_workspace_serves_fewer_queries(L, B, H, H_kv):
    for d, dtype in ((64, kb.F32), (128, kb.BF16)):
        sh, last = _shape(L=L, B=B, H=H, H_kv=H_kv, d=d, dtype=dtype, T=0), 0
        for Tq in (1, 2, 5, 16, 17, 40, 48, 64, 100, 128, 129, 256, 257, 700, 1024):
            need = kb.page_workspace_bytes(kb.OP_PAGE_ATTENTION, sh, kb.make_pages(64, 100, 150), Tq)
            assert need >= last > -1 and need > 0, (d, dtype, Tq)
            last = need
        # rows of one run: nothing to join
        assert kb.page_workspace_bytes(kb.OP_PAGE_ATTENTION, sh, kb.make_pages(64, 100, 3), 1) == 0


def test_pool_size():
    assert kb.page_pool_bytes(_shape(), kb.make_pages(32, 10, 7)) == 2 * 10 * 4 * 32 * (128 + 8)
    assert kb.page_pool_bytes(_shape(d=64, H_kv=0), kb.make_pages(16, 3, 7)) == 2 * 3 * 8 * 16 * (64 + 4)
    assert kb.page_pool_bytes(_shape(), kb.make_pages(33, 10, 7)) == 0


def test_rotary_axes():
    def axes(n, sections, layout=0):
        return ctypes.byref(kb.RotaryAxes(n, (ctypes.c_int32 * 4)(*sections), layout))
    assert _call("rotary", axes=axes(4, (16, 16, 16, 16))) == kb.OK and _call("rotary", axes=axes(2, (0, 1, 99, 99))) == kb.OK
    for n, sections in ((0, (8, 0, 0, 0)), (5, (8, 8, 8, 8)), (3, (-1, 8, 8, 0)), (3, (32, 32, 1, 0)), (1, (0, 0, 0, 0)), (2, (1 << 30, 1 << 30, 0, 0))):
        assert _call("rotary", axes=axes(n, sections)) == kb.ERR_INVALID_ARG, (n, sections)
    assert _call("rotary", axes=axes(1, (8, 0, 0, 0), 2)) == kb.ERR_UNSUPPORTED
    assert _call("rotary", inverse=2) == kb.ERR_INVALID_ARG and _call("rotary", Q=None, Q_out=None, K=None, K_out=None) == kb.ERR_INVALID_ARG
    assert _call("rotary", Q=None) == kb.ERR_INVALID_ARG and _call("rotary", K_out=None) == kb.ERR_INVALID_ARG
    assert _call("rotary", Q=None, Q_out=None) == kb.OK and _call("rotary", K=None, K_out=None) == kb.OK
    assert _call("rotary", Tq=1 << 23) == kb.ERR_INVALID_ARG
    with pytest.raises(kb.KvevError):
        kb.make_rotary_axes(())
    with pytest.raises(kb.KvevError):
        kb.make_rotary_axes((1,) * 5)


def test_python_calls_say_what_is_wrong_with_a_tensor():
    """Element types, sizes and devices are checked in Python; nothing of it needs the GPU."""
    sh, pg = _shape(), kb.make_pages(32, 10, 7)
    K = torch.zeros(2, 3, 4, 5, 128, dtype=torch.bfloat16)
    t = dict(start=torch.zeros(3, dtype=torch.int32), table=torch.zeros(3, 7, dtype=torch.int32), pool=torch.zeros(348160, dtype=torch.uint8))

    def call(**kw):
        a = dict(t, K=K, V=K.clone(), n_new=None, **kw)
        kb.kvev_page_append(sh, pg, a["K"], a["V"], 5, a["start"], a["n_new"], a["table"], a["pool"])
    for kw, text in ((dict(), "K is not on the current device"),):
        with pytest.raises(kb.KvevError, match=text):
            call(**kw)
    a = kb._Args("kvev_page_append", sh, pg)
    for f, text in ((lambda: a.rows("K", K.float(), 4, 5), "K has to hold 15360 elements of torch.bfloat16"), (lambda: a.rows("K", K, 4, 6), "K has to hold"),
                    (lambda: a.ints("start", torch.zeros(3, dtype=torch.int64), 3), "start has to hold 3 elements of torch.int32"),
                    (lambda: a.ints("start", None, 3), "start is missing"), (lambda: a.table(torch.zeros(3, 6, dtype=torch.int32)), "table has to hold 21"),
                    (lambda: a.pool(torch.zeros(348159, dtype=torch.uint8)), "pool has to hold 348160")):
        with pytest.raises(kb.KvevError, match=text) as e:
            f()
        assert e.value.status == kb.ERR_INVALID_ARG
    assert a.ints("n_new", None, 3, True) is None
    with pytest.raises(kb.KvevError, match="no such cache"):
        kb.PagedCache(sh, 33, 10, 7, device="cpu")
    c = kb.PagedCache(sh, 32, 10, 7, device="cpu")
    assert c.pool.numel() == 348160 and (c.table == -1).all() and not c.refs.any()


def test_hooks():
    L, n = kb.lib(), ctypes.c_int()
    assert L.kvev_debug_page_frame_work(-1) == kb.ERR_INVALID_ARG and L.kvev_debug_page_frame_work(0) == kb.OK
    assert L.kvev_debug_page_pair_units(-1) == kb.ERR_INVALID_ARG and L.kvev_debug_page_pair_units(0) == kb.OK
    sh, pg, r = _shape(), kb.make_pages(32, 10, 7), ctypes.byref(n)
    f = L.kvev_debug_page_form
    assert f(ctypes.byref(sh), ctypes.byref(pg), 1, r, r, r) == kb.OK
    assert f(ctypes.byref(sh), ctypes.byref(pg), 0, r, r, r) == kb.ERR_INVALID_ARG and f(ctypes.byref(sh), ctypes.byref(pg), 1, None, r, r) == kb.ERR_INVALID_ARG
    assert f(ctypes.byref(sh), ctypes.byref(kb.make_pages(31, 10, 7)), 1, r, r, r) == kb.ERR_INVALID_ARG


def test_plain_form_of_the_cache():
    """The tests' plain form against itself: codes are nearest, halfway cases go to the even one, blocks that are not finite are lost."""
    import numpy as np
    from tests import pages_ref as ref
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 32)) * 10.0 ** rng.integers(-30, 30, (50, 1))
    y = ref.block_values(x)
    top = np.abs(x).max(1, keepdims=True)
    assert (np.abs(x - y) <= top / 7 * 2).all()                                  # half the widest step is the scale, top > 3.5 of it
    assert (np.abs(y).max(1) * 5 / 4 >= top[:, 0] * (1 - 1e-12)).all()
    assert (ref.block_values(y) == y).all()
    blk = np.array([[7.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25] + [0.0] * 24])
    assert ref.block_values(blk)[0, :8].tolist() == [6.0, 4.0, 4.0, 2.0, 2.0, 1.0, 1.0, 0.0]
    assert np.isnan(ref.block_values(np.array([[np.inf] + [1.0] * 31]))).all()
