"""The 4-bit key/value cache's entry points refuse what they cannot do before they touch the GPU (the addresses here are no device
memory), and their sizes are the documented ones."""
import ctypes as C

import pytest
import torch

FAKE = 0x10000
DIMS, PAGES = (64, 80, 96, 128, 256), (32, 64, 128, 256)


@pytest.fixture(scope="module")
def qp():
    import paper_2211_04515_amd as m
    m.lib()
    return m


def make(qp, **change):
    """Arguments that would be taken, with changes by name."""
    a = {"pages": FAKE, "layers": 2, "n_pages": 10, "heads": 4, "dim": 128, "page": 64, "c_reserved": 0, "bytes": None,
         "table": FAKE, "lengths": FAKE, "rows": 3, "per_row": 5, "layer": 1, "begin": FAKE, "first": None, "tokens": 7,
         "k": FAKE, "v": FAKE, "kt": 0, "vt": 0, "ts": 512, "hs": 128, "v_reserved": 0,
         "q": FAKE, "out": FAKE, "qt": 1, "ot": 1, "q_heads": 8, "q_ts": 1024, "q_hs": 128, "o_ts": 1024, "o_hs": 128,
         "scale": 0.1, "causal": 1, "window": 0, "ws": FAKE, "ws_bytes": 1 << 40, "books": FAKE, "pool": FAKE, "pool_bytes": 1 << 40}
    a.update(change)
    nb = a["bytes"]
    if nb is None:
        nb = a["layers"] * a["n_pages"] * a["heads"] * a["page"] * (a["dim"] + 16)
    a["cache"] = qp.qp_kv_cache_t(a["pages"], nb & (2 ** 64 - 1), a["layers"], a["n_pages"], a["heads"], a["dim"], a["page"], a["c_reserved"])
    a["row"] = qp.qp_kv_rows_t(a["table"], a["lengths"], a["rows"], a["per_row"])
    view = qp.qp_kv_view_t
    a["kv"], a["vv"] = view(a["k"], a["kt"], a["v_reserved"], a["ts"], a["hs"]), view(a["v"], a["vt"], 0, a["ts"], a["hs"])
    a["qv"], a["ov"] = view(a["q"], a["qt"], 0, a["q_ts"], a["q_hs"]), view(a["out"], a["ot"], 0, a["o_ts"], a["o_hs"])
    a["cfg"] = qp.qp_kv_attn_cfg_t(a["scale"], a["q_heads"], a["causal"], a["window"])
    return a


def append(qp, a):
    return qp.lib().qp_kv_append(C.byref(a["cache"]), C.byref(a["row"]), a["layer"], a["begin"], a["tokens"], C.byref(a["kv"]), C.byref(a["vv"]), None)


def read(qp, a):
    return qp.lib().qp_kv_read(C.byref(a["cache"]), C.byref(a["row"]), a["layer"], a["begin"], a["first"], a["tokens"], C.byref(a["kv"]), C.byref(a["vv"]), None)


def attention(qp, a):
    return qp.lib().qp_kv_attention(C.byref(a["cache"]), C.byref(a["row"]), a["layer"], a["begin"], a["tokens"], C.byref(a["qv"]), C.byref(a["ov"]),
                                    C.byref(a["cfg"]), a["ws"], a["ws_bytes"], None)


def books(name):
    def call(qp, a):
        return getattr(qp.lib(), name)(C.byref(a["cache"]), C.byref(a["row"]), a["books"], a["pool"], a["pool_bytes"], None)
    return call


def compact(qp, a):
    return qp.lib().qp_kv_compact(C.byref(a["cache"]), C.byref(a["row"]), a["pool"], a["pool_bytes"], None)


BOOKS = [books("qp_kv_reserve"), books("qp_kv_fork"), books("qp_kv_free")]
ROWS = [append, read]
ALL = BOOKS + [compact] + ROWS + [attention]

CACHE = [{"pages": None}, {"pages": FAKE + 8}, {"layers": 0}, {"layers": 65537, "bytes": 1 << 60}, {"n_pages": 0}, {"n_pages": (1 << 24) + 1}, {"heads": 0},
         {"heads": 1025, "q_heads": 1025}, {"dim": 0}, {"dim": 48}, {"dim": 72}, {"dim": 112}, {"dim": 512}, {"page": 0}, {"page": 16}, {"page": 48}, {"page": 512},
         {"c_reserved": 1}, {"table": None}, {"lengths": None}, {"table": FAKE + 2}, {"lengths": FAKE + 1}, {"rows": 0}, {"rows": 65537}, {"per_row": 0},
         {"per_row": 1 << 25}]
TOKENS = [{"layer": 2}, {"begin": None}, {"begin": FAKE + 2}, {"tokens": 1 << 31}, {"tokens": 1 << 29}]


@pytest.mark.parametrize("bad", CACHE, ids=lambda d: "_".join("%s_%s" % i for i in d.items()))
def test_caches_and_rows_that_are_refused(qp, bad):
    a = make(qp, **bad)
    for call in ALL:
        assert call(qp, a) == qp.QP_EINVAL


def test_buffers_that_are_too_small(qp):
    whole = 2 * 10 * 4 * 64 * 144
    for call in ALL:
        assert call(qp, make(qp, bytes=whole - 1)) == qp.QP_ENOSPC
        # sizes whose product passes 64 bits do not wrap round
        assert call(qp, make(qp, layers=65536, n_pages=1 << 24, heads=1024, q_heads=1024, dim=256, page=256, bytes=1 << 20)) == qp.QP_ENOSPC
    for call in BOOKS + [compact]:
        assert call(qp, make(qp, pool_bytes=4 * (16 + 60) - 1)) == qp.QP_ENOSPC
    a = make(qp)
    need = qp.qp_kv_attention_workspace_bytes(a["cache"], a["row"], 7, 8)
    assert need > 0 and attention(qp, make(qp, ws_bytes=need - 1)) == qp.QP_ENOSPC
    assert qp.lib().qp_kv_pool_init(10, FAKE, 4 * 76 - 1, None) == qp.QP_ENOSPC


@pytest.mark.parametrize("bad", TOKENS, ids=lambda d: "_".join("%s_%s" % i for i in d.items()))
def test_tokens_that_are_refused(qp, bad):
    a = make(qp, **bad)
    for call in ROWS + [attention]:
        assert call(qp, a) == qp.QP_EINVAL


@pytest.mark.parametrize("bad", [{"k": None}, {"v": None}, {"k": FAKE + 4}, {"kt": 2, "vt": 2}, {"kt": 0, "vt": 1}, {"ts": 510}, {"hs": 130}, {"ts": 1 << 40},
                                 {"v_reserved": 3}], ids=lambda d: "_".join("%s_%s" % i for i in d.items()))
def test_tensors_that_are_refused(qp, bad):
    for call in ROWS:
        assert call(qp, make(qp, **bad)) == qp.QP_EINVAL


@pytest.mark.parametrize("ts,hs", [(0, 128), (512, 0), (508, 128), (128, 128), (512, 124), (128, 508)])
def test_outputs_that_overlap_are_refused(qp, ts, hs):
    assert read(qp, make(qp, ts=ts, hs=hs)) == qp.QP_EINVAL
    assert attention(qp, make(qp, q_heads=4, qt=0, ot=0, o_ts=ts, o_hs=hs)) == qp.QP_EINVAL


@pytest.mark.parametrize("bad", [{"q": None}, {"out": None}, {"out": FAKE + 8}, {"qt": 0}, {"ot": 7, "qt": 7}, {"q_ts": 1020}, {"o_hs": 120}, {"o_ts": 0},
                                 {"scale": 0.0}, {"scale": -1.0}, {"scale": float("nan")}, {"scale": float("inf")}, {"causal": 2}, {"window": 1 << 31},
                                 {"window": 5, "causal": 0}, {"q_heads": 0}, {"q_heads": 6}, {"q_heads": 4 * 1025}, {"ws": None}, {"ws": FAKE + 8}],
                         ids=lambda d: "_".join("%s_%s" % i for i in d.items()))
def test_attention_that_is_refused(qp, bad):
    assert attention(qp, make(qp, **bad)) == qp.QP_EINVAL


def test_books_that_are_refused(qp):
    for call in BOOKS:
        assert call(qp, make(qp, books=None)) == qp.QP_EINVAL
        assert call(qp, make(qp, books=FAKE + 2)) == qp.QP_EINVAL
    for call in BOOKS + [compact]:
        assert call(qp, make(qp, pool=None)) == qp.QP_EINVAL
        assert call(qp, make(qp, pool=FAKE + 2)) == qp.QP_EINVAL
    assert qp.lib().qp_kv_pool_init(0, FAKE, 1 << 40, None) == qp.QP_EINVAL
    assert qp.lib().qp_kv_pool_init((1 << 24) + 1, FAKE, 1 << 40, None) == qp.QP_EINVAL
    assert qp.lib().qp_kv_pool_init(4, None, 1 << 40, None) == qp.QP_EINVAL


def test_null_structs_are_refused(qp):
    L, a = qp.lib(), make(qp)
    c, r = C.byref(a["cache"]), C.byref(a["row"])
    for name in ("qp_kv_reserve", "qp_kv_fork", "qp_kv_free"):
        assert getattr(L, name)(None, r, FAKE, FAKE, 1 << 40, None) == qp.QP_EINVAL
        assert getattr(L, name)(c, None, FAKE, FAKE, 1 << 40, None) == qp.QP_EINVAL
    assert L.qp_kv_append(None, r, 0, FAKE, 7, C.byref(a["kv"]), C.byref(a["vv"]), None) == qp.QP_EINVAL
    assert L.qp_kv_append(c, r, 0, FAKE, 7, None, C.byref(a["vv"]), None) == qp.QP_EINVAL
    assert L.qp_kv_read(c, r, 0, FAKE, None, 7, C.byref(a["kv"]), None, None) == qp.QP_EINVAL
    assert L.qp_kv_read(c, r, 0, FAKE, FAKE + 2, 7, C.byref(a["kv"]), C.byref(a["vv"]), None) == qp.QP_EINVAL
    assert L.qp_kv_attention(None, r, 0, FAKE, 7, C.byref(a["qv"]), C.byref(a["ov"]), C.byref(a["cfg"]), FAKE, 1 << 40, None) == qp.QP_EINVAL
    assert L.qp_kv_attention(c, r, 0, FAKE, 7, C.byref(a["qv"]), C.byref(a["ov"]), None, FAKE, 1 << 40, None) == qp.QP_EINVAL
    assert L.qp_kv_page_bytes(None) == 0 and L.qp_kv_attention_workspace_bytes(None, r, 7, 8) == 0 and L.qp_kv_attention_workspace_bytes(c, None, 7, 8) == 0


def test_no_tokens_is_no_work(qp):
    a = make(qp, tokens=0, k=None, v=None, q=None, out=None)
    assert append(qp, a) == read(qp, a) == attention(qp, a) == qp.QP_OK


def test_sizes(qp):
    for dim in DIMS:
        for page in PAGES:
            assert qp.qp_kv_page_bytes(make(qp, dim=dim, page=page, heads=3)["cache"]) == 3 * page * (dim + 16)
    assert qp.qp_kv_page_bytes(make(qp, dim=100)["cache"]) == 0
    assert qp.qp_kv_pool_bytes(1) == 88 and qp.qp_kv_pool_bytes(1 << 24) == 4 * (16 + 6 * (1 << 24)) and qp.qp_kv_pool_bytes(0) == 0
    assert [C.sizeof(t) for t in (qp.qp_kv_cache_t, qp.qp_kv_rows_t, qp.qp_kv_view_t, qp.qp_kv_attn_cfg_t)] == [40, 24, 32, 16]


def test_workspaces_of_refused_sizes_are_0(qp):
    a = make(qp)
    for tokens, heads in ((7, 0), (7, 6), (7, 4 * 1025), (1 << 31, 8), (1 << 29, 8)):
        assert qp.qp_kv_attention_workspace_bytes(a["cache"], a["row"], tokens, heads) == 0
    # rows too short to be split need next to nothing; the largest workspace does not grow with the tokens
    assert qp.qp_kv_attention_workspace_bytes(a["cache"], qp.qp_kv_rows_t(None, None, 3, 2), 7, 8) < 4096
    assert qp.qp_kv_attention_workspace_bytes(a["cache"], qp.qp_kv_rows_t(None, None, 3, 1 << 20), 1 << 20, 64) < 1 << 28


def test_the_binding_refuses_tensors_of_other_kinds(qp):
    with pytest.raises(ValueError):
        qp.kv_cache(torch.zeros(1, 2, 64, dtype=torch.uint8), 1, 64, 32)                       # not on a device
    with pytest.raises(ValueError):
        qp.kv_rows(torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        qp.kv_rows(torch.zeros(3, 2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32))
    with pytest.raises(qp.QuantPipeError):
        qp.alloc_kv_pages(4, 1, 65, 32, device="cpu")
    with pytest.raises(qp.QuantPipeError):
        qp.alloc_kv_pool(0, device="cpu")
    with pytest.raises(qp.QuantPipeError):
        qp.alloc_kv_pool(2 ** 32 + 5, device="cpu")


def test_the_binding_refuses_numbers_past_32_bits(qp):
    """ctypes would cut them down to their low 32 bits: 2^32 + 4 pages to 4, 2^32 + 8 heads to 8."""
    for n in (2 ** 32 + 4, -4, 0):
        with pytest.raises(qp.QuantPipeError):
            qp.qp_kv_pool_init(n, torch.zeros(1000, dtype=torch.int32))
    for kind in ((2 ** 32 + 1, 64, 32), (1, 2 ** 32 + 64, 32), (1, 64, 2 ** 32 + 32), (-1, 64, 32)):
        with pytest.raises(qp.QuantPipeError):
            qp.alloc_kv_pages(4, *kind, device="cpu")
    for n, layers in ((2 ** 32 + 4, 1), (4, 2 ** 32 + 1), (0, 1), (4, 0), (-1, 1), (4, -1), (2 ** 24 + 1, 1), (4, 65537)):
        with pytest.raises(qp.QuantPipeError):
            qp.alloc_kv_pages(n, 1, 64, 32, layers=layers, device="meta")
    a = make(qp)
    for tokens, heads in ((7, 2 ** 32 + 8), (2 ** 64 + 7, 8), (-1, 8), (7, -8)):
        assert qp.qp_kv_attention_workspace_bytes(a["cache"], a["row"], tokens, heads) == 0
