"""The 4-bit key/value cache on the GPU, through the package's calls, against the plain forms of kv_plain.py in 64 bits (codes and
books: equal; answers: within tolerances derived there from the roundings that the kernels make)."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import kv_plain as kp  # noqa: E402

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qp():
    import paper_2211_04515_amd as m
    m.lib()
    return m


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def ints(*a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U_OUT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


class Case:
    """A cache of one layer with rows of the given lengths, quantized by the plain form; behind the lengths the pages hold anything."""

    def __init__(self, qp, dim, page, heads, lengths, seed=0, layers=1, spare=3, per_row=None, fill=True):
        self.rng = np.random.default_rng([seed, dim, page, heads, *lengths])
        self.qp, self.dim, self.page, self.heads = qp, dim, page, heads
        rows = len(lengths)
        per_row = per_row or max(1, max(kp.pages_of(n, page) for n in lengths))
        self.n_pages = rows * per_row + spare
        self.table = self.rng.permutation(self.n_pages)[:rows * per_row].reshape(rows, per_row).astype(np.int32)
        self.lengths = np.array(lengths, np.int32)
        self.pages = kp.new_pages(layers, self.n_pages, heads, dim, page, self.rng)
        if fill:
            self.fill()
        self.up()

    def fill(self):
        """Keys with a few strong channels, values of different sizes: written with numpy for whole rows at once."""
        rng, dim, page = self.rng, self.dim, self.page
        kc, vc, gk, gv = kp.pieces(self.pages[0], dim, page)
        strong = np.where(rng.random((self.heads, dim)) < 0.05, 4, 1)
        for r, n in enumerate(self.lengths):
            if n == 0:
                continue
            t = np.arange(n)
            p, s = self.table[r, t // page], t % page
            for h in range(self.heads):
                for side, (codes, grids) in enumerate(((kc, gk), (vc, gv))):
                    x = (rng.standard_normal((n, dim)) * (strong[h] if side == 0 else np.exp(rng.standard_normal((n, 1))))).astype(np.float32)
                    lo, hi = x.min(1, keepdims=True), x.max(1, keepdims=True)
                    scale = ((hi - lo) / np.float32(15)).astype(np.float32)
                    c = np.clip(np.rint((x - lo) * (np.float32(1) / scale)), 0, 15).astype(np.uint32)
                    grids[p, h, s] = np.concatenate([lo, scale], 1)
                    if side == 0:
                        codes[p, h, s] = (c.reshape(n, -1, 8) << (4 * np.arange(8, dtype=np.uint32))).sum(2)
                    else:
                        sh = (4 * (s % 8)).astype(np.uint32)[:, None]
                        np.bitwise_and.at(codes, (p, h, s // 8), ~(np.uint32(15) << sh))
                        np.bitwise_or.at(codes, (p, h, s // 8), c << sh)

    def up(self):
        qp = self.qp
        self.d_pages, self.d_table, self.d_lengths = dev(self.pages), dev(self.table), dev(self.lengths)
        self.cache = qp.kv_cache(self.d_pages, self.heads, self.dim, self.page)
        self.rows = qp.kv_rows(self.d_table, self.d_lengths)

    def attend(self, counts, group, dtype, causal=True, window=0, scale=None, q=None, strided=False, check=True):
        qp = self.qp
        begin = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        tokens = int(begin[-1])
        heads = group * self.heads
        if q is None:
            q = self.rng.standard_normal((tokens, heads, self.dim)).astype(np.float32)
        t = dev(q).to(TYPES[dtype])
        if strided:       # heads outside tokens, and room between them
            wide = torch.zeros(heads, tokens + 1, self.dim + 16, dtype=TYPES[dtype], device="cuda")
            x = wide[:, :tokens, 16 if dtype == "f32" else 8:][:, :, :self.dim]
            x.copy_(t.transpose(0, 1))
            t = x.transpose(0, 1)
            out = torch.full_like(wide, 7)[:, :tokens, :self.dim].transpose(0, 1)
        else:
            out = torch.full_like(t, 7)
        ws = qp.alloc_kv_workspace(self.cache, self.rows, tokens, heads)
        ws.fill_(0xA5)
        scale = float(np.float32(scale or self.dim ** -0.5))
        qp.qp_kv_attention(self.cache, self.rows, 0, dev(begin), t, out, ws, scale=scale, causal=causal, window=window)
        if check:
            want, tol = kp.attention(self.pages[0], self.dim, self.page, self.table, self.lengths, begin, t.float().cpu().numpy(), scale, causal, window,
                                     U_OUT[dtype], dtype == "f32")
            close(out, want, tol)
        return out


def close(out, want, tol):
    o = out.float().cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isnan(o), np.isnan(want))
    bad = np.abs(o - want) > tol
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), o[bad][:4], want[bad][:4], tol[bad][:4])


# ---- attention -----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,page,heads,group,lengths", [
    (64, 32, 12, 1, [197]), (64, 64, 1, 8, [1]), (80, 32, 16, 1, [1, 31, 32, 33, 1500]), (96, 256, 2, 4, [700, 0, 129]),
    (128, 64, 8, 4, [4097, 1, 640, 2047]), (128, 128, 1, 16, [20000]), (256, 32, 2, 7, [515, 90]), (128, 64, 3, 20, [1000, 3])])
def test_single_tokens(qp, dim, page, heads, group, lengths, dtype):
    Case(qp, dim, page, heads, lengths).attend([1 if n else 0 for n in lengths], group, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,page,heads,group,lengths,counts,window", [
    (64, 32, 2, 2, [300, 77], [300, 70], 0),          # prompts
    (80, 64, 4, 1, [1100, 40, 500], [5, 3, 4], 1024),  # drafts in a window
    (128, 64, 2, 4, [900, 2000, 130], [150, 1, 33], 0),   # chunks beside a single token
    (128, 128, 1, 8, [3001], [129], 0),               # few items, many tokens: columns split and pieces joined
    (256, 32, 1, 3, [260], [260], 50),
    (96, 32, 2, 5, [64, 0, 1000], [70, 4, 13], 0),    # more tokens than the row has
])
def test_several_tokens(qp, dim, page, heads, group, lengths, counts, window, dtype):
    Case(qp, dim, page, heads, lengths).attend(counts, group, dtype, window=window)


def test_without_causality(qp):
    Case(qp, 64, 32, 3, [577, 20]).attend([100, 20], 2, "bf16", causal=False)
    Case(qp, 64, 32, 3, [577, 20]).attend([1, 2], 2, "f32", causal=False)


def test_many_rows(qp):
    """More rows than a block has lanes, most of them empty or without a token; with some long ones among them."""
    rng = np.random.default_rng(4)
    lengths = np.where(rng.random(700) < 0.3, rng.integers(0, 90, 700), 0)
    lengths[[0, 256, 511, 699]] = 3, 1000, 1, 640
    counts = np.minimum(lengths, rng.integers(0, 3, 700))
    counts[[256, 699]] = 2, 1
    Case(qp, 64, 32, 1, lengths.tolist()).attend(counts.tolist(), 2, "bf16")


def test_thousands_of_rows(qp):
    """One token each of 3000 rows, and prompts among them: where each row's work begins is found ahead of it."""
    rng = np.random.default_rng(9)
    lengths = rng.integers(0, 12, 3000)
    lengths[[5, 1023, 1024, 2999]] = 700, 300, 90, 64
    counts = np.minimum(lengths, 1)
    Case(qp, 64, 32, 1, lengths.tolist(), per_row=22).attend(counts.tolist(), 1, "bf16")
    counts[[5, 1024, 2999]] = 150, 90, 33
    Case(qp, 64, 32, 2, lengths.tolist(), per_row=22).attend(counts.tolist(), 32, "f32")


def test_scores_that_spread_far(qp):
    """Softmax from next to one-hot to flat, maxima that come late, queries that are tiny, huge, zero, or not finite."""
    c = Case(qp, 64, 32, 2, [1300, 1300])
    q = c.rng.standard_normal((8, 4, 64)).astype(np.float32)
    q[0] *= 30
    q[1] *= 1e-30
    q[2] = 0
    q[3] *= 1e-3
    q[4, 1, 3], q[5, 2, 5], q[6, 0, 0] = np.nan, np.inf, -np.inf
    for dtype in ("f32", "bf16"):
        c.attend([4, 4], 2, dtype, q=q)
    c.attend([4, 4], 2, "f32", q=q, scale=3.0)
    c.attend([4, 4], 2, "f32", q=q, scale=1e-20)


def test_value_scales_that_spread_far(qp):
    """Tokens whose values differ by many powers of ten: the normalization of the value scales moves on the way."""
    c = Case(qp, 64, 32, 1, [1000, 1000])
    _, _, _, gv = kp.pieces(c.pages[0], 64, 32)
    t = np.arange(1000)
    for r in range(2):
        up = 10.0 ** (t / 50.0 - 10) if r == 0 else 10.0 ** (10 - t / 50.0)
        gv[c.table[r, t // 32], 0, t % 32] *= up[:, None].astype(np.float32)
    gv[c.table[0, :4], 0, :] = 0                       # constant rows of zeros among them
    c.up()
    c.attend([1, 1], 4, "f32")
    c.attend([40, 20], 2, "f32")
    c.attend([1, 1], 4, "bf16")


def test_tables_that_point_nowhere(qp):
    c = Case(qp, 128, 32, 2, [400, 300, 64])
    c.table[0, 3], c.table[1, 0], c.table[2, :2] = -1, c.n_pages, 2 ** 31 - 1
    c.up()
    c.attend([1, 2, 1], 4, "bf16")                     # the last row sees nothing: 0
    c.attend([40, 70, 1], 4, "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides(qp, dtype):
    c = Case(qp, 64, 32, 2, [100, 333])
    assert torch.equal(c.attend([2, 40], 3, dtype, q=np.ones((42, 6, 64), np.float32), strided=True), c.attend([2, 40], 3, dtype, q=np.ones((42, 6, 64), np.float32)))
    c.attend([2, 40], 3, dtype, strided=True)
    # one query for all tokens and heads (strides of 0)
    q = dev(c.rng.standard_normal((1, 1, 64)).astype(np.float32)).to(TYPES[dtype])
    out, same = (torch.empty(42, 6, 64, dtype=TYPES[dtype], device="cuda") for _ in range(2))
    ws = qp.alloc_kv_workspace(c.cache, c.rows, 42, 6)
    begin = ints(0, 2, 42)
    qp.qp_kv_attention(c.cache, c.rows, 0, begin, q.expand(42, 6, 64), out, ws)
    qp.qp_kv_attention(c.cache, c.rows, 0, begin, q.expand(42, 6, 64).contiguous(), same, ws)
    assert torch.equal(out, same)


def test_answers_that_belong_to_no_row_stay(qp):
    c = Case(qp, 64, 32, 1, [50, 60])
    q = torch.randn(9, 2, 64, device="cuda")
    out = torch.full_like(q, 7)
    ws = qp.alloc_kv_workspace(c.cache, c.rows, 9, 2)
    qp.qp_kv_attention(c.cache, c.rows, 0, ints(2, 5, 7), q, out, ws)
    assert (out[:2] == 7).all() and (out[7:] == 7).all() and not (out[2:7] == 7).any()
    qp.qp_kv_attention(c.cache, c.rows, 0, ints(0, 0, 0), q[:0], out[:0], ws)        # nothing to do
    qp.qp_kv_append(c.cache, c.rows, 0, ints(0, 0, 0), q[:0, :1], q[:0, :1])
    qp.qp_kv_read(c.cache, c.rows, 0, ints(0, 0, 0), q[:0, :1], q[:0, :1])


def test_the_same_on_every_run_and_stream(qp):
    c = Case(qp, 128, 64, 4, [5000, 300, 2222])
    q = c.rng.standard_normal((12, 16, 128)).astype(np.float32)
    first = c.attend([1, 10, 1], 4, "bf16", q=q)
    for _ in range(5):
        assert torch.equal(c.attend([1, 10, 1], 4, "bf16", q=q, check=False), first)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = c.attend([1, 10, 1], 4, "bf16", q=q, check=False)
    s.synchronize()
    assert torch.equal(other, first)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_heads_share_a_key_head_than_a_block_has_columns(qp, dtype):
    Case(qp, 64, 32, 1, [300, 5]).attend([1, 2], 200, dtype)
    Case(qp, 64, 32, 1, [700]).attend([1], 1024, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths,counts", [([4000, 30], [1, 3]), ([1500, 300], [260, 1])])
def test_the_answer_may_take_the_query_s_place(qp, lengths, counts, dtype):
    c = Case(qp, 128, 64, 2, lengths)
    q = torch.from_numpy(c.rng.standard_normal((sum(counts), 8, 128))).to(TYPES[dtype]).cuda()
    begin = dev(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32))
    ws = qp.alloc_kv_workspace(c.cache, c.rows, sum(counts), 8)
    out = torch.empty_like(q)
    qp.qp_kv_attention(c.cache, c.rows, 0, begin, q, out, ws)
    qp.qp_kv_attention(c.cache, c.rows, 0, begin, q, q, ws)
    assert torch.equal(q, out)


def test_calls_and_graphs_at_once_with_a_workspace_each(qp):
    """Two streams, then two graphs on two streams, over one cache: each its own answers, replay after replay."""
    c = Case(qp, 128, 64, 4, [5000, 300, 2222])
    g = torch.Generator("cuda").manual_seed(6)
    jobs = []
    for counts in ([1, 1, 1], [90, 1, 40]):
        n = sum(counts)
        j = dict(q=torch.randn(n, 16, 128, device="cuda", generator=g).bfloat16(), begin=dev(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)),
                 ws=qp.alloc_kv_workspace(c.cache, c.rows, n, 16), stream=torch.cuda.Stream())
        j["out"], j["want"] = torch.empty_like(j["q"]), torch.empty_like(j["q"])
        qp.qp_kv_attention(c.cache, c.rows, 0, j["begin"], j["q"], j["want"], j["ws"])
        jobs.append(j)
    torch.cuda.synchronize()
    for _ in range(10):
        for j in jobs:
            qp.qp_kv_attention(c.cache, c.rows, 0, j["begin"], j["q"], j["out"], j["ws"], stream=j["stream"])
    torch.cuda.synchronize()
    assert all(torch.equal(j["out"], j["want"]) for j in jobs)
    for j in jobs:
        j["graph"] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(j["graph"]):
            for _ in range(3):
                qp.qp_kv_attention(c.cache, c.rows, 0, j["begin"], j["q"], j["out"], j["ws"])
    for _ in range(4):
        for j in jobs:
            j["out"].zero_()
        torch.cuda.synchronize()
        for j in jobs:
            with torch.cuda.stream(j["stream"]):
                j["graph"].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(j["out"], j["want"]) for j in jobs)


def test_numbers_past_32_bits_are_refused(qp):
    c = Case(qp, 64, 32, 1, [40])
    q = torch.ones(1, 1, 64, device="cuda")
    ws = qp.alloc_kv_workspace(c.cache, c.rows, 1, 1)
    for layer, window in ((2 ** 32, 0), (-1, 0), (0, 2 ** 32), (0, 2 ** 31), (0, -1)):
        with pytest.raises(qp.QuantPipeError):
            qp.qp_kv_attention(c.cache, c.rows, layer, ints(0, 1), q, q, ws, window=window)
    for call in (qp.qp_kv_append, qp.qp_kv_read):
        with pytest.raises(qp.QuantPipeError):
            call(c.cache, c.rows, 2 ** 32, ints(0, 1), q, q)
    assert (q == 1).all()


@pytest.mark.parametrize("dim,group,lengths,counts", [(128, 1, [1024] * 8, [1] * 8), (80, 4, [2000] * 4, [1] * 4), (64, 2, [600, 900], [200, 60])])
def test_fp32_answers_are_fp32(qp, dim, group, lengths, counts):
    """The 2-norm over all answers, where a single weight that lost its lower half (2^-12 of it) shows: the roundings of one answer are
    independent of each other, so that they add up like the square root of their number, at most dim + 2 log2(n) + 32 < 256 of 2^-24 B
    with B, the terms' size over the answer's, below 16 here: 16 sqrt(256) 2^-24 = 2^-16 of each answer."""
    c = Case(qp, dim, 64, 2, lengths)
    q = c.rng.standard_normal((sum(counts), 2 * group, dim)).astype(np.float32)
    o = c.attend(counts, group, "f32", q=q).double().cpu().numpy()
    begin = np.concatenate([[0], np.cumsum(counts)])
    want, _ = kp.attention(c.pages[0], dim, 64, c.table, c.lengths, begin, q, float(np.float32(dim ** -0.5)), True, 0, 2.0 ** -24, True)
    per = np.linalg.norm(o - want, axis=-1) / np.linalg.norm(want, axis=-1)
    assert per.max() <= 2.0 ** -16, per.max()


# ---- rows in and out ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,page,heads,counts", [(64, 32, 12, [1, 1, 0, 1]), (80, 64, 3, [13, 70, 1, 0]), (96, 128, 2, [200, 31]), (128, 64, 8, [129, 1, 64]),
                                                   (256, 256, 1, [300, 8])])
def test_rows_go_in_and_come_back(qp, dim, page, heads, counts, dtype):
    counts = np.array(counts)
    c = Case(qp, dim, page, heads, (counts + 37 * np.arange(len(counts))).tolist(), fill=False, per_row=kp.pages_of(int((counts + 37 * len(counts)).max()), page) + 1)
    begin = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    n = int(begin[-1])
    wide = torch.randn(n, 2 * heads + 3, dim, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(TYPES[dtype])
    k, v = wide[:, :heads], wide[:, heads + 3:]
    k[0, 0, :4] = torch.tensor([float("nan"), float("inf"), -float("inf"), 0.0])
    v[0, 0] = 1.5
    qp.qp_kv_append(c.cache, c.rows, 0, dev(begin), k, v)
    kp.append(c.pages[0], dim, page, c.table, c.lengths, begin, k.float().cpu().numpy(), v.float().cpu().numpy())
    assert np.array_equal(c.d_pages.cpu().numpy(), c.pages)
    first = c.lengths - counts
    ko, vo = torch.full((n + 2, heads, dim), 7, dtype=TYPES[dtype], device="cuda"), torch.full((heads, n + 2, dim), 7, dtype=TYPES[dtype], device="cuda").transpose(0, 1)
    qp.qp_kv_read(c.cache, c.rows, 0, dev(begin), ko, vo, first=dev(first.astype(np.int32)))
    a, b = np.zeros((n, heads, dim)), np.zeros((n, heads, dim))
    kp.read(c.pages[0], dim, page, c.table, c.lengths, begin, first, a, b)
    for x, y in ((ko, a), (vo, b)):
        assert (x[n:] == 7).all()
        x = x[:n].float().cpu().numpy().astype(np.float64)
        # one rounding to fp32, one more to bf16
        assert (np.abs(x - y) <= np.abs(y) * (U_OUT[dtype] + (2.0 ** -23 if dtype == "bf16" else 0)) + 2.0 ** -149).all()


def test_places_past_four_gigabytes(qp):
    """The last pages of the last layer of a cache of 9 GB."""
    heads, dim, page, layers, n_pages = 8, 128, 256, 3, 10240
    pages = torch.empty(layers, n_pages, heads, kp.slab_bytes(dim, page), dtype=torch.uint8, device="cuda")
    assert pages.numel() > 9e9
    cache = qp.kv_cache(pages, heads, dim, page)
    table = ints(n_pages - 1, 0, n_pages - 3).view(1, 3)
    rows = qp.kv_rows(table, ints(700))
    g = torch.Generator("cuda").manual_seed(2)
    k, v = (torch.randn(700, heads, dim, device="cuda", generator=g) for _ in range(2))
    q = torch.randn(3, 16, dim, device="cuda", generator=g)
    begin = ints(0, 700)
    qp.qp_kv_append(cache, rows, layers - 1, begin, k, v)
    mini = pages[layers - 1][table.view(-1).long()].cpu().numpy()
    want = np.zeros_like(mini)
    kp.append(want, dim, page, np.array([[0, 1, 2]]), np.array([700]), [0, 700], k.cpu().numpy(), v.cpu().numpy())
    for a, b in zip(kp.pieces(mini, dim, page), kp.pieces(want, dim, page)):
        assert np.array_equal(a[:2], b[:2])            # (the third page ends behind the length)
    out = torch.empty_like(q)
    qp.qp_kv_attention(cache, rows, layers - 1, ints(0, 3), q, out, qp.alloc_kv_workspace(cache, rows, 3, 16))
    close(out, *kp.attention(mini, dim, page, np.array([[0, 1, 2]]), np.array([700]), [0, 3], q.cpu().numpy(), float(np.float32(dim ** -0.5)), True, 0, 2.0 ** -24, True))
    # a page moves in every layer
    pool = qp.alloc_kv_pool(n_pages)
    pool[kp.HEADER + table.view(-1).long()] = 1
    before = pages[:, [n_pages - 1, n_pages - 3]].clone()
    qp.qp_kv_compact(cache, rows, pool)
    assert table.view(-1).tolist() == [2, 0, 1] and int(pool[3]) == 3
    assert torch.equal(pages[:, [2, 1]], before)


# ---- pages -----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("seed,rows,n_pages,per_row,page", [(0, 6, 40, 9, 32), (1, 300, 900, 5, 64), (2, 1500, 20000, 12, 32), (3, 3, 5, 4, 256)])
def test_the_books_against_one_row_after_the_other(qp, seed, rows, n_pages, per_row, page):
    rng = np.random.default_rng(seed)
    heads, dim, layers = 1, 64, 2
    pages = torch.randint(0, 256, (layers, n_pages, heads, kp.slab_bytes(dim, page)), dtype=torch.uint8, device="cuda")
    cache = qp.kv_cache(pages, heads, dim, page)
    table, lengths, refs = np.full((rows, per_row), -1, np.int32), np.zeros(rows, np.int32), np.zeros(n_pages, np.int32)
    d_table, d_lengths, pool = dev(table), dev(lengths), qp.alloc_kv_pool(n_pages)
    r = qp.kv_rows(d_table, d_lengths)
    shadow = pages.cpu().numpy()
    seen = set()
    for step in range(24):
        op = ("reserve", "fork", "reserve", "free", "reserve", "compact")[step % 6]
        head = None
        if op == "reserve":
            want = np.where(rng.random(rows) < 0.7, rng.integers(-1, page * 2, rows), 0).astype(np.int32)
            if rng.random() < 0.7:
                want = np.minimum(want, per_row * page - lengths).astype(np.int32)
            if step % 4 == 0:
                want = np.minimum(want, 1)
            qp.qp_kv_reserve(cache, r, pool, dev(want))
            short, out, moves = kp.reserve(table, lengths, refs, want, page)
            head = [short, out]
            seen |= {"short"} if short else {"out"} if out else {"copies"} if moves else set()
        elif op == "fork":
            parent = np.where((lengths == 0) | (rng.random(rows) < 0.05), rng.integers(-1, rows, rows), -1).astype(np.int32)
            refused = int(pool[2])
            qp.qp_kv_fork(cache, r, pool, dev(parent))
            assert int(pool[2]) - refused == kp.fork(table, lengths, refs, parent, page)
            moves = []
        elif op == "free":
            keep = np.where(rng.random(rows) < 0.5, rng.integers(0, 2, rows) * rng.integers(0, page * per_row, rows), -1).astype(np.int32)
            qp.qp_kv_free(cache, r, pool, dev(keep))
            kp.free(table, lengths, refs, keep, page)
            moves = []
        else:
            qp.qp_kv_compact(cache, r, pool)
            live, moves = kp.compact(table, lengths, refs, page)
            assert int(pool[3]) == live
            seen |= {"moves"} if moves else set()
        for a, b in moves:
            shadow[:, b] = shadow[:, a]
        got = pool.cpu().numpy()
        assert np.array_equal(d_lengths.cpu().numpy(), lengths), (step, op)
        assert np.array_equal(d_table.cpu().numpy(), table), (step, op)
        assert np.array_equal(got[kp.HEADER:kp.HEADER + n_pages], refs), (step, op)
        assert head is None or got[:2].tolist() == head, (step, op)
        assert not got[kp.HEADER + n_pages:kp.HEADER + 3 * n_pages].any()
        assert np.array_equal(pages.cpu().numpy(), shadow), (step, op)
    if rows >= 300:                                    # (enough of them for every way out)
        assert {"copies", "moves"} <= seen


# ---- together -----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_serving_loop(qp, dtype):
    """Two prompts, their beams forked and grown token by token, drafts rolled back, losers freed, the pool compacted: after each
    step the answers are those of the plain form on what the rows hold."""
    heads, group, dim, page, layers, rows, n_pages = 2, 3, 64, 32, 2, 6, 30
    pages = qp.alloc_kv_pages(n_pages, heads, dim, page, layers=layers)
    cache, pool = qp.kv_cache(pages, heads, dim, page), qp.alloc_kv_pool(n_pages)
    table, lengths = torch.full((rows, 6), -1, dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
    r = qp.kv_rows(table, lengths)
    g = torch.Generator("cuda").manual_seed(3)
    held = [[np.zeros((2, 0, heads, dim)) for _ in range(rows)] for _ in range(layers)]     # what each row's tokens come back as

    def step(new):
        qp.qp_kv_reserve(cache, r, pool, ints(*new))
        assert pool[:2].tolist() == [0, 0]
        begin = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        n = int(begin[-1])
        ws = qp.alloc_kv_workspace(cache, r, n, heads * group)
        L = lengths.cpu().numpy()
        for layer in range(layers):
            k, v = (torch.randn(n, heads, dim, device="cuda", generator=g).to(TYPES[dtype]) for _ in range(2))
            q = torch.randn(n, heads * group, dim, device="cuda", generator=g).to(TYPES[dtype])
            out = torch.empty_like(q)
            qp.qp_kv_append(cache, r, layer, dev(begin), k, v)
            qp.qp_kv_attention(cache, r, layer, dev(begin), q, out, ws)
            P, T = pages[layer].cpu().numpy(), table.cpu().numpy()
            close(out, *kp.attention(P, dim, page, T, L, begin, q.float().cpu().numpy(), float(np.float32(dim ** -0.5)), True, 0, U_OUT[dtype], dtype == "f32"))
            for row in range(rows):
                a, b = np.zeros((L[row], heads, dim)), np.zeros((L[row], heads, dim))
                full = np.zeros(rows + 1, np.int32)
                full[row + 1:] = L[row]
                kp.read(P, dim, page, T, L, full, None, a, b)
                was = held[layer][row]
                assert np.array_equal(np.stack([a, b])[:, :was.shape[1]], was)      # what was there is still what it was
                held[layer][row] = np.stack([a, b])

    def forget(keep):
        for layer in held:
            for row, n in enumerate(keep):
                if 0 <= n:
                    layer[row] = layer[row][:, :n]

    step([45, 0, 0, 70, 0, 0])
    qp.qp_kv_fork(cache, r, pool, ints(-1, 0, 0, -1, 3, 3))
    for layer in held:
        layer[1] = layer[2] = layer[0]
        layer[4] = layer[5] = layer[3]
    step([1, 1, 1, 1, 1, 1])
    step([1, 1, 1, 4, 1, 1])
    qp.qp_kv_free(cache, r, pool, ints(-1, 0, -1, 72, -1, 0))
    forget([-1, 0, -1, 72, -1, 0])
    step([1, 0, 20, 1, 1, 0])
    qp.qp_kv_free(cache, r, pool, ints(0, -1, -1, -1, 5, -1))
    forget([0, -1, -1, -1, 5, -1])
    qp.qp_kv_compact(cache, r, pool)
    live = int(pool[3])
    assert int(table.max()) < live and int((pool[kp.HEADER:kp.HEADER + n_pages] > 0).sum()) == live
    step([33, 0, 1, 1, 1, 2])


def test_as_many_rows_as_there_may_be(qp):
    """65536 rows, two tokens each, in two steps.  fp32: the weights of two tokens are off by at most (dim + 8) roundings of 2^-24 of a score
    below 64 in size, so 2^-11 of one (72 * 64 * 2^-24 < 2^-11), and the answer by that times the values' spread.  Its two parts, of
    (c - 8) s and of lo + 8 s, cancel where an element is small: they are rounded as they are, and with T the largest of the tokens' values
    15 s <= 2 T and -T <= lo <= T, so both are at most 1.1 T; weights in two halves (2^-22) and three sums of two (2^-24 each) for both
    parts come to less than 2 * 1.1 * (2^-22 + 3 * 2^-24) T < 2^-20 T."""
    rows, dim, page = 65536, 64, 32
    pages = qp.alloc_kv_pages(rows + 9, 1, dim, page)
    cache, pool = qp.kv_cache(pages, 1, dim, page), qp.alloc_kv_pool(rows + 9)
    table, lengths = torch.full((rows, 1), -1, dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
    r = qp.kv_rows(table, lengths)
    begin = torch.arange(rows + 1, dtype=torch.int32, device="cuda")
    g = torch.Generator("cuda").manual_seed(8)
    ws = qp.alloc_kv_workspace(cache, r, rows, 2)
    for step in (1, 2):
        qp.qp_kv_reserve(cache, r, pool, torch.ones(rows, dtype=torch.int32, device="cuda"))
        assert pool[:2].tolist() == [0, 0] and (lengths == step).all()
        k, v, q = (torch.randn(rows, n, dim, device="cuda", generator=g) for n in (1, 1, 2))
        out = torch.empty_like(q)
        qp.qp_kv_append(cache, r, 0, begin, k, v)
        qp.qp_kv_attention(cache, r, 0, begin, q, out, ws)
    assert torch.equal(table.view(-1), begin[:-1])                # (in order: the lowest free page first)
    ko, vo = (torch.empty(2 * rows, 1, dim, device="cuda") for _ in range(2))
    qp.qp_kv_read(cache, r, 0, 2 * begin, ko, vo)
    ko, vo, q = ko.view(rows, 1, 2, dim).double(), vo.view(rows, 1, 2, dim).double(), q.double()
    scores = (q.unsqueeze(2) * ko).sum(-1) * dim ** -0.5
    assert scores.abs().max() < 64
    want = (torch.softmax(scores, -1).unsqueeze(-1) * vo).sum(2)
    off, spread, top = (out.double() - want).abs(), (vo[:, :, 0] - vo[:, :, 1]).abs(), vo.abs().amax((2, 3)).unsqueeze(-1)
    worst = (off / (spread * 2.0 ** -11 + top * 2.0 ** -20)).max()
    assert worst <= 1, worst
    qp.qp_kv_free(cache, r, pool, torch.where(begin[:-1] % 2 == 0, 0, -1).int())
    qp.qp_kv_compact(cache, r, pool)
    assert int(pool[3]) == rows // 2 and int(table[1::2].max()) < rows // 2 and (table[::2] == -1).all()
    k2, v2 = (torch.empty(rows, 1, dim, device="cuda") for _ in range(2))
    qp.qp_kv_read(cache, r, 0, torch.cat([torch.zeros(1, device="cuda"), (2 * (begin[:-1] % 2)).cumsum(0)]).int(), k2, v2)
    assert torch.equal(k2.view(rows // 2, 2, dim).double(), ko[1::2, 0]) and torch.equal(v2.view(rows // 2, 2, dim).double(), vo[1::2, 0])


def test_a_step_replays_from_a_graph(qp):
    """Reserve, append, attention and free of one step in a captured graph, replayed with other inputs between the program's own eager
    calls, each replay against the same calls made eagerly on a copy."""
    heads, group, dim, page, rows, n_pages = 2, 4, 128, 32, 4, 64
    g = torch.Generator("cuda").manual_seed(4)

    def world():
        pages = torch.zeros(1, n_pages, heads, kp.slab_bytes(dim, page), dtype=torch.uint8, device="cuda")
        table, lengths = torch.full((rows, 12), -1, dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
        w = {"pages": pages, "table": table, "lengths": lengths, "pool": qp.alloc_kv_pool(n_pages), "cache": qp.kv_cache(pages, heads, dim, page), "rows": qp.kv_rows(table, lengths)}
        w["q"], w["out"] = torch.zeros(rows, heads * group, dim, device="cuda"), torch.zeros(rows, heads * group, dim, device="cuda")
        w["k"], w["v"] = torch.zeros(rows, heads, dim, device="cuda"), torch.zeros(rows, heads, dim, device="cuda")
        w["ws"] = qp.alloc_kv_workspace(w["cache"], w["rows"], rows, heads * group)
        w["keep"] = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
        return w

    begin, one = ints(0, 1, 2, 3, 4), ints(1, 1, 1, 1)

    def step(w):
        qp.qp_kv_free(w["cache"], w["rows"], w["pool"], w["keep"])
        qp.qp_kv_reserve(w["cache"], w["rows"], w["pool"], one)
        qp.qp_kv_append(w["cache"], w["rows"], 0, begin, w["k"], w["v"])
        qp.qp_kv_attention(w["cache"], w["rows"], 0, begin, w["q"], w["out"], w["ws"])

    a, b = world(), world()
    step(a)
    step(b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)                                        # (recorded, not run)
    for i in range(70):
        for n in ("q", "k", "v"):
            a[n].normal_(generator=g)
            b[n].copy_(a[n])
        for w in (a, b):
            w["keep"].fill_(-1)
            if i in (20, 50):
                w["keep"][1] = 3
        graph.replay()
        step(b)
        for n in ("out", "table", "lengths", "pool", "pages"):
            assert torch.equal(a[n], b[n]), (i, n)
    assert a["lengths"].tolist() == [71, 23, 71, 71]


def test_more_blocks_than_a_launch_has(qp):
    """One token for each of 65536 rows of 1024 heads: 2^24 blocks and more, for append, read and attention.  Three of the rows hold anything;
    theirs are the answers of calls with these three alone, to the bit, and the others' are 0."""
    rows, heads, dim, page = 65536, 1024, 64, 32
    some = torch.tensor([0, 40000, 65535], device="cuda")
    pages = qp.alloc_kv_pages(3, heads, dim, page)
    cache = qp.kv_cache(pages, heads, dim, page)
    table, lengths = torch.full((rows, 1), -1, dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
    table[some, 0], lengths[some] = ints(2, 0, 1), ints(20, 1, 32)
    r = qp.kv_rows(table, lengths)
    few = qp.kv_rows(table[some].contiguous(), lengths[some].contiguous())
    g = torch.Generator("cuda").manual_seed(12)
    k, v = (torch.randn(53, heads, dim, device="cuda", generator=g).bfloat16() for _ in range(2))
    qp.qp_kv_append(cache, few, 0, ints(0, 20, 21, 53), k, v)
    begin = torch.arange(rows + 1, dtype=torch.int32, device="cuda")
    x = torch.randn(1, heads, dim, device="cuda", generator=g).bfloat16()
    before = pages.clone()
    qp.qp_kv_append(cache, few, 0, ints(0, 1, 2, 3), x.expand(3, -1, -1), 2 * x.expand(3, -1, -1))
    want = pages.clone()
    pages.copy_(before)
    qp.qp_kv_append(cache, r, 0, begin, x.expand(rows, -1, -1), (2 * x).expand(rows, -1, -1))
    assert torch.equal(pages, want)

    def zero(t):
        t[some] = 0
        return int(torch.count_nonzero(t.view(torch.int32))) == 0

    q = x.expand(rows, -1, -1)
    out, same = torch.full((rows, heads, dim), 7, dtype=torch.bfloat16, device="cuda"), torch.empty(3, heads, dim, dtype=torch.bfloat16, device="cuda")
    qp.qp_kv_attention(cache, r, 0, begin, q, out, qp.alloc_kv_workspace(cache, r, rows, heads))
    qp.qp_kv_attention(cache, few, 0, ints(0, 1, 2, 3), q[:3], same, qp.alloc_kv_workspace(cache, few, 3, heads))
    assert torch.equal(out[some], same) and not (same == 0).all(-1).any() and zero(out)
    vo, first = torch.full_like(out, 7), torch.where(lengths > 0, lengths - 1, 0).int()
    qp.qp_kv_read(cache, r, 0, begin, out.fill_(7), vo, first=first)
    k3, v3 = torch.empty_like(same), torch.empty_like(same)
    qp.qp_kv_read(cache, few, 0, ints(0, 1, 2, 3), k3, v3, first=first[some].contiguous())
    assert torch.equal(out[some], k3) and torch.equal(vo[some], v3) and zero(out) and zero(vo)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_causality_of_more_tokens_than_the_row_has(qp, dtype):
    """Queries that are none of the row's tokens: each sees the whole row."""
    Case(qp, 64, 32, 3, [5, 0, 40, 700]).attend([6, 2, 100, 900], 2, dtype, causal=False)
    c = Case(qp, 128, 64, 1, [9])
    q = np.repeat(c.rng.standard_normal((1, 4, 128)).astype(np.float32), 12, 0)
    out = c.attend([12], 4, dtype, causal=False, q=q)
    assert torch.equal(out, out[:1].expand(12, 4, 128))
    assert (c.attend([12], 4, dtype, q=q)[:3] == 0).all()          # causal: three tokens ahead of the row's first


def test_sizes_past_32_bits_are_refused(qp):
    pages = qp.alloc_kv_pages(4, 1, 64, 32)
    for kind in ((2 ** 32 + 1, 64, 32), (1, 2 ** 32 + 64, 32), (1, 64, 2 ** 32 + 32)):
        with pytest.raises(qp.QuantPipeError):
            qp.kv_cache(pages, *kind)
    pool = torch.full((100,), 7, dtype=torch.int32, device="cuda")
    with pytest.raises(qp.QuantPipeError):
        qp.qp_kv_pool_init(2 ** 32 + 4, pool)
    assert (pool == 7).all()
