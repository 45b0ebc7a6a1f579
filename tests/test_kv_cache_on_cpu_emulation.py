"""The 4-bit key/value cache's kernels on the CPU emulation (tests/emu/kv), under AddressSanitizer and UBSan with every buffer
exactly as long as it has to be, against the plain forms of kv_plain.py: indexing and logic, page tables that point nowhere,
lengths and token ranges that make no sense, workspaces of exactly the size asked for."""
import os
import subprocess
import sys

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)
sys.path.insert(0, os.path.join(HERE, "emu", "kv"))
import build_emu_kv  # noqa: E402
import kv_plain as kp  # noqa: E402


@pytest.fixture(scope="module")
def driver():
    try:
        exe = build_emu_kv.build()
    except subprocess.CalledProcessError as e:
        pytest.fail("emulation build failed:\n" + e.stderr.decode()[-3000:])
    if exe is None:
        pytest.skip("no host clang++ to build the emulation with")
    return exe


class Emu:
    """A script for the driver: buffers by name, calls, and what the buffers hold afterwards."""

    def __init__(self, exe, path):
        self.exe, self.path, self.lines, self.shapes, self.calls = exe, str(path), [], {}, 0

    def buf(self, name, a):
        a = np.ascontiguousarray(a)
        a.tofile(os.path.join(self.path, name))
        self.lines.append("buf %s %d %s" % (name, a.nbytes, os.path.join(self.path, name)))
        self.shapes[name] = (a.dtype, a.shape)

    def do(self, *words):
        self.lines.append(" ".join(str(w) for w in words))
        self.calls += words[0] not in ("cache", "rows")

    def run(self, *names):
        for n in names:
            self.lines.append("dump %s %s.out" % (n, os.path.join(self.path, n)))
        p = subprocess.run([self.exe], input="\n".join(self.lines) + "\n", text=True, capture_output=True, timeout=1500,
                           env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0", UBSAN_OPTIONS="print_stacktrace=1"))
        assert p.returncode == 0, p.stderr[-4000:]
        assert [int(x) for x in p.stdout.split()] == [0] * self.calls
        out = []
        for n in names:
            dt, shape = self.shapes[n]
            out.append(np.fromfile(os.path.join(self.path, n) + ".out", dt).reshape(shape))
        return out


def bf16(x):
    """fp32 -> the nearest bf16, as its bits; half to even."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def widen(b):
    return (b.astype(np.uint32) << 16).view(np.float32)


def setup(rng, rows, per_row, n_pages):
    order = rng.permutation(n_pages)[:rows * per_row].reshape(rows, per_row)
    return order.astype(np.int32)


# ---- rows in and out ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dim,page,dtype", [(64, 32, 0), (80, 64, 1), (96, 32, 1), (128, 128, 0), (256, 32, 1)])
def test_rows_go_in_and_come_back(driver, tmp_path, dim, page, dtype):
    rng = np.random.default_rng(dim + page)
    heads, rows, n_pages, per_row = 3, 4, 9, 2
    pages = kp.new_pages(2, n_pages, heads, dim, page, rng)
    table = setup(rng, rows, per_row, n_pages)
    table[2, 0] = -1 if dim == 64 else n_pages        # a page that is not there
    counts = [1, 13, 5, 0]
    lengths = np.array([page + 3, 21, 9, 4], np.int32)
    begin = np.concatenate([[1], 1 + np.cumsum(counts)]).astype(np.int32)      # token 0 and the last two are no row's
    tokens = int(begin[-1]) + 2
    wide = rng.standard_normal((tokens, 2 * heads + 1, dim)).astype(np.float32)
    wide[3, 0, 5], wide[3, 0, 6], wide[4, 1, 0], wide[5, 2, :] = np.nan, np.inf, -np.inf, np.nan
    wide[6, 0, :] = 2.5
    wide[7, 0, :] = np.linspace(-3.4e38, 3.4e38, dim)
    wide[8, 0, :] = 1e-40 * np.arange(dim)
    data = wide if dtype == 0 else bf16(wide)
    values = wide if dtype == 0 else widen(data)
    e = Emu(driver, tmp_path)
    for n, a in (("pages", pages), ("table", table), ("lengths", lengths), ("begin", begin), ("kv", data)):
        e.buf(n, a)
    # (the second tensor starts where the first one's heads end: strides of a fused projection)
    e.buf("vv", np.ascontiguousarray(data[:, heads:].reshape(tokens, -1)))
    e.do("cache", "pages", 2, n_pages, heads, dim, page)
    e.do("rows", "table", "lengths", rows, per_row)
    vv = np.ascontiguousarray(np.concatenate([data[:, heads:], data[:, :heads]], 1))
    e.buf("vv", vv)
    e.do("append", 1, "begin", tokens, "kv", "vv", dtype, (2 * heads + 1) * dim, dim)
    want = pages.copy()
    kp.append(want[1], dim, page, table, lengths, begin, values[:, :heads], np.concatenate([values[:, heads:], values[:, :heads]], 1)[:, :heads])
    # ... and back: from different places, past the end, before the start
    first = np.array([page, 0, 2, -2], np.int32)
    rcounts = [6, 30, 9, 8]
    rbegin = np.concatenate([[0], np.cumsum(rcounts)]).astype(np.int32)
    rtok = int(rbegin[-1]) + 3
    dense = np.full((rtok, heads, dim), 7, np.float32 if dtype == 0 else np.uint16)
    for n, a in (("first", first), ("rbegin", rbegin), ("ko", dense), ("vo", dense)):
        e.buf(n, a)
    e.do("read", 1, "rbegin", "first", rtok, "ko", "vo", dtype, heads * dim, dim)
    got, ko, vo = e.run("pages", "ko", "vo")
    assert np.array_equal(got, want)
    k, v = np.full((rtok, heads, dim), np.nan), np.full((rtok, heads, dim), np.nan)
    with np.errstate(invalid="ignore"):
        kp.read(want[1], dim, page, table, lengths, rbegin, first, k, v)
    for a, b in ((ko, k), (vo, v)):
        assert (a[rbegin[-1]:] == 7).all()            # no row's: as they were
        a = (a if dtype == 0 else widen(a)).astype(np.float64)[:rbegin[-1]]
        b = b[:rbegin[-1]]
        fine = np.isfinite(b) & (np.abs(b) < 3e38)
        # fp32: one rounding; bf16: that and one to bf16; half a step of the smallest subnormals (2^-149, 2^-133) below those
        tol = np.abs(b) * (2.0 ** -24 if dtype == 0 else 2.0 ** -8 + 2.0 ** -23) + (2.0 ** -150 if dtype == 0 else 2.0 ** -134 + 2.0 ** -150)
        assert (np.abs(a - b)[fine] <= tol[fine]).all()


def test_prompts_of_many_octets_and_rows(driver, tmp_path):
    """Eight tokens a wave: rows that begin and end inside an octet, rows without tokens, more rows than one search takes."""
    rng = np.random.default_rng(5)
    heads, dim, page, rows, per_row = 1, 64, 32, 130, 2
    n_pages = rows * per_row
    pages = kp.new_pages(1, n_pages, heads, dim, page, rng)
    table = setup(rng, rows, per_row, n_pages)
    counts = np.where(np.arange(rows) % 13 == 0, rng.integers(1, 60, rows), 0)
    counts[5], counts[129], counts[70] = 64, 3, 64
    counts[0] = 60
    need = 8 * rows + 1 - counts.sum()
    for r in range(1, rows):
        if need <= 0:
            break
        add = min(64 - counts[r], max(0, need))
        counts[r] += add
        need -= add
    lengths = np.minimum(counts + rng.integers(0, 5, rows), per_row * page).astype(np.int32)
    lengths[0] = counts[0] - 7                        # more tokens than the length: the first seven have no place
    begin = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    tokens = int(begin[-1])
    assert tokens >= 8 * rows
    k = rng.standard_normal((tokens, heads, dim)).astype(np.float32)
    v = rng.standard_normal((tokens, heads, dim)).astype(np.float32)
    e = Emu(driver, tmp_path)
    out = np.zeros((tokens, heads, dim), np.float32)
    for n, a in (("pages", pages), ("table", table), ("lengths", lengths), ("begin", begin), ("k", k), ("v", v), ("ko", out), ("vo", out)):
        e.buf(n, a)
    e.do("cache", "pages", 1, n_pages, heads, dim, page)
    e.do("rows", "table", "lengths", rows, per_row)
    e.do("append", 0, "begin", tokens, "k", "v", 0, heads * dim, dim)
    e.do("read", 0, "begin", "-", tokens, "ko", "vo", 0, heads * dim, dim)
    got, ko, vo = e.run("pages", "ko", "vo")
    kp.append(pages[0], dim, page, table, lengths, begin, k, v)
    assert np.array_equal(got, pages)
    a, b = np.zeros((tokens, heads, dim)), np.zeros((tokens, heads, dim))
    with np.errstate(invalid="ignore"):
        kp.read(pages[0], dim, page, table, lengths, begin, None, a, b)
    fine = np.isfinite(a) & np.isfinite(b)
    assert (np.abs(ko - a)[fine] <= np.abs(a[fine]) * 2.0 ** -24).all() and (np.abs(vo - b)[fine] <= np.abs(b[fine]) * 2.0 ** -24).all()


@pytest.mark.parametrize("begin", [[0, 5, 2, 9, 9], [-3, 4, 100, 7, 2], [9, 9, 9, 9, 9], [3, 1, 0, -5, -9]])
def test_token_ranges_that_make_no_sense_stay_inside(driver, tmp_path, begin):
    """Ranges that overlap, go back or lie outside: whatever is computed, nothing is read or written out of bounds."""
    rng = np.random.default_rng(1)
    heads, dim, page, rows, per_row, n_pages, tokens = 2, 64, 32, 4, 6, 5, 9
    pages = kp.new_pages(1, n_pages, heads, dim, page)
    table = rng.integers(-2, n_pages + 2, (rows, per_row)).astype(np.int32)
    table[0, 0], table[0, 1] = np.iinfo(np.int32).min, np.iinfo(np.int32).max
    lengths = np.array([-7, 100, 2 ** 31 - 1, 40], np.int32)
    x = rng.standard_normal((tokens, heads, dim)).astype(np.float32)
    q = rng.standard_normal((tokens, 5 * heads, dim)).astype(np.float32)
    e = Emu(driver, tmp_path)
    for n, a in (("pages", pages), ("table", table), ("lengths", lengths), ("begin", np.array(begin, np.int32)), ("k", x), ("v", x),
                 ("ko", x), ("vo", x), ("q", q), ("o", q), ("first", np.array([2 ** 31 - 1, -2 ** 31, 30, 190], np.int32))):
        e.buf(n, a)
    e.do("cache", "pages", 1, n_pages, heads, dim, page)
    e.do("rows", "table", "lengths", rows, per_row)
    e.do("append", 0, "begin", tokens, "k", "v", 0, heads * dim, dim)
    e.do("read", 0, "begin", "first", tokens, "ko", "vo", 0, heads * dim, dim)
    e.do("attention", 0, "begin", tokens, "q", "o", 0, 5 * heads * dim, dim, 5 * heads, 0.125, 1, 0)
    e.run("o")


def test_ranges_of_many_rows_that_overlap_stay_inside(driver, tmp_path):
    """More rows than a wave has lanes, of which every second one has all of the call's tokens: far more work than the launch is for."""
    rng = np.random.default_rng(2)
    heads, dim, page, rows, per_row, n_pages, tokens = 1, 64, 32, 70, 6, 5, 30
    e = Emu(driver, tmp_path)
    q = rng.standard_normal((tokens, 2 * heads, dim)).astype(np.float32)
    begin = np.where(np.arange(rows + 1) % 2, tokens, 0).astype(np.int32)
    for n, a in (("pages", kp.new_pages(1, n_pages, heads, dim, page)), ("table", rng.integers(-2, n_pages + 2, (rows, per_row)).astype(np.int32)),
                 ("lengths", rng.integers(-9, 400, rows).astype(np.int32)), ("begin", begin), ("q", q), ("o", q)):
        e.buf(n, a)
    e.do("cache", "pages", 1, n_pages, heads, dim, page)
    e.do("rows", "table", "lengths", rows, per_row)
    e.do("attention", 0, "begin", tokens, "q", "o", 0, 2 * heads * dim, dim, 2 * heads, 0.125, 1, 0)
    e.run("o")


# ---- attention -----------------------------------------------------------------------------------------------------------

def attend(driver, path, dim, page, heads, group, lengths, counts, dtype, causal=1, window=0, scale=None, spoil=None, per_row=None, missing=()):
    rng = np.random.default_rng(dim + sum(lengths) + 7 * sum(counts))
    rows = len(lengths)
    per_row = per_row or max(1, max(kp.pages_of(n, page) for n in lengths))
    n_pages = rows * per_row + 1
    pages = kp.new_pages(1, n_pages, heads, dim, page, rng)        # behind the lengths: NaN and Inf grids
    table = setup(rng, rows, per_row, n_pages)
    for r, s in missing:
        table[r, s] = -1
    full = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    n = int(full[-1])
    k = rng.standard_normal((n, heads, dim)).astype(np.float32) * np.where(rng.random((1, heads, dim)) < 0.05, 4, 1).astype(np.float32)
    v = rng.standard_normal((n, heads, dim)).astype(np.float32) * np.exp(rng.standard_normal((n, 1, 1))).astype(np.float32)
    kp.append(pages[0], dim, page, table, np.array(lengths), full, k, v)
    begin = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    tokens = int(begin[-1])
    q = rng.standard_normal((tokens, heads * group, dim)).astype(np.float32)
    if spoil:
        spoil(q)
    data = q if dtype == 0 else bf16(q)
    q = q if dtype == 0 else widen(data)
    scale = scale or dim ** -0.5
    e = Emu(driver, path)
    for name, a in (("pages", pages), ("table", table), ("lengths", np.array(lengths, np.int32)), ("begin", begin), ("q", data), ("o", np.zeros_like(data))):
        e.buf(name, a)
    e.do("cache", "pages", 1, n_pages, heads, dim, page)
    e.do("rows", "table", "lengths", rows, per_row)
    e.do("attention", 0, "begin", tokens, "q", "o", dtype, heads * group * dim, dim, heads * group, repr(float(np.float32(scale))), causal, window)
    (o,) = e.run("o")
    o = (o if dtype == 0 else widen(o)).astype(np.float64)
    want, tol = kp.attention(pages[0], dim, page, table, lengths, begin, q, float(np.float32(scale)), causal, window, 2.0 ** -24 if dtype == 0 else 2.0 ** -8, dtype == 0)
    assert np.array_equal(np.isnan(o), np.isnan(want))
    bad = np.abs(o - want) > tol
    assert not bad.any(), (np.argwhere(bad)[:4], o[bad][:4], want[bad][:4], tol[bad][:4])


@pytest.mark.parametrize("dim,page,heads,group,lengths,counts,dtype", [
    (64, 32, 2, 1, [1], [1], 1),                      # one token that sees itself
    (64, 32, 1, 3, [197, 33], [1, 1], 0),             # single tokens, shared heads, a page that ends inside a tile
    (80, 64, 1, 2, [300, 0, 65], [1, 0, 1], 1),       # an empty row; pieces of several blocks
    (128, 32, 1, 8, [600], [1], 1),
    (96, 32, 1, 4, [40], [9], 0),                     # 36 columns: a whole wave of them and a rest
    (256, 32, 1, 1, [70], [2], 1),
    (64, 32, 1, 2, [150], [150], 0),                  # a prompt over itself
    (64, 64, 1, 1, [90, 260], [90, 140], 1),
])
def test_attention(driver, tmp_path, dim, page, heads, group, lengths, counts, dtype):
    attend(driver, tmp_path, dim, page, heads, group, lengths, counts, dtype)


def test_attention_of_more_rows_than_a_wave_has_lanes(driver, tmp_path):
    lengths = [0] * 70
    lengths[3], lengths[64], lengths[69] = 40, 300, 5
    attend(driver, tmp_path, 64, 32, 1, 1, lengths, [0, 0, 0, 1] + [0] * 60 + [20, 0, 0, 0, 0, 2], 1, per_row=10)


def test_attention_without_causality(driver, tmp_path):
    attend(driver, tmp_path, 64, 32, 1, 2, [45, 130], [20, 3], 0, causal=0)


def test_attention_in_a_window(driver, tmp_path):
    attend(driver, tmp_path, 64, 32, 1, 1, [200, 31], [40, 31], 0, window=37)


def test_attention_of_more_tokens_than_the_row_has(driver, tmp_path):
    """The tokens ahead of the row's start see nothing: 0."""
    attend(driver, tmp_path, 64, 32, 1, 1, [5, 0], [20, 3], 0)


def test_attention_past_a_missing_page(driver, tmp_path):
    attend(driver, tmp_path, 64, 32, 1, 2, [100, 40], [1, 2], 0, missing=((0, 1), (1, 0)))


def test_attention_with_a_query_that_is_not_finite(driver, tmp_path):
    def spoil(q):
        q[1, 0, 3], q[2, 1, 0], q[4, 0, :], q[0, 0, :] = np.nan, -np.inf, 0, 0
        q[3, 1] *= np.float32(1e-30)
    attend(driver, tmp_path, 64, 32, 1, 2, [60], [7], 0, spoil=spoil)


# ---- pages -----------------------------------------------------------------------------------------------------------------

def test_the_books_against_one_row_after_the_other(driver, tmp_path):
    """Reserve, fork, reserve with shared pages, free in part, run short, outgrow, compact: tables, lengths, counts and pages."""
    rng = np.random.default_rng(3)
    heads, dim, page, layers, rows, per_row, n_pages = 1, 64, 32, 2, 7, 4, 17
    pages = rng.integers(0, 256, (layers, n_pages, heads, kp.slab_bytes(dim, page)), dtype=np.uint8)
    table = np.full((rows, per_row), -1, np.int32)
    lengths = np.zeros(rows, np.int32)
    pool = np.full(kp.HEADER + 6 * n_pages, 99, np.int32)
    refs = np.zeros(n_pages, np.int32)
    e = Emu(driver, tmp_path)
    for n, a in (("pages", pages), ("table", table), ("lengths", lengths), ("pool", pool)):
        e.buf(n, a)
    e.do("cache", "pages", layers, n_pages, heads, dim, page)
    e.do("rows", "table", "lengths", rows, per_row)
    e.do("pool_init", n_pages, "pool")
    steps = [("reserve", [40, 0, 64, -3, 0, 0, 1]), ("fork", [-1, 0, -1, 2, 0, 1, 3]), ("fork", [-1, -1, -1, -1, -1, 0, 9]),
             ("reserve", [1, 2, 0, 30, 3, 24, 0]), ("reserve", [0, 0, 200, 0, 0, 0, 0]), ("reserve", [80, 80, 0, 0, 80, 0, 0]),
             ("free", [-1, 0, 32, 70, 41, -1, 0]), ("free", [40, 5, 32, 64, 64, 33, -1]), ("fork", [-1, 0, -1, -1, -1, -1, 0]),
             ("reserve", [1, 1, 5, 1, 1, 1, 1]), ("free", [0, -1, 0, -1, 33, -1, -1])]
    heads_of = [0, 0, 0]
    dumps = []
    for i, (op, a) in enumerate(steps):
        a = np.array(a, np.int32)
        e.buf("a%d" % i, a)
        e.do(op, "a%d" % i, "pool")
        if op == "reserve":
            short, out, moves = kp.reserve(table, lengths, refs, a, page)
            heads_of[:2] = short, out
            for x, y in moves:
                pages[:, y] = pages[:, x]
        elif op == "fork":
            heads_of[2] += kp.fork(table, lengths, refs, a, page)
        else:
            kp.free(table, lengths, refs, a, page)
        for n in ("table", "lengths", "pool"):
            e.lines.append("dump %s %s.%d" % (n, os.path.join(e.path, n), i))
        dumps.append((table.copy(), lengths.copy(), refs.copy(), list(heads_of)))
    e.do("compact", "pool")
    got_pages, got_table, got_lengths, got_pool = e.run("pages", "table", "lengths", "pool")
    live, moves = kp.compact(table, lengths, refs, page)
    assert moves                                      # (the steps leave holes)
    for x, y in moves:
        pages[:, y] = pages[:, x]
    for i, (t, l, r, h) in enumerate(dumps):
        read = lambda n: np.fromfile(os.path.join(e.path, "%s.%d" % (n, i)), np.int32)  # noqa: E731
        assert np.array_equal(read("lengths"), l), (i, steps[i])
        assert np.array_equal(read("table").reshape(t.shape), t), (i, steps[i])
        p = read("pool")
        assert np.array_equal(p[kp.HEADER:kp.HEADER + n_pages], r), (i, steps[i])
        assert p[:3].tolist() == h, (i, steps[i])
        assert not p[kp.HEADER + n_pages:kp.HEADER + 3 * n_pages].any()      # the room that has to be clear between calls
    assert np.array_equal(got_table, table) and np.array_equal(got_lengths, lengths)
    assert np.array_equal(got_pool[kp.HEADER:kp.HEADER + n_pages], refs) and got_pool[3] == live
    assert np.array_equal(got_pages, pages)


def test_books_that_make_no_sense_stay_inside(driver, tmp_path):
    rng = np.random.default_rng(8)
    heads, dim, page, layers, rows, per_row, n_pages = 1, 64, 32, 1, 5, 3, 6
    e = Emu(driver, tmp_path)
    table = rng.integers(-9, n_pages + 9, (rows, per_row)).astype(np.int32)
    pool = np.zeros(kp.HEADER + 6 * n_pages, np.int32)
    pool[kp.HEADER:kp.HEADER + n_pages] = rng.integers(-1, 4, n_pages)
    for n, a in (("pages", np.zeros((layers, n_pages, heads, kp.slab_bytes(dim, page)), np.uint8)), ("table", table),
                 ("lengths", np.array([2 ** 31 - 1, -5, 50, 96, 33], np.int32)), ("pool", pool),
                 ("want", np.array([1, 40, 2 ** 31 - 1, 1, 5], np.int32)), ("want2", np.array([0, 40, 1, 0, 5], np.int32)),
                 ("parent", np.array([9, 4, 2 ** 31 - 1, 1, -4], np.int32)), ("keep", np.array([2 ** 31 - 1, 0, 3, 95, 1], np.int32))):
        e.buf(n, a)
    e.do("cache", "pages", layers, n_pages, heads, dim, page)
    e.do("rows", "table", "lengths", rows, per_row)
    e.do("reserve", "want", "pool")
    e.do("reserve", "want2", "pool")
    e.do("fork", "parent", "pool")
    e.do("compact", "pool")
    e.do("free", "keep", "pool")
    e.do("compact", "pool")
    e.run("pool")


@pytest.mark.parametrize("lengths,counts,dtype", [([5, 0, 33], [6, 3, 2], 1), ([5, 40], [20, 50], 0)])
def test_attention_without_causality_of_more_tokens_than_the_row_has(driver, tmp_path, lengths, counts, dtype):
    """Queries that are none of the row's tokens: each sees the whole row."""
    attend(driver, tmp_path, 64, 32, 1, 1, lengths, counts, dtype, causal=0)
