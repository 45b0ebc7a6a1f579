"""Attention over the 4-bit cache where a few tokens' values are far larger than all others': an answer holds what its query sees and
weighs, to the precision that it has without the others, whatever the mask, the softmax, other rows, heads or queries leave out.  On the
CPU emulation and on the GPU, against 64 bits."""
import glob
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
from test_kv_cache_on_cpu_emulation import Emu, bf16, widen  # noqa: E402

U = 2.0 ** -24
BF16, F32 = 1, 0


@pytest.fixture(scope="module")
def driver():
    emu = build_emu_kv.build_emu
    exe = os.path.join(build_emu_kv.EMU, "_build", "kv", "emu_kv_driver")
    sources = [f for d in (os.path.join(emu.CSRC, "*"), os.path.join(emu.CSRC, "kv", "*"), os.path.join(emu.ROOT, "include", "*"),
                           os.path.join(HERE, "emu", "*.*"), os.path.join(HERE, "emu", "hip", "*"), os.path.join(HERE, "emu", "kv", "*.*"),
                           os.path.join(HERE, "emu", "kv", "hip", "*")) for f in glob.glob(d) if os.path.isfile(f)]
    if os.path.exists(exe) and os.path.getmtime(exe) > max(map(os.path.getmtime, sources)):
        return exe                                                     # (built by another test file)
    try:
        exe = build_emu_kv.build()
    except subprocess.CalledProcessError as e:
        pytest.fail("emulation build failed:\n" + e.stderr.decode()[-3000:])
    if exe is None:
        pytest.skip("no host clang++ to build the emulation with")
    return exe


class World:
    """Rows of the given lengths with keys k and values v [row][length, heads, dim], quantized by the plain form."""

    def __init__(self, dim, page, heads, lengths, seed=0):
        self.dim, self.page, self.heads, self.lengths = dim, page, heads, np.array(lengths, np.int32)
        rng = self.rng = np.random.default_rng([seed, dim, heads, *lengths])
        self.per_row = max(kp.pages_of(n, page) for n in lengths)
        self.n_pages = len(lengths) * self.per_row + 1
        self.table = rng.permutation(self.n_pages)[:len(lengths) * self.per_row].reshape(len(lengths), -1).astype(np.int32)
        self.k = [rng.standard_normal((n, heads, dim)).astype(np.float32) for n in lengths]
        self.v = [rng.standard_normal((n, heads, dim)).astype(np.float32) for n in lengths]
        self.trash = kp.new_pages(1, self.n_pages, heads, dim, page, rng)          # behind the lengths: NaN and Inf grids

    def pages(self):
        p = self.trash.copy()
        begin = np.concatenate([[0], np.cumsum(self.lengths)])
        kp.append(p[0], self.dim, self.page, self.table, self.lengths, begin, np.concatenate(self.k), np.concatenate(self.v))
        return p

    def expected(self, pages, counts, q, window, dtype):
        """(answer, tolerance) [tokens, q_heads, dim].  With p the softmax's weights, s and b = lo + 8 s a value's grid, W = sum p (8 s + |b|):
          weights     a score's roundings make p_t off by r_t of itself: (dim + 16) u B_t for the products and sums of its terms' size B_t,
                      2^-22 (a query split in two) or 2^-24 of B_t, 4 u of each number that goes into the exponent (the score, the largest one,
                      the reference, which is that less log2 of the largest p s); an answer moves by p_t r_t (|v_t| + W) at most, 1.1 for what
                      is of second order
          sums        n + 64 additions: 2 (n + 64) u W for numerator and denominator
          p s         to fp16, 2^-11 of it, or in two halves, 2^-22; at least 2^-25 where the largest p max(s, 2^-20 |b|) is 2^6 or more,
                      or the largest p 2^89
          range       weights below 2^-126, which are 0, are less than 2^-132 of the answer's largest p s and more, in its units; fp32's smallest step
          out         half a step of its type
        """
        dim, heads = self.dim, self.heads
        group = q.shape[1] // heads
        out, tol = np.zeros(q.shape), np.zeros(q.shape)
        split, u_out = (2.0 ** -22, U) if dtype == F32 else (2.0 ** -11, 2.0 ** -8)
        scale = float(np.float32(dim ** -0.5))
        at = 0
        for r, m in enumerate(counts):
            n = int(self.lengths[r])
            t = np.arange(n)
            for h in range(heads):
                (ck, lk, sk), (cv, lv, sv) = kp.get(pages[0], dim, self.page, self.table[r, t // self.page], t % self.page, h)
                K, V, b = lk + ck * sk, lv + cv * sv, np.abs(lv + 8 * sv)[:, 0]
                kb, s8 = np.abs(ck - 8) * sk + np.abs(lk + 8 * sk), 8 * sv[:, 0]
                for i in range(m):
                    pos = n - m + i
                    see = (t <= pos) & ((t > pos - window) if window else True)
                    x = q[at + i, h * group:(h + 1) * group].astype(np.float64)
                    z = scale * (x @ K[see].T)
                    p = np.exp(z - z.max(1, keepdims=True))
                    p /= p.sum(1, keepdims=True)
                    o = p @ V[see]
                    B = scale * (np.abs(x) @ kb[see].T)
                    W = p @ (s8 + b)[see]
                    most = (p * np.maximum(s8 / 8, 2.0 ** -20 * b)[see]).max(1)
                    L = np.abs(np.log2(np.maximum(most, 2.0 ** -104))) + 8     # (never further, whatever the sizes: p stays below 2^96)
                    rt = (dim + 16) * U * B + (2.0 ** -22 if dtype == F32 else 2.0 ** -24) * B + 4 * U * (1 + np.abs(z) + np.abs(z).max(1, keepdims=True) + L[:, None])
                    off = 1.1 * (p * rt * ((s8 + b)[see][None] + W[:, None])).sum(1) + 2 * (see.sum() + 64) * U * W
                    off += split * (p @ s8[see]) + see.sum() * 8 * np.maximum(2.0 ** -31 * most, 2.0 ** -114)
                    off += see.sum() * 2.0 ** -132 * most * ((s8 + b)[see].max() + W) + 2.0 ** -148
                    out[at + i, h * group:(h + 1) * group] = o
                    tol[at + i, h * group:(h + 1) * group] = off[:, None] + u_out * np.abs(o)
            at += m
        return out, tol


def on_emulation(driver, path):
    def attend(w, pages, counts, q, window, dtype):
        os.makedirs(str(path), exist_ok=True)
        e = Emu(driver, path)
        data = q if dtype == F32 else bf16(q)
        begin = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        for name, a in (("pages", pages), ("table", w.table), ("lengths", w.lengths), ("begin", begin), ("q", data), ("o", np.zeros_like(data))):
            e.buf(name, a)
        e.do("cache", "pages", 1, w.n_pages, w.heads, w.dim, w.page)
        e.do("rows", "table", "lengths", len(w.lengths), w.per_row)
        e.do("attention", 0, "begin", q.shape[0], "q", "o", dtype, q.shape[1] * w.dim, w.dim, q.shape[1], repr(float(np.float32(w.dim ** -0.5))), 1, window)
        (o,) = e.run("o")
        return (o if dtype == F32 else widen(o)).astype(np.float64)
    return attend


def on_gpu():
    torch = pytest.importorskip("torch")
    import paper_2211_04515_amd as qp

    def attend(w, pages, counts, q, window, dtype):
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        cache, rows = qp.kv_cache(dev(pages), w.heads, w.dim, w.page), qp.kv_rows(dev(w.table), dev(w.lengths))
        x = dev(q).to(torch.float32 if dtype == F32 else torch.bfloat16)
        out = torch.empty_like(x)
        begin = dev(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32))
        qp.qp_kv_attention(cache, rows, 0, begin, x, out, qp.alloc_kv_workspace(cache, rows, q.shape[0], q.shape[1]), scale=float(np.float32(w.dim ** -0.5)), window=window)
        return out.double().cpu().numpy()
    return attend


def check(attend, w, counts, q, window, dtype):
    pages = w.pages()
    if dtype == BF16:
        q = widen(bf16(q))                                             # (what the kernel is given)
    o = attend(w, pages, counts, q, window, dtype)
    want, tol = w.expected(pages, counts, q, window, dtype)
    bad = ~(np.abs(o - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), o[bad][:4], want[bad][:4], tol[bad][:4])
    return o


def queries(w, counts, group):
    return w.rng.standard_normal((sum(counts), w.heads * group, w.dim)).astype(np.float32)


def vast_last_token(attend, lengths, counts, group, factor, dtype):
    """Of each row, the last token's value: only the last query sees it."""
    w = World(64, 32, 1, lengths)
    q = queries(w, counts, group)
    plain = check(attend, w, counts, q, 0, dtype)
    for v in w.v:
        v[-1] *= np.float32(factor)
    o = check(attend, w, counts, q, 0, dtype)
    ahead = np.ones(len(q), bool)
    ahead[np.cumsum(counts) - 1] = False
    assert np.array_equal(o[ahead], plain[ahead])                      # nothing of it in the others


def vast_tokens_behind_a_window(attend, lengths, counts, window, factor, dtype):
    """Every token that no query's window reaches, and one that only the first ones' do."""
    w = World(64, 32, 1, lengths)
    q = queries(w, counts, 1)
    plain = check(attend, w, counts, q, window, dtype)
    for v, k, n, m in zip(w.v, w.k, lengths, counts):
        v[:max(0, n - m - window + 1)] *= np.float32(factor)
        k[:max(0, n - m - window + 1)] *= 7
    o = check(attend, w, counts, q, window, dtype)
    assert np.array_equal(o, plain)
    for v, n, m in zip(w.v, lengths, counts):
        v[max(0, n - m - window + 1 + m // 2)] *= np.float32(factor)
    check(attend, w, counts, q, window, dtype)


def vast_values_of_others(attend, counts, factor, dtype):
    """Another head's values, another row's, another query's elements: nothing of them shows."""
    w = World(64, 32, 2, [70, 45])
    q = queries(w, counts, 2)
    plain = check(attend, w, counts, q, 0, dtype)
    w.v[0][::3, 1] *= np.float32(factor)
    w.v[1][20, 0] *= np.float32(factor)
    w.k[0][5:9, 1] *= 20
    q[1::2, 0] = q[1::2, 0] * 50
    o = check(attend, w, counts, q, 0, dtype)
    assert np.array_equal(o[:counts[0]:2, :2], plain[:counts[0]:2, :2])
    assert np.array_equal(o[counts[0]:, 2:], plain[counts[0]:, 2:])


def vast_token_without_weight(attend, lengths, counts, group, factor, dtype):
    """A token that every query sees, with a score so low that its share of an answer is nothing: exp(-80) and less of it."""
    w = World(64, 32, 1, lengths)
    way = np.sign(w.rng.standard_normal(64)).astype(np.float32)
    q = queries(w, counts, group) * np.float32(0.25) + 2 * way
    for k, v in zip(w.k, w.v):
        for t in (3, len(k) - max(counts) - 1):
            k[t] = -6 * way
            v[t] *= np.float32(factor)
    check(attend, w, counts, q, 0, dtype)


def values_of_every_size(attend, lengths, counts, dtype, kinds=range(6)):
    """Rows of tiny values, of huge ones, of zeros, of one value for a token's whole head, and of all of them."""
    w = World(64, 32, 1, lengths)
    q = queries(w, counts, 3)
    keep = [v.copy() for v in w.v]
    for kind in kinds:
        for v, x in zip(w.v, keep):
            t = np.arange(len(v))[:, None, None]
            v[:] = (x * np.float32(1e-20), x * np.float32(1e25), x * (t % 3 == 0), x[:, :, :1] * 40 + 0 * x, np.where(t % 5 == 0, 1e4 + x, x * np.float32(1e-4)),
                    x * np.float32(10.0) ** ((t * 7) % 30 - 15))[kind]
        check(attend, w, counts, q, 0, dtype)


TYPES = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])


# ---- on the CPU emulation: both kernels (16 columns or fewer of a row, and more) --------------------------------------------

@TYPES
@pytest.mark.parametrize("lengths,counts,factor", [([40], [2], 1e6), ([40, 47], [3, 5], 1e30), ([40], [40], 1e9), ([70], [60], 1e30)])
def test_vast_last_token_emulated(driver, tmp_path, lengths, counts, factor, dtype):
    vast_last_token(on_emulation(driver, tmp_path), lengths, counts, 1, factor, dtype)


@TYPES
@pytest.mark.parametrize("lengths,counts,window,factor", [([60], [1], 16, 1e9), ([70], [40], 17, 1e30)])
def test_vast_tokens_behind_a_window_emulated(driver, tmp_path, lengths, counts, window, factor, dtype):
    vast_tokens_behind_a_window(on_emulation(driver, tmp_path), lengths, counts, window, factor, dtype)


@TYPES
@pytest.mark.parametrize("counts", [[3, 2], [30, 2]])
def test_vast_values_of_others_emulated(driver, tmp_path, counts, dtype):
    vast_values_of_others(on_emulation(driver, tmp_path), counts, 1e9, dtype)


@TYPES
@pytest.mark.parametrize("lengths,counts", [([50], [2]), ([60], [20])])
def test_vast_token_without_weight_emulated(driver, tmp_path, lengths, counts, dtype):
    vast_token_without_weight(on_emulation(driver, tmp_path), lengths, counts, 1, 1e9, dtype)


@TYPES
@pytest.mark.parametrize("lengths,counts", [([70], [2]), ([40], [17])])
def test_values_of_every_size_emulated(driver, tmp_path, lengths, counts, dtype):
    values_of_every_size(on_emulation(driver, tmp_path), lengths, counts, dtype, (0, 3, 5))


# ---- on the GPU --------------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@TYPES
@pytest.mark.parametrize("factor", [1e6, 1e9, 1e30])
@pytest.mark.parametrize("lengths,counts,group", [([40], [2], 1), ([700, 1, 97], [3, 1, 5], 1), ([150], [140], 1), ([900, 130], [150, 33], 4), ([3000], [4], 2)])
def test_vast_last_token(lengths, counts, group, factor, dtype):
    vast_last_token(on_gpu(), lengths, counts, group, factor, dtype)


@pytest.mark.gpu
@TYPES
@pytest.mark.parametrize("factor", [1e6, 1e30])
@pytest.mark.parametrize("lengths,counts,window", [([60], [1], 16), ([800, 333], [3, 1], 100), ([600], [400], 70)])
def test_vast_tokens_behind_a_window(lengths, counts, window, factor, dtype):
    vast_tokens_behind_a_window(on_gpu(), lengths, counts, window, factor, dtype)


@pytest.mark.gpu
@TYPES
@pytest.mark.parametrize("counts", [[3, 2], [30, 2], [1, 45]])
def test_vast_values_of_others(counts, dtype):
    vast_values_of_others(on_gpu(), counts, 1e9, dtype)


@pytest.mark.gpu
@TYPES
@pytest.mark.parametrize("lengths,counts,group", [([50], [2], 1), ([1000, 300], [1, 4], 2), ([400], [150], 2)])
def test_vast_token_without_weight(lengths, counts, group, dtype):
    vast_token_without_weight(on_gpu(), lengths, counts, group, 1e9, dtype)


@pytest.mark.gpu
@TYPES
@pytest.mark.parametrize("lengths,counts", [([70, 1000], [2, 1]), ([500], [100]), ([4000], [3])])
def test_values_of_every_size(lengths, counts, dtype):
    values_of_every_size(on_gpu(), lengths, counts, dtype)
