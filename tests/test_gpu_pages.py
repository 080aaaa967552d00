"""The paged cache's kernels against plain 64-bit implementations of their definitions.

Tolerances.  A result of type t is off by half a step, eps(t)/2 of its value (twice that absolutely in fp16's subnormal
range: 2^-24).  A rotary cosine or sine is an fp32 function of an angle reduced in 64 bits: 2^-21 covers its rounding,
the argument's (pi 2^-24) and that of the products.  An attention row o = sum_j p_j v_j of scores x_j off by d has
p_j (1 + 2 d): with products of hd terms in fp32, d = (hd + 8) 2^-24 max_j sum |q k_j| scale + 2^-20; its probabilities are
rounded to the pages' type where that is shorter (half a step), and its sums over n positions add n 2^-24, all
relative to sum_j p_j |v_j|.
"""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2604_18396_amd import binding as B, configs, inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": (torch.float32, torch.float32), "bf16": (torch.bfloat16, torch.bfloat16), "bf16-f16": (torch.bfloat16, torch.float16)}


def half_step(t):
    return torch.finfo(t).eps / 2


class Setup:
    """A cache of random contents, tables in random order, and the batch: lens[s] positions, new[s] of them new."""

    def __init__(self, kind, nkv, hd, ps, lens, new, seed=0, spare=2, layers=1, pad=0, extra_cols=1, ragged=True, pages_first=False, room=0):
        # room: pages that the table has place for beyond what is used, and the bound on lengths allows: the kernel and the
        # splits of the keys go by that bound
        self.act, self.kvt = TYPES[kind]
        self.nkv, self.hd, self.ps, self.lens, self.new = nkv, hd, ps, lens, new
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.g = g
        rng = np.random.default_rng(seed)
        need = [-(-max(n, 0) // ps) for n in lens]
        most = max(max(need), 1) + extra_cols + room
        n_pages = sum(need) + spare
        self.host = np.full((len(lens), most), -1, dtype=np.int32)
        order, at = rng.permutation(n_pages), 0
        for i, n in enumerate(need):
            self.host[i, :n] = order[at:at + n]
            at += n
        self.spare = order[at:]
        shape = (n_pages, layers, 2, nkv, ps, hd) if pages_first else (layers, 2, n_pages, nkv, ps, hd)
        both = self.randn(*shape, dtype=self.kvt)
        if pages_first:     # a page's layers, and its keys and values, next to each other
            self.k, self.v = both[:, :, 0].transpose(0, 1), both[:, :, 1].transpose(0, 1)
        else:
            self.k, self.v = both[:, 0], both[:, 1]
        self.table = torch.from_numpy(self.host).to(DEV)
        self.start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.tokens = int(self.start[-1]) + pad
        self.q_start = torch.from_numpy(self.start).to(DEV)
        self.dlens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        self.pages = B.Pages(self.k, self.v, self.act)
        self.batch = B.Batch(self.table, self.dlens, self.q_start if ragged else None, max_new=max(max(new), 1),
                             max_len=None if room else max(max(lens), 1))

    def randn(self, *shape, dtype=None, std=1.0):
        return torch.randn(*shape, generator=self.g, device=DEV).mul_(std).to(dtype or self.act)

    def positions(self):
        """(sequence, token, position) of every new token."""
        return [(s, int(self.start[s]) + i, self.lens[s] - m + i) for s, m in enumerate(self.new) for i in range(m)]

    def rows(self, s, layer=0):
        """Keys and values of a sequence's positions [n, nkv, hd] in 64 bits, and which positions have a page."""
        n = max(self.lens[s], 0)
        p = np.arange(n)
        entry = np.where(p // self.ps < self.host.shape[1], self.host[s][np.minimum(p // self.ps, self.host.shape[1] - 1)], -1)
        there = (entry >= 0) & (entry < self.k.shape[1])
        page = torch.from_numpy(np.where(there, entry, 0)).to(DEV).long()
        slot = torch.from_numpy(p % self.ps).to(DEV).long()
        return self.k[layer][page, :, slot].double(), self.v[layer][page, :, slot].double(), torch.from_numpy(there).to(DEV)


def attention(st, q, window=0, sinks=0, scale=None, layer=0):
    """(rows, tolerance of each element) in 64 bits; rows of tokens without a position are zero."""
    nq, hd = q.shape[1:]
    scale = scale or hd ** -0.5
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    tol = torch.zeros_like(out)
    rounded = half_step(st.kvt) if st.kvt != torch.float32 else 2.0 ** -22
    for s, m in enumerate(st.new):
        n, lo = st.lens[s], int(st.start[s])
        if m == 0 or n < 1:
            continue
        k, v, there = st.rows(s, layer)
        p = torch.arange(n - m, n, device=DEV)
        j = torch.arange(n, device=DEV)
        sees = (j <= p[:, None]) & there
        if window:
            sees &= (j > p[:, None] - window) | (j < sinks)
        for h in range(nq):
            kh, vh = k[:, h * st.nkv // nq], v[:, h * st.nkv // nq]
            kh = torch.where(there[:, None], kh, 0.0)
            qh = q[lo:lo + m, h].double()
            x = (torch.where(sees.any(0)[:, None], kh, 0.0) @ qh.t()).t() * scale
            x = torch.where(sees, x, -math.inf)
            top = x.amax(1, keepdim=True)
            w = torch.where(sees, (x - torch.where(top == -math.inf, 0.0, top)).exp(), 0.0)
            total = w.sum(1, keepdim=True)
            w = torch.where(total > 0, w / total, 0.0)
            vh = torch.where(sees.any(0)[:, None], vh, 0.0)
            o, a = w @ vh, w @ vh.abs()
            most = torch.where(sees, (qh.abs() @ torch.where(sees.any(0)[:, None], kh, 0.0).abs().t()) * scale, 0.0).amax(1, keepdim=True)
            d = (hd + 8) * 2.0 ** -24 * most + 2.0 ** -20
            out[lo:lo + m, h] = o
            tol[lo:lo + m, h] = half_step(q.dtype) * o.abs() + a * (rounded + 2 * d + n * 2.0 ** -24)
    return out, tol


def check(got, want, tol, what=""):
    bad = ~((got.double() - want).abs() <= tol * 1.01 + 1e-30)
    if bool(bad.any()):
        i = int(bad.flatten().nonzero()[0])
        assert False, (what, int(bad.sum()), "of", bad.numel(), "first", i, float(got.flatten()[i]), float(want.flatten()[i]), float(tol.flatten()[i]))


# ------------------------------------------------------------------ rotary positions and the store

def freqs(rot, scaling="plain"):
    f, m = B.river_rope_frequencies(rot, 500000.0, scaling, 8.0, 8192.0, 1.0, 32.0)
    return torch.from_numpy(f).to(DEV), m


def turned(x, pos, f, m, layout):
    """[n, heads, hd] at positions pos as complex numbers in 64 bits, and the tolerance without the last rounding."""
    r = 2 * f.numel()
    a = torch.tensor(pos, dtype=torch.float64, device=DEV)[:, None, None] * f
    x = x.double()
    i = torch.arange(r // 2, device=DEV)
    first, second = (i, i + r // 2) if layout == "half" else (2 * i, 2 * i + 1)
    z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.full_like(a, m), a)
    y, tol = x.clone(), torch.zeros_like(x)
    y[..., first], y[..., second] = z.real, z.imag
    tol[..., first] = tol[..., second] = (x[..., first].abs() + x[..., second].abs()) * m * 2.0 ** -21
    return y, tol


def run_store(st, nq, rot, layout, scaling="plain", layer=0, stride_pad=0, in_place=False):
    nkv, hd, T = st.nkv, st.hd, st.tokens
    row = st.randn(T, (nq + 2 * nkv) * hd + stride_pad, std=1.5)
    if stride_pad % 2:
        row = row[:, 1:]                       # rows that begin in the middle of a word
    heads = row[:, :(nq + 2 * nkv) * hd].unflatten(1, (-1, hd))
    q, k, v = heads[:, :nq], heads[:, nq:nq + nkv], heads[:, nq + nkv:]
    f, m = freqs(rot, scaling)
    before_k, before_v = st.k.clone(), st.v.clone()
    q0 = q.clone()
    out = q if in_place else torch.full((T, nq, hd), 7.0, dtype=st.act, device=DEV)
    back = B.river_rope_store(st.pages, layer, st.batch, q, k, v, B.Rope(f, layout, m), out=out)
    torch.cuda.synchronize()
    assert back is out
    todo = [(s, t, p) for s, t, p in st.positions() if p >= 0]
    tok = [t for _, t, _ in todo]
    if todo:
        want, tol = turned(q0[tok], [p for _, _, p in todo], f, m, layout)
        check(out[tok], want, tol + half_step(st.act) * want.abs(), "queries")
    rest = [t for t in range(T) if t not in set(tok)]
    assert torch.equal(out[rest], q0[rest] if in_place else torch.full_like(out[rest], 7.0))
    written = [(s, t, p) for s, t, p in todo if p // st.ps < st.host.shape[1] and 0 <= st.host[s, p // st.ps] < st.k.shape[1]]
    if written:
        tok = [t for _, t, _ in written]
        page = [int(st.host[s, p // st.ps]) for s, _, p in written]
        slot = [p % st.ps for _, _, p in written]
        want, tol = turned(k[tok], [p for _, _, p in written], f, m, layout)
        check(st.k[layer][page, :, slot], want, tol + half_step(st.kvt) * want.abs() + 2.0 ** -24 * (st.kvt == torch.float16), "keys")
        assert torch.equal(st.v[layer][page, :, slot], v[tok].to(st.kvt))
        before_k[layer][page, :, slot], before_v[layer][page, :, slot] = st.k[layer][page, :, slot], st.v[layer][page, :, slot]
    assert torch.equal(st.k, before_k) and torch.equal(st.v, before_v)          # nothing else was written


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("hd,rot", [(64, 64), (64, 20), (64, 2), (128, 128), (128, 64), (128, 126), (128, 32)])
def test_rope_store(kind, layout, hd, rot):
    # lengths of one, pages that end in the middle of the new tokens, a sequence without new tokens, padding behind the last
    st = Setup(kind, 2, hd, 16, [1, 45, 0, 200, 16], [1, 40, 0, 7, 16], seed=rot, pad=3)
    run_store(st, 6, rot, layout)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("pad", [0, 8, 1, 5])
def test_rope_store_strides(kind, pad):
    st = Setup(kind, 3, 128, 20, [33, 7], [33, 2], seed=pad, layers=3, pages_first=True)
    run_store(st, 3, 96, "half", "ramp", layer=1, stride_pad=pad)
    run_store(st, 12, 128, "interleaved", "bands", layer=2, stride_pad=pad, in_place=True)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_store_far_positions_one_token_each(layout):
    # 40 sequences, angles of up to 2^30 turns: the fraction is in bits that fp32 has not
    lens = [1 + 31 * i for i in range(38)] + [100000, 300001]
    st = Setup("bf16", 1, 64, 256, lens, [1] * 40, ragged=False, seed=3)
    run_store(st, 4, 64, layout, "linear")
    run_store(Setup("f32", 1, 64, 256, lens, [1] * 40, ragged=False, seed=4), 4, 64, layout)


def test_rope_store_where_there_is_no_page_or_position():
    st = Setup("bf16", 2, 64, 8, [30, 30, 3], [20, 30, 5], seed=9)      # the third has more new tokens than positions
    st.host[0, 2], st.host[1, 0], st.host[1, 3] = -1, 10 ** 6, -2 ** 31
    st.table.copy_(torch.from_numpy(st.host))
    run_store(st, 4, 64, "half")
    st = Setup("bf16", 2, 64, 8, [30, 11], [25, 4], seed=10, extra_cols=0)
    short = B.Batch(st.table[:, :2], st.dlens, st.q_start, max_new=25, max_len=30)       # positions from 16 on have no page
    st.batch, st.host = short, st.host[:, :2]
    run_store(st, 4, 64, "half")


# ------------------------------------------------------------------ attention

def run_attention(st, nq, window=0, sinks=0, scale=0.0, std=1.5, layer=0):
    q = st.randn(st.tokens, nq, st.hd, std=std)
    out = torch.full_like(q, 7.0)
    B.river_paged_attention(st.pages, layer, st.batch, q, window, sinks, scale, out=out)
    torch.cuda.synchronize()
    want, tol = attention(st, q, window, sinks, scale or None, layer)
    n = int(st.start[-1])
    check(out[:n], want[:n], tol[:n])
    assert bool((out[n:] == 7.0).all())                  # the rows of a padded batch's last tokens
    assert float((out[:n].double() - want[:n]).norm()) <= 2.0 ** -8 * float(want[:n].norm()) + 1e-30
    return q, out


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("nkv,rep", [(1, 1), (2, 4), (3, 7), (1, 24)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 3)])
def test_attention_single_tokens(kind, hd, nkv, rep, window, sinks):
    lens = [1, 2, 15, 16, 17, 0, 63, 64, 65, 300, 1000, 33]
    run_attention(Setup(kind, nkv, hd, 16, lens, [1] * len(lens), ragged=False, seed=rep), nkv * rep, window, sinks)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("ps", [1, 7, 20, 64, 1000])
def test_attention_page_sizes(kind, ps):
    run_attention(Setup(kind, 2, 64, ps, [517, 64, 130], [1, 1, 1], seed=ps), 8, 77, 5)
    run_attention(Setup(kind, 2, 128, ps, [517, 64, 130], [40, 64, 1], seed=ps), 4)
    run_attention(Setup(kind, 2, 128, ps, [517, 64, 130], [140, 64, 1], seed=ps, room=320000 // ps), 4)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("hd,nkv,rep", [(64, 2, 4), (128, 1, 8), (128, 2, 1), (64, 1, 3)])
@pytest.mark.parametrize("lens,new", [([5, 9, 2], [2, 3, 2]), ([40, 70], [16, 9]), ([300, 77, 1], [300, 77, 1]), ([700, 513, 64, 0], [129, 1, 64, 0]),
                                      ([1500], [257])], ids=str)
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (64, 0), (90, 4), (200, 130)])
@pytest.mark.parametrize("room", [0, 300, 20000])
def test_attention_prompts(kind, hd, nkv, rep, lens, new, window, sinks, room):
    run_attention(Setup(kind, nkv, hd, 16, lens, new, seed=window, pad=2, room=room), nkv * rep, window, sinks)


@pytest.mark.parametrize("kind", ["bf16", "bf16-f16"])
@pytest.mark.parametrize("hd,nkv,rep,lens,new", [(128, 8, 4, [1100, 513, 64, 0], [1100, 129, 64, 0]), (64, 8, 8, [2050, 1], [515, 1]),
                                                 (128, 4, 1, [3000], [1025]), (128, 2, 7, [9000, 300], [70, 33]), (64, 1, 16, [20000], [40])],
                         ids=str)
@pytest.mark.parametrize("window,sinks", [(0, 0), (500, 4)])
def test_attention_large_prompts(kind, hd, nkv, rep, lens, new, window, sinks):
    run_attention(Setup(kind, nkv, hd, 16, lens, new, seed=31, pad=1), nkv * rep, window, sinks)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n_seq,nkv", [(2, 8), (3, 3), (4, 8), (5, 1), (8, 2), (33, 1), (33, 8)])
@pytest.mark.parametrize("shape", ["single tokens", "prompts", "split prompts"])
def test_attention_of_many_ragged_sequences(kind, n_seq, nkv, shape):
    # every sequence's tiles and splits are worked on once, whatever the order in which they are handed out
    rng = np.random.default_rng(n_seq * 10 + nkv)
    lens = [int(n) for n in rng.integers(1, 900, n_seq)]
    lens[0], lens[n_seq // 2] = 1000, 0
    new = [min(n, 1) if shape == "single tokens" else int(rng.integers(0, n + 1)) for n in lens]
    new[0] = 1 if shape == "single tokens" else 300
    run_attention(Setup(kind, nkv, 64, 16, lens, new, seed=n_seq, room=20000 // 16 if shape == "split prompts" else 0), nkv * 4)


@pytest.mark.parametrize("kind", TYPES)
def test_attention_long_cache(kind):
    run_attention(Setup(kind, 1, 64, 64, [20011], [1], seed=1, ragged=False), 4)
    run_attention(Setup(kind, 2, 128, 64, [9000, 31, 4097], [1, 1, 1], seed=2, ragged=False), 8, 8000, 70)
    run_attention(Setup(kind, 1, 128, 32, [6000, 2], [5, 2], seed=3), 4)
    run_attention(Setup(kind, 1, 64, 32, [5000], [130], seed=4), 2)
    run_attention(Setup(kind, 2, 128, 32, [5000, 70], [257, 70], seed=4, room=10), 8)


@pytest.mark.parametrize("kind", TYPES)
def test_attention_lengths_beyond_their_bounds(kind):
    # max_len only divides the work; what is longer is still right
    for lens, new, bound in (([900, 40], [1, 1], 50), ([900, 300], [150, 90], 50), ([6000, 300], [600, 90], 2000)):
        st = Setup(kind, 2, 64, 16, lens, new, seed=5)
        st.batch = B.Batch(st.table, st.dlens, st.q_start, max_new=max(new), max_len=bound)
        run_attention(st, 16)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("std,scale", [(8.0, 0.0), (1.0, 3.0), (0.01, 0.05), (200.0, 0.0)])
def test_attention_scales(kind, std, scale):
    run_attention(Setup(kind, 2, 64, 16, [300, 5], [1, 1], seed=6), 8, scale=scale, std=std)
    run_attention(Setup(kind, 1, 128, 16, [300, 200], [200, 150], seed=6), 4, scale=scale, std=std)
    run_attention(Setup(kind, 1, 128, 16, [300, 200], [200, 150], seed=6, room=20000), 4, scale=scale, std=std)


def test_attention_of_queries_that_half_precision_does_not_hold():
    # bf16 queries beyond fp16's largest and below its smallest number over a cache in fp16
    for mult in (2.0 ** 20, 2.0 ** -40):
        for lens, new, room in (([200, 9], [1, 1], 0), ([200, 90], [150, 80], 0), ([200, 90], [150, 80], 20000)):
            st = Setup("bf16-f16", 1, 64, 16, lens, new, seed=7, room=room)
            st.k.mul_(2.0 ** -10)       # fp16's normal numbers, still
            q = (st.randn(st.tokens, 4, 64) * mult)
            got = B.river_paged_attention(st.pages, 0, st.batch, q, scale=2.0 ** 10 / mult / 8)
            want, tol = attention(st, q, scale=2.0 ** 10 / mult / 8)
            check(got, want, tol)


def test_attention_of_many_small_probabilities_in_half_precision():
    # one position 2^17 times as likely as each of 20000 others, which together still count
    st = Setup("bf16-f16", 1, 64, 64, [20000], [1], seed=8)
    st.k.zero_()
    st.k[0, int(st.host[0, 0]), 0, 0, 0] = 17 * math.log(2)
    q = torch.zeros(1, 1, 64, dtype=torch.bfloat16, device=DEV)
    q[..., 0] = 1.0
    got = B.river_paged_attention(st.pages, 0, st.batch, q, scale=1.0)
    want, tol = attention(st, q, scale=1.0)
    st.v.abs_()
    got = B.river_paged_attention(st.pages, 0, st.batch, q, scale=1.0)
    want, tol = attention(st, q, scale=1.0)
    check(got, want, tol)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lens,new", [([1000, 63, 64, 65, 1], [1, 1, 1, 1, 1]), ([333, 200], [4, 3]), ([400, 257, 64], [300, 257, 3])], ids=str)
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 1), (60, 0), (128, 9), (100000, 4)])
@pytest.mark.parametrize("room", [0, 20000])
def test_attention_sees_exactly_what_it_should(kind, hd, lens, new, window, sinks, room):
    # scores of zero: every visible position counts the same.  Position j has a one in element j mod hd: the row holds
    # how many of each residue are seen, divided by their number (exact before the division, which is rounded: fp32's
    # reciprocal and product, then the output's type)
    st = Setup(kind, 2, hd, 20, lens, new, seed=11, room=room)
    for s, n in enumerate(lens):
        for c0 in range(0, n, 20):
            page = int(st.host[s, c0 // 20])
            for slot in range(20):
                st.v[0, page, :, slot] = 0
                st.v[0, page, :, slot, (c0 + slot) % hd] = 1
    nq = 4
    q = torch.zeros(st.tokens, nq, hd, dtype=st.act, device=DEV)
    got = B.river_paged_attention(st.pages, 0, st.batch, q, window, sinks).double()
    for s, t, p in st.positions():
        j = np.arange(p + 1)
        if window:
            j = j[(j > p - window) | (j < sinks)]
        want = torch.from_numpy(np.bincount(j % hd, minlength=hd) / len(j)).to(DEV)
        assert bool(((got[t] - want).abs() <= want * (half_step(st.act) + 2.0 ** -21)).all()), (s, t, p)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("lens,new", [([130, 17, 0, 64], [1, 1, 1, 1]), ([300, 41], [5, 3]), ([300, 130], [290, 130])], ids=str)
@pytest.mark.parametrize("window,sinks", [(0, 0), (37, 2)])
@pytest.mark.parametrize("room", [0, 20000])
def test_attention_does_not_look_at_what_it_does_not_see(kind, bad, lens, new, window, sinks, room):
    st = Setup(kind, 2, 128, 16, lens, new, seed=12, room=room)
    q = st.randn(st.tokens, 8, 128)
    first = B.river_paged_attention(st.pages, 0, st.batch, q, window, sinks)
    # slots behind the sequences' ends, pages of nobody, and positions that every new token's window has left behind
    seen = torch.zeros(st.k.shape[1], 16, dtype=torch.bool, device=DEV)
    for s, n in enumerate(lens):
        for j in range(n):
            if not window or j < sinks or j > n - new[s] - window:
                seen[int(st.host[s, j // 16]), j % 16] = True
    st.k.copy_(torch.where(seen[None, :, None, :, None], st.k, bad))
    st.v.copy_(torch.where(seen[None, :, None, :, None], st.v, bad))
    again = B.river_paged_attention(st.pages, 0, st.batch, q, window, sinks)
    assert torch.equal(first, again)
    for s, n in enumerate(lens):
        if n == 0:
            assert bool((again[int(st.start[s]):int(st.start[s + 1])] == 0).all())


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lens,new", [([200], [6]), ([400], [390])], ids=str)
@pytest.mark.parametrize("room", [0, 20000])
def test_attention_a_later_token_is_no_part_of_an_earlier_row(kind, bad, where, hd, lens, new, room):
    # a value that is not finite in the middle of the new tokens: rows before it, and rows whose window has left it, are as
    # they were; those that see a bad value are bad in its element, those that see a bad key are NaN or without it
    st = Setup(kind, 1, hd, 16, lens, new, seed=13, room=room)
    n, m, window = lens[0], new[0], 100
    at = n - m // 2
    q = st.randn(m, 4, hd)
    page, slot = int(st.host[0, at // 16]), at % 16
    first = B.river_paged_attention(st.pages, 0, st.batch, q, window)
    (st.k if where == "k" else st.v)[0, page, 0, slot, 3] = bad
    again = B.river_paged_attention(st.pages, 0, st.batch, q, window)
    p = torch.arange(n - m, n, device=DEV)
    sees = (p >= at) & (p < at + window)
    assert torch.equal(first[~sees], again[~sees])
    if where == "v":
        hit = again[sees][..., 3].double()
        assert bool(torch.isnan(hit).all() if math.isnan(bad) else (hit == bad).all())
        rest = [e for e in range(hd) if e != 3]
        assert torch.equal(first[sees][..., rest], again[sees][..., rest])
    elif math.isnan(bad):
        assert bool(torch.isnan(again[sees]).all())


@pytest.mark.parametrize("kind", TYPES)
def test_attention_pages_that_are_not_there(kind):
    for lens, new, room in (([300, 100], [1, 1], 0), ([300, 100], [200, 60], 0), ([300, 100], [200, 60], 20000)):
        st = Setup(kind, 2, 64, 16, lens, new, seed=14, room=room)
        st.host[0, 0], st.host[0, 3], st.host[0, 18], st.host[1, :] = -1, 10 ** 6, -2 ** 31, -5
        st.table.copy_(torch.from_numpy(st.host))
        q, out = run_attention(st, 8, 120, 20)
        assert bool((out[int(st.start[1]):] == 0).all())
        cut = B.Batch(st.table[:, :4], st.dlens, st.q_start, max_new=max(new), max_len=300)     # positions from 64 on have no page
        st.host, st.batch = st.host[:, :4].copy(), cut
        run_attention(st, 8)


@pytest.mark.parametrize("kind", TYPES)
def test_attention_more_new_tokens_than_positions(kind):
    # a padded prompt whose length says that it is shorter: tokens without a position get zeros
    for n, m, room in ((3, 5, 0), (40, 100, 0), (40, 100, 20000), (-4, 2, 0)):
        st = Setup(kind, 1, 64, 16, [n, 20], [m, 2], seed=15, room=room)
        q = st.randn(st.tokens, 4, 64)
        got = B.river_paged_attention(st.pages, 0, st.batch, q)
        lost = min(m, m - n)
        assert bool((got[:lost] == 0).all())
        if n > 0:
            st.new = [n, 2]
            st.start = np.array([lost, m, m + 2])
            want, tol = attention(st, q)
            check(got[lost:], want[lost:], tol[lost:])


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("lens,new,bound", [([3000, 2500], [5, 3], 3), ([900, 800], [90, 33], 40), ([3000, 700], [300, 300], 131)], ids=str)
def test_attention_new_tokens_beyond_their_bound_are_left_out(kind, lens, new, bound):
    st = Setup(kind, 2, 64, 16, lens, new, seed=32)
    st.batch = B.Batch(st.table, st.dlens, st.q_start, max_new=bound, max_len=max(lens))
    q = st.randn(st.tokens, 8, 64)
    out = torch.full_like(q, 7.0)
    B.river_paged_attention(st.pages, 0, st.batch, q, out=out)
    want, tol = attention(st, q)
    for s, m in enumerate(new):
        lo, hi, end = int(st.start[s]), int(st.start[s]) + min(m, bound), int(st.start[s + 1])
        check(out[lo:hi], want[lo:hi], tol[lo:hi], s)
        assert bool((out[hi:end] == 7.0).all())


def test_attention_of_a_much_padded_batch():
    # the workspace goes by what the sequences may have, not by the call's tokens
    st = Setup("bf16", 1, 64, 64, [20000, 30], [1, 1], seed=33, pad=200000)
    run_attention(st, 4)
    run_store(st, 4, 64, "half")


def test_calls_without_sequences_or_tokens():
    st = Setup("bf16", 1, 64, 16, [20], [1], seed=34)
    f, _ = freqs(64)
    none = B.Batch(st.table[:0], st.dlens[:0], st.q_start[:1], max_new=1)
    empty = torch.empty(0, 4, 64, dtype=torch.bfloat16, device=DEV)
    for batch, q in ((none, empty), (st.batch, empty), (none, st.randn(3, 4, 64))):
        before = st.k.clone()
        out = torch.full_like(q, 7.0)
        B.river_paged_attention(st.pages, 0, batch, q, out=out)
        B.river_rope_store(st.pages, 0, batch, q, q[:, :1], q[:, 1:2], B.Rope(f), out=out)
        assert bool((out == 7.0).all()) and torch.equal(st.k, before)
    B.river_copy_pages(st.pages, [], [])


@pytest.mark.parametrize("kind", TYPES)
def test_attention_strides_and_layers(kind):
    for lens, new, room in (([100, 45], [1, 1], 0), ([100, 45], [80, 45], 0), ([100, 45], [80, 45], 20000)):
        st = Setup(kind, 2, 64, 16, lens, new, seed=16, layers=3, pages_first=True, room=room)
        wide = st.randn(st.tokens, 8 * 64 * 3)
        q = wide[:, 64 * 8:64 * 16].unflatten(1, (8, 64))
        room = torch.full((st.tokens, 12, 64), 7.0, dtype=st.act, device=DEV)
        out = room[:, 2:10]
        for layer in range(3):
            B.river_paged_attention(st.pages, layer, st.batch, q, out=out)
            want, tol = attention(st, q, layer=layer)
            check(out, want, tol)
            assert bool((room[:, :2] == 7.0).all()) and bool((room[:, 10:] == 7.0).all())


def test_attention_pages_beyond_32_bits():
    # 2^31 elements and 4 GiB into the pages; only the pages that are used are ever touched
    stride = 3 * 2 ** 28
    flat = torch.empty(6 * stride, dtype=torch.bfloat16, device=DEV)
    k = flat.as_strided((1, 6, 1, 16, 64), (6 * stride, stride, 1024, 64, 1))
    v = flat[stride // 2:].as_strided((1, 6, 1, 16, 64), (6 * stride, stride, 1024, 64, 1))
    g = torch.Generator(device=DEV)
    g.manual_seed(17)
    for x in (k, v):
        for p in range(6):
            x[0, p] = torch.randn(1, 16, 64, generator=g, device=DEV).to(torch.bfloat16)
    for m in (1, 70):
        st = Setup("bf16", 1, 64, 16, [75], [m], seed=17)
        st.k, st.v = k, v
        st.host = np.array([[5, 3, 4, 0, 1, -1]], dtype=np.int32)
        st.pages = B.Pages(k, v)
        for room in (0, 400000):        # (both kernels)
            st.table = torch.full((1, 6 + room), -1, dtype=torch.int32, device=DEV)
            st.table[0, :6] = torch.from_numpy(st.host[0])
            st.batch = B.Batch(st.table, st.dlens, st.q_start, max_new=m)
            run_attention(st, 4)
    B.river_copy_pages(st.pages, [5], [2])
    assert torch.equal(k[0, 2], k[0, 5]) and torch.equal(v[0, 2], v[0, 5])


def test_the_same_call_gives_the_same_bits():
    for kind in TYPES:
        for lens, new, room in (([3000, 70], [1, 1], 0), ([700, 300], [300, 300], 0), ([700, 300], [300, 300], 20000), ([4000], [90], 300)):
            st = Setup(kind, 2, 128, 16, lens, new, seed=18, room=room)
            q = st.randn(st.tokens, 8, 128)
            first = B.river_paged_attention(st.pages, 0, st.batch, q)
            for _ in range(5):
                assert torch.equal(first, B.river_paged_attention(st.pages, 0, st.batch, q))


@pytest.mark.parametrize("kind", ["bf16", "bf16-f16"])
@pytest.mark.parametrize("hd", [64, 128])
def test_a_full_card_gives_the_same_bits(kind, hd):
    # workgroups side by side on every CU, out of step with each other
    st = Setup(kind, 8, hd, 16, [2000, 1100, 513, 40], [2000, 900, 513, 3], seed=37)
    q = st.randn(st.tokens, 32, hd)
    for window, sinks in ((0, 0), (700, 4)):
        first = B.river_paged_attention(st.pages, 0, st.batch, q, window, sinks)
        for _ in range(5):
            assert torch.equal(first, B.river_paged_attention(st.pages, 0, st.batch, q, window, sinks))


# ------------------------------------------------------------------ streams and graphs

def test_on_another_stream():
    st = Setup("bf16", 2, 64, 16, [500, 90], [1, 1], seed=19)
    q = st.randn(2, 8, 64)
    want = B.river_paged_attention(st.pages, 0, st.batch, q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = B.river_paged_attention(st.pages, 0, st.batch, q)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


def test_captured_steps_follow_the_table():
    """A step is captured once; lengths, table and inputs change between replays, with eager work between them, and every
    replay equals the eager call.  Two graphs of one batch object, replayed in turn and on two streams."""
    nkv, nq, hd, ps = 2, 8, 64, 16
    lens = [30, 400, 1, 77]
    st = Setup("bf16", nkv, hd, ps, [2000] * 4, [1] * 4, ragged=False, seed=20)
    twin = Setup("bf16", nkv, hd, ps, [2000] * 4, [1] * 4, ragged=False, seed=20)
    f, m = freqs(hd)
    rope = B.Rope(f, "half", m)
    x = torch.zeros(4, (nq + 2 * nkv) * hd, dtype=torch.bfloat16, device=DEV).unflatten(1, (-1, hd))

    def step(s, x, window):
        q = B.river_rope_store(s.pages, 0, s.batch, x[:, :nq], x[:, nq:nq + nkv], x[:, nq + nkv:], rope)
        return B.river_paged_attention(s.pages, 0, s.batch, q, window, 2)

    st.dlens.copy_(torch.tensor(lens))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    with torch.cuda.stream(side):
        for window in (0, 100):
            step(st, x, window)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for window in (0, 100):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(st, x, window))
        graphs.append(g)
    st.k.copy_(twin.k)
    st.v.copy_(twin.v)
    for i in range(4):
        lens = [n + 1 + 31 * i for n in lens]
        order = torch.randperm(4, device=DEV)
        table = st.table[order].clone()
        for s in (st, twin):
            s.dlens.copy_(torch.tensor(lens))
            s.table.copy_(table)
        x.copy_(st.randn(4, nq + 2 * nkv, hd))
        want = [step(twin, x, w) for w in (0, 100)]
        torch.cuda.synchronize()
        if i % 2:
            for g in graphs:
                g.replay()
        else:                           # (both write the same keys and values)
            streams = [torch.cuda.Stream(), torch.cuda.Stream()]
            for s, g in zip(streams, graphs):
                with torch.cuda.stream(s):
                    g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)
        assert torch.equal(st.k, twin.k) and torch.equal(st.v, twin.v)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("lens,splits", [([1000, 3, 0, 640, 129], "few"), ([20000], "many")], ids=str)
def test_splits_are_joined_alike_with_tickets_and_without(kind, lens, splits):
    for hd in (64, 128):
        st = Setup(kind, 2, hd, 16, lens, [1] * len(lens), seed=29, ragged=False)
        q = st.randn(len(lens), 8, hd)
        ref, n = st.batch.bind(len(lens), st.pages), C.c_size_t()
        assert B.load().river_paged_attention_workspace(st.pages.ref, ref, 8, 0, 0, C.byref(n)) == 0 and n.value > 0
        ws = torch.full((n.value,), 255, dtype=torch.uint8, device=DEV)
        tickets = torch.zeros(B.TICKETS, dtype=torch.int32, device=DEV)
        outs = []
        for t in (None, tickets, tickets, None):
            out = torch.full_like(q, 7.0)
            assert B.load().river_paged_attention(st.pages.ref, 0, ref, 8, q.data_ptr(), 8 * hd, 0.0, 0, 0, out.data_ptr(), 8 * hd, ws.data_ptr(),
                                                  n.value, None if t is None else t.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
            torch.cuda.synchronize()
            outs.append(out)
            assert int(tickets.abs().sum()) == 0             # left as they were
        assert all(torch.equal(outs[0], o) for o in outs)
        want, tol = attention(st, q)
        check(outs[0], want, tol)


def test_two_streams_at_once():
    """Calls of one batch object on two streams, in flight together."""
    st = Setup("bf16", 2, 128, 16, [3000, 1500, 700], [1, 1, 1], seed=30, ragged=False)
    q = st.randn(3, 8, 128)
    want = B.river_paged_attention(st.pages, 0, st.batch, q)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for _ in range(30):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(B.river_paged_attention(st.pages, 0, st.batch, q))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_captured_copies():
    st = Setup("bf16", 2, 64, 16, [160], [1], seed=21, layers=3)
    src, dst = st.host[0, :4].tolist(), [int(st.host[0, 7]), int(st.host[0, 8]), int(st.host[0, 9]), int(st.spare[0])]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.river_copy_pages(st.pages, src, dst)
    for _ in range(3):
        st.k.copy_(torch.randn_like(st.k))
        want = st.k.clone()
        want[:, dst] = want[:, src]
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(st.k, want)


# ------------------------------------------------------------------ copies and the pool

@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("hd,ps,nkv,layers", [(64, 1, 1, 1), (64, 7, 3, 2), (128, 64, 8, 2)])
def test_copy_pages(kind, hd, ps, nkv, layers):
    st = Setup(kind, nkv, hd, ps, [ps * 30], [1], seed=22, layers=layers, pages_first=layers == 2)
    n = st.k.shape[1]
    rng = np.random.default_rng(ps)
    for count in (1, 5, 40, 500):           # (pages again as sources and destinations: one after the other)
        src, dst = rng.integers(0, n, count), rng.integers(0, n, count)
        want_k, want_v = st.k.clone(), st.v.clone()
        for a, b in zip(src, dst):
            want_k[:, b], want_v[:, b] = want_k[:, a].clone(), want_v[:, a].clone()
        B.river_copy_pages(st.pages, src, dst)
        assert torch.equal(st.k, want_k) and torch.equal(st.v, want_v)


def test_copy_more_pages_than_a_launch_holds():
    st = Setup("bf16", 1, 64, 4, [4 * 1200], [1], seed=23)
    order = np.random.default_rng(1).permutation(1200)
    want = st.k.clone()
    want[:, order[600:].tolist()] = want[:, order[:600].tolist()]
    B.river_copy_pages(st.pages, order[:600], order[600:])
    assert torch.equal(st.k, want)


def test_pool_keeps_the_device_current():
    pool = B.PagePool(700, 4, 6, 300)
    k = torch.zeros(2, 700, 1, 4, 64, dtype=torch.bfloat16, device=DEV)
    k += torch.arange(700, device=DEV).view(1, 700, 1, 1, 1).to(torch.bfloat16)
    pages = B.Pages(k, k.clone())

    def same():
        pool.flush(pages)
        torch.cuda.synchronize()
        assert pool.lens.tolist() == [pool.length(s) for s in range(6)]
        assert np.array_equal(pool.table.cpu().numpy(), np.stack([pool.row(s) for s in range(6)]))

    same()
    pool.extend(0, 1190)
    pool.extend(1, 3)
    same()
    pool.fork(0, 2)
    pool.extend(2, 1)                  # its half-full last page: a copy
    pool.extend(0, 5)
    before = k.clone()
    same()
    a, b = int(pool.row(0)[297]), int(pool.row(2)[297])
    assert a != b and torch.equal(k[:, b], before[:, a])
    pool.free(0)
    pool.trim(2, 50, 9)
    same()
    want = k[:, [int(p) for p in pool.row(2) if p >= 0]].clone()
    assert pool.compact() > 0
    pool.fork(2, 3)
    same()
    assert torch.equal(k[:, [int(p) for p in pool.row(2) if p >= 0]], want)
    with pytest.raises(B.RiverError) as e:
        pool.extend(4, 4 * 301)
    assert e.value.code == B.RIVER_ENOSPC
    pool.close()


def test_copies_that_are_queued_behind_each_other():
    # page 1 is copied for a fork, freed and taken again as the copy of another: the second copy waits for the first
    pool = B.PagePool(5, 4, 4, 2)
    k = torch.arange(5, device=DEV).view(1, 5, 1, 1, 1).expand(1, 5, 1, 4, 64).to(torch.bfloat16).contiguous()
    pages = B.Pages(k, k.clone())
    pool.extend(0, 2)                   # page 0
    pool.extend(1, 2)                   # page 1
    pool.fork(1, 2)
    pool.extend(2, 1)                   # a copy of 1 in 2
    pool.free(1)                        # 1 is free
    pool.fork(0, 1)
    pool.extend(1, 1)                   # a copy of 0 in 1
    pool.flush(pages)
    torch.cuda.synchronize()
    assert [int(pool.row(s)[0]) for s in range(3)] == [0, 1, 2]
    assert k[0, :, 0, 0, 0].tolist()[:3] == [0.0, 0.0, 1.0]


# ------------------------------------------------------------------ all of them, as a program uses them

@pytest.mark.parametrize("kind", TYPES)
def test_a_serving_loop(kind):
    """A prompt, forks that go on in different ways, a window with its pages given back, a compaction: every step's rows
    against attention over the whole history of its sequence."""
    act, kvt = TYPES[kind]
    nkv, nq, hd, ps, L, window, sinks = 2, 8, 64, 8, 2, 30, 3
    g = torch.Generator(device=DEV)
    g.manual_seed(24)
    pool = B.PagePool(60, ps, 4, 20)
    k, v = (torch.full((L, 60, nkv, ps, hd), math.nan, dtype=kvt, device=DEV) for _ in range(2))
    pages = B.Pages(k, v, act)
    f, m = freqs(hd, "ramp")
    rope = B.Rope(f, "half", m)
    history = [[] for _ in range(4)]        # rows (k, v) of all positions and layers, [L][2][n][nkv][hd] in 64 bits

    def step(new):
        for s, n in enumerate(new):
            if n:
                pool.extend(s, n)
        pool.flush(pages)
        start = torch.tensor(np.concatenate([[0], np.cumsum(new)]).astype(np.int32), device=DEV)
        batch = B.Batch(pool.table, pool.lens, start, max_new=max(new))
        T = sum(new)
        for l in range(L):
            x = torch.randn(T, nq + 2 * nkv, hd, generator=g, device=DEV).to(act)
            q = B.river_rope_store(pages, l, batch, x[:, :nq], x[:, nq:nq + nkv], x[:, nq + nkv:], rope)
            out = B.river_paged_attention(pages, l, batch, q, window, sinks)
            t = 0
            for s, n in enumerate(new):
                if not n:
                    continue
                have = len(history[s]) if l == 0 else len(history[s]) - n
                if l == 0:
                    history[s] += [[None] * L for _ in range(n)]
                pos = list(range(have, have + n))
                kk, _ = turned(x[t:t + n, nq:nq + nkv], pos, f, m, "half")
                for i in range(n):
                    history[s][have + i][l] = (kk[i].to(kvt).double(), x[t + i, nq + nkv:].to(kvt).double())
                K = torch.stack([h[l][0] for h in history[s]])
                V = torch.stack([h[l][1] for h in history[s]])
                j, p = torch.arange(have + n, device=DEV), torch.tensor(pos, device=DEV)[:, None]
                sees = (j <= p) & ((j > p - window) | (j < sinks))
                for h in range(nq):
                    w = torch.where(sees, q[t:t + n, h].double() @ K[:, h // 4].t() / 8, -math.inf).softmax(-1)
                    o, a = w @ V[:, h // 4], w @ V[:, h // 4].abs()
                    # keys of the cache and of this oracle may round to neighbours (a step of the pages' type): scores
                    # off by step |q| |k| / 8 besides what the module's tolerances say
                    most = (q[t:t + n, h].double().abs() @ K[:, h // 4].abs().t()).amax(1, keepdim=True) / 8
                    d = most * (2 * half_step(kvt) + (hd + 8) * 2.0 ** -24) + 2.0 ** -20
                    check(out[t:t + n, h], o, half_step(act) * o.abs() + a * (half_step(kvt) + 2 * d + 200 * 2.0 ** -24), (s, l, h))
                t += n

    step([50, 9, 0, 0])
    step([1, 1, 0, 0])
    pool.fork(0, 2)
    history[2] = [list(h) for h in history[0]]
    for _ in range(3):
        step([1, 1, 1, 0])
    pool.fork(1, 3)
    history[3] = [list(h) for h in history[1]]
    step([3, 0, 1, 12])
    for s in range(4):
        pool.trim(s, window, sinks)
    assert min(pool.row(0)[:7]) == -1
    step([1, 1, 1, 1])
    pool.free(1)
    history[1] = []
    used = 60 - pool.free_pages
    assert pool.compact() > 0 and max(max(pool.row(s)) for s in range(4)) == used - 1
    for i in range(6):
        step([1, 5 if i == 2 else 0, 1, 2])
    pool.close()


SAVE = configs.ModelConfig("save-bf16", 2, 512, 8, 2, 64, 1024, 500, 10000.0, 1e-5, configs.DTYPE_BF16, 96, 1, 2.0)


@pytest.mark.parametrize("cfg,max_batch", [(SAVE, 3), (SAVE.with_(kv_dtype=1), 3), (SAVE.with_(head_dim=128, n_q_heads=4), 1),
                                           (configs.TINY.with_(tau=2.0), 1)], ids=str)
def test_contexts_share_a_prompt_through_pages(cfg, max_batch):
    """A prompt prefilled by one context goes on in another sequence, or another context, to the bit."""
    w = inputs.make_weights(cfg, 5)
    dw = B.upload_weights(w)
    river = B.quantize_river(cfg, dw)
    prompt = inputs.make_prompt(cfg.vocab, 45, 6)
    a = B.River(cfg, dw, river, max_batch=max_batch)
    kvt = torch.float32 if cfg.dtype == 0 else (torch.float16 if cfg.kv_dtype else torch.bfloat16)
    act = torch.float32 if cfg.dtype == 0 else torch.bfloat16
    pages = B.Pages(*(torch.full((cfg.n_layers, 9, cfg.n_kv_heads, 7, cfg.head_dim), math.nan, dtype=kvt, device=DEV) for _ in range(2)), act)
    row = torch.tensor([4, 0, 8, 2, 7, 1, 5], dtype=torch.int32, device=DEV)
    tok = a.prefill(prompt)
    ka, va = a.kcache(), a.vcache()
    ka, va = (ka, va) if max_batch == 1 else (ka[0], va[0])
    a.save_pages(pages, row, 20)
    a.save_pages(pages, row, 25, first=20)
    for p in range(45):
        page, slot = int(row[p // 7]), p % 7
        for l in range(cfg.n_layers):
            assert np.array_equal(pages.k[l, page, :, slot].float().cpu().numpy().ravel(), ka[l, p])
            assert np.array_equal(pages.v[l, page, :, slot].float().cpu().numpy().ravel(), va[l, p])
    free = torch.ones(9, 7, dtype=torch.bool)
    for p in range(45):
        free[int(row[p // 7]), p % 7] = False
    assert bool(torch.isnan(pages.k.transpose(2, 3)[:, free]).all())            # nothing else was written
    b = B.River(cfg, dw, river, max_batch=max_batch)
    if max_batch == 1:
        b.load_pages(pages, row, 45, tok)
        assert b.pos == 45
        for e in (None, cfg.min_exit_layer, cfg.n_layers):
            ta, ea, sa = a.decode_step(None, e)
            tb, eb, sb = b.decode_step(None, e)
            assert (ta, ea) == (tb, eb) and np.array_equal(sa, sb, equal_nan=True)
            assert np.array_equal(a.logits(), b.logits())
    else:
        # sequence 2 takes the prompt over, sequence 1 keeps one of its own
        other = inputs.make_prompt(cfg.vocab, 12, 7)
        a.prefill(other, seq=1)
        a.load_pages(pages, row, 45, tok, seq=2)
        assert a.seq_pos(2) == 45 and a.seq_pos(1) == 12
        for e in (None, [2, 1, 2], [1, 2, 1]):
            t, ex, sims = a.decode_batch(3, None, e)
            assert t[0] == t[2] and ex[0] == ex[2] and np.array_equal(sims[0], sims[2], equal_nan=True)
            assert np.array_equal(a.batch_logits()[0], a.batch_logits()[2])
    for bad in (dict(n=49, first=0), dict(n=1, first=99), dict(n=-1), dict(n=5, first=-1)):
        with pytest.raises(B.RiverError):
            b.save_pages(pages, row, **bad)
    for bad in (dict(n=0, next_token=0), dict(n=97, next_token=0), dict(n=50, next_token=0), dict(n=5, next_token=cfg.vocab)):
        with pytest.raises(B.RiverError):
            b.load_pages(pages, row, **bad)
    with pytest.raises(B.RiverError) as e:
        b.load_pages(B.Pages(pages.k[:1], pages.v[:1], act), row, 5, 0)
    assert e.value.code == B.RIVER_EINVAL and "not the context's" in str(e.value)
    a.close()
    b.close()


def test_attention_over_a_context_s_own_cache():
    """A prompt's keys and values, saved from a context, read by the paged attention."""
    cfg = SAVE
    dw = B.upload_weights(inputs.make_weights(cfg, 8))
    a = B.River(cfg, dw, None)
    a.prefill(inputs.make_prompt(cfg.vocab, 70, 9))
    st = Setup("bf16", 2, 64, 16, [70], [1], seed=25, layers=2)
    a.save_pages(st.pages, st.table[0], 70)
    for layer in range(2):
        run_attention(st, 8, layer=layer)
    a.close()


def test_handles_stay_as_they_were_made():
    st = Setup("bf16", 1, 64, 16, [20], [1], seed=38)
    f, m = freqs(64)
    for handle, name in ((st.pages, "k"), (st.batch, "max_len"), (st.batch, "table"), (B.Rope(f, "half", m), "inv_freq")):
        with pytest.raises(AttributeError):
            setattr(handle, name, getattr(handle, name))


def test_the_binding_refuses():
    st = Setup("bf16", 2, 64, 16, [20, 5], [1, 1], seed=26)
    q = st.randn(2, 8, 64)
    f, _ = freqs(64)
    for bad in (q.float(), q[..., :32], q.cpu(), q.transpose(0, 1), q[:, ::2], q[0]):
        with pytest.raises(ValueError):
            B.river_paged_attention(st.pages, 0, st.batch, bad)
    with pytest.raises(ValueError):
        B.river_paged_attention(st.pages, 0, st.batch, q, out=torch.empty(3, 8, 64, dtype=torch.bfloat16, device=DEV))
    with pytest.raises(B.RiverError):
        B.river_paged_attention(st.pages, 0, st.batch, st.randn(2, 7, 64))
    with pytest.raises(B.RiverError):
        B.river_paged_attention(st.pages, 1, st.batch, q)
    with pytest.raises(ValueError):
        B.river_rope_store(st.pages, 0, st.batch, q, q, q, B.Rope(f))
    with pytest.raises(ValueError):
        B.Rope(f.float())
    with pytest.raises(ValueError):
        B.Pages(st.k.transpose(3, 4), st.v.transpose(3, 4))
    with pytest.raises(ValueError):
        B.Pages(st.k, st.v, torch.float32)
    with pytest.raises(ValueError):
        B.Pages(st.k.cpu(), st.v.cpu())
    with pytest.raises(ValueError):
        B.Batch(st.table.long(), st.dlens)
    with pytest.raises(ValueError):
        B.Batch(st.table, st.dlens[:1])
    with pytest.raises(ValueError):
        B.Batch(st.table, st.dlens, st.q_start[:2])
    with pytest.raises(ValueError):
        B.Batch(st.table, st.dlens, None, max_new=2)
    with pytest.raises(ValueError):
        B.river_copy_pages(st.pages, [0, 1], [2])
    with pytest.raises(ValueError):
        B.river_copy_pages(st.pages, [0.5], [2])
    with pytest.raises(B.RiverError):
        B.river_copy_pages(st.pages, [0], [10 ** 6])
    # a workspace that is too small, or missing, where one is needed
    pg, n = st.pages, C.c_size_t()
    big = Setup("bf16", 1, 64, 64, [20000], [1], seed=27, ragged=False)
    qq = big.randn(1, 4, 64)
    ref = big.batch.bind(1, big.pages)
    assert B.load().river_paged_attention_workspace(big.pages.ref, ref, 4, 0, 0, C.byref(n)) == 0
    if n.value:
        ws = torch.empty(n.value, dtype=torch.uint8, device=DEV)
        args = lambda p, b: (big.pages.ref, 0, ref, 4, qq.data_ptr(), 256, 0.0, 0, 0, torch.empty_like(qq).data_ptr(), 256, p, b, None, None)
        assert B.load().river_paged_attention(*args(ws.data_ptr(), n.value - 1)) == B.RIVER_ENOSPC
        assert B.load().river_paged_attention(*args(None, n.value)) == B.RIVER_EINVAL
        assert B.load().river_paged_attention(*args(ws.data_ptr() + 8, n.value)) == B.RIVER_EINVAL


def busy():
    """Some 20 ms of work on the current stream."""
    x = torch.ones(4096, 4096, device=DEV)
    for _ in range(20):
        x = x @ x
    return x


@pytest.mark.parametrize("max_batch", [1, 2])
def test_contexts_and_pages_on_another_stream(max_batch):
    """Pages and row are what the caller's stream has queued when a context loads them, and what a context saves is there for what the
    caller's stream does next, although the context has a stream of its own."""
    w = inputs.make_weights(SAVE, 5)
    dw = B.upload_weights(w)
    river = B.quantize_river(SAVE, dw)
    prompt = inputs.make_prompt(SAVE.vocab, 45, 6)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    a = B.River(SAVE, dw, river, max_batch=max_batch)
    with torch.cuda.stream(side):
        b = B.River(SAVE, dw, river, max_batch=max_batch)
    tok = a.prefill(prompt)
    one = lambda x: x if max_batch == 1 else x[0]
    want_k, want_v = one(a.kcache())[:, :45], one(a.vcache())[:, :45]
    good = torch.tensor([4, 0, 8, 2, 7, 1, 5], dtype=torch.int32, device=DEV)

    def cache():
        return B.Pages(*(torch.full((SAVE.n_layers, 9, SAVE.n_kv_heads, 7, SAVE.head_dim), math.nan, dtype=torch.bfloat16, device=DEV) for _ in range(2)))

    def rows(k):
        p = np.arange(45)
        return k.float().cpu().numpy()[:, good.cpu().numpy()[p // 7], :, p % 7].transpose(1, 0, 2, 3).reshape(SAVE.n_layers, 45, -1)

    # the context's stream is behind, the caller's is not
    pages = cache()
    torch.cuda.synchronize()
    x = busy()
    with torch.cuda.stream(side):
        a.save_pages(pages, good + 0, 45)
        got_k, got_v = pages.k.clone(), pages.v.clone()
    torch.cuda.synchronize()
    assert np.array_equal(rows(got_k), want_k) and np.array_equal(rows(got_v), want_v)
    # the caller's is behind: pages and row are not written yet
    for context, stream in ((b, torch.cuda.current_stream()), (a, side)):
        context.fill_cache(0)
        late, row = cache(), torch.full_like(good, -1)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            x = busy()
            late.k.copy_(got_k)
            late.v.copy_(got_v)
            row.copy_(good)
            context.load_pages(late, row + 0, 45, tok)
            late.k.zero_()                  # (behind the call)
            row.fill_(-1)
        torch.cuda.synchronize()
        assert np.array_equal(one(context.kcache())[:, :45], want_k) and np.array_equal(one(context.vcache())[:, :45], want_v)
    a.close()
    b.close()
    del x


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("lens,new", [([20, 7], [3, 1]), ([300, 0, 64], [290, 0, 64]), ([3000, 40], [1, 33])], ids=str)
def test_attention_without_a_bound_on_the_new_tokens(kind, lens, new):
    # every new token of every sequence has its row, also where the batch was made without max_new
    st = Setup(kind, 2, 64, 16, lens, new, seed=39, pad=3)
    st.batch = B.Batch(st.table, st.dlens, st.q_start)
    run_attention(st, 8)
    run_attention(st, 8, 50, 3)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("window,sinks", [(2**31 - 1, 0), (2**31 - 1, 2**31 - 1), (2**31 - 3, 3), (2**30, 2**30), (5, 2**31 - 1)])
@pytest.mark.parametrize("n,m,room", [(1, 5, 0), (40, 100, 0), (40, 100, 20000), (130, 300, 20000), (-2**31, 40, 0), (-2**31, 300, 20000)])
def test_attention_of_the_widest_windows(kind, window, sinks, n, m, room):
    # a window that holds all there is, as a number that no length reaches; new tokens that have no position among the others
    st = Setup(kind, 1, 64, 16, [n, 20, 300], [m, 2, 150], seed=40, room=room)
    q = st.randn(st.tokens, 4, 64)
    got = B.river_paged_attention(st.pages, 0, st.batch, q, window, sinks)
    lost = min(m, m - n)
    assert bool((got[:lost] == 0).all())
    st.new, st.start = [max(n, 0), 2, 150], np.array([lost, m, m + 2, m + 152])
    want, tol = attention(st, q, window, sinks)
    check(got[lost:], want[lost:], tol[lost:])


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lens,new", [([300], [1]), ([20000], [1]), ([300], [5]), ([400], [290]), ([1500, 700], [200, 300])], ids=str)
@pytest.mark.parametrize("room", [0, 20000])
def test_attention_of_scores_of_minus_infinity_alone(kind, bad, hd, lens, new, room):
    # keys that score -infinity count for nothing: a row that sees no others is zero, whatever their values are
    st = Setup(kind, 1, hd, 16, lens, new, seed=41, room=room)
    st.k[..., 0] = -math.inf
    st.v[..., 3] = bad
    q = torch.zeros(st.tokens, 4, hd, dtype=st.act, device=DEV)
    q[..., 0] = 1.0
    out = torch.full_like(q, 7.0)
    B.river_paged_attention(st.pages, 0, st.batch, q, out=out)
    assert bool((out == 0).all())


def test_a_batch_does_not_grow_with_its_calls():
    # (what it remembers of shapes of calls is bounded, whatever the windows)
    st = Setup("bf16", 1, 64, 16, [40, 9], [1, 1], seed=42, ragged=False)
    q = st.randn(2, 4, 64)
    for window in range(1, 700):
        B.river_paged_attention(st.pages, 0, st.batch, q, window)
    assert len(st.batch._bytes) <= 256 and len(st.batch._calls) <= 256
    run_attention(st, 4, 7)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_probabilities_of_single_tokens_are_more_than_their_type(kind, hd):
    # Two keys of scores 0 and -d and values 1 and -1: o = tanh(d / 2).  Rounded to bf16 alone the second probability, 1 - d to the maximum's 1,
    # would be off by up to 2^-9 (its numbers below 1 are 2^-8 apart), and o by half of that; as a sum of two such numbers it is off by
    # 2^-17 at most, scores and exponentials by 2^-20 (the module's tolerance of a score: products of one term, and the instruction's)
    st = Setup(kind, 1, hd, 16, [2] * 64, [1] * 64, seed=43, ragged=False)
    st.k.zero_()
    st.v.zero_()
    d = (torch.arange(64, device=DEV, dtype=torch.float64) + 0.5) / 64 * 2.0 ** -7
    q = torch.zeros(64, 1, hd, dtype=st.act, device=DEV)
    q[:, 0, 0] = d.to(st.act)
    d = q[:, 0, 0].double()
    for s in range(64):
        page = int(st.host[s, 0])
        st.k[0, page, 0, 1, 0] = -1.0
        st.v[0, page, 0, 0], st.v[0, page, 0, 1] = 1.0, -1.0
    got = B.river_paged_attention(st.pages, 0, st.batch, q, scale=1.0).double()[:, 0]
    want = torch.tanh(d / 2)[:, None].expand(64, hd)
    tol = half_step(st.act) * want + 2.0 ** -17 + 2.0 ** -19
    p = (-d).exp()
    once = (1 - p.to(torch.bfloat16).double()) / (1 + p)
    assert int(((once - want[:, 0]).abs() > tol[:, 0]).sum()) > 32        # (a single rounding would be seen)
    check(got, want, tol)
