"""Attention with common prefixes against a plain 64-bit implementation of its definition, and steps of all operators of the paged cache
together.  Tolerances: those of test_gpu_pages (its `attention` has them); the parts of a row that are joined add a rounding each, which its
n 2^-24 for n positions covers, since a part has 128 positions or is one of two."""
import math

import numpy as np
import pytest
import torch

from paper_2604_18396_amd import binding as B
from test_gpu_pages import DEV, TYPES, Setup, attention, check, freqs, half_step, turned

pytestmark = pytest.mark.gpu


class Shared(Setup):
    """Sequences of `lens` positions, `new` of them new; group g has the next groups[g][1] sequences, behind the first `lonely` ones, and a
    prefix of groups[g][0] positions.  The sequences' own entries of whole pages of a prefix name pages that do not exist.
    how: the bounds that are given, by which a call is divided.  "through": those of what is there (each sequence goes through its prefix, unless
    that is large); "rows" and "tiles": the prefixes' table has room for so many positions that prefixes have units of their own, of 16 rows, or of 128
    where the type has them."""

    def __init__(self, kind, nkv, hd, ps, lens, new, groups, lonely=0, seed=0, layers=1, pad=0, ragged=True, room=0, how="through"):
        self.how = how
        self.groups, self.of = groups, [-1] * lonely + [g for g, (_, n) in enumerate(groups) for _ in range(n)]
        self.of += [-1] * (len(lens) - len(self.of))
        self.common = [-(-p // ps) for p, _ in groups]
        super().__init__(kind, nkv, hd, ps, lens, new, seed=seed, spare=2 + sum(self.common), layers=layers, pad=pad, ragged=ragged, room=room)
        self.prefix_host = np.full((max(len(groups), 1), max(self.common + [1]) + 1), -1, dtype=np.int32)
        at = 0
        for g, n in enumerate(self.common):
            self.prefix_host[g, :n] = self.spare[at:at + n]
            at += n
        for s, g in enumerate(self.of):
            if g >= 0:
                self.host[s, :min(groups[g][0] // ps, self.host.shape[1])] = (-1, 10**9, self.k.shape[1], -2**31)[s % 4]
        self.table.copy_(torch.from_numpy(self.host))
        start = lonely + np.concatenate([[0], np.cumsum([n for _, n in groups])]).astype(np.int32)
        self.make(start, *((max([p for p, _ in groups] + [1]), max([n for _, n in groups] + [1])) if how == "through" else (None, None)))

    def make(self, start, max_len=None, max_seqs=None):
        n, seqs = len(self.groups), len(self.lens)
        self.prefix_table = torch.from_numpy(self.prefix_host[:n]).to(DEV) if n else torch.zeros(0, 1, dtype=torch.int32, device=DEV)
        if self.how != "through" and n:
            # 26 MB that sharing saves, or 2^20 positions
            key = 2 * self.nkv * self.hd * self.kvt.itemsize
            room = 1 << 20 if self.how == "tiles" else 26e6 / (key * max(1, min(n * (seqs - 1), seqs)))
            wide = torch.full((n, max(self.prefix_host.shape[1], int(room) // self.ps + 1)), -1, dtype=torch.int32, device=DEV)
            wide[:, :self.prefix_host.shape[1]] = self.prefix_table
            self.prefix_table = wide
        self.prefixes = B.Prefixes(self.prefix_table, torch.tensor([p for p, _ in self.groups], dtype=torch.int32, device=DEV),
                                   torch.tensor(start, dtype=torch.int32, device=DEV), max_len, max_seqs)

    def rows(self, s, layer=0):
        k, v, there = super().rows(s, layer)
        g = self.of[s]
        if g >= 0:
            p = np.arange(min(self.groups[g][0], len(k)))
            entry = self.prefix_host[g][np.minimum(p // self.ps, self.prefix_host.shape[1] - 1)]
            ok = (entry >= 0) & (entry < self.k.shape[1])
            page, slot = torch.from_numpy(np.where(ok, entry, 0)).to(DEV).long(), torch.from_numpy(p % self.ps).to(DEV).long()
            k[:len(p)], v[:len(p)] = self.k[layer][page, :, slot].double(), self.v[layer][page, :, slot].double()
            there[:len(p)] = torch.from_numpy(ok).to(DEV)
        return k, v, there


HOW = pytest.mark.parametrize("how", ["through", "rows", "tiles"])


def run(st, nq, scale=0.0, std=1.5, layer=0):
    q = st.randn(st.tokens, nq, st.hd, std=std)
    out = torch.full_like(q, 7.0)
    B.river_prefix_attention(st.pages, layer, st.batch, st.prefixes, q, scale, out)
    want, tol = attention(st, q, scale=scale or None, layer=layer)
    n = int(st.start[-1])
    check(out[:n], want[:n], tol[:n], (st.lens, st.new, st.groups))
    assert bool((out[n:] == 7.0).all())                          # tokens of no sequence
    return q, out


def behind(groups, own, new, lonely=()):
    """Lengths of the sequences: a prefix, then own[i] positions, then the new ones."""
    before = [0] * len(lonely) + [p for p, n in groups for _ in range(n)]
    own = list(lonely) + list(own)
    before += [0] * (len(own) - len(before))
    return [b + o + m for b, o, m in zip(before, own, new)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("nkv,rep", [(1, 1), (2, 4), (3, 7), (1, 24), (8, 4)])
@pytest.mark.parametrize("groups,own", [([(200, 5)], [0, 3, 40, 170, 1]), ([(1000, 2), (64, 0), (17, 3), (513, 1)], [9, 300, 0, 31, 64, 128, 5, 0]),
                                        ([(2500, 20)], list(range(0, 200, 10)))], ids=str)
@HOW
def test_single_tokens(kind, hd, nkv, rep, groups, own, how):
    new = [1] * len(own)
    run(Shared(kind, nkv, hd, 16, behind(groups, own, new), new, groups, ragged=False, how=how), nkv * rep)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("hd,nkv,rep", [(64, 2, 4), (128, 1, 8), (128, 2, 1), (64, 1, 3)])
@pytest.mark.parametrize("groups,own,new,lonely", [([(100, 3)], [0, 7, 60], [2, 5, 1], ()), ([(300, 2), (40, 2)], [10, 200, 0, 5, 90], [4, 0, 9, 1, 2], (50, 3)),
                                                   ([(700, 4)], [0, 0, 33, 129], [130, 64, 1, 300], ()), ([(4000, 3), (130, 6)], [5] * 9, [3] * 9, (700,))], ids=str)
@HOW
@pytest.mark.parametrize("room", [0, 300])
def test_several_tokens(kind, hd, nkv, rep, groups, own, new, lonely, how, room):
    new = [1 + i for i in range(len(lonely))] + new
    run(Shared(kind, nkv, hd, 16, behind(groups, own, new, lonely), new, groups, lonely=len(lonely), pad=3, how=how, room=room), nkv * rep)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("ps", [1, 7, 20, 64, 1000])
@pytest.mark.parametrize("prefix", [1, 63, 64, 640, 1001])
@HOW
def test_page_sizes(kind, ps, prefix, how):
    groups, own, new = [(prefix, 4)], [0, 1, 63, 200], [1, 2, 1, 20]
    run(Shared(kind, 2, 64, ps, behind(groups, own, new), new, groups, seed=ps, how=how), 8)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
@HOW
def test_large_groups(kind, hd, how):
    # several tiles of rows, several splits of keys, several of them the sequences'
    groups, own = [(3000, 70), (800, 30)], [(i * 37) % 500 for i in range(101)]
    new = [1] * 101
    run(Shared(kind, 2, hd, 16, behind(groups, own, new), new, groups, ragged=False, seed=1, how=how), 16)
    new = [1 + i % 6 for i in range(101)]
    run(Shared(kind, 2, hd, 16, behind(groups, own, new), new, groups, seed=2, how=how), 8)


@pytest.mark.parametrize("kind", TYPES)
@HOW
def test_many_groups(kind, how):
    # more groups than a wavefront has lanes, some of them empty, some sequences in front of the first and behind the last
    groups = [(1 + (i * 97) % 300, (i * 7) % 4) for i in range(150)]
    n = 3 + sum(k for _, k in groups) + 2
    lonely, own = (7, 130, 1), [(i * 11) % 90 for i in range(n - 3)]
    for new in ([1] * n, [1 + i % 5 for i in range(n)]):
        run(Shared(kind, 1, 64, 16, behind(groups, own, new, lonely), new, groups, lonely=3, seed=14, how=how), 4)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@HOW
def test_queries_of_places_without_a_sequence(kind, bad, how):
    """A padded batch: places whose sequence has no positions, with whatever bits in their queries, are zeros, and all others have the bits that they
    have without them."""
    for new in ([1] * 9, [1, 2, 3, 4, 5, 1, 2, 3, 4]):
        lens = [260 + 9 * i + m for i, m in enumerate(new)]
        lens[1] = lens[4] = lens[8] = 0
        st = Shared(kind, 1, 64, 16, lens, new, [(250, 9)], seed=15, how=how)
        q = st.randn(st.tokens, 8, 64)
        places = torch.tensor([t for s, t, _ in st.positions() if s in (1, 4, 8)], device=DEV)
        q[places] = 0.0
        clean = B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, q)
        q[places] = bad
        assert torch.equal(B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, q), clean) and not bool(clean[places].any())


def least_ms(f, calls=10):
    f()
    best = math.inf
    for _ in range(7):
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        for _ in range(calls):
            f()
        end.record()
        end.synchronize()
        best = min(best, begin.elapsed_time(end) / calls)
    return best


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("prefix,n", [(30000, 24), (8191, 64), (8191, 6)])
def test_queries_of_places_without_a_sequence_cost_nothing(kind, prefix, n):
    """Not finite queries of such places leave the bits of all others (see above), and their time: a tile that is computed twice takes four to
    nineteen times as long; a call's best time over several tries differs by a few hundredths, under a clock that falls meanwhile by up to 1.5."""
    for new in ([1] * n, [1 + i % 3 for i in range(n)]):
        lens = [prefix + 9 + i + m for i, m in enumerate(new)]
        lens[1] = lens[n - 2] = 0
        st = Shared(kind, 8, 64, 16, lens, new, [(prefix, n)], ragged=max(new) > 1, seed=24)
        q = st.randn(st.tokens, 32, 64)
        call = lambda: B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, q)
        places = torch.tensor([t for s, t, _ in st.positions() if s in (1, n - 2)], device=DEV)
        q[places] = 0.0
        clean, usual = call(), least_ms(call)
        for bad in (math.nan, math.inf):
            q[places] = bad
            assert least_ms(call) < 2 * usual, (bad, usual)
            assert torch.equal(call(), clean)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("groups,own,new", [([(20000, 2)], [100, 3000], [1, 1]), ([(50, 2)], [20000, 10], [1, 1]), ([(9000, 2)], [100, 5], [20, 33])], ids=str)
@HOW
def test_long_caches(kind, groups, own, new, how):
    run(Shared(kind, 1, 128, 16, behind(groups, own, new), new, groups, seed=3, how=how), 4)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("hd,nkv,rep", [(64, 2, 4), (128, 1, 6)])
@pytest.mark.parametrize("groups,own,new,lonely", [([(20000, 1)], [100], [50], (0, 3, 40, 8, 300, 1)), ([(6000, 1), (9000, 1)], [0, 33], [8, 17], (200,) * 20)], ids=str)
def test_long_prefixes_beside_sequences_without_one(kind, hd, nkv, rep, groups, own, new, lonely):
    # (few long sequences do not fill the card by themselves: 16-bit types give their prefixes units of their own, though nobody shares them)
    new = [1 + i * 7 % 30 for i in range(len(lonely))] + new
    run(Shared(kind, nkv, hd, 16, behind(groups, own, new, lonely), new, groups, lonely=len(lonely), pad=2, seed=6), nkv * rep)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("hd,rep", [(64, 8), (128, 3), (128, 8)])
@pytest.mark.parametrize("new", [1, 3])
def test_prefixes_in_hundreds_of_splits(kind, hd, rep, new):
    # (one key head: as many splits as there are CUs, the last of them short)
    groups, own, tokens = [(45001, 9)], [0, 5, 130, 17, 300, 1, 2, 64, 33, 90], [1 + i % new for i in range(10)]
    run(Shared(kind, 1, hd, 64, behind(groups, own, tokens), tokens, groups, seed=8, ragged=new > 1), rep)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("hd,rep,new", [(64, 4, 1), (128, 2, 1), (128, 3, 5)])
def test_single_tokens_of_one_long_prefix_beside_sequences_without_one(kind, hd, rep, new):
    lonely, groups = tuple(i * 5 % 90 for i in range(30)), [(30000, 1)]
    tokens = [1 + i % new for i in range(30)] + [new]
    run(Shared(kind, 8, hd, 32, behind(groups, [70], tokens, lonely), tokens, groups, lonely=30, seed=7, ragged=new > 1), 8 * rep)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("max_len,max_seqs", [(1, 1), (1, 2), (64, 3), (10**6, 1000), (0, 0), (2000, 2)])
@HOW
def test_more_than_the_bounds_say(kind, max_len, max_seqs, how):
    groups = [(1500, 40), (333, 5)]
    for new in ([1] * 45, [1 + i % 4 for i in range(45)]):
        st = Shared(kind, 1, 64, 16, behind(groups, [i * 9 for i in range(45)], new), new, groups, seed=4, how=how)
        st.make([0, 40, 45], max_len, max_seqs)
        run(st, 8)
        st.batch = B.Batch(st.table, st.dlens, st.q_start, max_new=max(new), max_len=100)
        run(st, 8)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("lens,new", [([0, 300, 5, 128, 129, 1], [1] * 6), ([0, 200, 3, 128, 0, 40], [3, 90, 3, 128, 0, 7]), ([-5, 2, 130, -2**31, 127, 300], [2, 6, 1, 1, 140, 1])],
                         ids=str)
@HOW
def test_sequences_shorter_than_their_prefix(kind, lens, new, how):
    """What is below a token's position counts, up to it; a token without a position is zero."""
    for groups in ([(128, 6)], [(128, 2), (129, 3)], [(1000, 5)]):
        st = Shared(kind, 2, 64, 16, lens, new, groups, seed=5, how=how)
        q, out = run(st, 8)
        for s, t, p in st.positions():
            assert p >= 0 or not bool(out[t].any())


@pytest.mark.parametrize("kind", TYPES)
@HOW
def test_prefixes_of_no_positions_and_groups_of_no_sequences(kind, how):
    lens = [50, 1, 300, 0, 77]
    for new in ([1] * 5, [2, 1, 130, 0, 5]):
        for groups in ([(0, 5)], [(0, 2), (0, 0), (0, 1)], [(5, 0), (100, 0)], []):
            st = Shared(kind, 2, 64, 16, lens, new, groups, seed=6, how=how)
            q, out = run(st, 8)
            # nothing is shared: river_paged_attention's rows, up to what joining them in other parts rounds
            want, tol = attention(st, q)
            check(B.river_paged_attention(st.pages, 0, st.batch, q), want, tol)
    st.groups = [(-7, 3)]
    st.common, st.prefix_host = [0], np.full((1, 2), -1, dtype=np.int32)
    st.make([1, 4])
    run(st, 8)


@pytest.mark.parametrize("kind", TYPES)
@HOW
def test_pages_that_are_not_there(kind, how):
    groups, own = [(300, 3), (70, 2)], [40, 0, 200, 100, 3]
    for new in ([1] * 5, [3, 1, 40, 2, 3]):
        st = Shared(kind, 2, 64, 16, behind(groups, own, new), new, groups, seed=7, how=how)
        st.prefix_host[0, 3], st.prefix_host[0, 18] = -1, 2**31 - 1
        st.prefix_host[1, :] = -5                                 # a prefix of which nothing is there
        st.host[2, 25] = st.k.shape[1]
        st.table.copy_(torch.from_numpy(st.host))
        st.make([0, 3, 5], *((300, 3) if how == "through" else ()))
        run(st, 8)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("lens,new", [([130, 140, 200, 64, 33], [1] * 5), ([130, 300, 200, 64, 33], [2, 160, 60, 3, 1])], ids=str)
@HOW
def test_what_is_not_seen_has_no_influence(kind, bad, lens, new, how):
    """Places behind a row's position, of pages that nobody has, and of the prefix's last page behind its end, hold what is not finite."""
    st = Shared(kind, 2, 64, 16, lens, new, [(130, 4)], lonely=1, seed=8, how=how)
    q = st.randn(st.tokens, 8, 64)
    clean = B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, q)
    used = torch.zeros(st.k.shape[1], 16, dtype=torch.bool, device=DEV)
    for s, n in enumerate(st.lens):
        before = 130 if st.of[s] >= 0 else 0
        for p in range(before, n):
            used[int(st.host[s, p // 16]), p % 16] = True
    for p in range(130):
        used[int(st.prefix_host[0, p // 16]), p % 16] = True
    for x in (st.k, st.v):
        x[0] = torch.where(used[:, None, :, None], x[0], bad)
    assert torch.equal(B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, q), clean)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("hd", [64, 128])
@HOW
def test_a_later_position_is_no_part_of_an_earlier_row(kind, bad, where, hd, how):
    """A position holds what is not finite: rows below it are as without, others are not finite where the formula has it."""
    for lens, new, at in (([300, 320, 290], [40, 1, 3], 270), ([300, 90, 290], [290, 1, 3], 120), ([300, 300], [1, 1], 285), ([310, 300], [25, 1], 290)):
        st = Shared(kind, 1, hd, 16, lens, new, [(280, len(lens))], seed=9, how=how)
        q = st.randn(st.tokens, 4, hd)
        clean = B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, q)
        x = st.k if where == "k" else st.v
        in_prefix = at < 280
        page = st.prefix_host[0, at // 16] if in_prefix else st.host[0, at // 16]
        x[0, page, 0, at % 16, 5] = bad
        got = B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, q)
        for s, t, p in st.positions():
            if p < at or not (in_prefix or s == 0):
                assert torch.equal(got[t], clean[t]), (s, t, p)
            elif where == "v":
                assert not bool(got[t, :, 5].isfinite().any()) and torch.equal(got[t, :, 6:], clean[t, :, 6:])
            elif not math.isinf(bad):
                assert bool(got[t].isnan().all())


@pytest.mark.parametrize("kind", TYPES)
@HOW
def test_rows_that_see_only_scores_of_minus_infinity(kind, how):
    st = Shared(kind, 1, 64, 16, [140, 150, 145], [1, 1, 6], [(128, 3)], seed=10, how=how)
    q = st.randn(8, 4, 64).abs() + 0.5
    st.k[0, :, :, :, 0] = -math.inf
    st.v[0, :, :, :, 3] = math.inf
    assert not bool(B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, q).any())
    # one key of the prefix that counts, and is all that does
    page = int(st.prefix_host[0, 2])
    st.k[0, page, 0, 5] = 0.0
    st.v[0, :, :, :, 3] = 1.0
    got = B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, q)
    assert torch.equal(got, st.v[0, page, 0, 5].to(st.act).expand_as(got))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("std,scale", [(8.0, 0.0), (1.0, 3.0), (0.01, 0.05), (200.0, 0.0)])
@HOW
def test_scales(kind, std, scale, how):
    groups, own = [(400, 6)], [0, 100, 250, 3, 60, 31]
    for new in ([1] * 6, [3, 30, 1, 9, 20, 2], [3, 70, 1, 9, 40, 2]):
        run(Shared(kind, 2, 128, 16, behind(groups, own, new), new, groups, seed=11, how=how), 8, scale=scale, std=std)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("new", [1, 3])
@HOW
def test_probabilities_of_few_tokens_are_more_than_their_type(kind, hd, new, how):
    # As test_gpu_pages has it for single tokens, whose tolerance and its reasons hold here: two keys of the prefix with scores 0 and -d and values 1 and -1,
    # o = tanh(d / 2).  A sequence's own keys have scores below -42 and values of 0: they are below 2^-60 of the sum
    n, own = 64, 2.0 ** 21
    st = Shared(kind, 1, hd, 16, [2 + new] * n, [new] * n, [(2, n)], seed=23, ragged=new > 1, how=how)
    st.k[:, :, :, :, 0] = -own
    st.k[:, :, :, :, 1:] = 0.0
    st.v.zero_()
    page = int(st.prefix_host[0, 0])
    st.k[0, page, 0, 0, 0], st.k[0, page, 0, 1, 0] = 0.0, -1.0
    st.v[0, page, 0, 0], st.v[0, page, 0, 1] = 1.0, -1.0
    d = (torch.arange(n * new, device=DEV, dtype=torch.float64) + 0.5) / (n * new) * 2.0 ** -7
    q = torch.zeros(n * new, 1, hd, dtype=st.act, device=DEV)
    q[:, 0, 0] = d.to(st.act)
    d = q[:, 0, 0].double()
    assert float(d.min()) * own > 42
    got = B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, q, scale=1.0).double()[:, 0]
    want = torch.tanh(d / 2)[:, None].expand(n * new, hd)
    tol = half_step(st.act) * want + 2.0 ** -17 + 2.0 ** -19
    p = (-d).exp()
    once = (1 - p.to(torch.bfloat16).double()) / (1 + p)
    assert int(((once - want[:, 0]).abs() > tol[:, 0]).sum()) > n * new // 2        # (a single rounding would be seen)
    check(got, want, tol)


@pytest.mark.parametrize("kind", TYPES)
@HOW
@pytest.mark.parametrize("most", [20, 33])
def test_new_tokens_beyond_their_bound_are_left_out(kind, how, most):
    groups, own, new = [(200, 2), (90, 1)], [5, 60, 3], [7, 300, 40]
    st = Shared(kind, 2, 64, 16, behind(groups, own, new), new, groups, seed=12, how=how)
    st.batch = B.Batch(st.table, st.dlens, st.q_start, max_new=most)
    q = st.randn(st.tokens, 8, 64)
    out = torch.full_like(q, 7.0)
    B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, q, out=out)
    want, tol = attention(st, q)
    for s, n in enumerate(new):
        lo = int(st.start[s])
        m = min(n, most)
        check(out[lo:lo + m], want[lo:lo + m], tol[lo:lo + m])
        assert bool((out[lo + m:lo + n] == 7.0).all())


@pytest.mark.parametrize("kind", TYPES)
@HOW
def test_strides_and_layers(kind, how):
    groups, own = [(100, 2)], [45, 3]
    for new in ([1, 1], [20, 3], [80, 45]):
        st = Shared(kind, 2, 64, 16, behind(groups, own, new), new, groups, seed=13, layers=3, how=how)
        wide = st.randn(st.tokens, 8 * 64 * 3)
        q = wide[:, 64 * 8:64 * 16].unflatten(1, (8, 64))
        room = torch.full((st.tokens, 12, 64), 7.0, dtype=st.act, device=DEV)
        out = room[:, 2:10]
        for layer in range(3):
            B.river_prefix_attention(st.pages, layer, st.batch, st.prefixes, q, out=out)
            want, tol = attention(st, q, layer=layer)
            check(out, want, tol)
            assert bool((room[:, :2] == 7.0).all()) and bool((room[:, 10:] == 7.0).all())


@HOW
def test_pages_beyond_32_bits(how):
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
    for new in ([1, 1], [5, 30], [3, 20]):
        st = Shared("bf16", 1, 64, 16, [45, 60], new, [(30, 2)], seed=17, how=how)
        st.k, st.v, st.pages = k, v, B.Pages(k, v)
        st.prefix_host = np.array([[5, 4]], dtype=np.int32)
        st.host = np.array([[-1, 0, 3, -1], [-1, 1, 2, 5]], dtype=np.int32)
        st.table = torch.from_numpy(st.host).to(DEV)
        st.batch = B.Batch(st.table, st.dlens, st.q_start, max_new=max(new), max_len=60)
        st.make([0, 2], *((30, 2) if how == "through" else ()))
        run(st, 32)


@HOW
def test_the_same_call_gives_the_same_bits(how):
    for kind in TYPES:
        for hd in (64, 128):
            groups, own = [(3000, 20), (700, 12)], [(i * 53) % 400 for i in range(32)]
            for new in ([1] * 32, [1 + i % 9 for i in range(32)]):
                st = Shared(kind, 8, hd, 16, behind(groups, own, new), new, groups, seed=18, how=how)
                q = st.randn(st.tokens, 32, hd)
                first = B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, q)
                for _ in range(5):
                    assert torch.equal(first, B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, q))


@pytest.mark.parametrize("kind", TYPES)
@HOW
def test_a_captured_call_has_the_bits_of_an_eager_one(kind, how):
    """(A captured call has no tickets: its splits are joined by a launch of their own.)  Replayed with eager calls and synchronizations between, while
    lengths, prefixes and queries change."""
    groups, own = [(700, 3), (90, 2)], [300, 0, 41, 5, 200]
    for new in ([1] * 5, [2, 5, 1, 3, 4]):
        lens = behind(groups, own, new)
        st = Shared(kind, 2, 64, 16, lens, new, groups, ragged=new[1] > 1, seed=16, how=how)
        q, out = st.randn(st.tokens, 8, 64), torch.zeros(st.tokens, 8, 64, dtype=st.act, device=DEV)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, q, out=out)
        for i in range(5):
            q.copy_(st.randn(st.tokens, 8, 64))
            st.dlens.copy_(torch.tensor([n - i for n in lens], dtype=torch.int32))
            st.prefixes.lens.copy_(torch.tensor([700 - 32 * i, 90 - 7 * i], dtype=torch.int32))
            if i != 3:
                st.prefixes.seq_start.copy_(torch.tensor([0, 3 - i % 2, 5 - i % 2], dtype=torch.int32))
            want = B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, q)
            torch.cuda.synchronize()
            graph.replay()
            assert torch.equal(out, want), i


def test_calls_without_sequences_or_tokens():
    st = Shared("bf16", 2, 64, 16, [40, 30], [1, 1], [(10, 2)], seed=19)
    q = st.randn(0, 8, 64)
    assert B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, q).shape == (0, 8, 64)
    nobody = B.Batch(torch.zeros(0, 3, dtype=torch.int32, device=DEV), torch.zeros(0, dtype=torch.int32, device=DEV),
                     torch.zeros(1, dtype=torch.int32, device=DEV))
    q = st.randn(3, 8, 64)
    out = torch.full_like(q, 7.0)
    B.river_prefix_attention(st.pages, 0, nobody, st.prefixes, q, out=out)
    assert bool((out == 7.0).all())


@HOW
def test_on_another_stream_and_two_at_once(how):
    groups = [(900, 6)]
    st = Shared("bf16", 2, 64, 16, behind(groups, [0, 9, 90, 300, 31, 7], [1] * 6), [1] * 6, groups, ragged=False, seed=20, how=how)
    qs = [st.randn(6, 8, 64) for _ in range(2)]
    want = [B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, q) for q in qs]
    sides = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i in range(2):
            with torch.cuda.stream(sides[i]):
                got[i].append(B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, qs[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


def test_the_binding_refuses():
    st = Shared("bf16", 2, 64, 16, [40, 30], [1, 1], [(10, 2)], seed=21)
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32, device=DEV)
    for a in ((i32(2, 3), i32(1), i32(2)), (i32(1, 3), i32(1), i32(1)), (i32(1, 3).long(), i32(1), i32(2)), (i32(1, 3).cpu(), i32(1).cpu(), i32(2).cpu()),
              (i32(1, 3), i32(1), i32(4)[::2]), (i32(3, 2).t(), i32(2), i32(3)), (i32(1, 0), i32(1), i32(2))):
        with pytest.raises(ValueError):
            B.Prefixes(*a)
    with pytest.raises(AttributeError):
        st.prefixes.max_len = 5
    q = st.randn(2, 8, 64)
    for bad in (q.float(), q[:, :, :32], q.transpose(0, 1), q.cpu()):
        with pytest.raises(ValueError):
            B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, bad)
    for kw in (dict(scale=-1.0), dict(out=q)):
        with pytest.raises(B.RiverError):
            B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, q, **kw)
    with pytest.raises(B.RiverError):
        B.river_prefix_attention(st.pages, 1, st.batch, st.prefixes, q)
    with pytest.raises(B.RiverError):                             # heads that do not divide
        B.river_prefix_attention(st.pages, 0, st.batch, st.prefixes, st.randn(2, 7, 64))


# ------------------------------------------------------------------ all of them together

@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rotary", [True, False])
@HOW
def test_steps_of_a_server(kind, rotary, how):
    """Two system prompts are laid out, stored and read by sequences that come, grow, draft, give back and leave, layer by layer: the step
    is captured once, every replay's rows are those of attention over the whole history of each sequence, and in the end every page is free."""
    act, kvt = TYPES[kind]
    nkv, nq, hd, ps, L, n_pages, n = 2, 8, 64, 8, 2, 90, 6
    g = torch.Generator(device=DEV)
    g.manual_seed(22)
    r = np.random.default_rng(5)
    k, v = (torch.full((L, n_pages, nkv, ps, hd), math.nan, dtype=kvt, device=DEV) for _ in range(2))
    pages = B.Pages(k, v, act)
    f, m = freqs(hd, "ramp")
    rope = B.Rope(f, "half", m)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    # rows 0 and 1 are the prompts, the others sequences: 2, 3, 4 go on from the first, 5, 6 from the second, 7 from none
    shared = torch.zeros(n + 2, dtype=torch.int32, device=DEV)
    t = B.Tables.empty(n_pages, ps, n + 2, 16, n_shared=shared)
    # (rows of the prefixes with room for 2^20 positions, or what 26 MB are, and none: prefixes with units of their own or not, see Shared)
    wide = {"through": 16, "rows": 26000000 // (2 * nkv * hd * kvt.itemsize * 8 * ps) + 1, "tiles": (1 << 20) // ps}[how]
    prompts = torch.full((2, wide), -1, dtype=torch.int32, device=DEV)
    lens = [37, 16]
    group = [0, 0, 0, 1, 1, -1]
    history = [[] for _ in range(n + 2)]
    T = 64
    d, start = i32([0] * (n + 2)), i32([0] * (n + 3))
    slots, positions, refused = torch.zeros(T, dtype=torch.int64, device=DEV), i32([0] * T), i32([0])
    batch = B.Batch(t.table, t.lens, start, max_new=T, max_len=128)
    prefixes = B.Prefixes(prompts, t.lens[:2], i32([2, 5, 7]), *((40, 3) if how == "through" else ()))
    x = torch.zeros(L, T, nq + 2 * nkv, hd, dtype=act, device=DEV)
    outs = [torch.full((T, nq, hd), 7.0, dtype=act, device=DEV) for _ in range(L)]

    def step():
        B.river_build_batch(t, d, start, slots, positions, refused)
        prompts[:, :16] = t.table[:2]
        for l in range(L):
            q, kk, vv = x[l, :, :nq], x[l, :, nq:nq + nkv], x[l, :, nq + nkv:]
            if rotary:
                q = B.river_rope_store(pages, l, batch, q, kk, vv, rope, out=queries[l])
            else:
                B.river_store_slots(pages, l, slots, kk, vv)
            B.river_prefix_attention(pages, l, batch, prefixes, q, out=outs[l])

    queries = [torch.zeros(T, nq, hd, dtype=act, device=DEV) for _ in range(L)]
    graph = None

    def advance(want, expect_refused=0):
        """want: new positions of every row of the table."""
        nonlocal graph
        d.copy_(i32(want))
        x.copy_(torch.randn(x.shape, generator=g, device=DEV))
        for o in outs:
            o.fill_(7.0)
        if graph is None and len(history[2]):
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step()
        graph.replay() if graph is not None else step()
        assert refused.item() == expect_refused
        at = start.tolist()
        for s in range(n + 2):
            got = at[s + 1] - at[s]
            if want[s] < 0:
                history[s] = history[s][:max(0, len(history[s]) + want[s])]
                assert got == 0
            if not got:
                continue
            have = len(history[s])
            assert got == want[s] and positions[at[s]:at[s + 1]].tolist() == list(range(have, have + got))
            new = slice(at[s], at[s + 1])
            cols = []
            for l in range(L):
                kk, vv = x[l, new, nq:nq + nkv], x[l, new, nq + nkv:]
                if rotary:
                    kk = turned(kk, list(range(have, have + got)), f, m, "half")[0]
                cols.append((kk.to(kvt).double(), vv.to(kvt).double()))
            history[s] = history[s] + [[(cols[l][0][i], cols[l][1][i]) for l in range(L)] for i in range(got)]
            for l in range(L):
                K, V = (torch.stack([h[l][i] for h in history[s]]) for i in range(2))
                q = (queries[l] if rotary else x[l, :, :nq])[new]
                j, p = torch.arange(have + got, device=DEV), torch.arange(have, have + got, device=DEV)[:, None]
                for h in range(nq):
                    w = torch.where(j <= p, q[:, h].double() @ K[:, h // 4].t() / 8, -math.inf).softmax(-1)
                    o, a = w @ V[:, h // 4], w @ V[:, h // 4].abs()
                    # (rotated keys of the cache and of this oracle may round to neighbours: see test_gpu_pages.test_a_serving_loop)
                    most = (q[:, h].double().abs() @ K[:, h // 4].abs().t()).amax(1, keepdim=True) / 8
                    e = most * ((2 * half_step(kvt) if rotary else 0.0) + (hd + 8) * 2.0 ** -24) + 2.0 ** -20
                    check(outs[l][new, h], o, half_step(act) * o.abs() + a * (half_step(kvt) + 2 * e + 200 * 2.0 ** -24), (s, l, h))
        for o in outs:
            assert bool((o[at[-1]:] == 7.0).all())

    def join(s):
        """A sequence goes on from its prompt: whole pages are the prompt's, the last, half full one is copied."""
        p = group[s - 2]
        whole = lens[p] // ps
        t.table[s, :whole] = t.table[p, :whole]
        shared[s] = whole
        if lens[p] % ps:
            t.lens[s] = whole * ps
            d.copy_(i32([lens[p] % ps if i == s else 0 for i in range(n + 2)]))
            B.river_build_batch(t, d, start)
            src, dst = int(t.table[p, whole]), int(t.table[s, whole])
            B.river_copy_pages(pages, [src], [dst])
            assert t.lens[s].item() == lens[p]
        else:
            t.lens[s] = lens[p]
        history[s] = list(history[p])

    advance(lens + [0] * n)                                      # the prompts themselves, which are nobody's followers
    for s in range(2, 7):
        join(s)
    advance([0, 0, 5, 1, 9, 2, 1, 20])
    for i in range(3):
        advance([0, 0, 1, 1, 1, 1, 1, 1])
    advance([0, 0, 4, 4, 4, 4, 4, 4])                             # drafts, of which some are rejected
    advance([0, 0, -4, -1, 0, -2, -3, -4])
    advance([0, 0, 1, 1, 1, 1, 1, 1])
    advance([0, 0, -2**31, 0, 0, -2**31, 0, 0])                   # two leave (their prompts' pages stay), and come again
    history[2], history[5] = [], []
    assert t.table[2].tolist() == t.table[0, :4].tolist() + [-1] * 12 and t.table[5].tolist() == t.table[1, :2].tolist() + [-1] * 14
    for s in (2, 5):
        join(s)
    advance([0, 0, 7, 1, 1, 8, 1, 1])
    advance([0, 0, 1, 1, 1, 1, 1, 200], expect_refused=1)         # one has no room in its row and waits
    advance([0, 0, 1, 1, 1, 1, 1, 1])
    advance([0, 0] + [-2**31] * n)
    shared.zero_()
    t.table[2:].fill_(-1)
    advance([-2**31] * 2 + [0] * n)
    assert sorted(t.free_pages.tolist()) == list(range(n_pages)) and t.n_free.item() == n_pages and not bool(t.lens.any())
