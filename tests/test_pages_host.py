"""The paged cache's host side: refused arguments, rotary frequencies, the pool's bookkeeping (no GPU)."""
import ctypes as C
import heapq
import math
import os
import random
import subprocess
import sys
import types

import numpy as np
import pytest

from paper_2604_18396_amd import binding as B

P = 0x10000          # stands for a device address: every call below is refused, or ends, before it is used


def pages(**kw):
    d = dict(k=P, v=P, layer_stride=8 * 2048, page_stride=2048, n_layers=2, n_pages=8, page_size=16, n_kv_heads=2, head_dim=64,
             dtype=1, kv_dtype=0)
    d.update(kw)
    return B.river_pages(*(d[f] for f, _ in B.river_pages._fields_))


def batch(**kw):
    d = dict(table=P, lens=P, q_start=P, n_seq=2, n_tokens=4, max_pages=4, table_stride=4, max_new=2, max_len=64)
    d.update(kw)
    return B.river_batch(*(d[f] for f, _ in B.river_batch._fields_))


def rope(**kw):
    d = dict(inv_freq=P, rot_dim=64, layout=0, mscale=1.0)
    d.update(kw)
    return B.river_rope(*(d[f] for f, _ in B.river_rope._fields_))


BAD_PAGES = [dict(k=0), dict(v=0), dict(k=P + 8), dict(n_layers=0), dict(n_pages=0), dict(page_size=0), dict(page_size=65537),
             dict(n_kv_heads=0), dict(head_dim=96), dict(dtype=2), dict(kv_dtype=2), dict(dtype=0, kv_dtype=1), dict(page_stride=2047),
             dict(page_stride=2040), dict(layer_stride=7 * 2048), dict(layer_stride=8 * 2048 + 4), dict(page_stride=-2048),
             dict(page_stride=4096, layer_stride=0), dict(n_kv_heads=2**31 - 1, page_size=65536)]
BAD_BATCH = [dict(table=0), dict(lens=0), dict(lens=P + 2), dict(n_seq=-1), dict(n_tokens=-1), dict(max_pages=0), dict(table_stride=3),
             dict(max_new=-1), dict(max_len=-1), dict(q_start=0), dict(n_tokens=2**23)]


def text():
    return B.load().river_last_error(None).decode()


def store(pg=None, b=None, r=None, layer=0, nq=4, q=P, qs=256, k=P, ks=128, v=P, vs=128, qo=P, qos=256):
    return B.load().river_rope_store(C.byref(pg or pages()), layer, C.byref(b or batch()), C.byref(r or rope()), nq, q, qs, k, ks, v, vs,
                                     qo, qos, None)


def attend(pg=None, b=None, layer=0, nq=4, q=P, qs=256, scale=0.0, window=0, sinks=0, out=2 * P, os=256, ws=None, n=0):
    return B.load().river_paged_attention(C.byref(pg or pages()), layer, C.byref(b or batch()), nq, q, qs, scale, window, sinks, out, os,
                                          ws, n, None, None)


@pytest.mark.parametrize("bad", BAD_PAGES, ids=str)
def test_bad_pages_are_refused_everywhere(bad):
    pg = pages(**bad)
    one = (C.c_int32 * 1)(0)
    assert store(pg) == attend(pg) == B.load().river_copy_pages(C.byref(pg), one, one, 1, None) == B.RIVER_EINVAL
    assert text()


@pytest.mark.parametrize("bad", BAD_BATCH, ids=str)
def test_bad_batches_are_refused(bad):
    assert store(b=batch(**bad)) == attend(b=batch(**bad)) == B.RIVER_EINVAL
    assert text()


@pytest.mark.parametrize("bad", [dict(layer=2), dict(layer=-1), dict(nq=0), dict(q=0), dict(k=0), dict(v=0), dict(qo=0), dict(q=P + 1),
                                 dict(qs=255), dict(ks=127), dict(vs=0), dict(qos=192), dict(qs=512)], ids=str)
def test_store_refuses(bad):
    assert store(**bad) == B.RIVER_EINVAL and text()


@pytest.mark.parametrize("bad", [dict(inv_freq=0), dict(inv_freq=P + 4), dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=66), dict(layout=2)], ids=str)
def test_store_refuses_rotary_positions(bad):
    assert store(r=rope(**bad)) == B.RIVER_EINVAL and text()


@pytest.mark.parametrize("bad", [dict(layer=2), dict(nq=0), dict(nq=3), dict(q=0), dict(out=0), dict(q=P + 8), dict(out=P + 2), dict(qs=255),
                                 dict(qs=260), dict(os=128), dict(os=257), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf),
                                 dict(window=-1), dict(sinks=-1), dict(scale=3e38), dict(out=P, q=P),
                                 dict(nq=2**16 + 2)], ids=str)
def test_attention_refuses(bad):
    assert attend(**bad) == B.RIVER_EINVAL and text()


def test_calls_without_tokens_end_at_once():
    assert store(b=batch(n_tokens=0)) == attend(b=batch(n_tokens=0)) == 0
    assert store(b=batch(n_seq=0)) == attend(b=batch(n_seq=0)) == 0
    none = batch(n_seq=0, n_tokens=0, table=0, lens=0, q_start=0)         # (empty tensors have no address)
    assert store(b=none, q=0, k=0, v=0, qo=0) == attend(b=none, q=0, out=0) == 0
    assert B.load().river_copy_pages(C.byref(pages()), None, None, 0, None) == 0


def test_null_arguments_are_refused():
    L, n = B.load(), C.c_size_t()
    assert L.river_paged_attention_workspace(None, None, 4, 0, 0, C.byref(n)) == B.RIVER_EINVAL
    assert L.river_paged_attention_workspace(C.byref(pages()), C.byref(batch()), 4, 0, 0, None) == B.RIVER_EINVAL
    assert L.river_paged_attention_workspace(C.byref(pages()), C.byref(batch()), 4, 0, 0, C.byref(n)) == 0
    assert L.river_rope_store(None, 0, None, None, 4, P, 256, P, 128, P, 128, P, 256, None) == B.RIVER_EINVAL
    assert L.river_save_pages(None, 0, 0, 1, None, None, 0) == L.river_load_pages(None, 0, 1, 0, None, None, 0) == B.RIVER_EINVAL
    for f in (L.river_pool_extend, L.river_pool_fork, L.river_pool_rewind):
        assert f(None, 0, 0) == B.RIVER_EINVAL
    assert L.river_pool_destroy(None) == 0 and L.river_pool_length(None, 0) == L.river_pool_free_pages(None) == B.RIVER_EINVAL


@pytest.mark.parametrize("src,dst", [([8], [0]), ([0], [8]), ([-1], [0]), ([0], [-1])])
def test_copies_refuse_pages_that_do_not_exist(src, dst):
    a, b = (C.c_int32 * 1)(*src), (C.c_int32 * 1)(*dst)
    assert B.load().river_copy_pages(C.byref(pages()), a, b, 1, None) == B.RIVER_EINVAL and "page" in text()
    assert B.load().river_copy_pages(C.byref(pages()), None, b, 1, None) == B.RIVER_EINVAL


# ------------------------------------------------------------------ rotary frequencies

def test_frequencies():
    rot, base, factor, orig = 128, 500000.0, 8.0, 8192.0
    f = base ** (-2.0 * np.arange(rot // 2) / rot)
    for scaling in B.ROPE_SCALINGS:
        got, m = B.river_rope_frequencies(rot, base, scaling, factor, orig, 1.0, 32.0)
        assert got.shape == (64,)
        turns = orig * f / (2 * math.pi)
        if scaling == "plain":
            want = f
        elif scaling == "linear":
            want = f / factor
        elif scaling == "base":
            want = (base * factor ** (rot / (rot - 2))) ** (-2.0 * np.arange(rot // 2) / rot)
            np.testing.assert_allclose(want[-1], f[-1] / factor, rtol=1e-12)        # what the scaling is for
        elif scaling == "bands":
            want = np.where(turns >= 32, f, np.where(turns <= 1, f / factor, 0))
            s = (turns - 1) / 31
            want = np.where(want == 0, f * s + f / factor * (1 - s), want)
        else:
            at = [rot * math.log(orig / (n * 2 * math.pi)) / (2 * math.log(base)) for n in (32.0, 1.0)]
            t = np.clip((np.arange(rot // 2) - math.floor(at[0])) / (math.ceil(at[1]) - math.floor(at[0])), 0, 1)
            want = f * (1 - t) + f / factor * t
            assert turns[np.argmax(t > 0)] < 32 < turns[0] and want[0] == f[0] and abs(want[-1] / (f[-1] / factor) - 1) < 1e-12
        np.testing.assert_allclose(got, want, rtol=1e-13)
        assert m == (np.float32(0.1 * math.log(factor) + 1) if scaling == "ramp" else 1.0)
        one, m1 = B.river_rope_frequencies(rot, base, scaling, 1.0, orig, 1.0, 32.0)     # nothing to scale
        np.testing.assert_allclose(one, f, rtol=1e-13)
        assert m1 == 1.0


def test_frequencies_pass_between_the_usual_turns_by_default():
    # bands between 1 and 4 turns, the ramp between 1 and 32 (perf/operators.py has the same)
    rot, base, factor, orig = 128, 500000.0, 8.0, 8192.0
    for scaling, high in (("bands", 4.0), ("ramp", 32.0)):
        got, m = B.river_rope_frequencies(rot, base, scaling, factor, orig)
        want, m1 = B.river_rope_frequencies(rot, base, scaling, factor, orig, 1.0, high)
        assert got.tolist() == want.tolist() and m == m1
    f = base ** (-2.0 * np.arange(rot // 2) / rot)
    got, _ = B.river_rope_frequencies(rot, base, "bands", factor, orig)
    n = orig * f / (2 * math.pi)
    s = np.clip((n - 1) / 3, 0, 1)
    np.testing.assert_allclose(got, f * s + f / factor * (1 - s), rtol=1e-13)
    assert B.river_rope_frequencies(rot, base, "bands", factor, orig, high=32.0)[0].tolist() != got.tolist()


@pytest.mark.parametrize("args", [(0, 1e4), (7, 1e4), (64, 1.0), (64, math.nan), (64, 1e4, "linear", 0.5), (64, 1e4, "linear", math.inf),
                                  (2, 1e4, "base", 2.0), (64, 1e4, "bands", 2.0, 0.0), (64, 1e4, "ramp", 2.0, 8192.0, 32.0, 1.0),
                                  (64, 1e4, "ramp", 2.0, 8192.0, 0.0, 32.0)], ids=str)
def test_frequencies_refuse(args):
    with pytest.raises(B.RiverError) as e:
        B.river_rope_frequencies(*args)
    assert e.value.code == B.RIVER_EINVAL


# ------------------------------------------------------------------ the pool

class Pool:
    """The library's pool without the device (binding.PagePool holds its state there)."""

    def __init__(self, *a):
        self.h = C.c_void_p()
        self.rc = B.load().river_pool_create(*a, C.byref(self.h))
        self.max_pages = a[3]

    def __getattr__(self, name):
        f = getattr(B.load(), "river_pool_" + name)
        return lambda *a: f(self.h, *a)

    def entries(self, s):
        out = np.empty(self.max_pages, dtype=np.int32)
        assert self.row(s, out.ctypes.data) == 0
        return out.tolist()

    def __del__(self):
        B.load().river_pool_destroy(self.h)


@pytest.mark.parametrize("a", [(0, 16, 1, 1), (1, 0, 1, 1), (1, 65537, 1, 1), (1, 16, 0, 1), (1, 16, 1, 0), (1, 65536, 1, 32768),
                               (1, 1, 2**20, 2**10), (2**28 + 1, 16, 1, 1)])
def test_pool_refuses_sizes(a):
    assert Pool(*a).rc == B.RIVER_EINVAL and text()


def test_pool_by_hand():
    p = Pool(8, 4, 3, 5)
    assert p.rc == 0 and p.free_pages() == 8 and p.length(0) == 0 and p.length(3) == p.length(-1) == B.RIVER_EINVAL
    assert p.extend(0, 6) == 0 and p.entries(0) == [0, 1, -1, -1, -1] and p.length(0) == 6 and p.free_pages() == 6
    assert p.fork(0, 1) == 0 and p.entries(1) == [0, 1, -1, -1, -1] and p.free_pages() == 6
    assert p.fork(0, 1) == B.RIVER_ESTATE and p.fork(0, 0) == p.fork(0, 3) == B.RIVER_EINVAL
    assert p.extend(1, 0) == 0 and p.entries(1) == [0, 1, -1, -1, -1]          # nothing written, nothing copied
    assert p.extend(1, 1) == 0 and p.entries(1) == [0, 2, -1, -1, -1]          # its half-full last page is its own now
    assert p.extend(0, 3) == 0 and p.entries(0) == [0, 1, 3, -1, -1]           # and the other's is shared no longer
    assert p.extend(0, 12) == B.RIVER_ENOSPC and p.length(0) == 9 and p.entries(0) == [0, 1, 3, -1, -1]
    assert p.extend(2, 17) == B.RIVER_ENOSPC and p.extend(2, 16) == 0 and p.free_pages() == 0
    assert p.extend(0, 4) == B.RIVER_ENOSPC and p.extend(0, 3) == 0
    assert p.rewind(2, 17) == p.rewind(2, -1) == B.RIVER_EINVAL
    assert p.rewind(2, 5) == 0 and p.entries(2) == [4, 5, -1, -1, -1] and p.free_pages() == 2
    assert p.rewind(2, 0) == 0 and p.free_pages() == 4 and p.entries(2) == [-1] * 5
    assert p.trim(0, 0, 0) == p.trim(0, 4, -1) == p.trim(3, 4, 0) == B.RIVER_EINVAL
    assert p.trim(0, 4, 1) == 0 and p.entries(0) == [0, -1, 3, -1, -1]         # 12 positions: the last sees 8 .. 11, and 0
    assert p.rewind(0, 6) == B.RIVER_ESTATE and p.length(0) == 12              # its page is gone
    assert p.rewind(0, 8) == 0 and p.entries(0) == [0, -1, -1, -1, -1]
    assert p.extend(0, 1) == 0 and p.entries(0) == [0, -1, 1, -1, -1]
    assert p.compact() == 0 and p.rewind(0, 0) == 0 and p.entries(1) == [0, 2, -1, -1, -1]
    assert p.compact() == 1 and p.entries(1) == [0, 1, -1, -1, -1] and p.free_pages() == 6 and p.extend(2, 1) == 0
    assert p.entries(2) == [2, -1, -1, -1, -1]
    assert p.flush(None, None, None) == B.RIVER_EINVAL and p.flush(None, P, None) == B.RIVER_EINVAL      # a copy is queued: pages are needed
    bad = pages(n_pages=9, page_stride=1024, layer_stride=9 * 1024, page_size=4)
    assert p.flush(C.byref(bad), P, None) == B.RIVER_EINVAL and "not the pool's" in text()


class Model:
    """The same bookkeeping with contents: what every sequence's positions hold, page by page."""

    def __init__(self, n, ps, seqs, most):
        self.n, self.ps, self.most = n, ps, most
        self.free, self.rows, self.len = list(range(n)), [[] for _ in range(seqs)], [0] * seqs

    def refs(self, p):
        return sum(r.count(p) for r in self.rows)

    def extend(self, s, k):
        r, ps = self.rows[s], self.ps
        need = -(-(self.len[s] + k) // ps) - len(r)
        own = k > 0 and self.len[s] % ps and self.refs(r[-1]) > 1
        if self.len[s] + k > self.most * ps or need + bool(own) > len(self.free):
            return B.RIVER_ENOSPC
        if own:
            r[-1] = heapq.heappop(self.free)
        r += [heapq.heappop(self.free) for _ in range(need)]
        self.len[s] += k
        return 0

    def drop(self, s, i, to=None):
        p, r = self.rows[s][i], self.rows[s]
        r[i] = -1
        if p >= 0 and not self.refs(p):
            heapq.heappush(self.free, p)

    def rewind(self, s, n):
        keep = -(-n // self.ps)
        if n % self.ps and self.rows[s][n // self.ps] < 0:
            return B.RIVER_ESTATE
        for i in range(keep, len(self.rows[s])):
            self.drop(s, i)
        self.rows[s], self.len[s] = self.rows[s][:keep], n
        return 0

    def fork(self, a, b):
        if self.len[b]:
            return B.RIVER_ESTATE
        self.rows[b], self.len[b] = list(self.rows[a]), self.len[a]
        return 0

    def trim(self, s, w, k):
        for i, p in enumerate(self.rows[s]):
            at = range(i * self.ps, (i + 1) * self.ps)
            if all(k <= j <= self.len[s] - 1 - w for j in at):
                self.drop(s, i)
        return 0

    def compact(self):
        used = sorted({p for r in self.rows for p in r if p >= 0})
        holes = [p for p in range(len(used)) if p not in used]
        to = dict(zip([p for p in used if p >= len(used)], holes))
        self.rows = [[to.get(p, p) for p in r] for r in self.rows]
        self.free = list(range(len(used), self.n))
        return len(to)


@pytest.mark.parametrize("seed", range(6))
def test_pool_against_a_model(seed):
    rng = random.Random(seed)
    n, ps, seqs, most = rng.choice([(12, 4, 4, 6), (40, 1, 5, 12), (9, 16, 3, 5)])
    p, m = Pool(n, ps, seqs, most), Model(n, ps, seqs, most)
    for _ in range(600):
        s = rng.randrange(seqs)
        op = rng.choice(["extend"] * 5 + ["fork", "rewind", "rewind", "trim", "compact"])
        if op == "extend":
            k = rng.randrange(0, 3 * ps)
            assert p.extend(s, k) == m.extend(s, k)
        elif op == "fork":
            t = (s + 1) % seqs
            assert p.fork(s, t) == m.fork(s, t)
        elif op == "rewind":
            k = rng.choice([0, rng.randint(0, m.len[s])])
            assert p.rewind(s, k) == m.rewind(s, k)
        elif op == "trim":
            w, k = rng.randint(1, 3 * ps), rng.choice([0, 1, ps + 1])
            assert p.trim(s, w, k) == m.trim(s, w, k)
        else:
            assert p.compact() == m.compact()
        assert p.free_pages() == len(m.free)
        for i in range(seqs):
            assert p.length(i) == m.len[i] and p.entries(i) == m.rows[i] + [-1] * (most - len(m.rows[i]))


@pytest.mark.parametrize("ps", [1, 2, 16])
@pytest.mark.parametrize("window", [1, 2**31 - 1])
def test_pool_trims_nothing_where_every_position_is_a_sink(ps, window):
    # (the first page that is no sink's is beyond every row, and beyond an int at page size 1)
    p = Pool(64, ps, 2, 32)
    assert p.extend(0, 20) == 0
    before = p.entries(0)
    for sinks in (2**31 - 1, 2**31 - 2, 2**30, 20):
        assert p.trim(0, window, sinks) == 0 and p.entries(0) == before
    assert p.trim(0, 2**31 - 1, 0) == 0 and p.entries(0) == before


def test_the_binding_is_imported_where_torch_has_no_gpu_part():
    # (a torch built for the CPU: the byte model, the configurations and the host calls are of use there)
    code = ("import torch\n"
            "for name in [n for n in dir(torch._C) if n.startswith('_cuda_')]: delattr(torch._C, name)\n"
            "from paper_2604_18396_amd import binding as B\n"
            "assert B.river_rope_frequencies(4, 100.0)[0].tolist() == [1.0, 0.1]\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([sys.executable, "-c", code], check=True, cwd=root, timeout=300)


def test_threads_of_one_stream_share_its_tickets(monkeypatch):
    # another thread's first call comes in while this one's is making its tensor: both use the one that is kept
    made, others = [], []

    def zeros(n, dtype, device):
        a = np.zeros(n, dtype=np.int32)
        made.append(a)
        if len(made) == 1:
            others.append(B._tickets(0, 77))
        return Tensor(a)

    class Tensor:
        def __init__(self, a):
            self.a = a

        def data_ptr(self):
            return self.a.ctypes.data

    monkeypatch.setattr(B.torch._C, "_cuda_isCurrentStreamCapturing", lambda: False, raising=False)
    monkeypatch.setattr(B.torch, "zeros", zeros)
    monkeypatch.setattr(B, "_ticket_tensors", {})
    mine = B._tickets(0, 77)
    assert others == [mine] and B._tickets(0, 77) == mine and B._ticket_tensors[(0, 77)].data_ptr() == mine
    assert B._tickets(0, 78) != mine


def test_a_context_refuses_pages_of_another_device():
    # (its kernels would read another GPU's addresses; stand-ins for both, the call must not come as far as the library)
    r = B.River.__new__(B.River)
    r._h, r.workspace = None, B.torch.empty(1)
    pg = types.SimpleNamespace(device=B.torch.device("meta"), index=1, ref=None)
    row = B.torch.empty(3, dtype=B.torch.int32, device="meta")
    with pytest.raises(ValueError, match="different devices"):
        r.save_pages(pg, row, 1)
    with pytest.raises(ValueError, match="different devices"):
        r.load_pages(pg, row, 1, 0)
