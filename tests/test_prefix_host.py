"""The host side of a step laid out on the device and of attention with common prefixes: refused arguments, workspaces (no GPU)."""
import ctypes as C
import types

import pytest

from paper_2604_18396_amd import binding as B
from test_pages_host import BAD_BATCH, BAD_PAGES, P, batch, pages, text


def prefixes(**kw):
    d = dict(table=P, lens=P, seq_start=P, n_groups=2, max_pages=4, table_stride=4, max_len=64, max_seqs=2)
    d.update(kw)
    return B.river_prefixes(*(d[f] for f, _ in B.river_prefixes._fields_))


def tables(**kw):
    d = dict(table=P, lens=P, lens_out=P, free_pages=P, n_free=P, n_free_out=P, n_shared=0, n_seq=2, max_pages=4, table_stride=4, n_pages=8, page_size=16)
    d.update(kw)
    return B.river_tables(*(d[f] for f, _ in B.river_tables._fields_))


def attend(pg=None, b=None, x=None, layer=0, nq=4, q=P, qs=256, scale=0.0, out=2 * P, os=256, ws=None, n=0, tickets=None):
    return B.load().river_prefix_attention(C.byref(pg or pages()), layer, C.byref(b or batch()), C.byref(x or prefixes()), nq, q, qs, scale, out, os,
                                           ws, n, tickets, None)


def store(pg=None, layer=0, slots=P, n=4, k=P, ks=128, v=P, vs=128):
    return B.load().river_store_slots(C.byref(pg or pages()), layer, slots, n, k, ks, v, vs, None)


def build(t=None, n_new=P, n_tokens=4, q_start=P, slots=P, positions=P, refused=P):
    return B.load().river_build_batch(C.byref(t or tables()), n_new, n_tokens, q_start, slots, positions, refused, None)


def workspace(pg=None, b=None, x=None, nq=4):
    n = C.c_size_t()
    rc = B.load().river_prefix_attention_workspace(C.byref(pg or pages()), C.byref(b or batch()), C.byref(x or prefixes()), nq, C.byref(n))
    return rc or n.value


@pytest.mark.parametrize("bad", BAD_PAGES, ids=str)
def test_bad_pages_are_refused(bad):
    assert attend(pages(**bad)) == store(pages(**bad)) == workspace(pages(**bad)) == B.RIVER_EINVAL and text()


@pytest.mark.parametrize("bad", BAD_BATCH, ids=str)
def test_bad_batches_are_refused(bad):
    assert attend(b=batch(**bad)) == workspace(b=batch(**bad)) == B.RIVER_EINVAL and text()


@pytest.mark.parametrize("bad", [dict(table=0), dict(lens=0), dict(seq_start=0), dict(table=P + 1), dict(lens=P + 2), dict(seq_start=P + 3), dict(n_groups=-1),
                                 dict(n_groups=2**23), dict(max_pages=0), dict(table_stride=3), dict(max_len=-1), dict(max_seqs=-1)], ids=str)
def test_bad_prefixes_are_refused(bad):
    assert attend(x=prefixes(**bad)) == workspace(x=prefixes(**bad)) == B.RIVER_EINVAL and text()


BIG = prefixes(max_pages=1 << 20, table_stride=1 << 20, max_len=1 << 20)        # (a prefix that pays: it has parts, which need a workspace)


@pytest.mark.parametrize("bad", [dict(layer=-1), dict(layer=2), dict(nq=0), dict(nq=3), dict(nq=65538), dict(q=0), dict(out=0), dict(q=P + 8), dict(out=P + 4),
                                 dict(qs=255), dict(qs=260), dict(os=128), dict(out=P), dict(scale=-1.0), dict(scale=float("nan")),
                                 dict(scale=float("inf")), dict(scale=3e38), dict(x=BIG, ws=None, n=1 << 30), dict(x=BIG, ws=P + 8, n=1 << 30), dict(x=BIG, ws=P, n=1 << 30, tickets=P + 2)], ids=str)
def test_attention_refuses(bad):
    assert attend(**bad) == B.RIVER_EINVAL and text()


def test_a_workspace_that_is_too_small_is_refused():
    n = workspace(x=BIG)
    assert n > 0
    assert attend(x=BIG, ws=P, n=n - 1) == B.RIVER_ENOSPC and "workspace" in text()


def test_workspaces():
    # what nothing shares, or too little to pay, and nothing splits needs none; what is shared has a part of each row for the prefix and one of
    # its own at least
    assert workspace(x=prefixes(n_groups=0, table=0, lens=0, seq_start=0)) == 0
    assert workspace(x=prefixes(max_seqs=1)) == 0
    assert workspace() == 0
    assert workspace(x=BIG) >= 4 * 4 * 2 * (64 * 4 + 8)
    assert workspace(x=BIG, nq=8) == 2 * workspace(x=BIG)
    assert workspace(b=batch(n_tokens=0)) >= 0


def test_calls_without_tokens_end_at_once():
    assert attend(b=batch(n_tokens=0)) == attend(b=batch(n_seq=0)) == store(n=0, slots=0, k=0, v=0) == B.RIVER_OK


def test_calls_that_are_too_large_are_refused():
    assert attend(b=batch(n_tokens=1 << 22, max_new=1 << 22), nq=64, qs=4096, os=4096) == B.RIVER_EINVAL and "too many" in text()
    pg = pages(n_kv_heads=8, page_size=1, page_stride=512, layer_stride=8 * 512)
    assert attend(pg, batch(n_seq=1 << 22, n_tokens=1 << 22, max_new=1), BIG, nq=8, qs=512, os=512, ws=P, n=1 << 62) == B.RIVER_EINVAL
    assert "too many" in text()


@pytest.mark.parametrize("bad", [dict(layer=2), dict(layer=-1), dict(n=-1), dict(n=2**23), dict(slots=0), dict(k=0), dict(v=0), dict(slots=P + 4), dict(k=P + 1),
                                 dict(v=P + 1), dict(ks=127), dict(vs=0)], ids=str)
def test_store_refuses(bad):
    assert store(**bad) == B.RIVER_EINVAL and text()


def test_store_refuses_more_heads_than_it_counts():
    assert store(pages(n_kv_heads=8192, page_size=1, page_stride=8192 * 64, layer_stride=8 * 8192 * 64), ks=8192 * 64, vs=8192 * 64) == B.RIVER_EINVAL


@pytest.mark.parametrize("bad", [dict(n_seq=-1), dict(n_seq=4097), dict(n_pages=0), dict(n_pages=2**29), dict(page_size=0), dict(page_size=65537),
                                 dict(max_pages=0), dict(table_stride=3), dict(table=0), dict(lens=0), dict(lens_out=0), dict(free_pages=0), dict(n_free=0),
                                 dict(n_free_out=0), dict(table=P + 2), dict(lens=P + 1), dict(free_pages=P + 2), dict(n_shared=P + 2)], ids=str)
def test_build_refuses_tables(bad):
    assert build(tables(**bad)) == B.RIVER_EINVAL and text()


@pytest.mark.parametrize("bad", [dict(n_new=0), dict(n_tokens=-1), dict(n_tokens=2**23), dict(q_start=0), dict(q_start=P + 2), dict(slots=P + 4),
                                 dict(positions=P + 2), dict(refused=P + 1), dict(n_new=P + 2)], ids=str)
def test_build_refuses(bad):
    assert build(**bad) == B.RIVER_EINVAL and text()


def test_null_structs_are_refused():
    L, n = B.load(), C.c_size_t()
    assert L.river_build_batch(None, P, 4, P, P, P, P, None) == B.RIVER_EINVAL
    assert L.river_store_slots(None, 0, P, 4, P, 128, P, 128, None) == B.RIVER_EINVAL
    assert L.river_prefix_attention(C.byref(pages()), 0, C.byref(batch()), None, 4, P, 256, 0.0, 2 * P, 256, None, 0, None, None) == B.RIVER_EINVAL
    assert L.river_prefix_attention(C.byref(pages()), 0, None, C.byref(prefixes()), 4, P, 256, 0.0, 2 * P, 256, None, 0, None, None) == B.RIVER_EINVAL
    assert L.river_prefix_attention_workspace(C.byref(pages()), C.byref(batch()), C.byref(prefixes()), 4, None) == B.RIVER_EINVAL
    assert L.river_prefix_attention_workspace(C.byref(pages()), C.byref(batch()), None, 4, C.byref(n)) == B.RIVER_EINVAL


def test_the_binding_refuses_prefixes_of_another_device(monkeypatch):
    monkeypatch.setattr(B, "_device", lambda: 0)
    with pytest.raises(ValueError, match="different devices"):
        B.river_prefix_attention(types.SimpleNamespace(index=0), 0, None, types.SimpleNamespace(index=1), None)


def test_handles_ask_for_device_tensors():
    import torch
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)
    with pytest.raises(ValueError):
        B.Prefixes(i32(2, 3), i32(2), i32(3))
    with pytest.raises(ValueError):
        B.Tables(i32(2, 3), i32(2), i32(8), i32(1), 16)


def test_build_refuses_more_entries_than_it_counts():
    # pages given back are counted up to 2^30: more of them would stay in their rows
    assert build(tables(n_seq=4096, max_pages=2**18 + 1, table_stride=2**18 + 1)) == B.RIVER_EINVAL and "entries" in text()
    assert build(tables(n_seq=2, max_pages=2**29 + 1, table_stride=2**29 + 1)) == B.RIVER_EINVAL and "entries" in text()
