"""What the entry points on caller-held buffers refuse: checked on the host, before anything is enqueued, so no device is needed
(the addresses below are never followed)."""
import ctypes as C
import struct

import pytest

from paper_2407_19947_b200 import build as stairs_build
from paper_2407_19947_b200 import stairs as st

P = 0x10000   # stands for a device address
EINVAL, ENOSPC, EUNSUPPORTED = 1, 2, 6


@pytest.fixture(scope="module")
def lib():
    stairs_build.build()
    return st.load_library()


def cache(**kw):
    c = st.CPaged(P, P, 64 * 128, 128, 64, 4, 16, 2, 64, 1)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def said(lib, rc, want, text):
    assert rc == want and text in lib.stairs_last_error(None).decode()


@pytest.mark.parametrize("bad, code, text", [
    (dict(n_req=0), ENOSPC, "n_req"), (dict(n_req=4097), ENOSPC, "n_req"), (dict(n_seq=None), EINVAL, "NULL"), (dict(n_new=None), EINVAL, "NULL"),
    (dict(table=None), EINVAL, "NULL"), (dict(free=None), EINVAL, "NULL"), (dict(slot=None), EINVAL, "NULL"), (dict(served=None), EINVAL, "NULL"),
    (dict(page=0), EINVAL, "page_tokens"), (dict(blocks=0), EINVAL, "max_blocks"), (dict(blocks=1 << 27, page=16), EINVAL, "31 bits"),
    (dict(n_free=-1), EINVAL, "n_free"), (dict(rows=-1), EINVAL, "max_rows"), (dict(rows=2**31 - 1), EINVAL, "max_rows"),
    (dict(blocks_out=P + 4), EINVAL, "output is its input"), (dict(used_out=P + 8), EINVAL, "output is its input"),
    (dict(kv=P + 4), EINVAL, "output is its input"), (dict(off=P), EINVAL, "output is its input"),
    (dict(kv=P + 2), EINVAL, "aligned"), (dict(slot=P + 4), EINVAL, "aligned")])
def test_tables_refusals(lib, bad, code, text):
    a = dict(n_req=2, n_seq=P, n_new=P, blocks_in=P + 4, table=P, blocks=8, page=16, free=P, n_free=4, used_in=P + 8, rows=10, blocks_out=P + 12,
             used_out=P + 16, off=P + 20, kv=P + 40, req=P, pos=P, slot=P, served=P)
    a.update(bad)
    said(lib, lib.stairs_tables_static(*a.values(), None), code, text)


@pytest.mark.parametrize("bad, code, text", [
    (dict(c=None), EINVAL, "NULL"), (dict(c=cache(k_dev=None)), EINVAL, "NULL"), (dict(c=cache(dtype=3)), EINVAL, "dtype"), (dict(c=cache(head_dim=0)), EINVAL, "heads of 0"),
    (dict(c=cache(head_dim=257)), EUNSUPPORTED, "head_dim"), (dict(c=cache(page_stride=-1)), EINVAL, "stride"), (dict(c=cache(n_pages=0)), EINVAL, "pages"),
    (dict(rows=-1), EINVAL, "n_rows"), (dict(k=None), EINVAL, "NULL"), (dict(dtype=-1), EINVAL, "dtype"), (dict(row_stride=-2), EINVAL, "stride"), (dict(slot=None), EINVAL, "NULL"),
    (dict(k=P + 1), EINVAL, "aligned"), (dict(slot=P + 4), EINVAL, "aligned"), (dict(c=cache(v_dev=P + 1)), EINVAL, "aligned")])
def test_append_refusals(lib, bad, code, text):
    a = dict(c=cache(), rows=3, k=P, v=P, dtype=1, row_stride=128, head_stride=64, slot=P)
    a.update(bad)
    a["c"] = C.byref(a["c"]) if a["c"] is not None else None
    said(lib, lib.stairs_append_static(*a.values(), None), code, text)


def attend(lib, **bad):
    a = dict(c=cache(), table=P, blocks=8, n_req=2, off=P, kv=P, max_len=0, rows=3, heads=4, q=P, q_row=256, q_head=64, scale=0.125, o=P + 4096, o_row=256,
             o_head=64, ws=1 << 20, ws_bytes=1 << 40)
    a.update(bad)
    a["c"] = C.byref(a["c"]) if a["c"] is not None else None
    return lib.stairs_attend_static(*a.values(), None)


@pytest.mark.parametrize("bad, code, text", [
    (dict(c=None), EINVAL, "NULL"), (dict(table=None), EINVAL, "NULL"), (dict(off=None), EINVAL, "NULL"), (dict(q=None), EINVAL, "NULL"), (dict(o=None), EINVAL, "NULL"),
    (dict(n_req=0), ENOSPC, "n_req"), (dict(n_req=4097), ENOSPC, "n_req"), (dict(blocks=0), EINVAL, "max_blocks"), (dict(blocks=1 << 27), EINVAL, "max_blocks"),
    (dict(max_len=-1), EINVAL, "max_len"), (dict(rows=-1), EINVAL, "n_rows"), (dict(q_row=-1), EINVAL, "stride"), (dict(heads=3), EINVAL, "heads"),
    (dict(heads=0), EINVAL, "heads"), (dict(scale=float("nan")), EINVAL, "scale"), (dict(scale=float("inf")), EINVAL, "scale"), (dict(rows=1 << 30), ENOSPC, "rows"),
    (dict(c=cache(head_dim=264)), EUNSUPPORTED, "head_dim"), (dict(q=P + 1), EINVAL, "aligned"), (dict(o=P + 1), EINVAL, "aligned"), (dict(kv=P + 2), EINVAL, "aligned"),
    (dict(rows=4096, ws=None), EINVAL, "scratch"), (dict(rows=4096, ws=(1 << 20) + 64), EINVAL, "scratch"), (dict(rows=4096, ws_bytes=1000), ENOSPC, "scratch"),
    (dict(n_req=300, ws=None), EINVAL, "scratch"), (dict(n_req=300, ws_bytes=1000), ENOSPC, "scratch")])
def test_attend_refusals(lib, bad, code, text):
    said(lib, attend(lib, **bad), code, text)


def test_attend_scratch_grows_with_what_is_unknown(lib):
    c = cache(n_pages=64)
    ask = lambda rows, n, length: lib.stairs_attend_workspace_bytes(C.byref(c), 4, n, rows, length)  # noqa: E731
    assert ask(1, 1, 128) == 0                       # a small call needs none
    assert ask(1, 1, 0) > 0 and ask(4096, 1, 128) > 0
    assert ask(1, 1, -1) == 0 and ask(0, 1, 1) == 0 and lib.stairs_attend_workspace_bytes(C.byref(c), 3, 1, 1, 1) == 0
    for rows in (1, 9, 40, 300):                     # what is enough for a bound is enough for a smaller one, 0 standing for any
        assert ask(rows, 3, 0) >= ask(rows, 3, 100000) >= ask(rows, 3, 1000) >= ask(rows, 3, 10) >= 0


def test_calls_of_no_rows_enqueue_nothing(lib):
    assert attend(lib, rows=0, q=None, o=None) == 0
    c = cache()
    assert lib.stairs_append_static(C.byref(c), 0, None, None, 1, 0, 0, None, None) == 0
    assert lib.stairs_attend_workspace_bytes(None, 4, 1, 1, 0) == 0


@pytest.mark.parametrize("bad, code, text", [
    (dict(logits=None), EINVAL, "NULL"), (dict(u=None), EINVAL, "NULL"), (dict(dtype=5), EINVAL, "dtype"), (dict(vocab=0), EINVAL, "vocab"), (dict(ld=99), EINVAL, "ld"),
    (dict(vocab=(1 << 20) + 1, ld=1 << 21), EUNSUPPORTED, "2^20"), (dict(logits=P + 2, dtype=0), EINVAL, "aligned"), (dict(u=P + 2), EINVAL, "aligned"), (dict(n=0), ENOSPC, "n_req"), (dict(n=257), ENOSPC, "n_req"),
    (dict(k_max=64), EINVAL, "k_max"), (dict(k=5), EINVAL, "k[1]"), (dict(k=-1), EINVAL, "k[1]"), (dict(draft=None), EINVAL, "draft_dev"),
    (dict(t=-0.5), EINVAL, "temperature[1]"), (dict(t=float("nan")), EINVAL, "temperature[1]"), (dict(t=1e-7), EINVAL, "temperature[1]"), (dict(t=float("inf")), EINVAL, "temperature[1]"),
    (dict(top_k=-1), EINVAL, "top_k[1]"), (dict(top_p=0.0), EINVAL, "top_p[1]"), (dict(top_p=1.5), EINVAL, "top_p[1]"), (dict(top_p=float("nan")), EINVAL, "top_p[1]"),
    (dict(min_p=-0.1), EINVAL, "min_p[1]"), (dict(min_p=1.1), EINVAL, "min_p[1]"), (dict(min_p=float("nan")), EINVAL, "min_p[1]")])
def test_sample_refusals(lib, bad, code, text):
    a = dict(logits=P, dtype=1, vocab=100, ld=100, n=2, k=2, t=1.0, top_k=0, top_p=1.0, min_p=0.0, u=P, draft=P, k_max=4)
    a.update(bad)
    m = max(a["n"], 2)
    k = (C.c_int32 * m)(*([2, a["k"]] + [2] * (m - 2)))
    s = (st.CSampling * m)(*([(1.0, 0, 1.0, 0.0), (a["t"], a["top_k"], a["top_p"], a["min_p"])] + [(1.0, 0, 1.0, 0.0)] * (m - 2)))
    said(lib, lib.stairs_sample_static(a["logits"], a["dtype"], a["vocab"], a["ld"], a["n"], k, s, a["u"], a["draft"], a["k_max"], P, P, None), code, text)


def test_sample_refuses_more_rows_than_it_takes(lib):
    k, s = (C.c_int32 * 64)(*[16] * 64), (st.CSampling * 64)(*[(1.0, 0, 1.0, 0.0)] * 64)
    said(lib, lib.stairs_sample_static(P, 1, 100, 100, 64, k, s, P, P, 16, P, P, None), ENOSPC, "rows")


def test_binding_refuses_tensors_that_do_not_fit():
    import torch
    z = torch.zeros
    with pytest.raises(ValueError, match="CUDA device"):
        st.sample_static(z(1, 8), [0], None, 0, z(1))
    with pytest.raises(ValueError, match="top_p"):
        st._settings(2, 1.0, 0, [0.5], 0.0)
    with pytest.raises(ValueError, match="alike"):
        st._paged(z(2, 4, 1, 8), z(2, 4, 1, 16))
    with pytest.raises(ValueError, match="next to each other"):
        st._paged(z(2, 4, 8, 3).transpose(2, 3), z(2, 4, 8, 3).transpose(2, 3))
    with pytest.raises(ValueError, match="not supported"):
        st._dtype_code(z(1, dtype=torch.float64))


def test_binding_packs_the_structures_of_the_header():
    # the hand-packed structures against the ctypes ones, field by field
    import torch
    k, v = torch.zeros(3, 16, 2, 8, dtype=torch.float16), torch.zeros(3, 16, 2, 8, dtype=torch.float16)
    raw, heads, hd = st._paged(k.transpose(1, 2).contiguous().transpose(1, 2), v.transpose(1, 2).contiguous().transpose(1, 2))
    c = st.CPaged.from_buffer_copy(raw)
    assert (c.page_stride, c.token_stride, c.head_stride, c.n_pages, c.page_tokens, c.n_kv_heads, c.head_dim, c.dtype) == (256, 8, 128, 3, 16, 2, 8, 2)
    assert (heads, hd) == (2, 8)
    one = (st.CSampling * 3).from_buffer_copy(st._settings(3, 0.5, 7, 0.25, 0.125))
    many = (st.CSampling * 3).from_buffer_copy(st._settings(3, [0.5, 1.0, 2], 7, [0.25] * 3, 0.125))
    assert [(s.temperature, s.top_k, s.top_p, s.min_p) for s in one] == [(0.5, 7, 0.25, 0.125)] * 3
    assert [(s.temperature, s.top_k, s.top_p, s.min_p) for s in many] == [(0.5, 7, 0.25, 0.125), (1.0, 7, 0.25, 0.125), (2.0, 7, 0.25, 0.125)]
    for bad in ([1], 1.5, "x", 2**31):
        with pytest.raises((ValueError, TypeError, struct.error)):
            st._settings(3, 1.0, bad, 1.0, 0.0)
