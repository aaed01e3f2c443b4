"""The operators on caller-held buffers against plain 64-bit implementations (tests/operator_util.py)."""
import itertools
import math
import threading

import numpy as np
import pytest
import torch

from tests import operator_util as ou

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def st():
    from paper_2407_19947_b200 import build, stairs
    build.build()
    return stairs


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------------------------------------
# tables
# ------------------------------------------------------------------------------------------------
def check_tables(st, seq, new, had, table, free, used, page, max_rows):
    want = ou.tables_ref(seq, new, had, table, free, used, page, max_rows)
    t = i32(table)
    got = st.tables_static(i32(seq), i32(new), i32(had), t, i32(free), i32([used]), page_tokens=page, max_rows=max_rows)
    for name, v in got._asdict().items():
        assert v.tolist() == want[name], name
    assert t.tolist() == want["table"]


@pytest.mark.parametrize("n,page,seed", [(1, 16, 0), (3, 1, 1), (31, 7, 2), (33, 64, 3), (512, 16, 4), (513, 128, 5), (1024, 32, 6), (4096, 16, 7)])
def test_tables(st, n, page, seed):
    rng = np.random.default_rng(seed)
    seq, new = rng.integers(0, 300, n), rng.integers(-1, 12, n)          # (a negative number of new tokens is none)
    new[rng.random(n) < 0.2] = 0
    had = -(-seq // page) + rng.integers(0, 2, n)                        # some hold a page more than they need
    blocks = int(max(had.max(), (-(-(seq + 12) // page)).max())) + 1
    table = rng.integers(0, 1 << 20, (n, blocks))
    table[:, 0] = np.where(rng.random(n) < 0.1, -1, table[:, 0])         # (a page that is none gives slots that are none)
    free = rng.permutation(1 << 16)
    rows = int(np.maximum(new, 0).sum())
    args = [v.tolist() for v in (seq, new, had, table, free)]
    check_tables(st, *args, 5, page, rows + 3)
    check_tables(st, *args, 5, page, max(rows - 1, 0))                   # a row too few: the last requests wait
    check_tables(st, *args, len(free) - 2, page, rows + 3)               # two pages left
    check_tables(st, *args, len(free), page, rows)
    check_tables(st, *args, len(free) + 4, page, rows)                   # a count beyond the list
    check_tables(st, *args, -1, page, rows)


def test_tables_stop_at_lengths_that_are_none(st):
    for bad in (dict(seq=[4, -1, 4]), dict(had=[1, 9, 1]), dict(had=[1, -2, 1]), dict(new=[3, 200, 1]), dict(seq=[4, 2**31 - 1, 4]), dict(new=[1, 2**31 - 1, 1]), dict(seq=[-5, 4, 4])):
        a = dict(seq=[4, 4, 4], new=[3, 2, 1], had=[1, 1, 1])
        a.update(bad)
        table = [[7, -1, -1], [8, -1, -1], [9, -1, -1]]
        # (the reference's kv_len of a request that is not served is its n_seq)
        check_tables(st, a["seq"], a["new"], a["had"], table, [1, 2, 3], 0, 4, 40)
    check_tables(st, [0], [0], [0], [[-1]], [], 0, 16, 0)
    check_tables(st, [0, 3], [0, 0], [0, 0], [[-1], [-1]], [5], 0, 16, 0)


# ------------------------------------------------------------------------------------------------
# append
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("src", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("dst", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("heads,hd,layout,shift", [(2, 64, "NHD", 0), (5, 80, "HND", 0), (1, 128, "NHD", 1), (3, 7, "HND", 0), (2, 1, "NHD", 0), (4, 256, "HND", 0), (2, 20, "NHD", 0)])
def test_append(st, src, dst, heads, hd, layout, shift):
    g, pages, page, rows = gen(hd), 9, 16, 37
    x = torch.randn((rows, 2 * heads + 1, hd + shift), generator=g, device=DEV) * 3
    x[0, 0, 0], x[1, 0, 0], x[2, 0, 0] = math.inf, math.nan, 1e6        # (1e6: infinity in fp16)
    x = x.to(DTYPES[src])[:, :, shift:]
    k_new, v_new = x[:, :heads], x[:, heads: 2 * heads]
    mem = (2, pages, page, heads, hd + shift) if layout == "NHD" else (2, pages, heads, page, hd + shift)
    store = torch.randn(mem, generator=g, device=DEV).to(DTYPES[dst])
    views = [s[..., shift:] if layout == "NHD" else s[..., shift:].transpose(1, 2) for s in store]
    want = store.clone()
    wv = [s[..., shift:] if layout == "NHD" else s[..., shift:].transpose(1, 2) for s in want]
    slot = torch.randperm(pages * page, generator=g, device=DEV)[:rows]
    slot[5], slot[9], slot[11], slot[13] = -1, pages * page, 1 << 40, -(1 << 40)   # no slots
    for t, s in enumerate(slot.tolist()):
        if 0 <= s < pages * page:
            for w, new in zip(wv, (k_new, v_new)):
                w[s // page, s % page] = new[t].to(DTYPES[dst])
    st.append_static(k_new, v_new, views[0], views[1], slot)
    bits = torch.int32 if dst == "fp32" else torch.int16
    a, b = store, want
    same = (a.view(bits) == b.view(bits)) | (torch.isnan(a) & torch.isnan(b))
    assert bool(same.all())
    if src == dst:
        assert torch.equal(a.view(bits), b.view(bits))


def test_append_of_no_rows_and_refusals(st):
    c = torch.zeros((2, 4, 2, 8), device=DEV)
    e = torch.zeros((0, 2, 8), device=DEV)
    st.append_static(e, e, c, c.clone(), torch.zeros(0, dtype=torch.int64, device=DEV))
    k = torch.zeros((3, 2, 8), device=DEV)
    slot = torch.zeros(3, dtype=torch.int64, device=DEV)
    for bad in ((k, k, c, c[:, :, :1], slot), (k[:, :1], k[:, :1], c, c, slot), (k, k, c, c, slot[:2]), (k, k, c, c, slot.int()), (k, k.half(), c, c, slot),
                (k.cpu(), k, c, c, slot), (k.double(), k.double(), c, c, slot)):
        with pytest.raises(ValueError):
            st.append_static(*bad)


# ------------------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------------------
class Paged:
    """A pool whose pages lie in a random order, NaN wherever no request has a token."""

    def __init__(self, seed, dtype, hkv, hd, page, lens, layout="NHD", spare=3, shift=0):
        g = gen(seed)
        blocks = [-(-n // page) for n in lens]
        self.pages = sum(blocks) + spare
        pad = 16 // (4 if dtype == torch.float32 else 2) if shift == 0 else shift
        mem = (2, self.pages, page, hkv, hd + pad) if layout == "NHD" else (2, self.pages, hkv, page, hd + pad)
        store = torch.full(mem, math.nan, device=DEV, dtype=dtype)
        cut = (lambda s: s[..., shift:shift + hd]) if layout == "NHD" else (lambda s: s[..., shift:shift + hd].transpose(1, 2))
        self.k, self.v = cut(store[0]), cut(store[1])
        order = torch.randperm(self.pages, generator=g, device=DEV).tolist()
        self.table = torch.full((len(lens), max(blocks + [1]) + 1), -1, dtype=torch.int32, device=DEV)
        at = 0
        for r, n in enumerate(lens):
            mine = order[at: at + blocks[r]]
            at += blocks[r]
            self.table[r, : blocks[r]] = i32(mine)
            for c in (self.k, self.v):
                rows = torch.randn((blocks[r] * page, hkv, hd), generator=g, device=DEV).to(dtype)
                rows[n:] = math.nan
                if mine:
                    c[torch.tensor(mine, device=DEV)] = rows.view(blocks[r], page, hkv, hd)
        self.g = g


def check_attend(st, p, q, new, lens, scale=None, slack=0, max_len=0, out=None, rows_of=None):
    rows = sum(new)
    off, kv = i32(np.concatenate([[0], np.cumsum(new)]).tolist()), i32(lens)
    mark = 7.25
    if out is None:
        out = torch.full((rows + slack, q.shape[1], q.shape[2]), mark, dtype=q.dtype, device=DEV)
    s = scale if scale is not None else q.shape[2] ** -0.5
    padded = torch.cat([q, q[:slack]])                                   # (slack: rows behind the last request's)
    got = st.attend_static(padded if slack else q, p.k, p.v, p.table, off, kv, scale=scale, out=out, max_len=max_len)
    assert got is out
    torch.cuda.synchronize()
    want, tol = ou.attend_ref(q, p.k, p.v, p.table, off, kv, s, max_len or None, rows_of)
    asked = ~torch.isnan(want[:rows])
    assert bool((out[rows:] == mark).all()), "rows of no request were written"
    err = (out[:rows].double() - want[:rows]).abs()
    bad = asked & ~(err <= tol[:rows])
    assert not bool(bad.any()), (float(err[bad].max()) if bool(torch.isfinite(err[bad]).any()) else "NaN", int(bad.sum()), [int(v) for v in bad.nonzero()[0]])
    return out


SHAPES = [(4, 4, 64), (32, 8, 128), (8, 8, 80), (8, 1, 128), (6, 2, 16), (12, 4, 40), (4, 2, 96), (3, 3, 8), (2, 1, 256), (5, 5, 24), (4, 2, 192), (16, 1, 32), (64, 1, 64), (3, 1, 20), (2, 2, 7), (6, 3, 1)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("heads,hkv,hd", SHAPES)
def test_attend_shapes(st, dtype, heads, hkv, hd):
    lens, new = [1, 2, 17, 64, 65, 130, 300], [1, 2, 1, 9, 5, 0, 17]
    for layout, page in (("NHD", 16), ("HND", 64)):
        p = Paged(heads + hd, DTYPES[dtype], hkv, hd, page, lens, layout)
        q = (torch.randn((sum(new), heads, hd), generator=p.g, device=DEV) * 1.5).to(DTYPES[dtype])
        check_attend(st, p, q, new, lens)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("page", [1, 5, 16, 48, 128, 1000])
def test_attend_pages(st, dtype, page):
    lens, new = [3, 127, 1, 128, 129, 700, 999], [3, 2, 1, 64, 33, 1, 9]
    p = Paged(page, DTYPES[dtype], 2, 64, page, lens)
    q = torch.randn((sum(new), 8, 64), generator=p.g, device=DEV).to(DTYPES[dtype])
    check_attend(st, p, q, new, lens, scale=0.3)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("heads,hkv,hd,new,length", [(32, 8, 128, 1, 5000), (16, 16, 64, 9, 2057), (8, 2, 128, 200, 1000), (8, 2, 64, 129, 129), (4, 4, 80, 130, 700),
                                                     (8, 1, 128, 77, 1234), (4, 2, 96, 140, 300), (8, 8, 128, 257, 257), (2, 1, 64, 1000, 1600), (4, 4, 32, 150, 150)])
def test_attend_long_and_wide(st, dtype, heads, hkv, hd, new, length):
    p = Paged(new + length, DTYPES[dtype], hkv, hd, 64, [length])
    q = (torch.randn((new, heads, hd), generator=p.g, device=DEV) * 1.5).to(DTYPES[dtype])
    check_attend(st, p, q, [new], [length])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,hkv,hd,n,new,length", [(16, 8, 128, 6, 20, 5000), (32, 8, 128, 4, 9, 9000), (12, 12, 64, 12, 40, 3000), (8, 4, 80, 20, 33, 2500),
                                                       (8, 8, 128, 3, 600, 2500), (16, 16, 64, 2, 700, 1500), (4, 4, 128, 40, 140, 900)])
def test_attend_long_parts(st, dtype, heads, hkv, hd, n, new, length):
    # a CTA's share is long: dozens of chunks before the ones that some row does not see, several units
    lens = [length - (37 if n < 40 else 7) * r for r in range(n)]
    p = Paged(n + new, DTYPES[dtype], hkv, hd, 64, lens)
    q = (torch.randn((n * new, heads, hd), generator=p.g, device=DEV) * 1.5).to(DTYPES[dtype])
    check_attend(st, p, q, [new] * n, lens, rows_of=lambda t: t % 7 == 0 or t % new >= new - 2)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_attend_many_requests_of_every_length(st, dtype):
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 400, 150).tolist()
    new = [int(min(n, rng.integers(0, 12))) for n in lens]
    new[7], lens[7] = 120, 380                                           # one prompt chunk among single steps
    p = Paged(3, DTYPES[dtype], 2, 64, 16, lens, "HND")
    q = torch.randn((sum(new), 4, 64), generator=p.g, device=DEV).to(DTYPES[dtype])
    check_attend(st, p, q, new, lens)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n,hd,new", [(100, 64, 1), (40, 128, 3), (200, 32, 2)])
def test_attend_many_short_requests_of_one_key_head(st, dtype, n, hd, new):
    rng = np.random.default_rng(n)
    lens = rng.integers(1, 200, n).tolist()
    rows = [int(min(a, rng.integers(0, new + 1))) for a in lens]
    p = Paged(n, DTYPES[dtype], 1, hd, 32, lens)
    q = torch.randn((sum(rows), 4, hd), generator=p.g, device=DEV).to(DTYPES[dtype])
    check_attend(st, p, q, rows, lens, max_len=max(lens))
    check_attend(st, p, q, rows, lens, max_len=1 << 20, scale=-0.2)
    check_attend(st, p, q, rows, lens, scale=0.0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("hd,new", [(64, 5), (128, 5), (128, 150), (64, 150)])
def test_attend_rows_that_see_nothing(st, dtype, hd, new):
    # fewer tokens than new rows (the first rows lie before position 0), none at all, and tables without a page
    lens, rows = [3, 0, 20, 40], [new, 4, 4, 4]
    p = Paged(1, DTYPES[dtype], 1, hd, 16, [40, 40, 40, 40])
    p.table[2] = -1
    p.table[3, 1], p.table[3, 2] = p.pages, 1 << 30                      # beyond the pool: only the first page is seen
    q = torch.randn((sum(rows), 2, hd), generator=p.g, device=DEV).to(DTYPES[dtype])
    out = check_attend(st, p, q, rows, lens, slack=3)
    assert bool((out[: new - 3] == 0).all()) and bool((out[new: new + 8] == 0).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("hd,new", [(64, 9), (128, 9), (80, 9), (128, 200), (64, 200)])
@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
def test_attend_unseen_values_have_no_part(st, dtype, hd, new, what):
    # the values of a later new token do not reach the rows before it; its keys neither
    length = 230
    p = Paged(2, DTYPES[dtype], 2, hd, 16, [length])
    q = torch.randn((new, 4, hd), generator=p.g, device=DEV).to(DTYPES[dtype])
    clean = check_attend(st, p, q, [new], [length]).clone()
    for later in (length - 1, length - new // 2):
        at, tok = int(p.table[0, later // 16]), later % 16
        p.v[at, tok, :, ::3] = what
        p.k[at, tok, :, 1] = math.nan
    out = torch.zeros_like(clean)
    st.attend_static(q, p.k, p.v, p.table, i32([0, new]), i32([length]), out=out)
    seen = new - new // 2
    assert torch.equal(out[:seen], clean[:seen])
    assert bool(torch.isnan(out[new - 1]).all())


def test_attend_seen_infinities_arrive(st):
    # an infinite value of a position that a row sees: infinity of its sign in that element, as the formula has it
    for dtype in DTYPES.values():
        for new, hd in ((3, 64), (150, 128), (150, 64)):
            p = Paged(4, dtype, 1, hd, 16, [150])
            at, tok = int(p.table[0, 149 // 16]), 149 % 16
            p.v[at, tok, 0, 5] = -math.inf
            q = torch.randn((new, 2, hd), generator=p.g, device=DEV).to(dtype)
            out = st.attend_static(q, p.k, p.v, p.table, i32([0, new]), i32([150]))
            assert bool((out[new - 1, :, 5] == -math.inf).all()) and bool(torch.isfinite(out[new - 1, :, :5]).all()) and bool(torch.isfinite(out[new - 2]).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_attend_strides_and_alignment(st, dtype):
    d = DTYPES[dtype]
    for shift in (0, 1):
        p = Paged(6, d, 2, 64, 16, [50, 9], shift=shift)
        big = torch.randn((12, 3, 8, 64 + shift), generator=p.g, device=DEV).to(d)
        q = big[:, 1, :, shift:]                                         # rows of a wider projection, at an odd address
        check_attend(st, p, q, [8, 4], [50, 9])
        for width, at in ((65, 1), (72, 8)):                             # results at odd addresses, and with gaps between heads
            store = torch.full((12, 16, width), 3.0, dtype=d, device=DEV)
            check_attend(st, p, q, [8, 4], [50, 9], out=store[:, ::2, at:])
            assert bool((store[:, 1::2] == 3).all()) and bool((store[:, :, :at] == 3).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("order", list(itertools.permutations(range(3))))
@pytest.mark.parametrize("new", [4, 80])
def test_attend_caches_in_any_order(st, dtype, order, new):
    lens = [300, new]
    p = Paged(16, DTYPES[dtype], 2, 64, 16, lens)
    for name in ("k", "v"):                                              # pages, tokens and heads from the widest stride to the narrowest
        c = getattr(p, name)
        setattr(p, name, c.permute(*order, 3).contiguous().permute(*[order.index(i) for i in range(3)], 3))
    q = torch.randn((2 * new, 4, 64), generator=p.g, device=DEV).to(DTYPES[dtype])
    check_attend(st, p, q, [new, new], lens)
    for name in ("k", "v"):                                              # all heads of the cache in one place
        setattr(p, name, getattr(p, name)[:, :, :1].expand(-1, -1, 2, -1))
    check_attend(st, p, q, [new, new], lens)
    slots = torch.arange(3, device=DEV)                                  # and rows that all have the same keys
    rows = torch.randn((1, 1, 64), generator=p.g, device=DEV).to(DTYPES[dtype])
    k = torch.zeros((4, 16, 2, 64), dtype=DTYPES[dtype], device=DEV).permute(1, 0, 2, 3).contiguous().permute(1, 0, 2, 3)
    v = torch.zeros_like(k)
    st.append_static(rows.expand(3, 2, 64), rows.expand(3, 2, 64), k, v, slots)
    assert torch.equal(k[0, :3], rows.expand(3, 2, 64)) and torch.equal(v, k) and not bool(k[0, 3:].any()) and not bool(k[1:].any())


def test_calls_from_two_threads(st):
    p = Paged(17, torch.bfloat16, 2, 64, 16, [900, 2000])
    off, kv, rows = i32([0, 100, 200]), i32([900, 2000]), 200
    q = torch.randn((2, rows, 8, 64), generator=p.g, device=DEV).bfloat16()
    x, u = torch.randn((2, 6, 5000), generator=p.g, device=DEV), torch.rand(6, generator=p.g, device=DEV)
    attend = lambda i, **kw: st.attend_static(q[i], p.k, p.v, p.table, off, kv, **kw)   # noqa: E731
    sample = lambda i, **kw: st.sample_static(x[i], [0] * 6, None, 0, u, top_p=0.9, **kw)[0]   # noqa: E731
    want = [(attend(i), sample(i)) for i in range(2)]
    torch.cuda.synchronize()
    got, errors = [[], []], []

    def work(i):
        try:
            s = torch.cuda.Stream()
            for _ in range(30):
                got[i].append((attend(i, stream=s), sample(i, stream=s)))
            s.synchronize()
        except Exception as e:                                           # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for i in range(2):
        assert len(got[i]) == 30
        for o, tokens in got[i]:
            assert torch.equal(o, want[i][0]) and torch.equal(tokens, want[i][1])


def test_attend_refuses_to_write_over_its_queries(st):
    p = Paged(18, torch.bfloat16, 2, 64, 16, [30])
    q = torch.randn((2, 4, 64), generator=p.g, device=DEV).bfloat16()
    with pytest.raises(st.StairsError) as e:
        st.attend_static(q, p.k, p.v, p.table, i32([0, 2]), i32([30]), out=q)
    assert e.value.code == 1 and "over the queries" in str(e.value)


def test_sample_numbers_outside_their_range(st):
    x = torch.zeros((5, 100), device=DEV)
    u = torch.tensor([1.0, 2.0, math.inf, -1.0, math.nan], device=DEV)
    tokens, _ = st.sample_static(x, [0] * 5, None, 0, u)
    assert tokens[:, 0].tolist() == [99, 99, 99, 0, 0]


def test_attend_offsets_beyond_32_bits(st):
    pages, page, hkv, hd = 40000, 64, 8, 128                             # 2.6e9 elements of keys: their byte offsets pass 32 bits, their element offsets 31
    k = torch.empty((pages, page, hkv, hd), dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    g = gen(8)
    used = [39999, 0, 39998, 20001, 33000]
    for u in used:
        k[u], v[u] = torch.randn((2, page, hkv, hd), generator=g, device=DEV).bfloat16()
    p = Paged.__new__(Paged)
    p.k, p.v, p.table = k, v, i32([used])
    for new in (1, 9, 100):
        q = torch.randn((new, 32, hd), generator=g, device=DEV).bfloat16()
        check_attend(st, p, q, [new], [300])
    fresh = torch.randn((2, 3, hkv, hd), generator=g, device=DEV).bfloat16()
    slot = torch.tensor([39999 * 64 + 63, 39998 * 64 + 1, 17], device=DEV)
    st.append_static(fresh[0], fresh[1], k, v, slot)
    assert torch.equal(k.view(-1, hkv, hd)[slot], fresh[0]) and torch.equal(v.view(-1, hkv, hd)[slot], fresh[1])


def test_attend_bounds_of_lengths_and_rows(st):
    # kv_len above max_len counts as max_len, row_off as within the call's rows; what the table has no entry for is never read
    p = Paged(9, torch.bfloat16, 2, 64, 16, [60, 60])
    q = torch.randn((10, 4, 64), generator=p.g, device=DEV).bfloat16()
    check_attend(st, p, q, [6, 4], [60, 1 << 30], max_len=48)
    out = torch.full_like(q, 5.0)
    st.attend_static(q, p.k, p.v, p.table, i32([2, 6, 9]), i32([60, 60]), out=out)   # rows 0, 1 and 9 of no request
    assert bool((out[:2] == 5).all()) and bool((out[9:] == 5).all()) and bool(torch.isfinite(out[2:9]).all())
    a = st.attend_static(q[2:9], p.k, p.v, p.table, i32([0, 4, 7]), i32([60, 60]))
    assert torch.equal(out[2:9], a)


@pytest.mark.parametrize("captured", [False, True])
def test_attend_streams_and_graphs(st, captured):
    p = Paged(10, torch.bfloat16, 2, 128, 16, [3000, 700, 1])
    new, lens = [9, 1, 1], [3000, 700, 1]
    off = i32([0, 9, 10, 11])
    qs = torch.randn((4, 11, 8, 128), generator=p.g, device=DEV).bfloat16()
    want = [check_attend(st, p, q, new, lens).clone() for q in qs]
    q, kv = qs[0].clone(), i32(lens)
    side = torch.cuda.Stream()
    got = [torch.zeros_like(q) for _ in qs]
    if captured:
        graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
        outs = []
        for gr in graphs:
            with torch.cuda.graph(gr, stream=side):
                outs.append(st.attend_static(q, p.k, p.v, p.table, off, kv))
        for i in range(4):
            q.copy_(qs[i])
            for gr in graphs:                                            # (two graphs one behind another, with a scratch each)
                gr.replay()
            assert torch.equal(outs[0], outs[1])
            got[i].copy_(outs[0])
    else:
        for i in range(4):
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                q.copy_(qs[i])
            got[i] = st.attend_static(q, p.k, p.v, p.table, off, kv, stream=side)
            torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_attend_row_does_not_depend_on_the_call(st):
    # bit for bit the same when called twice
    p = Paged(11, torch.float16, 2, 64, 16, [900, 33])
    q = torch.randn((10, 4, 64), generator=p.g, device=DEV).half()
    a = check_attend(st, p, q, [9, 1], [900, 33]).clone()
    b = check_attend(st, p, q, [9, 1], [900, 33])
    assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------------
# sampling
# ------------------------------------------------------------------------------------------------
def check_sample(st, x, ks, u, settings, drafts=None):
    k_max = max(ks)
    tok, acc = st.sample_static(x, ks, drafts, k_max, u, temperature=[s[0] for s in settings], top_k=[s[1] for s in settings], top_p=[s[2] for s in settings],
                                min_p=[s[3] for s in settings])
    tok, acc, xs, us = tok.tolist(), acc.tolist(), x.double().cpu().numpy(), u.cpu().numpy()
    row = 0
    for i, k in enumerate(ks):
        want = [ou.sample_ref(xs[row + r], us[row + r], *settings[i]) for r in range(k + 1)]
        assert tok[i][: k + 1] == want, (i, settings[i])
        assert tok[i][k + 1:] == [0] * (k_max - k)
        d = drafts[i].tolist()[:k] if k else []
        a = next((r for r in range(k) if d[r] != want[r]), k)
        assert acc[i] == a
        row += k + 1


SETTINGS = [(1.0, 0, 1.0, 0.0), (0.7, 50, 0.9, 0.02), (1.3, 0, 0.99, 0.0), (0.0, 5, 0.5, 0.1), (0.8, 0, 0.6, 0.0), (1.0, 1, 1.0, 0.0), (1.0, 0, 1.0, 0.3), (1e6, 0, 0.5, 0.0),
            (1e-6, 3, 0.9, 0.0), (2.0, 1000, 0.8, 0.0), (1.0, 7, 1.0, 0.0), (1.0, 0, 1e-6, 0.0), (1.0, 0, 1.0, 1.0), (1e6, 20, 1.0, 0.0)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("vocab,pad", [(1, 0), (2, 1), (5, 3), (127, 0), (1000, 1), (2049, 0), (32000, 0), (32128, 8), (60001, 0), (151000, 2)])
def test_sample_settings(st, dtype, vocab, pad):
    g = gen(vocab)
    n = len(SETTINGS)
    ks = [1 + i % 2 for i in range(n)]
    rows = sum(ks) + n
    x = torch.randn((rows, vocab + pad), generator=g, device=DEV) * 2.5
    x[:, :4] += torch.rand((rows, min(4, vocab + pad)), generator=g, device=DEV) * 8
    x = x.to(DTYPES[dtype])[:, :vocab]
    u = torch.rand(rows, generator=g, device=DEV)
    u[0], u[1] = 0.0, 1 - 2.0**-24
    drafts = torch.randint(0, min(vocab, 3), (n, 2), generator=g, device=DEV, dtype=torch.int32)
    check_sample(st, x, ks, u, SETTINGS, drafts)


@pytest.mark.parametrize("vocab", [300, 32000])
@pytest.mark.parametrize("kind", ["equal", "two values", "masked", "lowest", "nan", "inf", "all masked", "close", "steps", "zeros", "one left"])
def test_sample_ties_masks_and_non_finite_scores(st, kind, vocab):
    g = gen(len(kind))
    n = len(SETTINGS)
    x = torch.randn((n, vocab), generator=g, device=DEV) * 2
    m = torch.rand((n, vocab), generator=g, device=DEV) < 0.7
    low = torch.finfo(torch.float32).min
    if kind == "equal":
        x[:] = -3.5
    elif kind == "two values":
        x = torch.where(m, 1.0, 1.5)
    elif kind == "masked":
        x[m] = -math.inf
    elif kind == "lowest":
        x[m] = low
        x[1] = low
    elif kind == "nan":
        x[m] = math.nan
        x[:, 0] = math.nan
    elif kind == "inf":
        x[:, vocab // 2] = math.inf
        x[::2, vocab // 3] = math.inf
        x[1::4, 5] = -math.inf
    elif kind == "all masked":
        x[:] = -math.inf
        x[1::3] = math.nan
        x[2] = 1.0
    elif kind == "close":                                                # neighbours in fp32, thousands of each
        x = (1.0 + torch.randint(0, 64, (n, vocab), generator=g, device=DEV) * 2.0**-23)
    elif kind == "steps":                                                # all magnitudes: few scores share an exponent
        x = 2.0 ** torch.randint(-120, 4, (n, vocab), generator=g, device=DEV).float() * torch.where(m, 1.0, -1.0)
    elif kind == "zeros":
        x = torch.where(m, 0.0, -0.0)
    else:
        x[:] = -math.inf
        x[torch.arange(n, device=DEV), torch.randint(0, vocab, (n,), generator=g, device=DEV)] = -1e30
    u = torch.rand(n, generator=g, device=DEV)
    check_sample(st, x, [0] * n, u, SETTINGS)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_sample_many_rows(st, dtype):
    # the largest calls: 256 requests, and 1024 rows of 64
    for n, k, vocab in ((256, 0, 3001), (64, 15, 1500), (16, 63, 700)):
        g = gen(n)
        rows = n * (k + 1)
        x = (torch.randn((rows, vocab), generator=g, device=DEV) * 3).to(DTYPES[dtype])
        u = torch.rand(rows, generator=g, device=DEV)
        drafts = x.float().argmax(1).view(n, k + 1)[:, : max(k, 1)].int().contiguous()
        check_sample(st, x, [k] * n, u, [SETTINGS[i % len(SETTINGS)] for i in range(n)], drafts)


@pytest.mark.parametrize("dtype,vocab", [("fp32", 1 << 20), ("bf16", 400001), ("fp32", 300000), ("bf16", 1 << 20)])
def test_sample_large_vocabularies(st, dtype, vocab):
    g = gen(vocab)
    n = 6
    x = torch.randn((n, vocab), generator=g, device=DEV) * 2
    x[0] = 1.0
    x[1, vocab - 1] = 30.0
    x[2, : vocab - 5] = -math.inf
    u = torch.rand(n, generator=g, device=DEV)
    check_sample(st, x.to(DTYPES[dtype]), [0] * n, u, [(1.0, 0, 0.7, 0.0), (1.0, 0, 1.0, 0.0), (1.0, 3, 1.0, 0.0), (0.8, 600, 0.95, 0.0), (1.5, 0, 0.98, 0.0), (0.7, 40, 1.0, 0.1)])


def test_sample_distribution(st):
    # 60000 draws of 8 tokens: frequencies within five standard deviations of the probabilities
    x = torch.tensor([0.3, -1.0, 2.0, 0.0, 1.0, -2.0, 0.5, 1.5], device=DEV)
    want = torch.softmax(x.double() / 0.9, dim=0)
    counts, g = torch.zeros(8, dtype=torch.float64, device=DEV), gen(1)
    rows = x.expand(1000, 8).contiguous()
    for _ in range(60):
        u = torch.rand(1000, generator=g, device=DEV)
        tok = torch.cat([st.sample_static(rows[a: a + 250], [0] * 250, None, 0, u[a: a + 250].contiguous(), temperature=0.9)[0].view(-1) for a in range(0, 1000, 250)])
        counts += torch.bincount(tok, minlength=8)
    n = 60000
    assert bool(((counts - n * want).abs() < 5 * (n * want * (1 - want)).sqrt()).all())


@pytest.mark.parametrize("captured", [False, True])
def test_sample_waits_for_the_kernels_before_it(st, captured):
    n, k, vocab, calls = 40, 3, 5000, 8
    g = gen(12)
    src = torch.randn((calls, n * (k + 1), vocab), generator=g, device=DEV) * 3
    us = torch.rand((calls, n * (k + 1)), generator=g, device=DEV)
    kw = dict(temperature=0.8, top_k=40, top_p=0.9)
    want = []
    for i in range(calls):
        d = src[i].argmax(1).view(n, k + 1)[:, :k].int().contiguous()
        want.append(tuple(v.clone() for v in st.sample_static(src[i], [k] * n, d, k, us[i], **kw)))
    torch.cuda.synchronize()
    x, u, d = torch.empty_like(src[0]), torch.empty_like(us[0]), torch.zeros((n, k), dtype=torch.int32, device=DEV)
    got = [(torch.zeros_like(a), torch.zeros_like(b)) for a, b in want]

    def one(i):
        x.copy_(src[i])
        u.copy_(us[i])
        d.copy_(src[i].argmax(1).view(n, k + 1)[:, :k])
        tok, acc = st.sample_static(x, [k] * n, d, k, u, **kw)
        got[i][0].copy_(tok)
        got[i][1].copy_(acc)

    one(0)
    if captured:
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            for i in range(calls):
                one(i)
        graph.replay()
        graph.replay()
    else:
        for i in range(calls):
            one(i)
    torch.cuda.synchronize()
    for (a, b), (c, e) in zip(got, want):
        assert torch.equal(a, c) and torch.equal(b, e)


def test_sample_greedy_equals_accept_static(st):
    g = gen(20)
    x = torch.randn((30, 4099), generator=g, device=DEV)
    d = x.argmax(1).view(6, 5)[:, :4].int().contiguous()
    d[2, 1] += 1
    a = st.accept_static(x, [4] * 6, d, 4)
    b = st.sample_static(x, [4] * 6, d, 4, torch.rand(30, generator=g, device=DEV), temperature=0)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ------------------------------------------------------------------------------------------------
# all of them, as a program with a model of its own uses them
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_stairs_steps_of_a_callers_own_model(st, dtype):
    # A one-layer model outside the library: embedding, projections, attention over the paged cache, head.  Three requests of different lengths do a prompt pass and
    # then sampled stairs steps whose lengths stay on the device; every step is compared with a dense 64-bit pass over the whole sequences.
    d_t = DTYPES[dtype]
    g = gen(30)
    vocab, d, heads, hkv, hd, page, k = 50, 64, 4, 2, 32, 16, 4
    emb = torch.randn((vocab, d), generator=g, device=DEV).to(d_t)
    wq, wk, wv = ((torch.randn((d, n * hd), generator=g, device=DEV) * d**-0.5).to(d_t) for n in (heads, hkv, hkv))
    wo = (torch.randn((heads * hd, vocab), generator=g, device=DEV) * 0.3).to(d_t)
    prompts = [torch.randint(0, vocab, (n,), generator=g, device=DEV).tolist() for n in (5, 33, 16)]
    n = len(prompts)
    kc, vc = (torch.full((24, page, hkv, hd), math.nan, dtype=d_t, device=DEV) for _ in range(2))
    free = torch.randperm(24, generator=g, device=DEV).int()
    table = torch.full((n, 8), -1, dtype=torch.int32, device=DEV)
    n_seq, n_blocks, n_used = i32([0] * n), i32([0] * n), i32([0])
    seqs = [list(p) for p in prompts]

    def layer(tokens, t):
        x = emb[tokens.clamp(min=0).long()]
        q, kn, vn = (x @ w for w in (wq, wk, wv))
        st.append_static(kn.view(-1, hkv, hd), vn.view(-1, hkv, hd), kc, vc, t.row_slot)
        o = torch.zeros((len(tokens), heads, hd), dtype=d_t, device=DEV)
        st.attend_static(q.view(-1, heads, hd), kc, vc, table, t.row_off, t.kv_len, out=o)
        return (o.flatten(1) @ wo).float()

    def dense(tokens):
        x = emb[torch.tensor(tokens, device=DEV)].double()
        q, kk, vv = (x @ w.double() for w in (wq, wk, wv))
        q, kk, vv = q.view(-1, heads, hd), kk.view(-1, hkv, hd).repeat_interleave(heads // hkv, 1), vv.view(-1, hkv, hd).repeat_interleave(heads // hkv, 1)
        s = torch.einsum("thd,phd->htp", q, kk) * hd**-0.5
        s = s.masked_fill(torch.ones_like(s[0]).triu(1).bool(), -math.inf)
        return torch.einsum("htp,phd->thd", torch.softmax(s, -1), vv).flatten(1) @ wo.double()

    # the prompts but for their last tokens, padded to a fixed number of rows
    t = st.tables_static(n_seq, i32([len(p) - 1 for p in prompts]), n_blocks, table, free, n_used, page_tokens=page, max_rows=64)
    flat = [tok for p in prompts for tok in p[:-1]]
    layer(i32(flat + [-1] * (64 - len(flat))), t)
    n_seq, n_blocks, n_used = t.kv_len, t.n_blocks, t.n_used
    # fp32: sums of at most 128 products in 32 bits, three of them behind each other: 3 * 128 * 2^-24 of scores of about 10; bf16: each of the four
    # roundings of an activation (x w, o, scores) is at most 2^-9 relative, through sums of 64 to 128 such terms at weight 0.3
    tol = 1e-3 if dtype == "fp32" else 0.25
    last = i32([p[-1] for p in prompts])
    rng = np.random.default_rng(1)
    for step in range(6):
        draft = torch.randint(0, vocab, (n, k), generator=g, device=DEV, dtype=torch.int32)
        # drafts that the sampled tokens will partly meet: the dense model's own drawn tokens, cut at a random place
        us = torch.rand(n * (k + 1), generator=g, device=DEV)
        for i in range(n):
            s = list(seqs[i])
            for j in range(int(rng.integers(0, k + 1))):
                tok = ou.sample_ref(dense(s)[-1].cpu().numpy(), float(us[i * (k + 1) + j]), 0.7, 20, 0.9, 0.0)
                draft[i, j] = tok
                s.append(tok)
        t = st.tables_static(n_seq, i32([k + 1] * n), n_blocks, table, free, n_used, page_tokens=page, max_rows=n * (k + 1) + 2)
        rows = torch.cat([last[:, None], draft], dim=1).flatten()
        logits = layer(torch.cat([rows, i32([-1, -1])]), t)
        assert int(t.n_served) == n
        tok, acc = st.sample_static(logits[: n * (k + 1)], [k] * n, draft, k, us, temperature=0.7, top_k=20, top_p=0.9)
        for i in range(n):
            want = dense(seqs[i] + draft[i].tolist())[-(k + 1):]
            assert float((logits[i * (k + 1): (i + 1) * (k + 1)].double() - want).abs().max()) < tol
            a = int(acc[i])
            seqs[i] += draft[i, :a].tolist() + [int(tok[i, a])]
        # the next pass's lengths, without the host: kept drafts and the row before them are cached, the token after them comes next
        n_seq = n_seq + acc + 1
        last = tok.gather(1, acc.long()[:, None])[:, 0]
        n_blocks, n_used = t.n_blocks, t.n_used
        assert n_seq.tolist() == [len(s) - 1 for s in seqs] and last.tolist() == [s[-1] for s in seqs]
    assert sum(len(s) for s in seqs) > sum(len(p) for p in prompts) + 6 * n   # some drafts were kept
