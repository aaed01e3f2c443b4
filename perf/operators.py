"""Performance cases of the stairs framework's operators on buffers that the caller holds: the steps of a stairs
pass for a program that runs its own model (its own projections, its own paged cache) and takes from the library
the block tables, the append, the attention over the cache and the sampled acceptance.

A case is a dict of plain values:
  op         tables | append | attend | sample
  dtype      fp32 | bf16 | fp16 of the cache, queries or logits
  heads, kv_heads, head_dim, page (tokens per page), layout (NHD: tokens before heads in a page, HND: heads first)
  requests   requests of one call; prefix: cached tokens of the longest one; new: new tokens of each
  ragged     1: the requests' prefixes (down to one token) and new tokens (down to none) differ
  vocab, k   sample: columns of the logits, drafted tokens of each request (k + 1 rows)
  temperature, top_k, top_p, min_p   sample: of the first request; 0, 0, 1 and 0 switch them off.  ragged: the
             other requests have others
"""
import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


# ------------------------------------------------------------------------------------------------
# the cases
# ------------------------------------------------------------------------------------------------
def _case(name=None, **kw):
    base = dict(op="attend", dtype="bf16", heads=32, kv_heads=8, head_dim=128, page=64, layout="NHD", requests=1, prefix=0, new=1,
                ragged=0, vocab=0, k=0, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    base.update(kw)
    return dict(base, name=name) if name else base


def listed():
    return [
        # lengths after one accepted step of four requests with long prefixes: tables for the next 9 rows each
        _case("tables 4 requests", op="tables", requests=4, prefix=16384, new=9),
        # a full serving batch, short pages, every length and number of new tokens different
        _case("tables 1024 requests", op="tables", requests=1024, prefix=2048, new=24, page=16, ragged=1),
        # the stair rows of one request of the 7B shape
        _case("append 9 rows", op="append", requests=1, prefix=1024, new=9),
        # a prefill pass of the 3B shape into a cache that keeps each head's tokens together
        _case("append 2048 rows", op="append", dtype="fp16", heads=32, kv_heads=32, head_dim=80, layout="HND", prefix=512, new=2048, page=16),
        # one token of the 7B shape: latency
        _case("attend 7B 1 token", requests=1, prefix=1023, new=1),
        # the validation call of the benchmark's default run: 9 rows after 2048 cached tokens
        _case("attend 0.4B p2048 k8", heads=16, kv_heads=16, head_dim=64, prefix=2048, new=9),
        # the tiny fp32 model: a chunk of its prompt
        _case("attend tiny fp32", dtype="fp32", heads=4, kv_heads=4, head_dim=64, page=16, prefix=32, new=64),
        # a serving batch of the 3B shape: requests of every length, some without a new token
        _case("attend 3B 16 requests", dtype="fp16", heads=32, kv_heads=32, head_dim=80, page=16, layout="HND", requests=16, prefix=960, new=7, ragged=1),
        # four requests with 16384 cached tokens each
        _case("attend 7B 4x16384 k8", requests=4, prefix=16384, new=9),
        # a chunk of a long prompt of the 7B shape
        _case("attend 7B chunk 2048", prefix=4096, new=2048),
        # the 5 rows of one request over a Llama-sized vocabulary, nucleus sampling
        _case("sample 5 rows", op="sample", dtype="fp32", requests=1, k=4, vocab=32000, temperature=0.8, top_p=0.95),
        # a full serving batch, each request with settings of its own
        _case("sample 576 rows", op="sample", dtype="bf16", requests=64, k=8, vocab=32128, temperature=0.7, top_k=50, top_p=0.9, min_p=0.02, ragged=1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


SHAPES = [(4, 4, 64), (16, 16, 64), (32, 32, 80), (32, 8, 128), (32, 8, 128), (8, 1, 128), (12, 4, 40), (20, 4, 96), (6, 2, 16)]


def draw(rng):
    op = rng.choice(["tables", "append", "attend", "attend", "attend", "sample", "sample"])
    heads, kv_heads, head_dim = rng.choice(SHAPES)
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    common = dict(op=op, dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=rng.choice([16, 32, 64, 128]),
                  layout=rng.choice(["NHD", "HND"]), ragged=rng.randint(0, 1))
    if op == "tables":
        return _case(**dict(common, requests=_log_int(rng, 1, 1024), prefix=_log_int(rng, 1, 2048), new=rng.randint(1, 24)))
    if op == "append":
        return _case(**dict(common, requests=_log_int(rng, 1, 8), prefix=_log_int(rng, 1, 512), new=_log_int(rng, 1, 256)))
    if op == "sample":
        k = rng.randint(0, 16)
        return _case(op=op, dtype=dtype, ragged=common["ragged"], requests=_log_int(rng, 1, max(1, min(64, 576 // (k + 1)))), k=k,
                     vocab=_log_int(rng, 1000, 32128), temperature=round(rng.uniform(0.5, 1.3), 3),
                     top_k=rng.choice([0, 1, 20, 50, 1000]), top_p=rng.choice([1.0, 0.99, 0.9, 0.6]), min_p=rng.choice([0.0, 0.0, 0.05, 0.3]))
    new = rng.choice([1, rng.randint(2, 17), _log_int(rng, 17, 1024)])
    # no more work than the listed chunk: rows x positions x heads x head size, a tenth of it where it is fp32
    budget = 2048 * 6144 * 32 * 128 // (10 if dtype == "fp32" else 1) // (new * heads * head_dim)
    prefix = _log_int(rng, 1, min(16384, budget))
    requests = _log_int(rng, 1, max(1, min(64, 65536 // (prefix + new), budget // (prefix + new))))
    return _case(**dict(common, requests=requests, prefix=prefix, new=new))


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _lengths(case):
    """Cached and new tokens of every request."""
    n, p, w = case["requests"], case["prefix"], case["new"]
    if not case["ragged"]:
        return [p] * n, [w] * n
    return [max(1, p - (r * p) // n) for r in range(n)], [(w - r) % (w + 1) if n > 1 else w for r in range(n)]


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    dtype, op = DTYPES[case["dtype"]], case["op"]
    if op == "sample":
        n, k, vocab = case["requests"], case["k"], case["vocab"]
        # a trained model's scores: a broad body and a handful of candidates that stand out of it
        x = torch.randn((n * (k + 1), vocab), generator=g, device=DEVICE) * 2.0
        at = torch.randint(0, vocab, (n * (k + 1), 8), generator=g, device=DEVICE)
        x.scatter_add_(1, at, torch.rand(at.shape, generator=g, device=DEVICE) * 6.0 + 4.0)
        best = x.argmax(dim=1).view(n, k + 1)[:, :k]
        keep = torch.rand((n, k), generator=g, device=DEVICE) < 0.75
        draft = torch.where(keep, best, (best + 1) % vocab).to(torch.int32).contiguous()
        s = {"temperature": [case["temperature"]] * n, "top_k": [case["top_k"]] * n, "top_p": [case["top_p"]] * n, "min_p": [case["min_p"]] * n}
        if case["ragged"]:   # in turn: as the first, without a filter, greedy, the smallest of the filters alone
            s["temperature"] = [case["temperature"] * (0.0 if r % 4 == 2 else 1.0) for r in range(n)]
            s["top_k"] = [case["top_k"] if r % 4 != 1 else 0 for r in range(n)]
            s["top_p"] = [case["top_p"] if r % 4 != 1 else 1.0 for r in range(n)]
            s["min_p"] = [case["min_p"] if r % 4 == 0 else 0.0 for r in range(n)]
        settings = torch.tensor([s["temperature"], s["top_k"], s["top_p"], s["min_p"]], dtype=torch.float32, device=DEVICE)
        return dict(s, case=case, logits=x.to(dtype), u=torch.rand(n * (k + 1), generator=g, device=DEVICE), k=[k] * n, k_max=k,
                    draft=draft if k else None, settings=settings)
    seq, new = _lengths(case)
    page = case["page"]
    n, rows = len(seq), sum(new)
    blocks = [-(-(p + w) // page) for p, w in zip(seq, new)]
    most, total = max(blocks), sum(blocks)
    pages = total + total // 8 + 1
    order = torch.randperm(pages, generator=g, device=DEVICE).to(torch.int32)   # pages in the order in which a used pool hands them out
    if op == "tables":
        had = [-(-p // page) for p in seq]
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEVICE)  # noqa: E731
        table = torch.full((n, most + 2), -1, dtype=torch.int32, device=DEVICE)
        first = torch.tensor(had, device=DEVICE).cumsum(0) - i32(had)
        b = torch.arange(most + 2, device=DEVICE)[None, :]
        held = b < i32(had)[:, None]
        table[held] = order[(first[:, None] + b)[held]]
        return {"case": case, "n_seq": i32(seq), "n_new": i32(new), "n_blocks": i32(had), "table": table, "free": order, "n_used": i32([sum(had)]),
                "max_rows": rows + 5}
    table = torch.full((n, most + 1), -1, dtype=torch.int32, device=DEVICE)
    first = torch.tensor([0] + blocks[:-1], device=DEVICE).cumsum(0)
    b = torch.arange(most + 1, device=DEVICE)[None, :]
    held = b < torch.tensor(blocks, device=DEVICE)[:, None]
    table[held] = order[(first[:, None] + b)[held]]
    hkv, hd = case["kv_heads"], case["head_dim"]
    mem = (pages, page, hkv, hd) if case["layout"] == "NHD" else (pages, hkv, page, hd)
    kc, vc = (torch.randn(mem, generator=g, device=DEVICE).to(dtype) for _ in range(2))
    if case["layout"] == "HND":
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    st = {"case": case, "k_cache": kc, "v_cache": vc, "table": table, "longest": max(p + w for p, w in zip(seq, new))}
    if op == "append":
        qkv = torch.randn((rows, case["heads"] + 2 * hkv, hd), generator=g, device=DEVICE).to(dtype)   # as a projection leaves it
        req = torch.tensor([r for r in range(n) for _ in range(new[r])], device=DEVICE)
        pos = torch.tensor([seq[r] + j for r in range(n) for j in range(new[r])], device=DEVICE)
        slot = table[req, pos // page].long() * page + pos % page
        return dict(st, k_new=qkv[:, case["heads"]: case["heads"] + hkv], v_new=qkv[:, case["heads"] + hkv:], slot=slot)
    off = torch.tensor([0] + new, device=DEVICE).cumsum(0).to(torch.int32)
    kv_len = torch.tensor([p + w for p, w in zip(seq, new)], dtype=torch.int32, device=DEVICE)
    q = (torch.randn((rows, case["heads"], hd), generator=g, device=DEVICE) * 1.5).to(dtype)
    return dict(st, q=q, row_off=off, kv_len=kv_len, most_new=max(new), scale=1.0 / math.sqrt(hd))


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def _tables(st):
    page, table, rows = st["case"]["page"], st["table"], st["max_rows"]
    seq, new, had = st["n_seq"].long(), st["n_new"].long().clamp(min=0), st["n_blocks"].long()
    need = ((seq + new + page - 1) // page - had).clamp(min=0)
    taken = st["n_used"].long() + need.cumsum(0)
    fits = (taken <= st["free"].numel()) & (new.cumsum(0) <= rows) & (had + need <= table.shape[1])
    served = fits.long().cumprod(0)
    need, new = need * served, new * served
    first = st["n_used"].long() + need.cumsum(0) - need
    b = torch.arange(table.shape[1], device=DEVICE)[None, :]
    fresh = (b >= had[:, None]) & (b < (had + need)[:, None])
    source = (first[:, None] + b - had[:, None]).clamp(0, st["free"].numel() - 1)
    table.copy_(torch.where(fresh, st["free"][source], table))
    off = torch.cat([torch.zeros_like(new[:1]), new.cumsum(0)])
    t = torch.arange(rows, device=DEVICE)
    req = torch.searchsorted(off[1:].contiguous(), t, right=True)
    real = req < new.numel()
    r = req.clamp(max=new.numel() - 1)
    pos = seq[r] + t - off[r]
    at = table[r, (pos // page).clamp(0, table.shape[1] - 1)].long()
    slot = torch.where(real & (at >= 0), at * page + pos % page, -1)
    i32 = lambda v: v.to(torch.int32)  # noqa: E731
    return {"table": table, "n_blocks": i32(had + need), "n_used": i32(st["n_used"].long() + need.sum()), "row_off": i32(off), "kv_len": i32(seq + new),
            "row_req": i32(torch.where(real, req, -1)), "row_pos": i32(torch.where(real, pos, -1)), "row_slot": slot, "n_served": i32(served.sum().view(1))}


def _attend(st):
    q, off, kv_len, page = st["q"].float(), st["row_off"].long(), st["kv_len"].long(), st["case"]["page"]
    hkv, hd = st["case"]["kv_heads"], st["case"]["head_dim"]
    rows, group, n, longest, most = q.shape[0], q.shape[1] // hkv, kv_len.numel(), st["longest"], st["most_new"]
    p = torch.arange(longest, device=DEVICE)
    at = st["table"].long()[:, p // page].clamp(min=0)                          # [requests, positions]
    k = st["k_cache"][at, p % page].float().permute(0, 2, 3, 1)                  # [requests, kv heads, head size, positions]
    t = torch.arange(rows, device=DEVICE)
    req = torch.searchsorted(off[1:].contiguous(), t, right=True)
    j = t - off[req]
    pos = kv_len[req] - (off[req + 1] - off[req]) + j
    padded = torch.zeros((n, most, hkv, group, hd), device=DEVICE)
    padded[req, j] = q.view(rows, hkv, group, hd)
    last = torch.full((n, most), -1, dtype=torch.long, device=DEVICE)
    last[req, j] = pos
    s = torch.matmul(padded.permute(0, 2, 3, 1, 4).reshape(n, hkv, group * most, hd), k) * st["scale"]
    seen = (p[None, None, :] <= last[:, :, None])[:, None, None]                 # [requests, 1, 1, rows, positions]
    s = s.view(n, hkv, group, most, longest).masked_fill_(~seen, -math.inf)
    e = torch.exp(s - s.amax(dim=-1, keepdim=True).clamp(min=-3e38))
    total = e.sum(dim=-1, keepdim=True)
    v = st["v_cache"][at, p % page].float().transpose(1, 2)
    v = torch.where((p[None, :] < kv_len[:, None])[:, None, :, None], v, 0.0)
    o = torch.matmul(e.view(n, hkv, group * most, longest), v).view(n, hkv, group, most, hd) / total.clamp(min=1e-38)
    return o.permute(0, 3, 1, 2, 4)[req, j].reshape(rows, hkv * group, hd).to(st["q"].dtype)


def _sample(st):
    n, k, x = len(st["k"]), st["k_max"], st["logits"].double()
    x = torch.where(torch.isnan(x), -math.inf, x)
    temperature, top_k, top_p, min_p = (v.double().repeat_interleave(k + 1)[:, None] for v in st["settings"])
    ordered, index = x.sort(dim=1, descending=True, stable=True)                 # ties: lowest index first
    best = ordered[:, :1]
    greedy = temperature == 0
    d = torch.where(ordered == best, 0.0, ordered - best) / torch.where(greedy, 1.0, temperature)
    w = torch.exp(d)
    rank = torch.arange(x.shape[1], device=DEVICE)[None, :]
    w = torch.where((w >= min_p) & ((top_k == 0) | (rank < top_k)), w, 0.0)
    before = w.cumsum(dim=1) - w
    w = torch.where((top_p >= 1) | (before < top_p * w.sum(dim=1, keepdim=True)), w, 0.0)
    kept = torch.zeros_like(w).scatter_(1, index, w).cumsum(dim=1)               # in the vocabulary's order
    token = (kept <= st["u"].double()[:, None] * kept[:, -1:]).sum(dim=1)
    token = torch.where(greedy[:, 0], index[:, 0], token)
    token = torch.where(best[:, 0] == -math.inf, -1, token).to(torch.int32).view(n, k + 1)
    if not k:
        return token, torch.zeros(n, dtype=torch.int32, device=DEVICE)
    return token, (token[:, :k] == st["draft"]).long().cumprod(dim=1).sum(dim=1).to(torch.int32)


def run(st):
    op = st["case"]["op"]
    if op == "tables":
        if not own:
            return _tables(st)
        from paper_2407_19947_b200 import stairs
        r = stairs.tables_static(st["n_seq"], st["n_new"], st["n_blocks"], st["table"], st["free"], st["n_used"], page_tokens=st["case"]["page"],
                                 max_rows=st["max_rows"])
        return dict(r._asdict(), table=st["table"])
    if op == "append":
        if own:
            from paper_2407_19947_b200 import stairs
            stairs.append_static(st["k_new"], st["v_new"], st["k_cache"], st["v_cache"], st["slot"])
        else:
            page = st["case"]["page"]
            st["k_cache"][st["slot"] // page, st["slot"] % page] = st["k_new"]
            st["v_cache"][st["slot"] // page, st["slot"] % page] = st["v_new"]
        return st["k_cache"], st["v_cache"]
    if op == "attend":
        if not own:
            return _attend(st)
        from paper_2407_19947_b200 import stairs
        return stairs.attend_static(st["q"], st["k_cache"], st["v_cache"], st["table"], st["row_off"], st["kv_len"], scale=st["scale"],
                                    max_len=st["longest"])
    if not own:
        return _sample(st)
    from paper_2407_19947_b200 import stairs
    return stairs.sample_static(st["logits"], st["k"], st["draft"], st["k_max"], st["u"], temperature=st["temperature"], top_k=st["top_k"],
                                top_p=st["top_p"], min_p=st["min_p"])


# ------------------------------------------------------------------------------------------------
# the same from the definitions, in 64 bits, and what a pass cannot do without
# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    if case["op"] not in ("append", "attend"):
        return None                                                              # whole numbers
    st = prepare(case, seed)
    page = case["page"]
    if case["op"] == "append":
        got = []
        for cache, fresh in ((st["k_cache"], st["k_new"]), (st["v_cache"], st["v_new"])):
            whole = cache.double().contiguous()
            whole.view(-1, *whole.shape[2:]).index_copy_(0, st["slot"], fresh.double())
            got.append(whole)
        return tuple(got)
    off, lens, table = st["row_off"].tolist(), st["kv_len"].tolist(), st["table"].tolist()
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEVICE)
    group = case["heads"] // case["kv_heads"]
    for r, length in enumerate(lens):
        a, b = off[r], off[r + 1]
        if a == b or length == 0:
            continue
        used = torch.tensor(table[r][: -(-length // page)], device=DEVICE)
        k = st["k_cache"][used].flatten(0, 1)[:length].double()
        v = st["v_cache"][used].flatten(0, 1)[:length].double()
        hidden = torch.arange(length, device=DEVICE)[None, :] - torch.arange(length - (b - a), length, device=DEVICE)[:, None] > 0
        for h in range(case["heads"]):
            s = st["q"][a:b, h].double() @ k[:, h // group].T / math.sqrt(case["head_dim"])
            s[hidden] = -math.inf
            out[a:b, h] = torch.softmax(s, dim=1) @ v[:, h // group]
    return out


def work(case):
    es = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "sample":
        rows = case["requests"] * (case["k"] + 1)
        return {"bytes": rows * (case["vocab"] * es + 4 + 4 + 4), "flops": rows * case["vocab"]}
    seq, new = _lengths(case)
    n, rows, page = len(seq), sum(new), case["page"]
    if case["op"] == "tables":
        held = sum(-(-(p + w) // page) for p, w in zip(seq, new))
        return {"bytes": 4 * (n * 6 + held) + 16 * (rows + 5), "flops": n + rows}
    row = case["kv_heads"] * case["head_dim"] * es
    if case["op"] == "append":
        return {"bytes": rows * (4 * row + 8), "flops": 2 * rows * case["kv_heads"] * case["head_dim"]}
    kv = sum(p + w for p, w in zip(seq, new) if w) * 2 * row
    pairs = sum(w * p + w * (w + 1) // 2 for p, w in zip(seq, new))
    return {"bytes": kv + rows * 2 * case["heads"] * case["head_dim"] * es, "flops": 4 * pairs * case["heads"] * case["head_dim"]}
