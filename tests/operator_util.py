"""Plain 64-bit implementations of the operators on caller-held buffers (include/stairs.h), written from their definitions."""
import numpy as np
import torch


def tables_ref(n_seq, n_new, n_blocks, table, free, n_used, page, max_rows):
    table = [list(r) for r in table]
    max_blocks, rows, used, served, stopped = len(table[0]), 0, n_used, 0, n_used < 0
    out = dict(n_blocks=[], row_off=[0], kv_len=[], row_req=[], row_pos=[], row_slot=[])
    for i, (seq, new, had) in enumerate(zip(n_seq, n_new, n_blocks)):
        new = max(new, 0)
        need = max(-(-(seq + new) // page) - had, 0)
        if seq < 0 or not 0 <= had <= max_blocks or had + need > max_blocks or used + need > len(free) or rows + new > max_rows:
            stopped = True
        if stopped:
            out["n_blocks"].append(had)
            out["kv_len"].append(seq)
            out["row_off"].append(rows)
            continue
        served += 1
        table[i][had: had + need] = free[used: used + need]
        used += need
        for p in range(seq, seq + new):
            at = table[i][p // page]
            out["row_req"].append(i)
            out["row_pos"].append(p)
            out["row_slot"].append(at * page + p % page if at >= 0 else -1)
        rows += new
        out["n_blocks"].append(had + need)
        out["kv_len"].append(seq + new)
        out["row_off"].append(rows)
    for name in ("row_req", "row_pos", "row_slot"):
        out[name] += [-1] * (max_rows - rows)
    return dict(out, table=table, n_used=[used], n_served=[served])


def attend_ref(q, k_cache, v_cache, table, row_off, kv_len, scale, max_len=None, rows_of=None):
    """(o in 64 bits, the bound of its error by the score's and the weights' roundings) - row by row, only of what a row sees.
    Rows of no request, and those that rows_of (a choice of rows) leaves out, are NaN in o."""
    pages, page, hkv, hd = k_cache.shape
    rows, heads, _ = q.shape
    group = heads // hkv
    o = torch.full((rows, heads, hd), float("nan"), dtype=torch.float64, device=q.device)
    off = torch.zeros((rows, heads, 1), dtype=torch.float64, device=q.device)
    two_bytes = q.dtype != torch.float32
    half = torch.finfo(q.dtype).eps / 2
    for r, length in enumerate(kv_len.tolist()):
        a, b = int(row_off[r]), int(row_off[r + 1])
        length = max(0, length if max_len is None else min(length, max_len))
        for t in range(a, min(b, rows)):
            if rows_of is not None and not rows_of(t):
                continue
            last = length - (b - a) + (t - a)
            p = torch.arange(max(last + 1, 0), device=q.device)
            at = table[r][p // page].long()
            ok = (at >= 0) & (at < pages)
            p, at = p[ok], at[ok]
            if not len(p):
                o[t] = 0.0
                continue
            k = k_cache[at, p % page].double().repeat_interleave(group, dim=1)     # [positions, heads, hd]
            v = v_cache[at, p % page].double().repeat_interleave(group, dim=1)
            qk = q[t].double()[None] * k
            s = qk.sum(dim=2) * scale
            w = torch.softmax(s, dim=0)[:, :, None]
            o[t] = (w * v).sum(dim=0)
            # scores: products and sums of head_dim terms in 32 bits, scaled (each step half a unit of 2^-23), the exponential's
            # argument and value a few units more; an error e of every exponent moves the weighted mean by at most 2 e max |v|
            e = (abs(qk).sum(dim=2) * abs(scale)).amax(dim=0) * (hd + 8) * 2.0 ** -24 + 8 * 2.0 ** -24
            # sums over the positions in 32 bits, in chunks: at most 2^-24 for each of the additions that one value passes through
            chain = (64 + len(p) ** 0.5 + len(p) / 64) * 2.0 ** -24
            # 16-bit weights: half a step each, of numerator alone; a weight below the type's normal range (fp16) by 2^-25 of the largest
            weights = half + (2.0 ** -25 * len(p) if q.dtype == torch.float16 else 0.0) if two_bytes else 0.0
            big = abs(v).amax(dim=(0, 2))
            off[t, :, 0] = (2 * e + chain + weights) * big
    return o, off + half * abs(o).nan_to_num()


def sample_ref(x, u, temperature, top_k, top_p, min_p):
    """The drawn token of one row of scores (numpy, 64 bits)."""
    x = np.asarray(x, np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    best = x.max()
    if best == -np.inf:
        return -1
    if temperature == 0:
        return int(np.argmax(x))
    order = np.argsort(-x, kind="stable")
    with np.errstate(invalid="ignore"):
        w = np.exp(np.where(x == best, 0.0, x - best) / np.float64(np.float32(temperature)))[order]
    w[w < np.float64(np.float32(min_p))] = 0.0
    if top_k:
        w[top_k:] = 0.0
    if top_p < 1:
        before = np.cumsum(w) - w
        w[before >= np.float64(np.float32(top_p)) * w.sum()] = 0.0
    kept = np.zeros_like(w)
    kept[order] = w
    c = np.cumsum(kept)
    return int(np.argmax(c > np.float64(u) * c[-1]))
