"""Plain 64-bit implementations, on the CPU, of the operators for several sequences behind one prompt, written from their
definitions, and how far a correct fp32 / bf16 computation may be from them."""
import math

import torch

F64 = torch.float64
STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}     # half a rounding step, relative


def rope_table(n_pos, dh, base=10000.0):
    at = torch.arange(n_pos, dtype=F64)[:, None] * base ** (-torch.arange(dh // 2, dtype=F64) * 2 / dh)
    return torch.stack([at.cos(), at.sin()], -1)


def norm_rotate(x, gain, eps, cs_sn):
    """x: [heads, dh] float64 of one row; returns the head rows and the magnitude that their rounding errors scale with."""
    if gain is not None:
        x = x / (x.pow(2).mean(-1, keepdim=True) + eps).sqrt() * gain.to(F64)
    size = x.abs()
    if cs_sn is not None:
        half = x.shape[-1] // 2
        a, b = x[:, :half], x[:, half:]
        c, s = cs_sn[:, 0].to(F64), cs_sn[:, 1].to(F64)
        x = torch.cat([a * c - b * s, b * c + a * s], -1)
        size = torch.cat([size[:, :half] + size[:, half:]] * 2, -1)
    return x, size


def key_at(pages, page, head, off, pt, dh):
    return pages[page, 0, head].view(pt, dh)[off]


def val_at(pages, page, head, off, pt, dh):
    return pages[page, 1, head].view(dh, pt)[:, off]


def gather(pages, table, n, head, pt, dh):
    """Keys and values of positions 0 .. n - 1 of a table, float64; NaN where a page is outside the pool."""
    k, v = torch.full((n, dh), math.nan, dtype=F64), torch.full((n, dh), math.nan, dtype=F64)
    for p in range(0, n, pt):
        page, m = int(table[p // pt]), min(pt, n - p)
        if 0 <= page < pages.shape[0]:
            k[p:p + m] = pages[page, 0, head].view(pt, dh)[:m].to(F64)
            v[p:p + m] = pages[page, 1, head].view(dh, pt)[:, :m].T.to(F64)
    return k, v


def attention(q, n_tok, nq, nkv, dh, pt, pages, tables, lens, prefix_pages, prefix_table, prefix_len, scale):
    """out, lse, and per output the size that errors scale with: sum_j p_j |v_j|, and per row the bound of a score's error in units of 2^-24."""
    rows, grp = q.shape[0], nq // nkv
    out, size = torch.zeros(rows, nq, dh, dtype=F64), torch.zeros(rows, nq, dh, dtype=F64)
    lse, e_s = torch.full((rows, nq), -math.inf, dtype=F64), torch.zeros(rows, nq, dtype=F64)
    qd = q.to(F64).view(rows, nq, dh)
    for kvh in range(nkv):
        pk, pv = gather(prefix_pages, prefix_table, prefix_len, kvh, pt, dh) if prefix_len else (torch.zeros(0, dh, dtype=F64),) * 2
        hs = slice(kvh * grp, (kvh + 1) * grp)
        for b in range(rows // n_tok):
            ok, ov = gather(pages, tables[b], max(0, min(int(lens[b]), tables.shape[1] * pt)), kvh, pt, dh)
            for t in range(n_tok):
                n = max(0, min(ok.shape[0], int(lens[b]) - n_tok + 1 + t))
                k, v = torch.cat([pk, ok[:n]]), torch.cat([pv, ov[:n]])
                if k.shape[0] == 0:
                    continue
                r = b * n_tok + t
                s = qd[r, hs] @ k.T * scale
                z = torch.logsumexp(s, -1, keepdim=True)
                p = (s - z).exp()
                out[r, hs], size[r, hs], lse[r, hs] = p @ v, p @ v.abs(), z[:, 0]
                # dh products and their sum, the factors' third bf16 term, scaling, exp2 of a rounded argument
                e_s[r, hs] = ((qd[r, hs].abs() @ k.abs().T * scale).amax(-1) * (dh + 8) + 3 * s.abs().amax(-1) + 8)
    return out.view(rows, nq * dh), lse, size.view(rows, nq * dh), e_s.repeat_interleave(dh, 1), e_s


def attention_bounds(dtype, out, lse, size, e_out, e_lse, n_pos):
    """Elementwise bounds: scores (twice: numerator and sum), fp32 sums over n_pos positions, and for bf16 the rounding of the probabilities and
    of the result."""
    u = 2.0 ** -24
    tol = size * (2 * e_out + 2 * n_pos + 16) * u
    if dtype == torch.bfloat16:
        tol = tol + STEP[dtype] * size + STEP[dtype] * out.abs()
    return tol + 1e-30, (e_lse + n_pos + 16) * u + 4 * u * torch.where(lse.isfinite(), lse.abs(), torch.zeros_like(lse))


def select(logits, scores, groups, beams, k, done=None, end_token=-1):
    """(tokens, parents, scores, done) as nested lists, from float64 keys."""
    got = []
    for g in range(groups):
        cand, bad = [], False
        for b in range(beams):
            row = g * beams + b
            s = float(scores[row])
            if math.isnan(s) or s == math.inf:
                bad = True
            if done is not None and int(done[row]):
                cand.append((-s, b, end_token))
                continue
            x = logits[row].to(F64)
            if x.isnan().any() or (x == math.inf).any():
                bad = True
                continue
            key = s + x - torch.logsumexp(x, 0)
            # (stable: equal keys stay in the order of their index; inside a row the order is that of the logits)
            for v in x.sort(descending=True, stable=True).indices[:k].tolist():
                cand.append((-float(key[v]), b, v))
        cand = sorted(c for c in cand if c[0] < math.inf)[:k]
        if bad:
            got.append([(-1, -1, math.nan, 1)] * k)
            continue
        row = [(v, b, -m, int((done is not None and bool(done[g * beams + b])) or v == end_token)) for m, b, v in cand]
        got.append(row + [(-1, -1, -math.inf, 1)] * (k - len(row)))
    return got


def reorder(pool, tables, parents, groups, beams, length, pt):
    """(tables_out, pool), by the definition, one sequence after another."""
    out, pool, full, live = tables.clone(), pool.clone(), length // pt, length % pt
    before = pool.clone()
    for g in range(groups):
        par = [int(p) if 0 <= int(p) < beams else b for b, p in enumerate(parents[g * beams:(g + 1) * beams])]
        free, seen = [b for b in range(beams) if b not in par], set()
        for b, p in enumerate(par):
            row, src = g * beams + b, g * beams + p
            out[row, :full] = tables[src, :full]
            if not live:
                continue
            if p not in seen:
                seen.add(p)
                out[row, full] = tables[src, full]
                continue
            page, dst = int(tables[src, full]), int(tables[g * beams + free.pop(0), full])
            out[row, full] = dst
            if 0 <= page < pool.shape[1] and 0 <= dst < pool.shape[1]:
                pool[:, dst] = before[:, page]
    return out, pool
