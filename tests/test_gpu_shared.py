"""The operators for several sequences behind one prompt against 64-bit implementations (tests/shared_ref.py), with bounds derived there."""
import math

import pytest
import torch

from paper_2405_04304_amd import binding as B
import shared_ref as R

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def dev():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch.device("cuda:0")


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _cache(g, n_seqs, cols, pt, nkv, dh, prefix, spare=2):
    """(pages, tables, prefix pages, prefix table) on the host: pages in random order, more of them than the tables name."""
    n = n_seqs * cols + spare
    pages = torch.randn(n, 2, nkv, pt * dh, generator=g).to(BF16)
    tables = torch.randperm(n, generator=g)[:n_seqs * cols].to(torch.int32).view(n_seqs, cols)
    n_p = -(-prefix // pt) + 1
    return pages, tables, torch.randn(n_p, 2, nkv, pt * dh, generator=g).to(BF16), torch.randperm(n_p, generator=g).to(torch.int32)


def _attn(q, n_tok, nq, nkv, dh, pt, pages, tables, lens, ppages, ptable, prefix, max_len=0, stride=0, scale=None):
    d = dev()
    kv = B.SharedKV(pages.to(d), tables.to(d), torch.tensor(lens, dtype=torch.int32, device=d), pt, nkv, dh, prefix_pages=ppages.to(d),
                    prefix_len=prefix, prefix_table=ptable.to(d))
    wide = torch.full((q.shape[0], nq * dh + stride), 3.0, dtype=q.dtype, device=d)
    wide[:, :nq * dh] = q.to(d)
    out = torch.full((q.shape[0] + 1, nq * dh + stride), 5.0, dtype=q.dtype, device=d)
    lse = torch.full((q.shape[0] + 1, nq), 7.0, dtype=F32, device=d)
    ws = torch.empty(B.disco_attn_shared_bytes(kv, n_tok, nq, max_len), dtype=torch.uint8, device=d).fill_(0xFF)
    B.disco_attn_shared(kv, wide[:, :nq * dh], n_tok, nq, out[:, :nq * dh], ws, lse=lse, scale=scale, max_len=max_len)
    torch.cuda.synchronize()
    assert bool((out[-1] == 5.0).all()) and bool((out[:, nq * dh:] == 5.0).all()) and bool((lse[-1] == 7.0).all())
    return out[:-1, :nq * dh].cpu(), lse[:-1].cpu()


def _check_attn(got, want, dtype, n_pos):
    (out, lse), (w_out, w_lse, size, e_out, e_lse) = got, want
    tol, tol_lse = R.attention_bounds(dtype, w_out, w_lse, size, e_out, e_lse, n_pos)
    nan = w_out.isnan()
    assert bool((out.isnan() == nan).all())
    diff = (out.double() - w_out).abs()
    assert bool((diff <= tol)[~nan].all()), float((diff / tol)[~nan].max())
    fin = w_lse.isfinite()
    assert bool((lse.double() == w_lse)[~fin & ~w_lse.isnan()].all())
    assert bool(((lse.double() - w_lse).abs() <= tol_lse)[fin].all()), float(((lse.double() - w_lse).abs() / tol_lse)[fin].max())


ATTN = [
    # heads, K / V heads, d_head, page, sequences, tokens, prompt, own lengths
    (2, 2, 64, 16, 1, 1, 0, [1]),
    (2, 1, 64, 4, 3, 1, 5, [0, 1, 9]),                       # an empty sequence of its own
    (4, 2, 128, 16, 2, 1, 0, [0, 17]),                       # and one that sees nothing at all
    (4, 1, 64, 12, 3, 3, 31, [1, 3, 40]),                    # fewer own positions than tokens; pages that are no power of two
    (8, 2, 128, 32, 5, 2, 64, [2, 33, 64, 65, 31]),
    (6, 2, 64, 20, 4, 5, 257, [5, 6, 100, 20]),              # groups of three, a page that ends inside a tile
    (16, 1, 128, 16, 3, 6, 100, [6, 77, 130]),               # 96 rows of a sequence on one K / V head
    (48, 1, 64, 16, 2, 6, 40, [6, 300]),                     # 288 rows: several row tiles of one sequence
    (8, 8, 64, 64, 40, 1, 300, [1 + (7 * b) % 90 for b in range(40)]),
    (16, 2, 128, 16, 33, 1, 1000, [1 + (5 * b) % 40 for b in range(33)]),
    (4, 4, 128, 64, 2, 16, 700, [16, 900]),
    (32, 8, 64, 16, 70, 1, 130, [3] * 70),                   # 280 rows
    (2, 2, 128, 16, 1, 1, 3001, [1500]),
]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("case", ATTN, ids=[f"{c[0]}on{c[1]}x{c[2]}p{c[3]}s{c[4]}t{c[5]}n{c[6]}" for c in ATTN])
def test_attention(case, dtype):
    nq, nkv, dh, pt, s, t, prefix, lens = case
    g = _gen(nq * dh + s * t + prefix)
    cols = max(1, -(-max(lens) // pt))
    pages, tables, ppages, ptable = _cache(g, s, cols, pt, nkv, dh, prefix)
    q = (1.5 * torch.randn(s * t, nq * dh, generator=g)).to(dtype)
    got = _attn(q, t, nq, nkv, dh, pt, pages, tables, lens, ppages, ptable, prefix, stride=8)
    want = R.attention(q, t, nq, nkv, dh, pt, pages, tables, lens, ppages, ptable, prefix, dh ** -0.5)
    _check_attn(got, want, dtype, prefix + max(lens))


@pytest.mark.parametrize("max_len", [1, 64, 100000])
def test_attention_expected_length_changes_no_meaning(max_len):
    g, lens = _gen(3), [700, 5, 260]
    pages, tables, ppages, ptable = _cache(g, 3, 44, 16, 2, 64, 90)
    q = torch.randn(3, 4 * 64, generator=g)
    got = _attn(q, 1, 4, 2, 64, 16, pages, tables, lens, ppages, ptable, 90, max_len=max_len)
    _check_attn(got, R.attention(q, 1, 4, 2, 64, 16, pages, tables, lens, ppages, ptable, 90, 0.125), F32, 790)


@pytest.mark.parametrize("t", [1, 4])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
def test_attention_what_a_row_does_not_see_does_not_touch_it(t, dtype):
    """Infinities and NaN behind the prompt's end, behind a sequence's end, in unnamed pages, and in the newest positions, which the
    call's earlier tokens do not see."""
    nq, nkv, dh, pt, prefix, lens = 4, 2, 64, 16, 37, [21, 64, 5]
    g = _gen(11 + t)
    pages, tables, ppages, ptable = _cache(g, 3, 5, pt, nkv, dh, prefix)
    for head in range(nkv):
        for pos, x in ((prefix, math.nan), (prefix + 5, math.inf)):
            R.key_at(ppages, int(ptable[pos // pt]), head, pos % pt, pt, dh)[:] = x
            R.val_at(ppages, int(ptable[pos // pt]), head, pos % pt, pt, dh)[:] = x
        for b, n in enumerate(lens):
            for pos, x in ((n, math.nan), (n + 3, -math.inf)):
                R.key_at(pages, int(tables[b, pos // pt]), head, pos % pt, pt, dh)[:] = x
                R.val_at(pages, int(tables[b, pos // pt]), head, pos % pt, pt, dh)[:] = x
        if t > 1:                                    # the last token's own value entry
            R.val_at(pages, int(tables[0, (lens[0] - 1) // pt]), head, (lens[0] - 1) % pt, pt, dh)[:8] = math.inf
            R.val_at(pages, int(tables[1, (lens[1] - 2) // pt]), head, (lens[1] - 2) % pt, pt, dh)[3:5] = math.nan
    used = {int(x) for x in tables.flatten()}
    for page in range(pages.shape[0]):
        if page not in used:
            pages[page] = math.nan
    q = torch.randn(3 * t, nq * dh, generator=g).to(dtype)
    got = _attn(q, t, nq, nkv, dh, pt, pages, tables, lens, ppages, ptable, prefix)
    want = R.attention(q, t, nq, nkv, dh, pt, pages, tables, lens, ppages, ptable, prefix, dh ** -0.5)
    finite = want[0].isfinite()
    assert bool((got[0].isfinite() == finite).all()) and (t == 1) == bool(finite.all())
    _check_attn((torch.where(finite, got[0], torch.zeros_like(got[0])), got[1]),
                (torch.where(finite, want[0], torch.zeros_like(want[0])), want[1], torch.where(finite, want[2], torch.zeros_like(want[2])), want[3], want[4]),
                dtype, prefix + max(lens))


def test_attention_pages_outside_the_pool_are_not_read():
    nq, nkv, dh, pt, prefix, lens = 4, 2, 64, 16, 50, [40, 40, 40, 40]
    g = _gen(21)
    pages, tables, ppages, ptable = _cache(g, 4, 3, pt, nkv, dh, prefix)
    tables[1, 1], tables[2, 2], tables[3, 0] = -1, pages.shape[0], 1 << 30
    tables[2, 1] = tables[0, 1]                      # (two sequences may share a page)
    q = torch.randn(4, nq * dh, generator=g)
    got = _attn(q, 1, nq, nkv, dh, pt, pages, tables, lens, ppages, ptable, prefix)
    assert bool(got[0][1:].isnan().all()) and bool(got[0][0].isfinite().all())
    lens = [40, 16, 32, 0]                           # shorter: nobody sees them
    got = _attn(q, 1, nq, nkv, dh, pt, pages, tables, lens, ppages, ptable, prefix)
    _check_attn(got, R.attention(q, 1, nq, nkv, dh, pt, pages, tables, lens, ppages, ptable, prefix, 0.125), F32, 90)
    ptable[2] = ppages.shape[0] + 7
    got = _attn(q, 1, nq, nkv, dh, pt, pages, tables, lens, ppages, ptable, prefix)
    assert bool(got[0].isnan().all())


def test_attention_scores_far_apart():
    """Scores up to a few hundred: the running maximum moves, old sums vanish; a length larger than a table holds is cut."""
    nq, nkv, dh, pt, prefix = 2, 1, 128, 16, 600
    g = _gen(5)
    pages, tables, ppages, ptable = _cache(g, 2, 4, pt, nkv, dh, prefix)
    q = 25.0 * torch.randn(2, nq * dh, generator=g)
    got = _attn(q, 1, nq, nkv, dh, pt, pages, tables, [64, 1000], ppages, ptable, prefix)
    _check_attn(got, R.attention(q, 1, nq, nkv, dh, pt, pages, tables, [64, 64], ppages, ptable, prefix, dh ** -0.5), F32, 664)


APPEND = [
    # heads, K / V heads, d_head, page, sequences, tokens, prompt, own lengths
    (2, 2, 64, 16, 1, 1, 0, [1]),
    (4, 1, 128, 4, 3, 1, 5, [1, 4, 5]),
    (6, 2, 64, 12, 4, 5, 33, [5, 17, 30, 48]),
    (8, 8, 128, 64, 2, 16, 7, [16, 100]),
    (32, 8, 128, 16, 70, 1, 300, [1 + b % 40 for b in range(70)]),
]


def _append_want(qkv, places, nq, nkv, dh, pt, pages, tables, prefix, rope, q_gain, k_gain, eps, q0):
    """Queries and pages after the rows, with elementwise bounds (rounding of the result; norm and rotation in fp32)."""
    q, pages = q0.double().clone(), pages.double().clone()
    q_tol, p_tol = torch.zeros_like(q), torch.zeros_like(pages)
    u = 2.0 ** -24
    n_ops = (dh // 2 + 16 if q_gain is not None or k_gain is not None else 0) + (6 if rope is not None else 0)
    for i, (b, pos) in enumerate(places):
        if not (0 <= b < tables.shape[0] and 0 <= pos < tables.shape[1] * pt):
            continue
        x = qkv[i].double().view(-1, dh)
        cs = rope[prefix + pos] if rope is not None else None
        xq, sq = R.norm_rotate(x[:nq], q_gain, eps, cs)
        xk, sk = R.norm_rotate(x[nq:nq + nkv], k_gain, eps, cs)
        q[i] = xq.reshape(-1)
        q_tol[i] = (sq * n_ops * u).reshape(-1) + (xq.abs().reshape(-1) * R.STEP[qkv.dtype] if n_ops else 0.0)
        page, off = int(tables[b, pos // pt]), pos % pt
        if not 0 <= page < pages.shape[0]:
            continue
        for h in range(nkv):
            R.key_at(pages, page, h, off, pt, dh)[:] = xk[h]
            R.key_at(p_tol, page, h, off, pt, dh)[:] = sk[h] * n_ops * u + xk[h].abs() * R.STEP[BF16]
            R.val_at(pages, page, h, off, pt, dh)[:] = x[nq + nkv + h]
            R.val_at(p_tol, page, h, off, pt, dh)[:] = x[nq + nkv + h].abs() * R.STEP[BF16]
    return q, q_tol + 1e-30, pages, p_tol


def _append(qkv, nq, nkv, dh, pt, pages, tables, lens, prefix, rope, q_gain, k_gain, places=None, stride=0):
    d = dev()
    put = lambda x: None if x is None else x.to(d)  # noqa: E731
    pages = pages.to(d)
    kv = B.SharedKV(pages, tables.to(d), None if lens is None else torch.tensor(lens, dtype=torch.int32, device=d), pt, nkv, dh, prefix_len=prefix)
    wide = torch.full((qkv.shape[0], qkv.shape[1] + stride), 3.0, dtype=qkv.dtype, device=d)
    wide[:, :qkv.shape[1]] = qkv.to(d)
    q = torch.full((qkv.shape[0] + 1, nq * dh + stride), 5.0, dtype=qkv.dtype, device=d)
    seq = pos = None
    if places is not None:
        seq, pos = (torch.tensor([p[j] for p in places], dtype=torch.int32, device=d) for j in (0, 1))
    B.disco_append(kv, wide[:, :qkv.shape[1]], nq, q[:-1, :nq * dh], seq=seq, pos=pos, rope=put(rope), q_gain=put(q_gain), k_gain=put(k_gain), eps=1e-6)
    torch.cuda.synchronize()
    assert bool((q[-1] == 5.0).all()) and bool((q[:, nq * dh:] == 5.0).all())
    return q[:-1, :nq * dh].cpu(), pages.cpu()


@pytest.mark.parametrize("rope,gains", [(True, "both"), (True, ""), (False, ""), (False, "k")])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("case", APPEND, ids=[f"{c[0]}on{c[1]}x{c[2]}p{c[3]}s{c[4]}t{c[5]}" for c in APPEND])
def test_append_last_tokens(case, dtype, rope, gains):
    nq, nkv, dh, pt, s, t, prefix, lens = case
    g = _gen(nq + dh + s)
    cols = -(-max(lens) // pt)
    pages, tables, _, _ = _cache(g, s, cols, pt, nkv, dh, 0)
    qkv = torch.randn(s * t, (nq + 2 * nkv) * dh, generator=g).to(dtype)
    tab = R.rope_table(prefix + cols * pt, dh).to(F32) if rope else None
    q_gain = 1 + 0.2 * torch.randn(dh, generator=g) if gains == "both" else None
    k_gain = 1 + 0.2 * torch.randn(dh, generator=g) if gains else None
    q, after = _append(qkv, nq, nkv, dh, pt, pages, tables, lens, prefix, tab, q_gain, k_gain, stride=16)
    places = [(b, lens[b] - t + j) for b in range(s) for j in range(t)]
    w_q, q_tol, w_p, p_tol = _append_want(qkv, places, nq, nkv, dh, pt, pages, tables, prefix, tab, q_gain, k_gain, 1e-6, torch.full_like(q, 5.0))
    assert bool(((q.double() - w_q).abs() <= q_tol).all())
    assert bool(((after.double() - w_p).abs() <= p_tol).all())      # untouched entries bit for bit


@pytest.mark.parametrize("pt", [4, 12, 16, 64])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
def test_append_ragged_rows_in_any_order(pt, dtype):
    """Runs that start and end inside pages, single rows, rows in descending order, padding, places outside the tables, pages outside the pool."""
    nq, nkv, dh, prefix = 4, 2, 128, 9
    g = _gen(pt)
    cols = -(-200 // pt)
    pages, tables, _, _ = _cache(g, 5, cols, pt, nkv, dh, 0)
    places = [(0, p) for p in range(3, 95)] + [(-1, -1)] * 3 + [(1, p) for p in range(30, 10, -1)] + [(2, 7)] + [(3, p) for p in range(150)]
    places += [(4, -1), (5, 0), (4, cols * pt), (1 << 30, 2), (4, 1 << 30), (2, 8), (2, 9)] + [(4, p) for p in range(0, 60, 3)] + [(0, p) for p in range(95, 130)]
    tables[3, 1], tables[2, 0] = -1, pages.shape[0]
    qkv = torch.randn(len(places), (nq + 2 * nkv) * dh, generator=g).to(dtype)
    tab = R.rope_table(prefix + cols * pt, dh).to(F32)
    q, after = _append(qkv, nq, nkv, dh, pt, pages, tables, None, prefix, tab, None, None, places=places)
    w_q, q_tol, w_p, p_tol = _append_want(qkv, places, nq, nkv, dh, pt, pages, tables, prefix, tab, None, None, 1e-6, torch.full_like(q, 5.0))
    assert bool(((q.double() - w_q).abs() <= q_tol).all())
    assert bool(((after.double() - w_p).abs() <= p_tol).all())


def test_append_keeps_infinities_and_nan_of_a_head_to_itself():
    nq, nkv, dh, pt = 4, 2, 64, 16
    g = _gen(2)
    pages, tables, _, _ = _cache(g, 2, 2, pt, nkv, dh, 0)
    qkv = torch.randn(2, (nq + 2 * nkv) * dh, generator=g)
    clean = _append(qkv, nq, nkv, dh, pt, pages, tables, [3, 20], 0, None, None, torch.ones(dh))
    qkv[0, dh + 3], qkv[1, (nq + 1) * dh] = math.nan, math.inf
    q, after = _append(qkv, nq, nkv, dh, pt, pages, tables, [3, 20], 0, None, None, torch.ones(dh))
    hit = q[0].view(nq, dh)
    assert bool(hit[1, 3].isnan()) and torch.equal(hit[[0, 2, 3]], clean[0][0].view(nq, dh)[[0, 2, 3]]) and torch.equal(q[1], clean[0][1])
    page = int(tables[1, 1])
    same = (after == clean[1]) | (after.isnan() & clean[1].isnan())
    same[page, 0, 1].view(pt, dh)[3] = True
    assert bool(same.all()) and bool(R.key_at(after, page, 1, 3, pt, dh)[0].isnan())


def test_rope_table():
    t = B.disco_rope_table(5000, 128, 10000.0)
    assert float((t.cpu().double() - R.rope_table(5000, 128)).abs().max()) <= 2.0 ** -24


def _select(logits, scores, groups, beams, k, done=None, end=-1, ld=0):
    d = dev()
    wide = torch.full((logits.shape[0], logits.shape[1] + ld), math.nan, dtype=logits.dtype, device=d)
    wide[:, :logits.shape[1]] = logits.to(d)
    tok, par, don = (torch.full((groups + 1, k), -9, dtype=torch.int32, device=d) for _ in range(3))
    sc = torch.full((groups + 1, k), 9.0, dtype=F32, device=d)
    ws = torch.empty(B.disco_beam_select_bytes(groups, beams, logits.shape[1], k), dtype=torch.uint8, device=d).fill_(0xFF)
    B.disco_beam_select(wide[:, :logits.shape[1]], scores.to(d), groups, beams, k, tok, par, sc, ws, done=None if done is None else done.to(d),
                        done_out=don, end_token=end)
    torch.cuda.synchronize()
    assert bool((tok[-1] == -9).all()) and bool((sc[-1] == 9.0).all()) and bool((par[-1] == -9).all()) and bool((don[-1] == -9).all())
    return tok[:-1].tolist(), par[:-1].tolist(), sc[:-1].tolist(), don[:-1].tolist()


def _check_select(got, want):
    for g, row in enumerate(want):
        for j, (v, b, s, d) in enumerate(row):
            assert (got[0][g][j], got[1][g][j], got[3][g][j]) == (v, b, d), (g, j, got[0][g], got[1][g], row)
            x = got[2][g][j]
            # one rounding to fp32 of a key whose logsumexp is within 2^-22 (fp32 exponentials, sums of up to 16 by lane)
            assert (math.isnan(s) and math.isnan(x)) or x == s or abs(x - s) <= 2.0 ** -24 * abs(s) + 2.0 ** -22, (g, j, x, s)


SELECT = [(1, 1, 1, 1), (1, 1, 7, 3), (1, 4, 5, 20), (2, 3, 100, 7), (1, 4, 32000, 4), (3, 8, 4096, 16), (2, 5, 4097, 10), (5, 2, 49153, 4), (1, 64, 1000, 64),
          (1, 2, 131072, 128), (2, 16, 33333, 16), (1, 64, 300, 128), (33, 5, 60000, 12), (1, 1, 1048576, 128)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("groups,beams,vocab,k", SELECT)
def test_select(groups, beams, vocab, k, dtype):
    """bf16 logits hold many equal values: the lowest index goes first."""
    g = _gen(vocab + k)
    logits = (2.5 * torch.randn(groups * beams, vocab, generator=g)).to(dtype)
    scores = -20 * torch.rand(groups * beams, generator=g)
    _check_select(_select(logits, scores, groups, beams, k, ld=3), R.select(logits, scores, groups, beams, k))


def test_select_equal_candidates():
    """All logits equal, and equal rows: lower beam, then lower token."""
    logits, scores = torch.zeros(6, 5000), torch.tensor([-1.0, -1.0, -2.0, -3.0, -1.0, -1.0])
    logits[:, 4990:] = 1.0
    _check_select(_select(logits, scores, 2, 3, 40), R.select(logits, scores, 2, 3, 40))
    logits[:, 100:200], logits[:, 150:160] = 2.0, 2.0
    logits[1, 4000:] = 3.0 * torch.tensor([1.0, -0.0]).repeat(500)       # zeros of both signs are equal
    logits[0], logits[0, ::3] = 0.0, -0.0
    _check_select(_select(logits, scores, 2, 3, 100), R.select(logits, scores, 2, 3, 100))
    logits, scores = torch.full((2, 9000), 0.25), torch.zeros(2)
    _check_select(_select(logits, scores, 1, 2, 64), R.select(logits, scores, 1, 2, 64))


def test_select_masked_tokens_and_finished_beams():
    g = _gen(1)
    logits = torch.randn(8, 777, generator=g)
    logits[0, 5:] = -math.inf                        # five tokens left
    logits[1] = -math.inf                            # none
    logits[2, ::2] = torch.finfo(F32).min
    logits[3, 7] = math.nan                          # of a finished beam: not looked at
    scores = torch.tensor([0.0, -0.5, -1.0, -2.0, -math.inf, -math.inf, -math.inf, -0.25])
    done = torch.tensor([0, 0, 0, 1, 0, 0, 1, 0], dtype=torch.int32)
    for groups, beams in ((1, 8), (2, 4)):
        _check_select(_select(logits, scores, groups, beams, 12, done, 2), R.select(logits, scores, groups, beams, 12, done, 2))
    few = logits[:2, :9].contiguous()                # fewer candidates than places
    _check_select(_select(few, scores[:2], 1, 2, 12, None, 3), R.select(few, scores[:2], 1, 2, 12, None, 3))
    _check_select(_select(few, torch.full((2,), -math.inf), 1, 2, 3), R.select(few, torch.full((2,), -math.inf), 1, 2, 3))


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_select_says_so_where_a_number_is_none(bad):
    g = _gen(4)
    for where in (0, 5000, 8190):
        logits = torch.randn(6, 8191, generator=g)
        logits[2, where] = bad
        scores = -torch.rand(6, generator=g)
        got = _select(logits, scores, 3, 2, 4)
        _check_select(got, R.select(logits, scores, 3, 2, 4))
        assert got[0][1] == [-1] * 4 and min(got[0][0] + got[0][2]) >= 0
    scores[0] = bad
    got = _select(torch.randn(6, 100, generator=g), scores, 3, 2, 4)
    assert got[0][0] == [-1] * 4 and all(math.isnan(x) for x in got[2][0]) and min(got[0][1] + got[0][2]) >= 0


@pytest.mark.parametrize("groups,beams,length,pt,cols", [(1, 1, 5, 4, 2), (1, 4, 37, 16, 4), (3, 8, 64, 16, 5), (2, 5, 1, 12, 1), (1, 64, 100, 16, 9), (4, 3, 48, 16, 3), (2, 2, 0, 4, 1)])
def test_reorder(groups, beams, length, pt, cols):
    g = _gen(beams + length)
    n, nkv, dh, layers = groups * beams, 2, 64, 3
    pool = torch.randn(layers, n * cols + 1, 2, nkv, pt * dh, generator=g).to(BF16)
    tables = torch.randperm(n * cols + 1, generator=g)[:n * cols].to(torch.int32).view(n, cols)
    for parents in (torch.randint(0, beams, (n,), generator=g), torch.arange(beams).repeat(groups), torch.full((n,), beams - 1),
                    torch.arange(beams - 1, -1, -1).repeat(groups), torch.randint(-2, beams + 2, (n,), generator=g)):
        d = dev()
        p, out = pool.to(d), torch.full((n + 1, cols), -5, dtype=torch.int32, device=d)
        B.disco_beam_reorder(p, tables.to(d), parents.to(torch.int32).to(d), out, groups, beams, length, pt)
        torch.cuda.synchronize()
        w_t, w_p = R.reorder(pool, tables, parents.tolist(), groups, beams, length, pt)
        assert torch.equal(out[:-1].cpu(), w_t) and bool((out[-1] == -5).all())
        assert torch.equal(p.cpu().view(torch.int16), w_p.view(torch.int16))


def test_reorder_pages_outside_the_pool_and_strided_layers():
    g = _gen(9)
    wide = torch.randn(2, 14, 2, 1, 16 * 64, generator=g).to(BF16)
    pool = wide[:, :12]
    tables = torch.randperm(12, generator=g).to(torch.int32).view(4, 3)
    tables[0, 1], tables[3, 1] = -1, 13
    for parents in ([1, 1, 0, 0], [2, 2, 2, 2], [3, 3, 1, 1]):
        d = dev()
        p, out = wide.to(d), torch.empty(4, 3, dtype=torch.int32, device=d)
        B.disco_beam_reorder(p[:, :12], tables.to(d), torch.tensor(parents, dtype=torch.int32, device=d), out, 1, 4, 20, 16)
        w_t, w_p = R.reorder(pool, tables, parents, 1, 4, 20, 16)
        assert torch.equal(out.cpu(), w_t)
        assert torch.equal(p[:, :12].cpu().view(torch.int16), w_p.view(torch.int16)) and torch.equal(p[:, 12:].cpu(), wide[:, 12:])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("kind", ["random", "few ranges", "rising", "equal", "steps"])
@pytest.mark.parametrize("beams,vocab,k", [(3, 70001, 128), (64, 140003, 64), (2, 3000, 128)])
def test_select_where_the_best_lie_close_together(beams, vocab, k, kind, dtype):
    """Many candidates: the best of a row in a few ranges of its vocabulary (a mask), all in its last one, all equal, a few values only."""
    g = _gen(vocab + k)
    logits = torch.randn(beams, vocab, generator=g)
    if kind == "few ranges":
        mask = torch.ones(vocab, dtype=torch.bool)
        for first in (100, vocab // 2, vocab - 900):
            mask[first:first + 700] = False
        logits[:, mask] = -math.inf
    elif kind == "rising":
        logits = torch.linspace(-4.0, 4.0, vocab).repeat(beams, 1)
    elif kind == "equal":
        logits = torch.full((beams, vocab), -1.25)
    elif kind == "steps":
        logits = torch.randint(-3, 3, (beams, vocab), generator=g).float()
    logits = logits.to(dtype)
    scores = -torch.arange(beams, dtype=F32) / 8
    _check_select(_select(logits, scores, 1, beams, k), R.select(logits, scores, 1, beams, k))
