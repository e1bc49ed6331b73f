"""Decoding steps of several sequences behind one prompt, and beam search built on them, against the 64-bit oracle: every sequence's logits
are those of its own tokens read from the start, whatever beams it shared pages with on the way."""
import dataclasses
import math

import pytest
import torch

from paper_2405_04304_amd import binding as B
from paper_2405_04304_amd.engine import SpecEngine
from oracle import disco_oracle as O
from workloads import synth as W

pytestmark = pytest.mark.gpu

REL = 2e-3           # of a row's largest logit: the bound that the forwards of one sequence are held to (test_gpu_parity.py)
SHAPES = {
    "LayerNorm, own heads": W.ModelShape("A", 2, 256, 4, 64, 4, 512, 1024, max_pos=256),
    "LayerNorm, one K / V head": W.ModelShape("A", 2, 384, 6, 64, 1, 768, 512, max_pos=256),
    "RMSNorm, own heads": W.ModelShape("B", 2, 256, 2, 128, 2, 512, 1024),
    "RMSNorm, grouped": W.ModelShape("B", 3, 512, 8, 64, 2, 1024, 512),
}


def dev():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch.device("cuda:0")


def _models(shape, seed=0):
    w = W.make_weights(shape, seed, "bf16")
    return B.DiscoModel(shape, w, dev()), O.Model(shape, w, kv_bf16=True)


def _oracle_logits(om, tokens):
    return om.forward(tokens, om.new_cache(len(tokens)))[-1]


@pytest.mark.parametrize("n_prompt,n_seqs,pt", [(1, 1, 16), (38, 3, 16), (21, 16, 4), (65, 9, 32)])
@pytest.mark.parametrize("name", SHAPES)
def test_steps_match_the_oracle(name, n_prompt, n_seqs, pt):
    """Steps with reorderings between them that copy pages, share full ones and leave sequences where they are."""
    shape, d = SHAPES[name], dev()
    gm, om = _models(shape)
    prompt = W.make_prompt(1, n_prompt, shape.vocab).tolist()
    steps = 7
    kv = B.DiscoKV(gm, n_prompt + 2 * pt + 64, pt, page_order=list(reversed(range(-(-(n_prompt + 2 * pt + 64) // pt)))))
    if n_prompt > 1:
        ws_one, am = gm.workspace(16, n_prompt + 96), torch.zeros(16, dtype=torch.int32, device=d)
        toks = torch.tensor(prompt, dtype=torch.int32, device=d)
        for i in range(0, n_prompt - 1, 16):
            B.disco_verify(gm, kv, toks.data_ptr() + 4 * i, min(16, n_prompt - 1 - i), am, None, ws_one)
    seqs = B.Sequences(gm, n_seqs, steps, pt)
    seqs.pages.fill_(math.nan)                       # nothing but what steps have written may be read
    ws = gm.step_workspace(kv, seqs)
    logits = torch.empty(n_seqs, shape.vocab, dtype=torch.float32, device=d)
    g = torch.Generator().manual_seed(n_prompt + n_seqs)
    history = [[prompt[-1]] for _ in range(n_seqs)]
    for t in range(steps):
        B.disco_step(gm, kv, seqs, torch.tensor([h[-1] for h in history], dtype=torch.int32, device=d), logits, ws)
        got = logits.cpu().double()
        for b in range(n_seqs) if t in (0, 3, steps - 1) else (0, n_seqs - 1):
            want = _oracle_logits(om, prompt[:-1] + history[b])
            scale = float(want.abs().max())
            assert float((got[b] - want).abs().max()) <= REL * scale, (t, b)
        parents = torch.randint(0, n_seqs, (n_seqs,), generator=g) if t != 2 else torch.arange(n_seqs)
        new = torch.randint(0, shape.vocab, (n_seqs,), generator=g)
        if t + 1 < steps:
            B.disco_step_reorder(seqs, parents.to(torch.int32).to(d))
            history = [history[int(p)] + [int(x)] for p, x in zip(parents, new)]
    assert kv.len == n_prompt - 1


def test_step_is_the_forward_of_one_sequence():
    """One sequence: logits as disco_verify gives them for the same tokens, to the order of fp32 sums."""
    shape, d = W.ModelShape("B", 2, 768, 12, 64, 12, 2048, 4096), dev()
    gm, _ = _models(shape)
    toks = W.make_prompt(3, 40, shape.vocab).to(torch.int32).to(d)
    am, ws_one = torch.zeros(16, dtype=torch.int32, device=d), gm.workspace(16, 160)
    one, kv = B.DiscoKV(gm, 96, 16), B.DiscoKV(gm, 96, 16)
    for i in (0, 16):
        B.disco_verify(gm, one, toks.data_ptr() + 4 * i, 16, am, None, ws_one)
        B.disco_verify(gm, kv, toks.data_ptr() + 4 * i, 16, am, None, ws_one)
    seqs = B.Sequences(gm, 1, 8, 16)
    ws, a, b = gm.step_workspace(kv, seqs), torch.empty(1, shape.vocab, device=d), torch.empty(1, shape.vocab, device=d)
    for i in range(32, 40):
        B.disco_verify(gm, one, toks[i:i + 1], 1, am, a, ws_one)
        B.disco_step(gm, kv, seqs, toks[i:i + 1].contiguous(), b, ws)
        torch.cuda.synchronize()
        assert float((a - b).abs().max()) <= 1e-4 * float(a.abs().max())


def _follow(om, prompt, res, n_beams, end):
    """Checks a beam search's result against the oracle's own search, as far as the logits' bound decides: returned scores, their order, and that
    no hypothesis of the oracle's search is better than the worst returned one by more than the bound allows."""
    vocab = om.shape.vocab
    beams = [(0.0, [], False)]
    steps = max(len(r["tokens"]) for r in res)
    bound = 0.0
    for _ in range(steps):
        cand = []
        for s, toks, done in beams:
            if done:
                cand.append((s, toks, True))
                continue
            x = _oracle_logits(om, prompt + toks)
            bound = max(bound, 2 * REL * float(x.abs().max()))
            logp = torch.log_softmax(x, 0) + s
            for v in logp.topk(min(n_beams + 1, vocab)).indices.tolist():
                cand.append((float(logp[v]), toks + [v], v == end))
        beams = sorted(cand, key=lambda c: -c[0])[:n_beams]
    return beams, bound * steps


@pytest.mark.parametrize("name,n_beams,max_new,end", [("LayerNorm, own heads", 4, 12, -1), ("RMSNorm, grouped", 5, 9, -1), ("RMSNorm, own heads", 1, 6, -1),
                                                      ("LayerNorm, one K / V head", 16, 5, -1)])
def test_beam_search_matches_the_oracle(name, n_beams, max_new, end):
    shape = SHAPES[name]
    gm, om = _models(shape, 5)
    prompt = W.make_prompt(2, 35, shape.vocab).tolist()
    eng = SpecEngine(gm, None, None, max_ctx=96)
    res = eng.beam_search(prompt, n_beams, max_new, end)
    assert len(res) == n_beams and all(len(r["tokens"]) == max_new for r in res)
    assert [r["score"] for r in res] == sorted((r["score"] for r in res), reverse=True)
    assert len({tuple(r["tokens"]) for r in res}) == n_beams
    want, bound = _follow(om, prompt, res, n_beams, end)
    for r in res:                                    # scores: the oracle's log probabilities of the same tokens
        s, toks = 0.0, list(prompt)
        for v in r["tokens"]:
            s += float(torch.log_softmax(_oracle_logits(om, toks), 0)[v])
            toks.append(v)
        assert abs(s - r["score"]) <= bound, (s, r["score"], bound)
    for got, (s, toks, _) in zip(res, want):
        assert got["tokens"] == toks or abs(got["score"] - s) <= 2 * bound
    if n_beams == 1:
        assert res[0]["tokens"] == eng.greedy(prompt, max_new)
    again = eng.beam_search(prompt, n_beams, max_new, end)
    assert again == res                              # sums in a fixed order: the same bits


def test_beam_search_ends():
    """An end token that the best beam takes: it keeps its score, the others go on; a search whose beams have all ended stops."""
    shape = SHAPES["RMSNorm, grouped"]
    gm, om = _models(shape, 5)
    prompt = W.make_prompt(2, 20, shape.vocab).tolist()
    eng = SpecEngine(gm, None, None, max_ctx=96)
    free = eng.beam_search(prompt, 3, 8)
    end = free[0]["tokens"][3]
    res = eng.beam_search(prompt, 3, 24, end)
    for r in res:
        assert end not in r["tokens"][:-1] and (r["tokens"][-1] == end or len(r["tokens"]) == 24)
        s, toks, bound = 0.0, list(prompt), 0.0
        for v in r["tokens"]:
            x = _oracle_logits(om, toks)
            bound += 2 * REL * float(x.abs().max())
            s += float(torch.log_softmax(x, 0)[v])
            toks.append(v)
        assert abs(s - r["score"]) <= bound
    with pytest.raises(ValueError, match="positions"):
        eng.beam_search(prompt, 3, 200)


def test_a_captured_step_replays():
    """Step, selection and reordering in graphs (one for each direction between the two tables), replayed with eager work in between: the
    same tokens and scores as without graphs.  Two captured searches with workspaces of their own share nothing."""
    shape, d = SHAPES["RMSNorm, own heads"], dev()
    gm, _ = _models(shape, 1)
    prompt = W.make_prompt(7, 30, shape.vocab).to(torch.int32).to(d)
    am, ws_one = torch.zeros(16, dtype=torch.int32, device=d), gm.workspace(16, 96)
    kv = B.DiscoKV(gm, 96, 16)
    for i in (0, 16):
        B.disco_verify(gm, kv, prompt.data_ptr() + 4 * i, min(16, 29 - i), am, None, ws_one)
    nb, steps = 4, 5

    class Search:
        def __init__(self):
            self.seqs = B.Sequences(gm, nb, 16, 16)
            self.ws, self.logits = gm.step_workspace(kv, self.seqs), torch.empty(nb, shape.vocab, device=d)
            self.tokens = [torch.empty(nb, dtype=torch.int32, device=d) for _ in range(2)]
            self.scores = [torch.empty(nb, device=d) for _ in range(2)]
            self.parents, self.sel = torch.empty(nb, dtype=torch.int32, device=d), torch.empty(B.disco_beam_select_bytes(1, nb, shape.vocab, nb), dtype=torch.uint8, device=d)

        def start(self, seed):
            self.seqs.reset()
            self.tokens[0].copy_(torch.randint(0, shape.vocab, (nb,), generator=torch.Generator().manual_seed(seed)).to(torch.int32))
            self.scores[0].copy_(torch.tensor([0.0, -0.5, -1.0, -float("inf")]))

        def step(self, t):
            a, b = t & 1, 1 - (t & 1)
            B.disco_step(gm, kv, self.seqs, self.tokens[a], self.logits, self.ws)
            B.disco_beam_select(self.logits, self.scores[a], 1, nb, nb, self.tokens[b], self.parents, self.scores[b], self.sel)
            B.disco_step_reorder(self.seqs, self.parents)

        def result(self):
            torch.cuda.synchronize()
            return self.tokens[steps & 1].tolist(), self.scores[steps & 1].tolist(), self.logits.cpu().clone()

    one, two = Search(), Search()
    want = {}
    for seed in (1, 2):
        one.start(seed)
        for t in range(steps):
            one.step(t)
        want[seed] = one.result()
    graphs = {}
    side = torch.cuda.Stream()
    for s in (one, two):
        s.start(1)
        torch.cuda.synchronize()
        graphs[s] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[s], stream=side):
            for t in range(steps):
                s.step(t)
    for seeds in ((1, 2), (2, 1), (1, 1)):
        for s, seed in zip((one, two), seeds):
            s.start(seed)
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        for s, st in zip((one, two), streams):
            with torch.cuda.stream(st):
                graphs[s].replay()
        torch.randn(1000, device=d).sum().item()     # eager work beside them
        for s, seed in zip((one, two), seeds):
            got = s.result()
            assert got[0] == want[seed][0] and got[1] == want[seed][1] and torch.equal(got[2], want[seed][2])


def test_step_on_another_stream_than_the_current():
    shape, d = SHAPES["LayerNorm, own heads"], dev()
    gm, _ = _models(shape)
    kv, seqs = B.DiscoKV(gm, 64, 16), B.Sequences(gm, 2, 8, 16)
    ws, tok = gm.step_workspace(kv, seqs), torch.tensor([5, 9], dtype=torch.int32, device=d)
    out = [torch.empty(2, shape.vocab, device=d) for _ in range(2)]
    B.disco_step(gm, kv, seqs, tok, out[0], ws)
    torch.cuda.synchronize()
    seqs.reset()
    s = torch.cuda.Stream()
    B.disco_step(gm, kv, seqs, tok, out[1], ws, stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(*out)


def test_step_refusals():
    shape, d = SHAPES["RMSNorm, grouped"], dev()
    gm, _ = _models(shape)
    other, _ = _models(dataclasses.replace(shape, n_layers=1))
    kv, seqs = B.DiscoKV(gm, 64, 16), B.Sequences(gm, 2, 20, 16)
    ws, tok, out = gm.step_workspace(kv, seqs), torch.tensor([5, 9], dtype=torch.int32, device=d), torch.empty(2, shape.vocab, device=d)

    def code(f, *a, **k):
        with pytest.raises(B.DiscoError) as e:
            f(*a, **k)
        return e.value.code

    assert code(B.disco_step, other, kv, seqs, tok, out, ws) == B.ESTATE
    assert code(B.disco_step, gm, kv, seqs, tok.long(), out, ws) == B.EINVAL
    assert code(B.disco_step, gm, kv, seqs, tok[:1], out, ws) == B.EINVAL
    assert code(B.disco_step, gm, kv, seqs, tok, out[:1], ws) == B.EINVAL
    assert code(B.disco_step, gm, kv, seqs, tok.cpu(), out, ws) == B.EINVAL
    small = B.Workspace(ws.nbytes - 256, d)
    assert code(B.disco_step, gm, kv, seqs, tok, out, small) == B.EINVAL
    assert code(B.disco_step, gm, kv, B.Sequences(gm, 17, 20, 16), torch.zeros(17, dtype=torch.int32, device=d), torch.empty(17, shape.vocab, device=d), ws) == B.EINVAL
    assert code(B.disco_step, gm, kv, B.Sequences(gm, 2, 20, 32), tok, out, ws) == B.EINVAL       # another page size than the prompt's
    assert code(B.disco_step, gm, B.DiscoKV(gm, 16, 16), seqs, tok, out, ws) == B.ECAP            # its rotary table ends before the tables do
    seqs.len = 32
    assert code(B.disco_step, gm, kv, seqs, tok, out, ws) == B.ECAP and seqs.len == 32
    seqs.len = 0
    B.disco_step(gm, kv, seqs, tok, out, ws)
    torch.cuda.synchronize()
    assert bool(out.isfinite().all())
