"""The operators for several sequences behind one prompt refuse bad arguments on the host, before any launch (fake device addresses are
never dereferenced), and calls without rows are no-ops."""
import ctypes as C

import pytest
import torch

from paper_2405_04304_amd import binding as B

FAKE = 0x7F0000000000
GB = 1 << 30
F32, BF16 = 0, 1


def _kv(**over):
    d = dict(dev_prefix=FAKE, dev_prefix_table=None, n_prefix_pages=8, prefix_len=100, dev_pages=FAKE + GB, dev_tables=FAKE + 2 * GB, dev_lens=FAKE + 3 * GB,
             n_pages=64, table_ld=4, n_seqs=4, page_tokens=16, n_kv_heads=2, d_head=64)
    d.update(over)
    return B.SharedKVDesc(**d)


LONG = dict(prefix_len=1000, n_prefix_pages=63)


BAD_SHAPES = [dict(d_head=96), dict(d_head=0), dict(page_tokens=6), dict(page_tokens=0), dict(n_kv_heads=0), dict(n_seqs=-1), dict(n_seqs=65536),
              dict(prefix_len=-1), dict(n_prefix_pages=-1), dict(table_ld=0), dict(n_pages=0), dict(table_ld=1 << 30)]


def _append(kv=None, **over):
    d = dict(qkv=FAKE + 4 * GB, dtype=F32, ld_qkv=8 * 64, n_rows=4, n_heads=4, seq=None, pos=None, rope=FAKE + 5 * GB, n_rope=164, q_gain=None, k_gain=None,
             eps=1e-6, q=FAKE + 6 * GB, ld_q=256)
    d.update(over)
    return B.lib().disco_append(C.byref(kv if kv is not None else _kv()), *d.values(), None)


@pytest.mark.parametrize("over", BAD_SHAPES, ids=str)
def test_bad_caches(over):
    kv = _kv(**over)
    assert _append(kv) == B.EINVAL
    assert B.lib().disco_attn_shared_bytes(C.byref(kv), 1, 4, 0) == 0
    assert _attn(kv) == B.EINVAL


def test_append_refusals():
    assert B.lib().disco_append(None, *([None, 0, 0, 1, 4] + [None] * 3 + [0, None, None, 1e-6, None, 0, None])) == B.EINVAL
    for over in (dict(n_rows=-1), dict(n_rows=(1 << 24) + 4), dict(n_heads=0), dict(n_heads=3), dict(n_heads=2048), dict(dtype=2), dict(qkv=None), dict(q=None),
                 dict(qkv=FAKE + 4 * GB + 8), dict(q=FAKE + 8), dict(ld_qkv=508), dict(ld_qkv=514), dict(ld_q=255), dict(ld_q=252), dict(ld_q=258),
                 dict(seq=FAKE + 7 * GB), dict(pos=FAKE + 7 * GB), dict(n_rows=6), dict(seq=FAKE + 1, pos=FAKE), dict(rope=FAKE + 8),
                 dict(q_gain=FAKE, eps=0.0), dict(k_gain=FAKE, eps=float("nan")), dict(q_gain=FAKE + 4), dict(q=FAKE + 4 * GB), dict(q=FAKE + 4 * GB + 2048),
                 dict(dtype=BF16, ld_qkv=516), dict(dtype=BF16, ld_q=260)):
        assert _append(**over) == B.EINVAL, over
    assert _append(n_rope=163) == B.ECAP
    assert "rotary" in B.last_error()
    assert _append(_kv(dev_lens=None)) == B.EINVAL
    for over in (dict(dev_pages=None), dict(dev_tables=None), dict(dev_pages=FAKE + 8), dict(dev_tables=FAKE + 2), dict(dev_lens=FAKE + 1), dict(n_seqs=0)):
        assert _append(_kv(**over)) == B.EINVAL, over


def _attn(kv=None, **over):
    d = dict(q=FAKE + 4 * GB, dtype=F32, ld_q=256, n_tok=1, n_heads=4, scale=0.125, out=FAKE + 5 * GB, ld_out=256, lse=None, max_len=0, ws=FAKE + 6 * GB, ws_bytes=GB)
    d.update(over)
    return B.lib().disco_attn_shared(C.byref(kv if kv is not None else _kv()), *d.values(), None)


def test_attention_refusals():
    assert B.lib().disco_attn_shared_bytes(C.byref(_kv()), 1, 4, 0) == 256            # one launch, no parts
    need = B.lib().disco_attn_shared_bytes(C.byref(_kv(**LONG)), 1, 4, 0)
    assert need > 256
    assert _attn(_kv(**LONG), ws_bytes=need - 1024) == B.EINVAL and "workspace" in B.last_error()
    assert _attn(_kv(**LONG), ws=None) == B.EINVAL and _attn(_kv(**LONG), ws=FAKE + 6 * GB + 128) == B.EINVAL
    for over in (dict(n_tok=0), dict(n_tok=17), dict(n_heads=3), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
                 dict(max_len=-1), dict(q=None), dict(out=None), dict(q=FAKE + 4), dict(out=FAKE + 4), dict(ld_q=252), dict(ld_out=258), dict(dtype=7),
                 dict(out=FAKE + 4 * GB), dict(lse=FAKE + 2)):
        assert _attn(**over) == B.EINVAL, over
    for over in (dict(dev_prefix=None), dict(dev_prefix=FAKE + 8), dict(dev_prefix_table=FAKE + 2), dict(dev_lens=None), dict(dev_pages=None), dict(dev_tables=None)):
        assert _attn(_kv(**over)) == B.EINVAL, over
    assert _attn(_kv(n_prefix_pages=6)) == B.ECAP


def test_attention_workspace_follows_the_plan():
    size = lambda n_tok=1, heads=4, max_len=0, **over: B.lib().disco_attn_shared_bytes(C.byref(_kv(**{**LONG, **over})), n_tok, heads, max_len)  # noqa: E731
    assert size(prefix_len=0, table_ld=1) == 256                     # one range: nothing to put together
    assert size(n_tok=2) > size() and size(heads=8) > size()
    assert size(n_seqs=0) == 256
    assert size(max_len=1 << 29) == size()                           # a table holds 64 positions


def test_no_rows_is_no_work():
    empty = _kv(n_seqs=0, dev_tables=None, dev_lens=None)
    assert _append(n_rows=0, qkv=None, q=None) == 0
    assert _attn(empty, q=None, out=None, ws=None, ws_bytes=0) == 0
    assert _select(n_groups=0, logits=None, tokens=None) == 0
    assert _reorder(n_groups=0, pages=None, tables=None) == 0


def _select(**over):
    d = dict(logits=FAKE, dtype=F32, ld=1000, n_groups=2, n_beams=4, vocab=1000, k=8, scores=FAKE + GB, done=None, end=-1, tokens=FAKE + 2 * GB, parents=FAKE + 3 * GB,
             scores_out=FAKE + 4 * GB, done_out=None, ws=FAKE + 5 * GB, ws_bytes=GB)
    d.update(over)
    return B.lib().disco_beam_select(*d.values(), None)


def test_select_refusals():
    for over in (dict(n_groups=-1), dict(n_beams=0), dict(n_beams=65), dict(n_groups=65535), dict(vocab=0), dict(vocab=(1 << 20) + 1), dict(k=0), dict(k=129), dict(dtype=2),
                 dict(ld=999), dict(end=1000), dict(end=-2), dict(done=FAKE, end=-1), dict(logits=None), dict(scores=None), dict(tokens=None), dict(parents=None),
                 dict(scores_out=None), dict(ws=None), dict(ws=FAKE + 128), dict(ws_bytes=256), dict(logits=FAKE + 2), dict(tokens=FAKE + 2), dict(done=FAKE + 2, end=1)):
        assert _select(**over) == B.EINVAL, over
    assert B.lib().disco_beam_select_bytes(1, 65, 10, 1) == 0 and B.lib().disco_beam_select_bytes(2, 4, 1000, 8) > 256


def _reorder(**over):
    d = dict(pages=FAKE, n_layers=2, layer_stride=64 * 4096, n_pages=64, page_elems=4096, tables=FAKE + GB, tables_out=FAKE + 2 * GB, table_ld=4, parents=FAKE + 3 * GB,
             n_groups=2, n_beams=4, len=20, page_tokens=16)
    d.update(over)
    return B.lib().disco_beam_reorder(*d.values(), None)


def test_reorder_refusals():
    for over in (dict(n_groups=-1), dict(n_beams=0), dict(n_beams=65), dict(table_ld=0), dict(page_tokens=6), dict(n_layers=0), dict(n_layers=65536), dict(n_pages=0),
                 dict(page_elems=4), dict(page_elems=4100), dict(layer_stride=63 * 4096), dict(layer_stride=64 * 4096 + 4), dict(layer_stride=-8), dict(pages=None),
                 dict(tables=None), dict(tables_out=None), dict(parents=None), dict(pages=FAKE + 8), dict(tables=FAKE + 2), dict(tables_out=FAKE + GB + 64)):
        assert _reorder(**over) == B.EINVAL, over
    assert _reorder(len=65) == B.ECAP and _reorder(len=-1) == B.ECAP


def test_rope_table_refusals():
    f = B.lib().disco_rope_table
    assert f(FAKE, 0, 64, 10000.0, None) == 0
    for args in ((FAKE, -1, 64, 1e4), (FAKE, 10, 63, 1e4), (FAKE, 10, 0, 1e4), (FAKE, 10, 64, 0.0), (FAKE, 10, 64, float("inf")), (FAKE, 10, 64, float("nan")),
                 (None, 10, 64, 1e4), (FAKE + 8, 10, 64, 1e4)):
        assert f(*args, None) == B.EINVAL, args


def test_binding_refuses_tensors_it_cannot_hand_over():
    """Host tensors (no device here), whatever else they are."""
    pages, tables = torch.zeros(4, 2, 2, 16 * 64, dtype=torch.bfloat16), torch.zeros(2, 2, dtype=torch.int32)
    with pytest.raises(B.DiscoError, match="device"):
        B.SharedKV(pages, tables, None, 16, 2, 64)
    with pytest.raises(B.DiscoError, match="device"):
        B.disco_beam_select(torch.zeros(4, 10), torch.zeros(4), 1, 4, 4, tables, tables, torch.zeros(4), torch.zeros(256, dtype=torch.uint8))
    with pytest.raises(B.DiscoError, match="device"):
        B.disco_beam_reorder(pages[None], tables, tables, tables, 1, 2, 3, 16)


def test_select_refuses_results_that_overlap():
    """A group's results are written while another group's scores are read (and its own flags, by other lanes)."""
    base = dict(n_groups=2, n_beams=4, k=8, end=1, scores=FAKE + 8 * GB, done=FAKE + 9 * GB, tokens=FAKE + 10 * GB, parents=FAKE + 11 * GB, scores_out=FAKE + 12 * GB,
                done_out=FAKE + 13 * GB)
    for over in (dict(scores_out=base["scores"]), dict(scores_out=base["scores"] + 28), dict(scores_out=base["scores"] - 60), dict(done_out=base["done"]),
                 dict(tokens=base["done"] + 4), dict(tokens=base["parents"]), dict(parents=base["scores_out"] + 60), dict(done_out=base["tokens"] - 4)):
        assert _select(**{**base, **over}) == B.EINVAL and "overlap" in B.last_error(), over


def test_calls_larger_than_a_launch():
    """More threads than 2^32 are refused, not cut off."""
    for heads, d in ((512, 128), (1024, 64)):           # 2^24 rows of 2^16 and more elements
        kv = _kv(d_head=d, n_kv_heads=heads, n_seqs=1, dev_prefix=None, prefix_len=0)
        assert _append(kv, n_heads=heads, n_rows=1 << 24, ld_qkv=3 * heads * d, ld_q=heads * d, qkv=FAKE, q=FAKE + (1 << 46), n_rope=1 << 20) == B.EINVAL
        assert "2^33" in B.last_error()
    wide = _kv(d_head=128, n_kv_heads=1024, n_seqs=65535, dev_prefix=None, prefix_len=0)
    assert _attn(wide, n_heads=1024, ld_q=1 << 17, ld_out=1 << 17, out=FAKE + (1 << 46), ws_bytes=1 << 60) == B.EINVAL and "launch" in B.last_error()
    assert _reorder(page_elems=1 << 40, layer_stride=1 << 46) == B.EINVAL
    assert _reorder(n_layers=65535, n_beams=64, page_elems=1 << 20, layer_stride=1 << 26) == B.EINVAL and "launch" in B.last_error()


def test_attention_plan_holds_over_its_arguments():
    """Workspaces of calls from one token of one sequence to many: never none, whole multiples of 256 bytes."""
    for seqs in (1, 3, 40, 900):
        for prefix in (0, 1, 129, 4097, 70000):
            for tok in (1, 7, 16):
                got = [B.lib().disco_attn_shared_bytes(C.byref(_kv(n_seqs=seqs, prefix_len=prefix, n_prefix_pages=5000, n_kv_heads=kvh, table_ld=300)), tok, 4 * kvh, n)
                       for kvh in (1, 8) for n in (0, 1, 300)]
                assert all(x >= 256 and x % 256 == 0 for x in got)
