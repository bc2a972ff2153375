"""Refusals of the calls around the pass - sampled acceptance, probabilities, paged cache - and the sizes of their
scratch.  Nothing here reaches a GPU: arguments are checked before anything would be launched."""
import ctypes as C

import pytest
import torch

from paper_2507_22424_amd import binding as sv

ONE = C.c_void_p(4096)          # a non-null, aligned pointer that the host never follows
NAN, INF = float("nan"), float("inf")


def test_token_probs_refusals():
    f = sv.lib().sv_token_probs
    assert f(None, 1, 5, 1.0, ONE, None) == -1 and f(ONE, 1, 5, 1.0, None, None) == -1
    for rows, n in ((0, 5), (-1, 5), (1 << 21, 5), (1, 0), (1, sv.SV_MAX_SAMPLED_VOCAB + 1)):
        assert f(ONE, rows, n, 1.0, ONE, None) == -2, (rows, n)
    for t in (0.0, -1.0, NAN, INF, 1e-39):
        assert f(ONE, 1, 5, t, ONE, None) == -4, t


def _accept(tree=None, n_vocab=100, lo=0, B=1, d_cap=7, null=None, draft=ONE):
    p = [ONE] * 11
    if null is not None:
        p[null] = None
    tree = sv.Tree(4096, None, None, 15, 0) if tree is None else tree
    return sv.lib().sv_sampled_accept(C.byref(tree), p[0], p[1], draft, n_vocab, lo, p[2], p[3], B, d_cap, p[4], p[5], p[6],
                                      p[7], p[8], p[9], None)


def test_sampled_accept_refusals():
    for i in range(10):
        assert _accept(null=i) == -1, i
    assert _accept(tree=sv.Tree(None, 4096, 4096, 15, 1)) == -1
    assert sv.lib().sv_sampled_accept(None, *[ONE] * 3, 5, 0, ONE, ONE, 1, 7, *[ONE] * 6, None) == -1
    for T in (0, 129):
        assert _accept(tree=sv.Tree(4096, 4096, 4096, T, 1)) == -2
    for kw in (dict(B=0), dict(B=(1 << 15) + 1), dict(d_cap=-1), dict(d_cap=32), dict(n_vocab=0),
               dict(n_vocab=sv.SV_MAX_SAMPLED_VOCAB + 1)):
        assert _accept(**kw) == -2, kw
    for lo in (-1, 2 ** 31 - 100):
        assert _accept(lo=lo) == -4


def _view(**kw):
    f = dict(k=4096, v=4096, block_table=4096, dtype=sv.SV_BF16, n_seqs=4, max_pages=8, n_pages=20, page_size=16, n_kv_heads=2,
             head_dim=64)
    f.update(kw)
    return sv.PagedView(*[f[n] for n, _ in sv.PagedView._fields_])


BAD_VIEWS = [(dict(k=None), -1), (dict(v=None), -1), (dict(block_table=None), -1), (dict(dtype=sv.SV_BF16_W8), -6),
             (dict(dtype=7), -6), (dict(n_seqs=0), -2), (dict(n_seqs=(1 << 15) + 1), -2), (dict(max_pages=0), -2), (dict(n_pages=0), -2),
             (dict(page_size=0), -2), (dict(page_size=8), -2), (dict(page_size=24), -2), (dict(max_pages=1 << 27), -2),
             (dict(n_kv_heads=0), -2), (dict(head_dim=4), -2), (dict(head_dim=100), -2), (dict(head_dim=264), -2),
             (dict(k=4104), -2), (dict(v=4098), -2)]


def _append(view=None, n=3, seq=ONE, pos=ONE, q=ONE, n_q=4, qs=256, k=ONE, ks=128, v=ONE, vs=128, theta=1e4, q_out=ONE, status=None):
    view = _view() if view is None else view
    return sv.lib().sv_paged_append(C.byref(view), n, seq, pos, q, n_q, qs, k, ks, v, vs, theta, q_out, status, None)


def _attend(view=None, lens=ONE, max_len=100, q=ONE, n_q=4, scale=0.125, window=0, sink=0, out=ONE, ws=ONE, ws_bytes=1 << 40):
    view = _view() if view is None else view
    return sv.lib().sv_paged_attention(C.byref(view), lens, max_len, q, n_q, scale, window, sink, out, None, None, ws, ws_bytes, None)


@pytest.mark.parametrize("change,status", BAD_VIEWS)
def test_paged_caches_that_are_refused(change, status):
    view, n = _view(**change), C.c_size_t(0)
    assert _append(view) == status and _attend(view) == status
    assert sv.lib().sv_paged_workspace_bytes(C.byref(view), 4, 100, C.byref(n)) == status


def test_paged_append_refusals():
    for kw in (dict(seq=None), dict(pos=None), dict(k=None), dict(v=None), dict(q=None), dict(q_out=None)):
        assert _append(**kw) == -1, kw
    other = C.c_void_p(4096 + 4)
    for kw in (dict(n=0), dict(n=(1 << 22) + 1), dict(n_q=0), dict(n_q=-1), dict(n_q=(1 << 15) + 1), dict(qs=252), dict(qs=258),
               dict(ks=124), dict(ks=130), dict(vs=0), dict(vs=-128), dict(q=other), dict(k=other), dict(v=other),
               dict(q_out=other), dict(q=ONE, q_out=ONE, qs=512), dict(theta=0.0), dict(theta=-1.0), dict(theta=NAN), dict(theta=INF),
               dict(q=None, q_out=None, n_q=4)):
        assert _append(**kw) == -2, kw


def test_paged_attention_refusals():
    for kw in (dict(lens=None), dict(q=None), dict(out=None), dict(ws=None)):
        assert _attend(**kw) == -1, kw
    other = C.c_void_p(4096 + 8)
    for kw in (dict(max_len=-1), dict(max_len=129), dict(n_q=0), dict(n_q=3), dict(n_q=(1 << 15) + 2), dict(scale=NAN), dict(scale=INF),
               dict(window=-1), dict(sink=-1), dict(q=other), dict(out=other)):
        assert _attend(**kw) == -2, kw
    view = _view(max_pages=4096, n_seqs=1)
    n = C.c_size_t(0)
    assert sv.lib().sv_paged_workspace_bytes(C.byref(view), 4, 65536, C.byref(n)) == 0 and n.value > 256
    assert _attend(view, max_len=65536, ws_bytes=n.value - 1) == -5 and _attend(view, max_len=65536, ws=C.c_void_p(4096 + 128)) == -5
    assert sv.lib().sv_paged_workspace_bytes(C.byref(view), 4, 65536, None) == -1
    # more threads than a launch can have: n_seqs * n_q_heads * ceil(max_len / 4096) above 2^23
    for seqs, n_q, length, ok in ((1 << 15, 256, 4096, True), (1 << 15, 258, 4096, False), (1 << 15, 256, 4097, False), (1 << 15, 256, 0, True),
                                  (1 << 10, 32, 1 << 20, True), (1 << 10, 34, 1 << 20, False)):
        view = _view(max_pages=1 << 16, n_seqs=seqs)
        assert sv.lib().sv_paged_workspace_bytes(C.byref(view), n_q, length, C.byref(n)) == (0 if ok else -2), (seqs, n_q, length)
        if not ok:
            assert _attend(view, n_q=n_q, max_len=length) == -2


@pytest.mark.parametrize("n_seqs,n_kv,n_q,d", [(1, 1, 1, 64), (1, 8, 32, 128), (3, 2, 80, 256), (64, 8, 32, 128), (700, 5, 35, 96)])
def test_scratch_never_falls_as_sequences_grow(n_seqs, n_kv, n_q, d):
    view, n, last = _view(n_seqs=n_seqs, n_kv_heads=n_kv, head_dim=d, max_pages=1 << 14), C.c_size_t(0), 0
    for length in sorted({0, 1, 15, 16, 17, 255, 256, 257, 1000, 4095, 4096, 5000, 30000, 30001, 131072, 262144} | set(range(200, 2000, 97))):
        assert sv.lib().sv_paged_workspace_bytes(C.byref(view), n_q, length, C.byref(n)) == 0
        assert n.value >= last
        last = n.value


def test_the_holder_refuses_tensors_that_are_no_cache():
    k = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16)
    table = torch.zeros(1, 2, dtype=torch.int32)
    for a in ((k, k[:2], table), (k[0], k[0], table), (k, k.float(), table), (k.half(), k.half(), table), (k, k, table[0]),
              (k, k, table)):                       # the last: on the host
        with pytest.raises(ValueError):
            sv.PagedCache(*a)


def test_numbers_past_32_bits_are_refused():
    """Not taken modulo 2^32, as an int argument of the C call would be."""
    cache = type("Cache", (), {"struct": _view(n_seqs=1, n_kv_heads=2, head_dim=64, max_pages=4)})()
    q, ws, one = torch.zeros(1, 2, 64), torch.zeros(256, dtype=torch.uint8), torch.zeros(1, dtype=torch.int32)
    big = 1 << 32
    for max_len, window, n_sink in ((big + 5, 0, 0), (5, big, 0), (5, big + 4, 0), (5, 3, big + 1), (-big + 5, 0, 0), (5, -big, 0)):
        with pytest.raises(ValueError, match="32-bit"):
            sv.sv_paged_attention(cache, one, max_len, q, 0.1, window, n_sink, q, None, None, ws)
    for n_q, max_len in ((big + 2, 5), (2, big + 5)):
        with pytest.raises(ValueError, match="32-bit"):
            sv.sv_paged_workspace_bytes(cache, n_q, max_len)
    wide = torch.zeros(1, 1).expand(big + 1, 1)
    with pytest.raises(ValueError, match="rows, vocabulary"):
        sv.sv_token_probs(wide, 1.0, wide)
    tree, nodes, out = sv.Tree(4096, 4096, 4096, 2, 1), torch.zeros(2), torch.zeros(8, dtype=torch.int32)
    for p, lo in ((torch.zeros(1, 1).expand(2, big + 1), 0), (torch.zeros(2, 5), big), (torch.zeros(2, 5), -big)):
        with pytest.raises(ValueError, match="sizes"):
            sv.sv_sampled_accept(tree, nodes.int(), p, None, lo, nodes, nodes[:1], 1, 7, nodes.byte(), out[:1], out[:1], out, out, out[:1])


def test_sizes_past_32_bits_are_refused():
    """Sizes of tensors too: a page of 2^32 + 16 rows is none of 16."""
    big = 1 << 32
    page, table = torch.zeros(1, 1, 16, 8), torch.zeros(1, 1, dtype=torch.int32)
    for k, t in ((page.expand(big + 1, 1, 16, 8), table), (page.expand(1, big + 1, 16, 8), table),
                 (page[:, :, :1].expand(1, 1, big + 16, 8), table), (page[..., :1].expand(1, 1, 16, big + 8), table),
                 (page, table.expand(big + 1, 1)), (page, table.expand(1, big + 1))):
        with pytest.raises(ValueError, match="32-bit"):
            sv.PagedCache(k, k, t)
    cache = type("Cache", (), {"struct": _view(n_seqs=1, n_kv_heads=1, head_dim=8, max_pages=4)})()
    ids, x, ws = torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1, 8), torch.zeros(256, dtype=torch.uint8)
    many, heads = x.expand(big + 1, 1, 8), x.expand(1, big + 1, 8)
    with pytest.raises(ValueError, match="32-bit"):
        sv.sv_paged_append(cache, ids.expand(big + 1), ids.expand(big + 1), None, many, many, None, 1e4)
    with pytest.raises(ValueError, match="32-bit"):
        sv.sv_paged_append(cache, ids, ids, heads, x, x, heads, 1e4)
    with pytest.raises(ValueError, match="32-bit"):
        sv.sv_paged_attention(cache, ids, 5, heads, 0.1, 0, 0, heads, None, None, ws)
    tree, f, i, m = sv.Tree(4096, 4096, 4096, 1, 1), torch.zeros(1).expand(big + 1), ids.expand(big + 1), ws[:1].expand(big + 1)
    with pytest.raises(ValueError, match="sizes"):
        sv.sv_sampled_accept(tree, i, f[:, None], None, 0, f, f, big + 1, 0, m, i, i, i, i, i)


def test_scales_that_float32_does_not_hold_in_base_two_are_refused():
    """3e38 log2(e) is infinite: queries of zeros would become NaN."""
    for scale in (3e38, -3e38, 2.4e38):
        assert _attend(scale=scale) == -2
    for scale in (2.3e38, -2.3e38):
        assert _attend(scale=scale, ws_bytes=0) == -5        # past the check of the scale
