"""Host-only checks of the operators over a paged KV cache: refusals come before any launch (no GPU), and the helpers that run on the host."""
import ctypes as C

import pytest

from paper_2504_08791_amd import _ffi
from paper_2504_08791_amd.paged import draft_tree

FAKE = 0x7f0000001000  # never dereferenced: every call below must fail validation first


def _pages(**kw):
    p = dict(k=FAKE, v=FAKE, page_stride=2 * 16 * 128, head_stride=16 * 128, row_stride=128, n_pages=10, page_rows=16, n_kv_heads=2, head_dim=128, dtype=1)
    p.update(kw)
    return _ffi.KVPages(*[p[f[0]] for f in _ffi.KVPages._fields_])


def _step(n_past=(40,), n_tok=(3,), n_seqs=None, table_stride=4, table=FAKE, tree=FAKE, positions=FAKE):
    arr = lambda v: None if v is None else (C.c_int32 * len(v))(*v)
    a, b = arr(n_past), arr(n_tok)
    s = _ffi.PagedStep(len(n_past or n_tok) if n_seqs is None else n_seqs, table_stride, a and C.cast(a, C.POINTER(C.c_int32)), b and C.cast(b, C.POINTER(C.c_int32)),
                       table, tree, positions)
    s.keep = (a, b)
    return s


def _append(pages=None, step=None, dtype=0, k=FAKE, ldk=256, v=FAKE, ldv=256, rope=FAKE, rows=100, mode=0, heads=4, q=FAKE, ldq=512, q_out=FAKE, ldqo=512):
    p, s = pages or _pages(), step or _step()
    return _ffi.lib().prima_paged_append(C.byref(p), C.byref(s), dtype, k, ldk, v, ldv, rope, rows, mode, heads, q, ldq, q_out, ldqo, None)


def _attn(pages=None, step=None, heads=4, dtype=0, q=FAKE, ldq=512, scale=0.1, o=FAKE, ldo=512, ws=FAKE, n=1 << 30):
    p, s = pages or _pages(), step or _step()
    return _ffi.lib().prima_tree_attn(C.byref(p), C.byref(s), heads, dtype, q, ldq, scale, o, ldo, ws, n, None)


@pytest.mark.parametrize("call", [_append, _attn], ids=["append", "attn"])
def test_pages_and_steps_that_are_refused(call):
    assert call(pages=_pages(k=None)) == 1 and call(pages=_pages(v=None)) == 1
    for bad in (dict(dtype=0), dict(dtype=3), dict(head_dim=96), dict(n_kv_heads=0), dict(n_pages=0), dict(page_rows=12), dict(page_rows=4), dict(page_rows=2048),
                dict(row_stride=120), dict(head_stride=0), dict(page_stride=-256), dict(row_stride=2 ** 24 + 8)):
        assert call(pages=_pages(**bad)) == 2, bad
    for bad in (dict(k=FAKE + 8), dict(v=FAKE + 2), dict(row_stride=132), dict(head_stride=2050), dict(page_stride=4100)):
        assert call(pages=_pages(**bad)) == 3, bad
    assert call(step=_step(n_past=None)) == 1 and call(step=_step(n_tok=None)) == 1 and call(step=_step(table=None)) == 1
    for bad in (dict(n_seqs=0), dict(n_past=[1] * 65, n_tok=[1] * 65), dict(n_tok=(65,)), dict(n_tok=(-1,)), dict(n_past=(-1,)), dict(n_past=(2 ** 31 - 2,)),
                dict(n_past=(62,)), dict(table_stride=2)):
        assert call(step=_step(**bad)) == 4, bad
    for bad in (dict(table=FAKE + 2), dict(tree=FAKE + 4), dict(positions=FAKE + 1)):
        assert call(step=_step(**bad)) == 3, bad
    assert call(pages=_pages(dtype=2), dtype=0) == 2 and call(pages=_pages(dtype=2), dtype=1) == 2 and call(dtype=2) == 2


def test_append_refusals():
    assert _append(k=None) == 1 and _append(v=None) == 1 and _append(q_out=None) == 1
    assert _append(mode=2) == 2 and _append(heads=0) == 2 and _append(ldk=255) == 2 and _append(ldv=128) == 2 and _append(ldq=508) == 2 and _append(ldqo=508) == 2
    assert _append(rows=0) == 4 and _append(rows=42, step=_step(positions=None)) == 4
    assert _append(k=FAKE + 4) == 3 and _append(v=FAKE + 8) == 3 and _append(q=FAKE + 4) == 3 and _append(q_out=FAKE + 4) == 3 and _append(rope=FAKE + 8) == 3
    assert _append(ldk=258) == 3 and _append(ldq=514) == 3 and _append(dtype=1, ldk=260) == 3
    assert _append(step=_step(n_tok=(0,))) == 0 and _append(step=_step(n_past=(40, 0), n_tok=(0, 0))) == 0  # nothing to do, nothing launched


def test_attention_refusals():
    assert _attn(q=None) == 1 and _attn(o=None) == 1 and _attn(ws=None) == 1
    assert _attn(heads=0) == 2 and _attn(heads=3) == 2 and _attn(ldq=508) == 2 and _attn(ldo=508) == 2
    assert _attn(q=FAKE + 4) == 3 and _attn(o=FAKE + 8) == 3 and _attn(ldq=514) == 3 and _attn(ws=FAKE + 16) == 3
    assert _attn(n=0, step=_step(n_past=(5000,), table_stride=400)) == 5
    for scale in (0.0, -1.0, float("nan"), float("inf"), 2e6):
        assert _attn(scale=scale) == 4
    assert _attn(step=_step(n_tok=(0,))) == 0
    ws = lambda p, s, h: _ffi.lib().prima_tree_attn_workspace_bytes(C.byref(p), C.byref(s), h)
    assert ws(_pages(), _step(), 4) >= 0 and ws(_pages(dtype=0), _step(), 4) == 0 and ws(_pages(), _step(n_tok=(65,)), 4) == 0 and ws(_pages(), _step(), 3) == 0


def test_attention_refuses_more_heads_than_a_group_may_have():
    one, s = _pages(n_kv_heads=1), _step()
    size = lambda heads: _ffi.lib().prima_tree_attn_workspace_bytes(C.byref(one), C.byref(s), heads)
    assert _attn(pages=one, heads=1025, ldq=1025 * 128, ldo=1025 * 128) == 2 and size(1025) == 0
    assert _attn(pages=_pages(n_kv_heads=2), heads=3) == 2 and _attn(heads=0) == 2 and _attn(heads=65538, ldq=65538 * 128, ldo=65538 * 128) == 2


def test_accept_refusals():
    f = lambda pages=None, ls=8192, L=2, step=None, path=FAKE, ld=8, n=FAKE: \
        _ffi.lib().prima_tree_accept(C.byref(pages or _pages()), ls, L, C.byref(step or _step()), path, ld, n, None)
    assert f(path=None) == 1 and f(n=None) == 1 and f(step=_step(table=None)) == 1
    assert f(L=0) == 2 and f(L=40000) == 2 and f(ls=-8) == 2 and f(ld=-1) == 2 and f(pages=_pages(head_dim=32)) == 2
    assert f(ls=4) == 3 and f(path=FAKE + 2) == 3 and f(n=FAKE + 1) == 3
    assert f(step=_step(n_tok=(0,))) == 0 and f(ld=0) == 0


def test_select_refusals():
    f = lambda dtype=0, logits=FAKE, ld=100, B=2, W=3, V=100, scores=FAKE, done=FAKE, eos=1, K=3, o=FAKE, w=FAKE, t=FAKE, ws=FAKE, n=1 << 30: \
        _ffi.lib().prima_beam_select(dtype, logits, ld, B, W, V, scores, done, eos, K, o, w, t, ws, n, None)
    for name in ("logits", "scores", "o", "w", "t", "ws"):
        assert f(**{name: None}) == 1, name
    for bad in (dict(dtype=3), dict(B=0), dict(W=0), dict(W=65), dict(V=0), dict(K=0), dict(K=65), dict(ld=99), dict(B=65535, W=2), dict(W=64, V=2 ** 25, ld=2 ** 25), dict(V=2, ld=2, K=7)):
        assert f(**bad) == 2, bad
    assert f(eos=-1) == 4 and f(eos=100) == 4
    assert f(logits=FAKE + 2) == 3 and f(dtype=1, logits=FAKE + 1) == 3 and f(scores=FAKE + 2) == 3 and f(ws=FAKE + 64) == 3
    need = _ffi.lib().prima_beam_select_workspace_bytes(2, 3, 100, 3)
    assert need > 0 and f(n=need - 1) == 5 and _ffi.lib().prima_beam_select_workspace_bytes(2, 65, 100, 3) == 0


def test_reorder_refusals():
    def f(pages=None, ls=8192, L=2, B=1, W=3, n_rows=(20,), parents=FAKE, table=FAKE, out=FAKE + (1 << 20), stride=4):
        rows = None if n_rows is None else (C.c_int32 * len(n_rows))(*n_rows)
        return _ffi.lib().prima_beam_reorder(C.byref(pages or _pages()), ls, L, B, W, rows, parents, table, out, stride, None)
    assert f(n_rows=None) == 1 and f(parents=None) == 1 and f(table=None) == 1 and f(out=None) == 1
    assert f(L=0) == 2 and f(L=20000) == 2 and f(ls=-1) == 2 and f(stride=0) == 2 and f(pages=_pages(page_rows=7)) == 2
    assert f(B=0) == 4 and f(B=65, n_rows=[1] * 65) == 4 and f(W=0) == 4 and f(W=65) == 4 and f(n_rows=(-1,)) == 4 and f(n_rows=(65,)) == 4
    assert f(out=FAKE) == 4 and f(out=FAKE + 44) == 4 and f(out=FAKE - 44) == 4
    assert f(ls=4) == 3 and f(parents=FAKE + 2) == 3 and f(table=FAKE + 1) == 3


def test_rope_table_refusals():
    f = lambda n=4, D=128, theta=1e4, tab=FAKE: _ffi.lib().prima_rope_table(n, D, theta, tab, None)
    assert f(tab=None) == 1 and f(n=-1) == 2 and f(D=96) == 2 and f(theta=0.0) == 2 and f(tab=FAKE + 4) == 3 and f(n=0) == 0


def test_draft_tree():
    bits, depth = draft_tree([-1, 0, 0, 1, -1])
    assert bits == [1, 3, 5, 11, 16] and depth == [0, 1, 1, 2, 0]
    chain, depth = draft_tree(list(range(-1, 63)))
    assert chain[-1] == -1 and chain[62] == 2 ** 63 - 1 and depth[-1] == 63   # (64 bits as a signed number)
    assert draft_tree([]) == ([], [])
    for bad in ([0], [-1, 1], [-2], [-1] * 65):
        with pytest.raises(ValueError):
            draft_tree(bad)


def _plan(pages=None, step=None, heads=4, dtype=0):
    p, s = pages or _pages(), step or _step()
    n = s.n_seqs
    few, many, ranges, rows = C.c_int32(-1), C.c_int32(-1), (C.c_int32 * max(n, 1))(), (C.c_int32 * max(n, 1))()
    code = _ffi.lib().prima_tree_attn_plan(C.byref(p), C.byref(s), heads, dtype, C.byref(few), C.byref(many), ranges, rows)
    return code, few.value, many.value, list(ranges)[:n], list(rows)[:n]


def test_attention_plans():
    """Host logic, no GPU: which kernel a step goes to, and ranges that cover every sequence's rows, each of which has some."""
    seen = set()
    for Hkv, G in ((1, 1), (2, 5), (8, 4), (8, 8), (1, 64)):
        pages = _pages(n_kv_heads=Hkv, page_rows=64, head_stride=64 * 128, page_stride=Hkv * 64 * 128)
        for dtype in (0, 1):
            for tok in (1, 3, 7, 16, 33, 63):
                for n in (1, 5, 64):
                    for past in (0, 63, 500, 7001, 50000):
                        pasts, toks = [past - past * b // (3 * n) for b in range(n)], [tok - (b % 3) * tok // 3 if b else tok for b in range(n)]
                        code, few, many, ranges, rows = _plan(pages, _step(n_past=pasts, n_tok=toks, table_stride=1000), Hkv * G, dtype)
                        assert code == 0 and (few in (1, 2) and many == 0 or few == 0 and many in ((2, 4) if dtype == 0 else (2, 4, 8)))
                        assert few or tok * G > 32
                        for p, t, k, r in zip(pasts, toks, ranges, rows):
                            assert (k == 0) if t == 0 else (1 <= k <= 256 and r % 64 == 0 and (k - 1) * r < p + t <= k * r)
                        seen.add((few, many))
    assert seen == {(1, 0), (2, 0), (0, 2), (0, 4), (0, 8)}
    assert _plan(step=_step(n_tok=(0,)))[:4] == (0, 0, 0, [0])
    assert _plan(pages=_pages(dtype=0))[0] == 2 and _plan(heads=3)[0] == 2 and _plan(dtype=2)[0] == 2 and _plan(step=_step(n_tok=(65,)))[0] == 4
    p, s, x = _pages(), _step(), C.c_int32()
    for null in range(4):
        assert _ffi.lib().prima_tree_attn_plan(C.byref(p), C.byref(s), 4, 0, *(None if i == null else C.byref(x) for i in range(4))) == 1


@pytest.mark.parametrize("Hkv,G", [(1, 1), (1, 60), (8, 8), (600, 1)])
@pytest.mark.parametrize("tok", [1, 64])
def test_attention_plans_of_the_longest_sequences(Hkv, G, tok):
    """Up to the most cached rows that a step may name, 2^31 - 1 - 1024 - 64: ranges, which end behind 32 bits, cover all rows."""
    pages = _pages(n_kv_heads=Hkv, page_rows=1024, head_stride=1024 * 128, page_stride=Hkv * 1024 * 128)
    for past in (2 ** 31 - 1089, 2 ** 31 - 2000, 2 ** 31 - 16400, 2 ** 30):
        code, few, many, ranges, rows = _plan(pages, _step(n_past=(past, 10), n_tok=(tok, 0), table_stride=2 ** 21), Hkv * G, 0)
        assert code == 0 and bool(few) != bool(many) and ranges[1] == 0
        assert 1 <= ranges[0] <= 256 and 0 < rows[0] and (ranges[0] - 1) * rows[0] < past + tok <= ranges[0] * rows[0]
        if Hkv == 1 and G == 1:
            assert ranges[0] > 128 and (past < 2 ** 31 - 2000 or ranges[0] * rows[0] >= 2 ** 31)


def test_attention_scratch_is_never_nothing_for_a_call_that_is_taken():
    """A caller that allocates what it is told has something to pass; 0 is for what is refused."""
    size = lambda pages, step, heads: _ffi.lib().prima_tree_attn_workspace_bytes(C.byref(pages), C.byref(step), heads)
    for step in (_step(), _step(n_past=(0,), n_tok=(1,)), _step(n_tok=(0,)), _step(n_past=(40, 0), n_tok=(0, 0))):
        assert size(_pages(), step, 4) == 256 and _attn(step=_step(n_tok=(0,)), n=256) == 0
    long = _step(n_past=(5000,), table_stride=400)
    need = size(_pages(), long, 4)
    ranges = _plan(step=long)[3][0]
    assert ranges > 1 and need >= 3 * 4 * ranges * (4 + 128) * 4 and need % 256 == 0
    assert _attn(step=long, n=need - 256) == 5
    for pages, step, heads in ((_pages(dtype=0), _step(), 4), (_pages(), _step(n_tok=(65,)), 4), (_pages(), _step(), 3), (_pages(), _step(n_past=None), 4), (_pages(k=None), _step(), 4)):
        assert size(pages, step, heads) == 0
