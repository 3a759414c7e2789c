"""The beam search's choice and the pages' bookkeeping: argument checks without a GPU, documented codes before any device work."""
import ctypes as C

import pytest

from paper_2504_10724_amd import capi as ee

DUMMY = C.c_void_p(4096)
BAD, SHAPE, CAPACITY = ee.EE_ERR_INVALID_ARG, ee.EE_ERR_SHAPE, ee.EE_ERR_CAPACITY


def _beams(**kw):
    c = dict(n_groups=2, beams=4, keep=4, vocab=1000, dtype=ee.EE_F32, end_token=-1)
    c.update(kw)
    return ee.ee_beam_config(**c)


@pytest.mark.parametrize("kw,code", [
    (dict(n_groups=-1), BAD), (dict(beams=0), SHAPE), (dict(beams=65), SHAPE), (dict(keep=0), SHAPE), (dict(keep=129), SHAPE),
    (dict(vocab=0), SHAPE), (dict(vocab=2 ** 30 + 1), SHAPE), (dict(dtype=2), ee.EE_ERR_DTYPE), (dict(end_token=-2), BAD),
    (dict(end_token=1000), BAD), (dict(n_groups=2 ** 31 - 1), SHAPE), (dict(n_groups=2 ** 20, vocab=2 ** 30), SHAPE)])
def test_searches_of_no_such_kind(kw, code):
    lib, c, out = ee.load(), _beams(**kw), ee.ee_beam_choice(4096, 4096, 4096, None)
    assert lib.ee_beam_workspace(C.byref(c)) == 0
    assert lib.ee_beam_select(C.byref(c), DUMMY, 1000, DUMMY, None, C.byref(out), DUMMY, 1 << 60, None) == code
    assert lib.ee_last_error()


def test_choices():
    lib, c = ee.load(), _beams(end_token=3)
    need = lib.ee_beam_workspace(C.byref(c))
    assert need > 0 and lib.ee_beam_workspace(None) == 0
    args = lambda **kw: ee.ee_beam_choice(*[kw.get(k, 8192) for k in ("score", "parent", "token", "done")])      # noqa: E731

    def call(c=c, logits=DUMMY, score=C.c_void_p(4096), done=None, out=args(), ws=DUMMY, n=need):
        return lib.ee_beam_select(None if c is None else C.byref(c), logits, 1000, score, done, None if out is None else C.byref(out), ws, n, None)
    assert call(c=None) == BAD and call(out=None) == BAD and call(logits=None) == BAD and call(score=None) == BAD
    for k in ("score", "parent", "token"):
        assert call(out=args(**{k: None})) == BAD
    assert call(n=need - 1) == CAPACITY and call(ws=None) == BAD and call(ws=C.c_void_p(4097)) == BAD
    assert call(logits=C.c_void_p(4098)) == BAD
    assert call(c=_beams(), done=DUMMY) == BAD                                     # ended beams without a token to go on with
    wide = _beams(keep=8, end_token=3)
    n = lib.ee_beam_workspace(C.byref(wide))
    assert call(c=wide, n=n, out=args(score=4096)) == BAD                          # in place of fewer
    assert call(c=wide, n=n, done=C.c_void_p(12288), out=args(done=12288)) == BAD
    assert call(c=_beams(n_groups=0), logits=None, score=None, out=args(score=None), ws=None, n=0) == ee.EE_OK


def _cache(lib, **kw):
    c = dict(n_layers=2, n_pages=100, n_kv_heads=2, head_dim=128, page_size=64, dtype=ee.EE_BF16)
    c.update(kw)
    cfg, p = ee.ee_paged_config(**c), C.c_void_p()
    assert lib.ee_paged_bind(C.byref(cfg), DUMMY, 1 << 60, C.byref(p)) == ee.EE_OK
    return p


def test_bookkeeping_handles():
    lib, h = ee.load(), C.c_void_p()
    p = _cache(lib)
    need = lib.ee_pages_state_bytes(p, 8)
    assert need >= 4 * 100 and lib.ee_pages_state_bytes(None, 8) == 0
    for n in (0, -1, 4097):
        assert lib.ee_pages_state_bytes(p, n) == 0 and lib.ee_pages_bind(p, n, DUMMY, 1 << 60, C.byref(h)) == SHAPE
    assert lib.ee_pages_bind(None, 8, DUMMY, need, C.byref(h)) == BAD and lib.ee_pages_bind(p, 8, None, need, C.byref(h)) == BAD
    assert lib.ee_pages_bind(p, 8, DUMMY, need - 1, C.byref(h)) == CAPACITY and lib.ee_pages_bind(p, 8, C.c_void_p(4097), need, C.byref(h)) == BAD
    many = _cache(lib, n_layers=1, n_pages=2 ** 21 + 1, n_kv_heads=1, head_dim=64, page_size=32)
    assert lib.ee_pages_state_bytes(many, 8) == 0 and lib.ee_pages_bind(many, 8, DUMMY, 1 << 60, C.byref(h)) == SHAPE
    lib.ee_paged_destroy(many)
    assert not h.value and lib.ee_pages_reset(None, None) == BAD
    assert lib.ee_pages_destroy(None) == ee.EE_OK
    lib.ee_paged_destroy(p)


def _table(**kw):
    c = dict(n_seqs=4, pages_per_seq=3, dev_pages=4096, dev_kv_len=8192)
    c.update(kw)
    return ee.ee_page_table(**c)


@pytest.mark.parametrize("kw,code", [
    (dict(n_seqs=-1), BAD), (dict(pages_per_seq=-1), BAD), (dict(pages_per_seq=2 ** 25), CAPACITY), (dict(dev_pages=None), BAD),
    (dict(dev_kv_len=None), BAD)])
def test_tables_of_no_such_kind(kw, code):
    lib, g = ee.load(), C.c_void_p()
    p = _cache(lib)
    assert lib.ee_pages_bind(p, 8, DUMMY, 1 << 40, C.byref(g)) == ee.EE_OK
    t = _table(**kw)
    assert lib.ee_pages_grow(g, C.byref(t), None, None, None) == code
    assert lib.ee_pages_fork(g, C.byref(t), None, DUMMY, None, 0, None, 0, None, None) == code
    assert lib.ee_pages_compact(g, C.byref(t), 1, None) == code
    lib.ee_pages_destroy(g)
    lib.ee_paged_destroy(p)


def test_bookkeeping_calls():
    lib, g = ee.load(), C.c_void_p()
    p = _cache(lib)
    assert lib.ee_pages_bind(p, 8, DUMMY, 1 << 40, C.byref(g)) == ee.EE_OK
    t, none, wide = _table(), _table(n_seqs=0), _table(n_seqs=9)
    T = C.byref
    assert lib.ee_pages_grow(None, T(t), None, None, None) == BAD and lib.ee_pages_grow(g, None, None, None, None) == BAD
    assert lib.ee_pages_grow(g, T(wide), None, None, None) == CAPACITY and lib.ee_pages_grow(g, T(none), None, None, None) == ee.EE_OK

    def fork(to=t, source=None, parent=C.c_void_p(32768), keep=None, group=0, states=(), n=None):
        a = (ee.ee_rows * 9)(*states)
        return lib.ee_pages_fork(g, T(to), None if source is None else T(source), parent, keep, group, a if states else None,
                                 len(states) if n is None else n, None, None)
    other = dict(dev_pages=16384, dev_kv_len=20480)
    assert lib.ee_pages_fork(None, T(t), None, DUMMY, None, 0, None, 0, None, None) == BAD
    assert fork(parent=None) == BAD and fork(group=-1) == BAD and fork(n=-1) == BAD and fork(n=2) == BAD
    assert fork(to=none, parent=None) == ee.EE_OK
    assert fork(group=3) == SHAPE                                                  # 4 rows in groups of 3
    assert fork(source=_table(n_seqs=8, **other), group=4) == SHAPE                # groups of unlike tables
    assert fork(source=_table(pages_per_seq=4, **other)) == SHAPE                  # rows that do not fit
    assert fork(source=_table(dev_pages=16384)) == BAD and fork(source=_table(dev_kv_len=16384)) == BAD and fork(source=_table(n_seqs=3)) == BAD
    assert fork(to=_table(n_seqs=4097)) == SHAPE and fork(to=_table(n_seqs=8194), group=4097) == SHAPE
    rows = ee.ee_rows(65536, 64, 64)
    assert fork(states=[rows] * 9) == SHAPE and fork(source=_table(**other), states=[rows]) == BAD
    assert fork(states=[ee.ee_rows(65536, 63, 64)]) == BAD and fork(states=[ee.ee_rows(65536, 64, -1)]) == BAD
    assert fork(states=[ee.ee_rows(None, 64, 64)]) == BAD and fork(states=[rows, rows]) == BAD
    own = [C.c_void_p(t.dev_pages), C.c_void_p(t.dev_kv_len)]
    assert all(fork(parent=a) == BAD and fork(parent=C.c_void_p(24576), keep=a) == BAD for a in own)            # of the table that is written
    for a in (t.dev_pages, t.dev_kv_len, 24576, 28672):
        assert fork(parent=C.c_void_p(24576), keep=C.c_void_p(28672), states=[ee.ee_rows(a, 4, 4)]) == BAD
    assert lib.ee_pages_compact(None, T(t), 1, None) == BAD and lib.ee_pages_compact(g, None, 1, None) == BAD
    assert lib.ee_pages_compact(g, T(t), -1, None) == BAD and lib.ee_pages_compact(g, T(t), 9, None) == SHAPE
    assert lib.ee_pages_compact(g, (ee.ee_page_table * 2)(t, t), 2, None) == BAD
    for kw, code in ((dict(head_dim=64), SHAPE), (dict(page_size=32), SHAPE), (dict(n_layers=1), SHAPE), (dict(n_kv_heads=1), SHAPE),
                     (dict(dtype=ee.EE_F32), ee.EE_ERR_DTYPE)):
        q = _cache(lib, **kw)
        assert lib.ee_pages_copy(p, q, DUMMY, DUMMY, 1, None, None) == code
        lib.ee_paged_destroy(q)
    assert lib.ee_pages_copy(None, p, DUMMY, DUMMY, 1, None, None) == BAD and lib.ee_pages_copy(p, p, DUMMY, DUMMY, -1, None, None) == BAD
    assert lib.ee_pages_copy(p, p, None, DUMMY, 1, None, None) == BAD and lib.ee_pages_copy(p, p, None, None, 0, None, None) == ee.EE_OK
    lib.ee_pages_destroy(g)
    lib.ee_paged_destroy(p)


def test_default_streams_are_those_of_the_current_device(monkeypatch):
    """their handle is 0 on every device; a stream that was made knows its device"""
    from paper_2504_10724_amd import beams, paged
    handles = {0: 0, 1: 0, 2: 0x5000}
    monkeypatch.setattr(paged, "_stream_of", handles.__getitem__)
    monkeypatch.setattr(paged, "_current_device", lambda: 0)
    assert beams._stream is paged._stream
    assert paged._stream(0) == 0 and paged._stream(2) == 0x5000
    with pytest.raises(ee.EEError, match="device 0 is current"):
        paged._stream(1)


@pytest.mark.parametrize("dtype", [ee.EE_F32, ee.EE_BF16])
@pytest.mark.parametrize("kw", [dict(n_groups=2 ** 22, beams=4, keep=4, vocab=8), dict(n_groups=2 ** 24, beams=1, keep=1, vocab=1),
                                dict(n_groups=2 ** 11, beams=2 ** 5, keep=1, vocab=2 ** 20), dict(n_groups=2 ** 11, beams=2 ** 5, keep=1, vocab=2 ** 20 - 4095)])
def test_choices_of_more_slices_than_a_launch_holds(kw, dtype):
    """2^24 workgroups of 256 threads are 2^32 threads, which no grid has; a request less is fine"""
    lib, c, out = ee.load(), _beams(dtype=dtype, **kw), ee.ee_beam_choice(4096, 4096, 4096, None)
    assert lib.ee_beam_workspace(C.byref(c)) == 0
    assert lib.ee_beam_select(C.byref(c), DUMMY, c.vocab, DUMMY, None, C.byref(out), DUMMY, 1 << 60, None) == SHAPE
    c.n_groups -= 1
    assert lib.ee_beam_workspace(C.byref(c)) > 0


def test_forks_of_more_workgroups_than_a_launch_holds():
    """rows that are groups of one: a workgroup for each one's lengths and one for its column"""
    lib, g = ee.load(), C.c_void_p()
    p = _cache(lib)
    assert lib.ee_pages_bind(p, 8, DUMMY, 1 << 40, C.byref(g)) == ee.EE_OK
    far = [C.c_void_p(k << 32) for k in (1, 2, 3, 4)]
    t = ee.ee_page_table(2 ** 23, 1, far[0], far[1])
    assert lib.ee_pages_fork(g, C.byref(t), None, far[2], None, 1, None, 0, None, None) == SHAPE
    t = ee.ee_page_table(2 ** 22, 2, far[0], far[1])
    states = (ee.ee_rows * 1)(ee.ee_rows(far[3], 8192, 8192))
    assert lib.ee_pages_fork(g, C.byref(t), None, far[2], None, 1, states, 1, None, None) == SHAPE
    lib.ee_pages_destroy(g)
    lib.ee_paged_destroy(p)


def test_choices_whose_arrays_overlap():
    """a request's workgroup writes its results while others still read: results lie apart from each other and from what is read, but for the
    scores and the ended beams themselves in place"""
    lib, c = ee.load(), _beams(end_token=3)                                        # 2 requests of 4 beams, 4 kept: arrays of 32 and of 8 bytes
    need = lib.ee_beam_workspace(C.byref(c))
    base = dict(score=1 << 20, parent=2 << 20, token=3 << 20, done=4 << 20, in_score=5 << 20, in_done=6 << 20, ws=1 << 30)

    def call(**kw):
        a = dict(base, **kw)
        out = ee.ee_beam_choice(a["score"], a["parent"], a["token"], a["done"])
        return lib.ee_beam_select(C.byref(c), DUMMY, 1000, C.c_void_p(a["in_score"]), C.c_void_p(a["in_done"]), C.byref(out), C.c_void_p(a["ws"]), need, None)
    sizes = dict(score=32, parent=32, token=32, done=8, in_score=32, in_done=8)
    assert need % 256 == 0
    for one, n in sizes.items():
        for other, m in sizes.items():
            if one == other or {one, other} == {"in_score", "in_done"}:            # both only read
                continue
            for by in (4 - n, 4, m - 4, *(() if {one, other} in ({"score", "in_score"}, {"done", "in_done"}) else (0,))):
                assert call(**{one: base[other] + by}) == BAD, (one, other, by)
                assert b"memory" in lib.ee_last_error()
        for by in (4 - n, 0, need - 4):
            assert call(**{one: base["ws"] + by}) == BAD, (one, by)


def test_forks_whose_arrays_overlap():
    """workgroups read parents, lengths to keep and the other table while others write: these, the table and the states lie apart, to the byte"""
    lib, g = ee.load(), C.c_void_p()
    p = _cache(lib)
    assert lib.ee_pages_bind(p, 8, DUMMY, 1 << 40, C.byref(g)) == ee.EE_OK
    n, width = 6, 5
    base = dict(pages=1 << 20, kv_len=2 << 20, parent=3 << 20, keep=4 << 20, other_pages=5 << 20, other_len=6 << 20)
    sizes = dict(pages=4 * n * width, kv_len=4 * n, parent=4 * n, keep=4 * n, other_pages=4 * n * width, other_len=4 * n)

    def fork(states=(), source=False, **kw):
        a = dict(base, **kw)
        t, s = ee.ee_page_table(n, width, a["pages"], a["kv_len"]), ee.ee_page_table(n, width, a["other_pages"], a["other_len"])
        rows = (ee.ee_rows * max(len(states), 1))(*states)
        return lib.ee_pages_fork(g, C.byref(t), C.byref(s) if source else None, C.c_void_p(a["parent"]), C.c_void_p(a["keep"]), 0, rows, len(states), None, None)

    def refused(*a, **kw):
        code = fork(*a, **kw)
        assert code == BAD and b"memory" in lib.ee_last_error(), (a, kw, code)
    for one in ("pages", "kv_len"):
        for other in ("parent", "keep", "other_pages", "other_len"):
            for by in (4 - sizes[one], 0, sizes[other] - 4):
                refused(source=True, **{one: base[other] + by})
    refused(pages=base["kv_len"] - 4)
    for a, at in base.items():                                                     # rows of 12 bytes every 16
        if not a.startswith("other"):
            for by in (1 - (16 * (n - 1) + 12), -28, 0, sizes[a] - 1):
                refused(states=[ee.ee_rows(at + by, 16, 12)])
    x = 8 << 20
    for b in ((x + 1, 16, 4), (x + 11, 16, 1), (x + 12, 16, 5), (x - 4, 16, 5), (x + 5 * 16 + 11, 16, 4), (x - 5 * 16, 16, 1), (x + 12, 20, 4), (x + 13, 17, 1),
              (x - 100, 24, 24), (x - 1000, 200, 5)):
        refused(states=[ee.ee_rows(x, 16, 12), ee.ee_rows(*b)])
        refused(states=[ee.ee_rows(*b), ee.ee_rows(x, 16, 12)])
    lib.ee_pages_destroy(g)
    lib.ee_paged_destroy(p)
