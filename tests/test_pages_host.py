"""What the paged-pool and prefix-attention entry points refuse before anything is launched (no GPU needed), and the host mirror's
own bookkeeping."""
import ctypes as C

import numpy as np
import pytest

import pages_reference as ref


@pytest.fixture(scope="module")
def vb():
    from paper_2502_02175_b200 import build
    build.build()
    from paper_2502_02175_b200 import binding
    return binding


FAKE = 1 << 20          # an address that is never read: every call here is refused on the host


def _struct(vb, **over):
    f = dict(k=FAKE, v=FAKE, dtype=0, n_layers=2, n_pages=40, page_size=16, n_kv_heads=4, head_dim=64, n_slots=6, max_pages=9,
             table=FAKE, len=FAKE, refs=FAKE, work=FAKE, work_bytes=1 << 30)
    f.update(over)
    return vb.vlac_pages(**f)


def _calls(vb, p):
    """Every entry point on pool `p` with otherwise valid arguments."""
    r = C.byref(p) if p is not None else None
    plan = vb.vlac_prefix(2, 2, 4, FAKE, 1 << 40)
    return {
        "resize": lambda n=2, a=FAKE, b=FAKE, st=FAKE: vb.lib.vlac_pages_resize(r, a, b, n, st, None),
        "free": lambda n=2, a=FAKE, b=FAKE, st=FAKE: vb.lib.vlac_pages_free(r, a, n, st, None),
        "fork": lambda n=2, a=FAKE, b=FAKE, st=FAKE: vb.lib.vlac_pages_fork(r, a, b, n, 0, st, None),
        "compact": lambda n=2, a=FAKE, b=FAKE, st=FAKE: vb.lib.vlac_pages_compact(r, a, b, n, FAKE, FAKE, 4, st, None),
        "write": lambda n=2, a=FAKE, b=FAKE, st=FAKE: vb.lib.vlac_pages_write(r, 0, a, None, b, n, 4, FAKE, 256, FAKE, 256, st, None),
        "plan": lambda n=2, a=FAKE, b=FAKE, st=FAKE: vb.lib.vlac_prefix_plan(r, C.byref(vb.vlac_prefix(n, 2, 4, FAKE, 1 << 40)), a, b, st, None),
        "attention": lambda: vb.lib.vlac_prefix_attention(r, 0, C.byref(plan), FAKE, 256, 1.0, FAKE, 256, None, None),
        "from_cache": lambda: vb.lib.vlac_pages_from_cache(r, None, 0, 0, 1, FAKE, None),
    }


BAD_POOLS = [dict(k=None), dict(v=None), dict(table=None), dict(len=None), dict(refs=None), dict(work=None), dict(k=FAKE + 8), dict(refs=FAKE + 4),
             dict(work=FAKE + 8), dict(dtype=2), dict(head_dim=96), dict(n_layers=0), dict(n_pages=0), dict(n_slots=0), dict(max_pages=0),
             dict(n_kv_heads=0), dict(page_size=12), dict(page_size=4), dict(page_size=512), dict(n_pages=1 << 28), dict(max_pages=1 << 28),
             dict(work_bytes=64)]


@pytest.mark.parametrize("over", BAD_POOLS, ids=lambda o: "-".join(f"{k}{v}" for k, v in o.items()))
def test_a_pool_that_cannot_be_is_refused_by_every_call(vb, over):
    for name, call in _calls(vb, _struct(vb, **over)).items():
        assert call() == -1, name
    for name, call in _calls(vb, None).items():
        assert call() == -1, name


def test_lists(vb):
    calls = _calls(vb, _struct(vb))
    for name in ("resize", "free", "fork", "compact", "write", "plan"):
        call = calls[name]
        assert call(n=-1) == -1 and call(n=1025) == -6, name
        assert call(n=0, a=None, b=None, st=None) == 0, name
        assert call(a=None) == -1 and call(st=None) == -1, name
        if name != "free":
            assert call(b=None) == -1, name


def test_arguments_of_single_calls(vb):
    p = _struct(vb)
    r = C.byref(p)
    assert vb.lib.vlac_pages_fork(r, FAKE, FAKE, 1, 2, FAKE, None) == -1
    assert vb.lib.vlac_pages_compact(r, FAKE, FAKE, 1, FAKE, None, 3, FAKE, None) == -1
    assert vb.lib.vlac_pages_compact(r, FAKE, FAKE, 1, None, FAKE, 3, FAKE, None) == -1
    assert vb.lib.vlac_pages_compact(r, FAKE, FAKE, 1, FAKE, FAKE, -1, FAKE, None) == -1
    write = lambda layer=0, rows=4, k=FAKE, ks=256, v=FAKE, vs=256: vb.lib.vlac_pages_write(r, layer, FAKE, None, FAKE, 1, rows, k, ks, v, vs, FAKE, None)
    for bad in (dict(layer=-1), dict(layer=2), dict(rows=-1), dict(k=None), dict(v=None), dict(ks=255), dict(ks=248), dict(vs=260), dict(k=FAKE + 8), dict(v=FAKE + 2)):
        assert write(**bad) == -1, bad

    def attention(layer=0, n=2, rows=2, heads=4, mem=FAKE, size=1 << 40, q=FAKE, qs=256, scale=1.0, out=FAKE, os=256, lse=None):
        plan = vb.vlac_prefix(n, rows, heads, mem, size)
        return vb.lib.vlac_prefix_attention(r, layer, C.byref(plan), q, qs, scale, out, os, lse, None)
    for bad in (dict(layer=2), dict(layer=-1), dict(n=-1), dict(rows=-1), dict(heads=6), dict(heads=0), dict(mem=None), dict(mem=FAKE + 4), dict(size=100), dict(q=None),
                dict(qs=248), dict(qs=260), dict(out=None), dict(os=248), dict(q=FAKE + 2), dict(out=FAKE + 8), dict(lse=FAKE + 2), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(rows=1 << 28, heads=4)):
        assert attention(**bad) == -1, bad
    assert attention(n=1025) == -6
    assert attention(rows=0, q=None, out=None) == 0 and attention(n=0, q=None, out=None, mem=None) == 0
    assert vb.lib.vlac_prefix_attention(r, 0, None, FAKE, 256, 1.0, FAKE, 256, None, None) == -1


def test_sizes(vb):
    p = _struct(vb)
    assert vb.vlac_pages_work_bytes(p) > 4 * (p.n_pages + p.n_slots * p.max_pages)
    assert vb.lib.vlac_pages_work_bytes(None) == 0 and vb.vlac_pages_work_bytes(_struct(vb, n_pages=0)) == 0
    size = lambda n=2, rows=3, heads=8: vb.lib.vlac_prefix_bytes(C.byref(p), n, rows, heads)
    assert size() > 2 * 3 * 8 * 64 * 4 and size(rows=300) > size()
    assert size(n=0) == size(rows=0) == size(heads=0) == size(heads=6) == size(n=1025) == size(rows=1 << 27) == 0


def test_mirror_keeps_its_books():
    """The host mirror itself: whatever the calls, refs count the slots that hold a page, and rows read back as they were."""
    rng = np.random.default_rng(0)
    k = rng.integers(0, 1 << 16, (1, 24, 8, 2, 4)).astype(np.uint16)
    h = ref.HostPool(k, k, np.full((7, 5), -1, np.int32), np.zeros(7, np.int32), np.zeros(24, np.int32))
    for _ in range(200):
        op = rng.integers(3)
        a, b = (list(rng.choice(7, 2, replace=False)) for _ in range(2))
        before = [(h.len[s], [h.k[0, h.table[s, x // 8], x % 8].copy() for x in range(h.len[s])]) for s in range(7)]
        if op == 0:
            st = h.resize(a, [int(x) for x in rng.integers(0, 41, 2)])
        elif op == 1:
            st = h.fork(a, b, bool(rng.integers(2)))
            want = [list(range(before[s][0])) for s in a]
        else:
            want = [sorted(rng.choice(before[s][0], rng.integers(0, before[s][0] + 1), replace=False).tolist()) for s in a]
            st = h.compact(a, b, want)
        if op:
            for s, d, w, c in zip(a, b, want, st):
                if c == ref.OK:
                    assert h.len[d] == len(w)
                    assert all(np.array_equal(h.k[0, h.table[d, x // 8], x % 8], before[s][1][y]) for x, y in enumerate(w))
        held = np.zeros(24, int)
        for s in range(7):
            n = h.pages(h.len[s])
            held[h.table[s, :n]] += 1
            assert np.all(h.table[s, n:] == -1)
            assert h.len[s] % 8 == 0 or h.refs[h.table[s, n - 1]] == 1      # a partly filled last page is never shared
        assert np.array_equal(held, h.refs)


def test_tables_whose_positions_would_leave_32_bits_are_not_attended(vb):
    """Keys are taken in units: behind the last position of a sequence there has to be room for one in an int."""
    for page in (8, 256):
        p = _struct(vb, page_size=page, max_pages=(2 ** 31 - 1024 + page - 1) // page, n_pages=40, work_bytes=1 << 62)
        calls = _calls(vb, p)
        assert calls["plan"]() == -1 and calls["attention"]() == -1


@pytest.mark.parametrize("scale,code", [(3.0e38, -1), (-3.0e38, -1), (2.36e38, -1), (float("-inf"), -1)])
def test_scales_that_overflow_in_powers_of_two_are_refused(vb, scale, code):
    """Exponentials are taken to the base 2: the scale times log2(e) has to be finite too."""
    plan = vb.vlac_prefix(2, 2, 4, FAKE, 1 << 40)
    assert vb.lib.vlac_prefix_attention(C.byref(_struct(vb)), 0, C.byref(plan), FAKE, 256, scale, FAKE << 4, 256, None, None) == code


def test_results_over_the_queries_are_refused(vb):
    plan = vb.vlac_prefix(2, 3, 4, FAKE, 1 << 40)
    for q, qs, out, os in ((FAKE, 256, FAKE, 256), (FAKE, 256, FAKE + 16, 256), (FAKE + 1024, 256, FAKE, 256), (FAKE, 512, FAKE + 256, 512), (FAKE, 256, FAKE + 1520, 1024),
                           (FAKE + 3056, 256, FAKE, 1280), (FAKE, 1 << 40, FAKE + (1 << 42) + 496, 256)):
        assert vb.lib.vlac_prefix_attention(C.byref(_struct(vb)), 0, C.byref(plan), q, qs, 1.0, out, os, None, None) == -1, (q, qs, out, os)
