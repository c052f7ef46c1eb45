"""What the calls for speculative decoding refuse before anything is launched (no GPU needed), and the host forms' own arithmetic."""
import ctypes as C

import numpy as np
import pytest

import speculate_reference as ref
from test_pages_host import BAD_POOLS, FAKE, _struct, vb  # noqa: F401

SIDE = FAKE + (1 << 30)
INVALID, TOO_LARGE = -1, -6


def _rope(vb, **over):
    f = dict(cos=FAKE, sin=FAKE, n_pos=100, rot_dim=64, interleaved=0, q_gain=None, k_gain=None, eps=1e-6)
    f.update(over)
    return vb.vlac_rope(**f)


def _append(vb, p=None, rope=None, **over):
    f = dict(layer=0, seqs=FAKE, start=None, row_ptr=FAKE, n=2, rows=4, pos=None, heads=4, q=FAKE, q_stride=256, q_out=SIDE, out_stride=256, k=FAKE, k_stride=256, v=FAKE,
             v_stride=256, status=FAKE)
    f.update(over)
    p = _struct(vb) if p is None else p
    rope = _rope(vb) if rope is None else rope
    return vb.lib.vlac_pages_append(C.byref(p), f["layer"], f["seqs"], f["start"], f["row_ptr"], f["n"], f["rows"], C.byref(rope) if rope != "none" else None, f["pos"],
                                    f["heads"], f["q"], f["q_stride"], f["q_out"], f["out_stride"], f["k"], f["k_stride"], f["v"], f["v_stride"], f["status"], None)


def _tree(vb, **over):
    f = dict(n=2, rows=4, max_rows=8, q_ptr=FAKE, parent=FAKE, mask=FAKE, pos=FAKE, entry=FAKE)
    f.update(over)
    return vb.vlac_tree(**f)


@pytest.mark.parametrize("over", BAD_POOLS, ids=lambda o: "-".join(f"{k}{v}" for k, v in o.items()))
def test_impossible_pools(vb, over):
    p = _struct(vb, **over)
    t, plan = _tree(vb), vb.vlac_prefix(2, 4, 4, FAKE, 1 << 40)
    assert _append(vb, p) == INVALID
    assert vb.lib.vlac_tree_plan(C.byref(p), C.byref(t), FAKE, FAKE, None) == INVALID
    assert vb.lib.vlac_tree_attention(C.byref(p), 0, C.byref(plan), C.byref(t), FAKE, 256, 1.0, SIDE, 256, None, None) == INVALID
    assert vb.lib.vlac_tree_accept(C.byref(p), C.byref(t), *[FAKE] * 8, 4, FAKE, None) == INVALID


def test_tables(vb):
    good = dict(rot_dim=64, theta=1e4, factor=1.0, original_len=0.0, turns_low=1.0, turns_high=32.0, amplitude=1.0)
    call = lambda first=0, n=4, cos=FAKE, sin=FAKE, **o: vb.lib.vlac_rope_tables(C.byref(vb.vlac_rope_scaling(**dict(good, **o))), first, n, cos, sin, None)  # noqa: E731
    for bad in (dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=258), dict(theta=0.0), dict(theta=float("nan")), dict(theta=float("inf")), dict(theta=1e-30), dict(factor=1e-9), dict(factor=0.0), dict(factor=-1.0),
                dict(original_len=-1.0), dict(original_len=float("inf")), dict(original_len=64.0, turns_low=2.0, turns_high=2.0), dict(amplitude=float("nan")), dict(first=-1), dict(n=-1),
                dict(first=2 ** 31 - 2, n=3), dict(cos=None), dict(sin=None), dict(cos=FAKE + 2)):
        assert call(**bad) == INVALID, bad
    assert vb.lib.vlac_rope_tables(None, 0, 4, FAKE, FAKE, None) == INVALID
    assert call(n=0, cos=None, sin=None) == 0


def test_append(vb):
    for bad in (dict(layer=-1), dict(layer=2), dict(n=-1), dict(rows=-1), dict(heads=-1), dict(seqs=None), dict(row_ptr=None), dict(status=None), dict(k=None), dict(v=None), dict(q=None),
                dict(q_out=None), dict(q_stride=248), dict(out_stride=248), dict(k_stride=248), dict(v_stride=260), dict(q_stride=257), dict(q=FAKE + 8), dict(q_out=SIDE + 8),
                dict(k=FAKE + 2), dict(v=FAKE + 8), dict(q_out=FAKE + 256), dict(q_out=FAKE, out_stride=264), dict(q=SIDE, q_out=FAKE + 512), dict(q=SIDE, q_out=FAKE + 2048 - 512)):
        assert _append(vb, **bad) == INVALID, bad
    for bad in (dict(rot_dim=8), dict(rot_dim=-16), dict(rot_dim=80), dict(interleaved=2), dict(cos=None), dict(sin=FAKE + 4), dict(n_pos=-1), dict(q_gain=FAKE + 8),
                dict(k_gain=FAKE, eps=-1.0), dict(k_gain=FAKE, eps=float("nan"))):
        assert _append(vb, rope=_rope(vb, **bad)) == INVALID, bad
    assert _append(vb, rope="none") == INVALID
    assert _append(vb, n=1025) == TOO_LARGE
    assert _append(vb, n=0, seqs=None, row_ptr=None, status=None) == 0


def test_trees(vb):
    p, plan = _struct(vb), vb.vlac_prefix(2, 4, 4, FAKE, 1 << 40)
    r, attend = C.byref(p), lambda t, **k: vb.lib.vlac_tree_attention(C.byref(p), 0, C.byref(plan), t, FAKE, 256, 1.0, k.get("out", SIDE), 256, None, None)  # noqa: E731
    for bad in (dict(n=-1), dict(rows=-1), dict(max_rows=0), dict(max_rows=1025), dict(q_ptr=None), dict(parent=None), dict(q_ptr=FAKE + 2)):
        t = C.byref(_tree(vb, **bad))
        assert vb.lib.vlac_tree_plan(r, t, FAKE, FAKE, None) == INVALID, bad
        assert vb.lib.vlac_tree_accept(r, t, *[FAKE] * 8, 4, FAKE, None) == INVALID, bad
    for bad in (dict(mask=None), dict(pos=None), dict(entry=None), dict(mask=FAKE + 1)):
        assert vb.lib.vlac_tree_plan(r, C.byref(_tree(vb, **bad)), FAKE, FAKE, None) == INVALID, bad
    for bad in (dict(n=1), dict(rows=5), dict(max_rows=0), dict(max_rows=2000), dict(mask=None), dict(mask=FAKE + 2)):
        assert attend(C.byref(_tree(vb, **bad))) == INVALID, bad
    assert attend(None) == INVALID and attend(C.byref(_tree(vb)), out=FAKE + 512) == INVALID
    t = C.byref(_tree(vb))
    assert vb.lib.vlac_tree_plan(r, None, FAKE, FAKE, None) == INVALID and vb.lib.vlac_tree_plan(r, t, None, FAKE, None) == INVALID
    assert vb.lib.vlac_tree_plan(None, t, FAKE, FAKE, None) == INVALID and vb.lib.vlac_tree_plan(r, t, FAKE, None, None) == INVALID
    assert vb.lib.vlac_tree_plan(r, C.byref(_tree(vb, n=1025)), FAKE, FAKE, None) == TOO_LARGE
    assert vb.lib.vlac_tree_plan(None, C.byref(_tree(vb, n=0)), None, None, None) == 0
    good = [FAKE] * 8
    for i in range(8):
        assert vb.lib.vlac_tree_accept(r, t, *[None if j == i else FAKE for j in range(8)], 4, FAKE, None) == INVALID, i
    assert vb.lib.vlac_tree_accept(r, t, *good, 4, None, None) == INVALID
    assert vb.lib.vlac_tree_accept(r, t, *good, -1, FAKE, None) == INVALID and vb.lib.vlac_tree_accept(r, t, *good, 2 ** 31 - 1, FAKE, None) == INVALID
    assert vb.lib.vlac_tree_accept(r, C.byref(_tree(vb, n=0)), *[None] * 8, 0, None, None) == 0


def test_logits(vb):
    def call(rows=4, vocab=100, dtype=2, x=FAKE, stride=100, out=SIDE, out_stride=100, picked=FAKE, status=FAKE, rules=True, **u):
        r = vb.vlac_logits_rules(**u)
        return vb.lib.vlac_logits_adjust(rows, vocab, dtype, x, stride, C.byref(r) if rules else None, out, out_stride, picked, status, None)
    tree = lambda **o: C.addressof(call.keep.setdefault(str(o), _tree(vb, **o)))  # noqa: E731
    call.keep = {}
    for bad in (dict(rows=-1), dict(vocab=0), dict(vocab=2 ** 30 + 1, stride=2 ** 31), dict(dtype=3), dict(dtype=-1), dict(x=None), dict(x=FAKE + 2), dict(out=SIDE + 1), dict(stride=99),
                dict(out_stride=99), dict(status=None), dict(picked=FAKE + 2), dict(status=FAKE + 1), dict(rules=False), dict(out=FAKE + 4), dict(out=FAKE, out_stride=101),
                dict(span=FAKE, n_tokens=3), dict(n_tokens=-1), dict(n_tokens=2 ** 30 + 1), dict(n_bias=-1), dict(n_bias=2 ** 30 + 1), dict(n_allow=-1), dict(bias_ptr=FAKE, n_bias=2, bias=FAKE), dict(bias_ptr=FAKE, n_bias=2, bias_token=FAKE),
                dict(allow=FAKE, n_allow=3), dict(allow=FAKE + 2, n_allow=4), dict(span=FAKE + 1), dict(repetition=FAKE + 2), dict(tree=tree()), dict(drafted=FAKE),
                dict(tree=tree(rows=5), drafted=FAKE), dict(tree=tree(n=1025), drafted=FAKE), dict(tree=tree(max_rows=0), drafted=FAKE), dict(tree=tree(mask=None), drafted=FAKE),
                dict(tree=tree(entry=None), drafted=FAKE), dict(tree=tree(q_ptr=FAKE + 2), drafted=FAKE)):
        assert call(**bad) == INVALID, bad
    assert call(rows=65536) == TOO_LARGE
    assert call(rows=0, x=None, status=None) == 0


def test_host_forms():
    """The references' own arithmetic, by hand."""
    assert ref.path([-1, 0, 0, 2, 1], 3) == [3, 2, 0]
    assert ref.accept([-1, 0, 0, 2, 2, 1], [0, 5, 6, 7, 8, 9], [6, 0, 8, 0, 1, 0]) == [0, 2, 4]
    assert ref.accept([-1, 0, 0], [0, 5, 5], [5, 1, 1]) == [0, 1] and ref.accept([-1, 0], [0, -1], [-1, 0]) == [0]
    x, at = ref.logits(np.array([2.0, -2.0, 1.0, 4.0], np.float32), [0, 99], [1, 1], 2.0, 0.5, 0.25, [(2, 9.0), (2, 1.0)], np.array([1, 1, 1, 0], bool))
    assert x.tolist() == [1.0, -5.25, 2.0, -np.inf] and at == 2
    assert ref.logits(np.zeros(3, np.float32), [], [], 1, 0, 0, [], np.zeros(3, bool))[1] == -1
    c, s = ref.tables(3, 1, 4, 100.0)
    assert np.allclose(c, [[np.cos(3.0), np.cos(0.3)]]) and np.allclose(s, [[np.sin(3.0), np.sin(0.3)]])
    # by parts: one frequency kept (many turns), one divided
    c, s = ref.tables(3, 1, 4, 1e6, factor=4.0, original_len=1000.0)
    assert np.allclose(s, [[np.sin(3.0), np.sin(0.003 / 4)]])
    y, _ = ref.turned(np.array([[[1.0, 2.0, 3.0, 4.0]]]), None, 0, np.array([[0.0]]), np.array([[1.0]]), False, 0, 0)
    assert y.tolist() == [[[-2.0, 1.0, 3.0, 4.0]]]


def test_queries_into_the_pool_are_refused(vb):
    """Rotated queries written over K or V: any layer, the pool's first and last bytes, rows on both sides of it."""
    side, far = FAKE + (1 << 32), FAKE + (1 << 33)
    p = _struct(vb, v=side)
    layer = 40 * 16 * 4 * 64 * 2
    for begin in (FAKE, side):
        for at in (begin, begin + layer, begin + 2 * layer - 16, begin + layer - 512, begin - 3 * 512 - 16, begin - 2048 + 16):
            assert _append(vb, p, q=far, q_out=at, k=far + (1 << 20), v=far + (1 << 21)) == INVALID, (begin, at)
        # queries that live there, in place; a row of a wide buffer that lies inside the pool
        assert _append(vb, p, q=begin, q_out=begin, k=far, v=far) == INVALID
        assert _append(vb, p, q=far, q_out=begin - (1 << 19), out_stride=1 << 18, k=far + (1 << 24), v=far + (1 << 24)) == INVALID


def test_attention_results_over_the_pool_or_the_sums_are_refused(vb):
    """Rows of out share no memory with K, V or lse (plain and with a tree)."""
    side, far = FAKE + (1 << 32), FAKE + (1 << 33)
    p, plan, tree = _struct(vb, v=side), vb.vlac_prefix(2, 4, 4, FAKE, 1 << 40), _tree(vb)
    layer = 40 * 16 * 4 * 64 * 2

    def call(out, stride=256, lse=None):
        head = C.byref(p), 1, C.byref(plan)
        return {vb.lib.vlac_prefix_attention(*head, far, 256, 1.0, out, stride, lse, None), vb.lib.vlac_tree_attention(*head, C.byref(tree), far, 256, 1.0, out, stride, lse, None)}
    for begin in (FAKE, side):
        for at in (begin, begin + layer, begin + 2 * layer - 16, begin - 3 * 512 - 16):
            assert call(at) == {INVALID}, (begin, at)
        assert call(begin - (1 << 19), stride=1 << 18) == {INVALID}
    out = far + (1 << 20)
    for lse in (out, out - 60, out + 3 * 512 + 508, out + 512):                  # (4 rows of 4 sums: 64 bytes)
        assert call(out, lse=lse) == {INVALID}, lse - out
    assert call(out, stride=1 << 12, lse=out + 3 * (1 << 13) - 4) == {INVALID}


def test_lists_off_their_alignment_are_refused(vb):
    """A list of ints that does not begin at a multiple of 4 bytes would be a misaligned read on the device."""
    p, t = _struct(vb), _tree(vb)
    for name in ("seqs", "row_ptr", "status", "start", "pos"):
        assert _append(vb, **{name: FAKE + 2}) == INVALID, name
    for seqs, status in ((FAKE + 1, FAKE), (FAKE, FAKE + 2)):
        assert vb.lib.vlac_tree_plan(C.byref(p), C.byref(t), seqs, status, None) == INVALID
    for i in range(9):
        a = [FAKE + 2 if j == i else FAKE for j in range(9)]
        assert vb.lib.vlac_tree_accept(C.byref(p), C.byref(t), *a[:8], 4, a[8], None) == INVALID, i
