"""Rotary tables, append, tree attention, logits and acceptance against their definitions (speculate_reference), and a run of them together."""
import math

import numpy as np
import pytest
import torch

import pages_reference as pref
import speculate_reference as ref
from test_gpu_prefix_attention import HALF, Case, dev

pytestmark = pytest.mark.gpu
TINY = {torch.bfloat16: 1e-38, torch.float16: 2.0 ** -25}
TYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def vb():
    from paper_2502_02175_b200 import binding
    return binding


def ints(n, value=77):
    return torch.full((n,), value, dtype=torch.int32, device="cuda")


def host(t):
    return t.double().cpu().numpy()


# ------------------------------------------------------------------------------------------------ tables
@pytest.mark.parametrize("first,n_pos,rot,kw", [
    (0, 1, 2, {}), (0, 300, 128, {}), (7, 33, 16, dict(theta=500000.0)), (1000003, 17, 64, {}), (2 ** 31 - 20, 19, 256, dict(theta=1e6)), (5, 40, 6, dict(amplitude=0.0)),
    (0, 100, 128, dict(factor=4.0)), (65000, 700, 128, dict(factor=8.0, original_len=8192.0)), (3, 50, 96, dict(factor=40.0, original_len=4096.0, turns=(0.5, 4.0), amplitude=1.37)),
    (3, 16, 64, dict(factor=0.5)), (31, 15, 34, dict(theta=0.5))])
def test_tables(vb, first, n_pos, rot, kw):
    kw = dict(dict(theta=10000.0), **kw)
    cos, sin = (torch.full((n_pos + 2, rot // 2), 9.0, device="cuda") for _ in range(2))
    vb.vlac_rope_tables(cos[1:-1], sin[1:-1], first=first, **kw)
    for got, want in zip((cos, sin), ref.tables(first, n_pos, rot, **kw)):
        # one rounding to fp32, and what 64 bits leave of an angle (the reference's own sine of it among that)
        assert np.all(np.abs(host(got[1:-1]) - want) <= 2.0 ** -24 * np.abs(want) + 1e-9 * kw.get("amplitude", 1.0))
        assert torch.all(got[0] == 9) and torch.all(got[-1] == 9)


def test_tables_are_those_of_the_decoder(vb):
    from paper_2502_02175_b200 import synth
    cfg = synth.llama7b_config(2)
    cos, sin = (torch.zeros((cfg.max_seq, cfg.head_dim // 2), device="cuda") for _ in range(2))
    vb.vlac_rope_tables(cos, sin, cfg.rope_theta)
    for got, want in zip((cos, sin), synth.rope_tables(cfg)):
        assert np.max(np.abs(got.cpu().numpy() - want)) <= 2.0 ** -24


# ------------------------------------------------------------------------------------------------ append
class Append:
    """A pool whose slot i has lens[i] rows, and new rows for its end (or for `start`)."""

    def __init__(self, vb, lens, new, heads, kv, d, page=16, dtype=torch.bfloat16, rot=0, inter=False, norm="", seed=0, layers=2, far=None, start=None):
        self.vb, self.rng, self.d, self.dtype, self.rot, self.inter, self.page, self.kv = vb, np.random.default_rng(seed), d, dtype, rot, inter, page, kv
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        most = max(-(-n // page) for n in lens) + 2
        self.pages = vb.Pages.empty(layers, sum(-(-n // page) for n in lens) + 4, page, kv, d, len(lens), most, dtype)
        st = ints(len(lens))
        vb.vlac_pages_resize(self.pages, dev(range(len(lens))), dev(lens), st)
        assert st.tolist() == [0] * len(lens)
        self.lens, self.new, self.seqs = lens, new, [int(x) for x in self.rng.permutation(len(lens))]
        self.count = [new[s] for s in self.seqs]
        self.ptr = np.concatenate([[0], np.cumsum(self.count)])
        self.rows = int(self.ptr[-1])
        self.start = None if start is None else [start[s] for s in self.seqs]
        make = lambda h: (torch.empty((self.rows, h, d), device="cuda").normal_(generator=g) * 3).to(dtype)  # noqa: E731
        self.q, self.k, self.v = make(heads), make(kv), make(kv)
        gain = lambda: (1 + 0.3 * torch.empty(d, device="cuda").normal_(generator=g)).to(dtype)  # noqa: E731
        self.q_gain, self.k_gain = gain() if "q" in norm else None, gain() if "k" in norm else None
        n_pos = far or max(lens) + 1
        self.cos, self.sin = (torch.from_numpy(x.astype(np.float32)).to("cuda") for x in ref.tables(0, n_pos, max(rot, 2), 10000.0))
        self.rope = vb.Rope(self.cos if rot else None, self.sin if rot else None, inter, self.q_gain, self.k_gain, 1e-5)

    def places(self, i):
        s, c = self.seqs[i], self.count[i]
        a = self.lens[s] - c if self.start is None else self.start[i]
        return np.arange(a, a + c)

    def want(self, pos=None):
        """Values and bounds of q and of the whole pool."""
        rows = [self.places(i) for i in range(len(self.seqs))]
        at = np.clip(np.concatenate(rows) if pos is None else np.asarray(pos), 0, len(self.cos) - 1)      # (refused rows may lie outside)
        c, s = (host(t)[at][:, :self.rot // 2] if self.rot else np.zeros((len(at), 0)) for t in (self.cos, self.sin))
        turn = lambda x, g: ref.turned(host(x), None if g is None else host(g), 1e-5, c, s, self.inter, HALF[self.dtype], TINY[self.dtype])  # noqa: E731
        q, k = turn(self.q, self.q_gain), turn(self.k, self.k_gain)
        return q, k, rows

    def run(self, layer=1, pos=None, q=None, q_out=None, k=None, v=None, seqs=None, status=None):
        st = ints(len(self.seqs)) if status is None else status
        q_out = torch.full_like(self.q, 5.0) if q_out is None else q_out
        self.vb.vlac_pages_append(self.pages, layer, dev(self.seqs if seqs is None else seqs), None if self.start is None else dev(self.start), dev(self.ptr), self.rope,
                                  None if pos is None else dev(pos), self.q if q is None else q, q_out, self.k if k is None else k, self.v if v is None else v, st)
        return q_out, st

    def check(self, q_out, before, layer=1, pos=None, skip=()):
        (q, eq), (k, ek), rows = self.want(pos)
        got_k, got_v, want_k, want_v = host(self.pages.k), host(self.pages.v), before[0].copy(), before[1].copy()
        bound = np.zeros_like(want_k)
        for i, at in enumerate(rows):
            a, b, t = self.ptr[i], self.ptr[i + 1], self.pages.table[self.seqs[i]].cpu().numpy()
            if i in skip:
                assert torch.all(q_out[a:b] == 5)
                continue
            assert np.all(np.abs(host(q_out[a:b]) - q[a:b]) <= eq[a:b])
            pg, r = t[at // self.page], at % self.page
            want_k[layer, pg, r], bound[layer, pg, r], want_v[layer, pg, r] = k[a:b], ek[a:b], host(self.v[a:b])
        assert np.all(np.abs(got_k - want_k) <= bound) and np.array_equal(got_v, want_v)


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "fp16"])
@pytest.mark.parametrize("heads,kv,d,rot,inter,norm", [(4, 4, 64, 64, False, ""), (4, 2, 64, 32, True, "qk"), (5, 1, 128, 128, False, "qk"), (32, 8, 128, 32, True, ""),
                                                      (3, 3, 128, 96, False, "q"), (7, 1, 64, 48, False, "k"), (2, 1, 64, 16, True, "qk"), (6, 2, 128, 0, False, "qk"),
                                                      (40, 20, 64, 0, False, ""), (0, 3, 64, 64, False, "k"), (33, 3, 64, 64, True, "q")])
@pytest.mark.parametrize("lens,new", [([1], [1]), ([17, 5, 40], [1, 1, 1]), ([33, 16, 70, 1], [33, 0, 20, 1]), ([300], [299])], ids=["one", "tokens", "ragged", "long"])
def test_append(vb, lens, new, heads, kv, d, rot, inter, norm, dtype):
    a = Append(vb, lens, new, heads, kv, d, dtype=dtype, rot=rot, inter=inter, norm=norm, seed=heads)
    before = host(a.pages.k), host(a.pages.v)
    q_out, st = a.run()
    assert st.tolist() == [0] * len(lens)
    a.check(q_out, before)


@pytest.mark.parametrize("page", [8, 64, 256])
def test_append_many_rows(vb, page):
    """More rows than warps: every form of sharing rows out, entries of all lengths, start in the middle of the slots."""
    for n, most in ((3, 2000), (70, 60)):
        lens = [most - 7 * (i % 5) for i in range(n)]
        new = [(most - 40) // (1 + i % 3) for i in range(n)]
        a = Append(vb, lens, new, 4, 2, 64, page=page, rot=64, norm="qk", seed=n, start=[i % 4 for i in range(n)])
        before = host(a.pages.k), host(a.pages.v)
        q_out, st = a.run(layer=0)
        assert st.tolist() == [0] * n
        a.check(q_out, before, layer=0)


def test_append_in_place_strides_and_positions(vb):
    """Columns of one fused buffer, queries rotated in place, positions of the caller's own."""
    a = Append(vb, [40, 33], [9, 4], 4, 2, 64, rot=64, norm="qk", seed=3, far=5000)
    pos = a.rng.integers(0, 5000, a.rows)
    fused = torch.cat([a.q, a.k, a.v], 1).contiguous()
    q, k, v = fused[:, :4], fused[:, 4:6], fused[:, 6:]
    before = host(a.pages.k), host(a.pages.v)
    _, st = a.run(q=q, q_out=q, k=k, v=v, pos=pos)
    assert st.tolist() == [0, 0] and torch.equal(k, a.k) and torch.equal(v, a.v)
    a.check(q, before, pos=pos)


def test_append_refusals_on_the_device(vb):
    """An entry that cannot be written changes nothing, in q_out either; the others stand."""
    for kind, code in (("slot", -1), ("twice", -1), ("position", -1), ("pos", -1), ("page", -2), ("shared", -2), ("len", -2), ("start", -1)):
        a = Append(vb, [40, 33, 20], [9, 4, 5], 4, 2, 64, rot=64, seed=4, far=39 if kind == "position" else None, start=[31, 29, 15])
        seqs, pos, bad = list(a.seqs), None, 1
        if kind == "slot":
            seqs[1] = 3
        elif kind == "twice":
            seqs[1] = seqs[0]
        elif kind == "position":
            bad = a.seqs.index(0)                                                # (its last row is the 40th)
        elif kind == "pos":
            pos = np.concatenate([a.places(i) for i in range(3)])
            pos[a.ptr[1]] = -1
        elif kind == "page":
            a.pages.table[seqs[1], a.places(1)[0] // 16] = 10 ** 6
        elif kind == "shared":
            a.pages.refs[a.pages.table[seqs[1], a.places(1)[0] // 16].long()] = 2
        elif kind == "len":
            a.pages.len[seqs[1]] = -3
        else:
            a.start[1] += 5000
        before = host(a.pages.k), host(a.pages.v)
        q_out, st = a.run(seqs=seqs, pos=pos)
        assert st.tolist() == [code if i == bad else 0 for i in range(3)], kind
        a.check(q_out, before, pos=pos, skip=(bad,))


def test_append_lists_that_fall(vb):
    """A falling row_ptr would rotate rows twice: nothing is done; entries that run out of the rows, and none at all."""
    a = Append(vb, [40, 33, 20], [9, 4, 5], 4, 2, 64, rot=64, seed=4)
    before, ptr = (host(a.pages.k), host(a.pages.v)), a.ptr
    for bad, want in (([0, 9, 4, 18], [-1] * 3), ([0, 2, 4, 19], None), ([-1, 2, 2, 2], None)):
        a.ptr = np.array(bad)
        q_out, st = a.run()
        if want is None:
            assert st.tolist()[0 if bad[0] < 0 else 2] == -1
            q_out, st = a.run(seqs=[9, 9, 9])
            assert set(st.tolist()) == {-1}
        else:
            assert st.tolist() == want and torch.equal(a.pages.k.double().cpu(), torch.from_numpy(before[0])) and torch.equal(a.pages.v.double().cpu(), torch.from_numpy(before[1]))
        assert torch.all(q_out == 5)
    st = ints(0)
    vb.vlac_pages_append(a.pages, 0, dev([]), None, dev([0]), a.rope, None, a.q, a.q.clone(), a.k, a.v, st)
    a.ptr, a.rows = ptr, 0
    none, st = a.q[:0], ints(3)
    vb.vlac_pages_append(a.pages, 0, dev(range(3)), None, dev([0] * 4), a.rope, None, none, none, a.k[:0], a.v[:0], st)
    assert st.tolist() == [0, 0, 0]


def test_append_far_pages_and_layers(vb):
    """Element offsets beyond 2^31 in K and V of the last layer, table rows beyond 2^31 bytes."""
    n_pages, kv, d = 5000, 16, 64
    k = torch.zeros((2, n_pages, 256, kv, d), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    assert k.numel() > 2 ** 31
    pages = vb.Pages(k, v, dev([[n_pages - 1, 7]]), dev([300]), torch.ones(n_pages, dtype=torch.int32, device="cuda"))
    far = 9_000_000
    cos, sin = (torch.empty((far, 64), device="cuda")[:, :32].contiguous() for _ in range(2))
    vb.vlac_rope_tables(cos[far - 5:], sin[far - 5:], 10000.0, first=far - 5)
    x = torch.randn((300, kv, d), device="cuda").to(torch.bfloat16)
    pos, st, q_out = np.full(300, far - 1), ints(1), torch.zeros_like(x)
    pos[::2] = far - 3
    vb.vlac_pages_append(pages, 1, dev([0]), None, dev([0, 300]), vb.Rope(cos, sin), dev(pos), x, q_out, x, x, st)
    assert st.item() == 0 and not torch.any(k[0]) and torch.equal(v[1, n_pages - 1], x[:256]) and torch.equal(v[1, 7, :44], x[256:])
    c, s = (t[pos - (far - 5)] for t in ref.tables(far - 5, 5, 64, 10000.0))
    y, e = ref.turned(host(x), None, 0, c, s, False, 2.0 ** -8, 1e-38)
    got = torch.cat([k[1, n_pages - 1], k[1, 7, :44]])
    assert np.all(np.abs(host(got) - y) <= e) and torch.equal(got, q_out)


# ------------------------------------------------------------------------------------------------ trees
def tree_of(vb, nq, parents, max_rows=None):
    return vb.Tree(dev(np.concatenate([[0], np.cumsum(nq)])), dev(np.concatenate([np.array(p, np.int64) for p in parents])), max_rows or max(nq + [1]))


def mask_rows(tree):
    return np.unpackbits(tree.mask.cpu().numpy().view(np.uint8).reshape(tree.rows, -1), axis=1, bitorder="little").astype(bool)


@pytest.mark.parametrize("nq,max_rows", [([1], 1), ([5, 0, 33, 64, 1], 64), ([1024], 1024), ([100, 31, 32], 100), ([1000] + [3] * 40, 1024)])
@pytest.mark.parametrize("reach", [1, 3, 2000])
def test_tree_plan(vb, nq, max_rows, reach):
    rng = np.random.default_rng(len(nq))
    parents = [ref.random_tree(n, rng, reach) for n in nq]
    lens = [n + int(rng.integers(0, 50)) for n in nq]
    pages = vb.Pages.empty(1, 200, 16, 1, 64, len(nq), 70)
    pages.len.copy_(dev(lens))
    tree = tree_of(vb, nq, parents, max_rows)
    for pool in (True, False):
        st = ints(len(nq))
        tree.mask.fill_(-1)
        vb.vlac_tree_plan(pages if pool else None, tree, dev(range(len(nq))) if pool else None, st)
        assert st.tolist() == [0] * len(nq)
        got, r = mask_rows(tree), 0
        for i, p in enumerate(parents):
            for j in range(nq[i]):
                up = ref.path(p, j)
                assert np.nonzero(got[r])[0].tolist() == sorted(up)
                assert tree.pos[r].item() == (lens[i] - nq[i] if pool else 0) + len(up) - 1 and tree.entry[r].item() == i
                r += 1


def test_tree_plan_refusals(vb):
    """Each bad entry gets its code and blank rows; rows of no entry are blank; a falling list refuses all."""
    pages = vb.Pages.empty(1, 20, 16, 1, 64, 4, 4)
    pages.len.copy_(dev([10, 20, 3, 99]))
    parent = dev([0, -1, 0, 0, -1, 0, 5, -1, 0, 1, -1, 0])
    seqs = [0, 1, 2, 3, 9, 0]
    #       rows     1..3    4..6: parent 5 of row 2    7..9: three rows    two: len 99    slot 9   none
    ptr = [1, 4, 7, 10, 12, 12, 12]
    tree = vb.Tree(dev(ptr), parent, 3)
    st = ints(6)
    vb.vlac_tree_plan(pages, tree, dev(seqs), st)
    assert st.tolist() == [0, -1, 0, -2, -1, 0]
    assert tree.entry.tolist() == [-1, 0, 0, 0, -1, -1, -1, 2, 2, 2, -1, -1]
    assert tree.pos.tolist() == [-1, 7, 8, 8, -1, -1, -1, 0, 1, 2, -1, -1]
    assert not np.any(mask_rows(tree)[[0, 4, 5, 6, 10, 11]])
    pages.len[2] = 2                                                             # fewer rows than the tree
    small = vb.Tree(dev(ptr), parent, 2)
    vb.vlac_tree_plan(pages, small, dev(seqs), st)
    assert st.tolist() == [-6, -6, -1, -2, -1, 0]
    for bad, want in (([1, 4, 3, 10, 12, 12, 12], [-1] * 6), ([-1, 1, 1, 1, 1, 1, 1], [-1, 0, 0, -2, -1, 0]), ([1, 1, 1, 1, 1, 1, 13], [0, 0, 0, -2, -1, -1])):
        t = vb.Tree(dev(bad), parent, 12)
        vb.vlac_tree_plan(pages, t, dev(seqs), st)
        assert st.tolist() == want
        assert set(t.entry.tolist()) == {-1} and set(t.pos.tolist()) == {-1} and not torch.any(t.mask)


# (common rows, [(own rows, drafted rows among them)])
TREES = {
    "one_row": [(0, [(1, 1)])],
    "alone": [(0, [(25, 25)]), (0, [(300, 25)]), (0, [(7, 3)])],
    "candidates": [(96, [(13, 9), (20, 13), (5, 5), (1, 1)])],
    "words": [(64, [(40, 31), (40, 32), (40, 33), (70, 64), (70, 65)])],
    "page_ends": [(16, [(16, 16), (17, 16), (15, 8)]), (160, [(33, 33)])],
    "large": [(1000, [(257, 200)]), (0, [(400, 400)])],
    "long": [(4100, [(70, 61)]), (2000, [(9, 7), (40, 33)])],
    "crowd": [(200, [(n % 7 + 4, n % 4 + 1) for n in range(40)])],
}


class TreeCase(Case):
    def __init__(self, vb, groups, *a, reach=4, **kw):
        super().__init__(vb, groups, *a, **kw)
        rng = np.random.default_rng(7)
        self.parents = [ref.random_tree(n, rng, reach) for n in self.nq]
        self.tree = tree_of(vb, self.nq, self.parents)

    def run(self, q=None, layer=0, out=None, lse=True, plan=None, mask=None):
        n, q = len(self.seqs), self.q if q is None else q
        plan = plan or self.vb.PrefixPlan(self.pages, n, self.rows, self.heads)
        out = torch.full((self.rows, self.heads, self.d), 5.0, dtype=self.dtype, device="cuda") if out is None else out
        l = torch.full((self.rows, self.heads), 5.0, device="cuda") if lse else None
        st, st2 = self.st(n), self.st(n)
        self.vb.vlac_tree_plan(self.pages, self.tree, dev(self.seqs), st2)
        self.vb.vlac_prefix_plan(self.pages, plan, dev(self.seqs), self.tree.q_ptr, st)
        if mask is not None:
            self.tree.mask.copy_(mask)
        self.vb.vlac_tree_attention(self.pages, layer, plan, self.tree, q, self.scale, out, l)
        assert st.tolist() == [0] * n and st2.tolist() == [0] * n and self.vb.vlac_prefix_error(plan) == 0
        return out, l

    def want(self, i, layer=0, q=None):
        slot, nq = self.seqs[i], self.nq[i]
        n = int(self.pages.len[slot])
        t = self.pages.table[slot, :-(-n // self.page)].long()
        k, v = (host(x[layer, t].reshape(-1, self.kv_heads, self.d)[:n]) for x in (self.pages.k, self.pages.v))
        r0 = sum(self.nq[:i])
        q = host((self.q if q is None else q)[r0:r0 + nq])
        seen = np.ones((nq, n), bool)
        seen[:, n - nq:] = mask_rows(self.tree)[r0:r0 + nq, :nq]
        return ref.tree_attention(k, v, q, n, nq, self.heads // self.kv_heads, self.scale, HALF[self.dtype], seen)


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "fp16"])
@pytest.mark.parametrize("heads,kv_heads,d", [(4, 4, 64), (4, 1, 128), (6, 2, 64), (2, 2, 128), (15, 3, 64)])
@pytest.mark.parametrize("groups", TREES, ids=str)
@pytest.mark.parametrize("columns", [0, 30000], ids=["narrow_tables", "wide_tables"])
def test_tree_attention(vb, columns, groups, heads, kv_heads, d, dtype):
    c = TreeCase(vb, TREES[groups], heads, kv_heads, d, dtype=dtype, seed=len(groups), columns=columns)
    first = c.run()
    c.check(*first)
    again = c.run()
    assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


@pytest.mark.parametrize("columns", [0, 30000], ids=["narrow_tables", "wide_tables"])
def test_a_chain_is_a_causal_chunk(vb, columns):
    """A tree without branches gives the bits of vlac_prefix_attention."""
    c = TreeCase(vb, [(100, [(40, 33), (9, 7)]), (0, [(70, 64)])], 6, 2, 128, seed=1, reach=1, columns=columns)
    out, lse = c.run()
    o2, l2 = Case.run(c)
    assert torch.equal(out, o2) and torch.equal(lse, l2)


@pytest.mark.parametrize("columns", [0, 30000], ids=["narrow_tables", "wide_tables"])
@pytest.mark.parametrize("page", [8, 256])
def test_any_mask(vb, page, columns):
    """Masks of the caller's own: random bits, later rows too, none (a row that sees only the sequence, or nothing at all), and bits behind the entry's rows."""
    c = TreeCase(vb, [(page * 2, [(40, 33), (50, 40), (35, 35)]), (0, [(33, 33), (64, 64), (1, 1)])], 4, 2, 64, seed=page, page=page, columns=columns)
    rng = np.random.default_rng(page)
    bits = rng.random((c.rows, 64)) < 0.3
    bits[::5] = False
    m = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32)).to("cuda")
    out, lse = c.run(mask=m)
    c.check(out, lse)
    empty = [r for r in range(108, 141) if not bits[r, :33].any()]
    assert empty and torch.all(out[empty] == 0) and torch.all(torch.isneginf(lse[empty]))


@pytest.mark.parametrize("columns", [0, 30000], ids=["narrow_tables", "wide_tables"])
def test_tree_values_a_row_does_not_see_never_reach_it(vb, columns):
    for d, heads in ((64, 1), (128, 3)):
        c = TreeCase(vb, [(40, [(40, 35), (9, 9)])], heads, 1, d, seed=d, columns=columns)
        c.parents[0] = [-1] + [0] * 34                                           # a root and 34 leaves
        c.tree = tree_of(vb, c.nq, c.parents)
        clean, clean_lse = c.run()
        n = int(c.pages.len[c.seqs[0]])
        for row, what in ((34, float("nan")), (20, float("inf")), (3, float("-inf"))):
            at = n - 35 + row
            pg = int(c.pages.table[c.seqs[0], at // 16])
            c.pages.v[0, pg, at % 16, 0, 5] = what
            if row == 34:
                c.pages.k[0, pg, at % 16, 0, 3] = what
        out, lse = c.run()
        same = [r for r in range(44) if r not in (34, 20, 3)]
        assert torch.equal(out[same], clean[same]) and torch.equal(lse[[20, 3] + same], clean_lse[[20, 3] + same])
        assert torch.all(torch.isnan(out[34])) and torch.all(torch.isposinf(out[20, :, 5])) and torch.all(torch.isneginf(out[3, :, 5]))
        assert torch.equal(out[20, :, 6:], clean[20, :, 6:])


def test_tree_layers_strides_scales(vb):
    c = TreeCase(vb, [(300, [(30, 20), (40, 33)]), (400, [(9, 8)] * 12)], 4, 2, 128, layers=3, seed=2, q_scale=0.5)
    wide = torch.full((c.rows, 3, c.heads, c.d), 3.0, dtype=c.dtype, device="cuda")
    wide[:, 1] = c.q
    for layer, scale in ((2, -0.2), (0, 0.0), (1, 3.0)):
        c.scale = scale
        out = torch.full((c.rows + 2, 2 * c.heads, c.d), 7.0, dtype=c.dtype, device="cuda")
        c.run(q=wide[:, 1], layer=layer, out=out[1:-1, :c.heads], lse=False)
        c.check(out[1:-1, :c.heads], None, layer)
        assert torch.all(out[0] == 7) and torch.all(out[-1] == 7) and torch.all(out[:, c.heads:] == 7)


def test_tree_refused_entries(vb):
    """What the prefix plan refuses keeps its rows; what only the tree plan refuses sees what lies in front of the tree."""
    c = TreeCase(vb, [(48, [(9, 5), (20, 11), (7, 4)])], seed=4)
    clean, clean_lse = c.run()
    plan, st, st2 = vb.PrefixPlan(c.pages, 3, c.rows, c.heads), ints(3), ints(3)
    c.tree.parent[6] = 9                                                         # of entry 1
    out, lse = torch.full_like(clean, 5.0), torch.full_like(clean_lse, 5.0)
    vb.vlac_tree_plan(c.pages, c.tree, dev(c.seqs), st2)
    vb.vlac_prefix_plan(c.pages, plan, dev([c.seqs[0], c.seqs[1], 10 ** 6]), c.tree.q_ptr, st)
    vb.vlac_tree_attention(c.pages, 0, plan, c.tree, c.q, c.scale, out, lse)
    assert st.tolist() == [0, 0, -1] and st2.tolist() == [0, -1, 0]
    assert torch.all(out[16:] == 5) and torch.all(lse[16:] == 5)
    c.check(out, lse, only=(0, 1))


# ------------------------------------------------------------------------------------------------ acceptance
def accept(vb, nq, lens, parents, drafted, chosen, room=0, max_rows=None, pages=None, seqs=None):
    n, rows = len(nq), sum(nq)
    if pages is None:
        pages = vb.Pages.empty(1, 2000, 16, 1, 64, n, 700)
        pages.len.copy_(dev(lens))
    tree = tree_of(vb, nq, parents, max_rows)
    out = dict(count=ints(n), path=ints(rows), tokens=ints(rows), keep_ptr=ints(n + 1), keep=ints(max(0, sum(max(x, 0) for x in lens) + room)), status=ints(n))
    vb.vlac_tree_accept(pages, tree, dev(range(n) if seqs is None else seqs), dev(drafted), dev(chosen), *out.values())
    return {k: v.tolist() for k, v in out.items()}


@pytest.mark.parametrize("nq,front", [([1], [0]), ([25], [290]), ([5, 0, 33, 64, 1], [0, 9, 100, 7, 0]), ([1024, 700], [3, 10000]), ([7 + i % 9 for i in range(200)], [i for i in range(200)]),
                                      ([2] * 1024, [5] * 1024)], ids=["one", "tree", "ragged", "largest", "many", "list"])
def test_accept(vb, nq, front):
    rng = np.random.default_rng(len(nq))
    parents = [ref.random_tree(n, rng, 3) for n in nq]
    rows, lens = sum(nq), [a + b for a, b in zip(nq, front)]
    for likely in (1, 2, 1000):
        drafted, chosen = rng.integers(-1 if likely == 2 else 0, likely, rows), rng.integers(-1 if likely == 2 else 0, likely, rows)   # (-1: no token)
        got = accept(vb, nq, lens, parents, drafted, chosen, room=3)
        keep, r = [], 0
        assert got["status"] == [0] * len(nq) and got["keep_ptr"][0] == 0
        for i, p in enumerate(parents):
            d, c = drafted[r:r + nq[i]], chosen[r:r + nq[i]]
            up = ref.accept(p, d, c)
            assert got["count"][i] == len(up)
            assert got["path"][r:r + nq[i]] == up + [-1] * (nq[i] - len(up))
            assert got["tokens"][r:r + nq[i]] == [c[x] for x in up] + [-1] * (nq[i] - len(up))
            keep += list(range(front[i])) + [front[i] + x for x in up]
            assert got["keep_ptr"][i + 1] == len(keep)
            r += nq[i]
        assert got["keep"][:len(keep)] == keep and set(got["keep"][len(keep):]) <= {77}


def test_accept_refusals(vb):
    """A refused entry keeps all its rows; a list that does not fit is refused by vlac_pages_compact too."""
    pages = vb.Pages.empty(1, 40, 16, 1, 64, 5, 4)
    st = ints(4)
    vb.vlac_pages_resize(pages, dev(range(4)), dev([10, 20, 5, 30]), st)
    parents = [[-1, 0, 0], [-1, 1, 0], [-1, 0], [-1, 0]]
    got = accept(vb, [3, 3, 2, 2], [10, 20, 5, 30], parents, [0] * 10, [0] * 10, pages=pages, seqs=[0, 1, 9, 3])
    assert got["status"] == [0, -1, -1, 0] and got["count"] == [2, 0, 0, 2] and got["keep_ptr"] == [0, 9, 29, 29, 59]
    assert got["keep"][:59] == list(range(9)) + list(range(20)) + list(range(30))
    assert got["path"] == [0, 1, -1] + [-1] * 5 + [0, 1] and got["tokens"] == [0, 0, -1] + [-1] * 5 + [0, 0]
    tree = tree_of(vb, [3, 3, 2, 2], [[-1, 0, 0], [-1, 0, 0], [-1, 0], [-1, 0]])
    count, path, tokens, ptr, keep, st = ints(4), ints(10), ints(10), ints(5), ints(30), ints(4)
    vb.vlac_tree_accept(pages, tree, dev(range(4)), dev([0] * 10), dev([0] * 10), count, path, tokens, ptr, keep, st)
    assert st.tolist() == [0, 0, -6, -6] and ptr.tolist() == [0, 9, 28, 33, 63] and keep.tolist() == list(range(9)) + list(range(19)) + [77, 77]
    vb.vlac_pages_compact(pages, dev(range(4)), dev(range(4)), ptr, keep, st)
    assert st.tolist() == [0, 0, -1, -1] and pages.len.tolist() == [9, 19, 5, 30, 0]
    for bad, code in (([0, 3, 2, 8, 10], [-1] * 4), ([-1, 3, 6, 8, 10], [-1, 0, 0, 0]), ([0, 3, 6, 8, 11], [0, 0, 0, -1])):
        t = vb.Tree(dev(bad), tree.parent, 4)
        vb.vlac_tree_accept(pages, t, dev(range(4)), dev([0] * 10), dev([0] * 10), count, path, tokens, ptr, keep, st)
        assert [min(0, x) if x != -6 else 0 for x in st.tolist()] == code


# ------------------------------------------------------------------------------------------------ logits
class Logits:
    def __init__(self, vb, rows, vocab, dtype=torch.float32, seed=0, hist=40, bias=5, masks=2, tree=(), drop=(), allow=0.5):
        self.vb, self.rows, self.vocab, self.dtype = vb, rows, vocab, dtype
        r = self.rng = np.random.default_rng(seed)
        self.x = torch.from_numpy((r.standard_normal((rows, vocab)) * 3).astype(np.float32)).to(dtype).to("cuda")
        few = r.integers(0, vocab, 8)
        self.history = np.where(r.random(hist * 2) < 0.6, few[r.integers(0, 8, hist * 2)], r.integers(-2, vocab + 3, hist * 2))   # some outside the vocabulary
        a = np.sort(r.integers(0, hist * 2 + 1, (rows, 3)), 1)
        self.span = a
        self.rep, self.freq, self.pres = (r.uniform(*w, rows).astype(np.float32) for w in ((0.7, 1.6), (-0.2, 0.5), (-0.1, 0.6)))
        cnt = r.integers(0, bias + 1, rows)
        self.bptr = np.concatenate([[0], np.cumsum(cnt)])
        self.btok, self.bval = r.integers(-1, min(vocab + 1, 12), self.bptr[-1]), r.uniform(-5, 5, self.bptr[-1]).astype(np.float32)   # many twice
        self.bits = r.random((masks, -(-vocab // 32) * 32)) < allow
        self.arow = r.integers(-1, masks, rows) if masks else None
        self.parents = [ref.random_tree(n, r) for n in tree]
        self.nq, self.drafted = list(tree), few[r.integers(0, 8, rows)]
        d = lambda x, t: torch.from_numpy(np.ascontiguousarray(x, t)).to("cuda")  # noqa: E731
        kw = dict(history=d(self.history, np.int32), span=d(self.span, np.int32), repetition=d(self.rep, np.float32), frequency=d(self.freq, np.float32),
                  presence=d(self.pres, np.float32), bias_ptr=d(self.bptr, np.int32), bias_token=d(self.btok, np.int32), bias=d(self.bval, np.float32))
        if masks:
            kw.update(allow=d(np.packbits(self.bits, axis=1, bitorder="little").view(np.int32), np.int32), allow_row=d(self.arow, np.int32))
        if tree:
            t = tree_of(vb, self.nq, self.parents)
            vb.vlac_tree_plan(None, t, None, ints(len(tree)))
            kw.update(tree=t, drafted=d(self.drafted, np.int32))
        for name in drop:
            kw.pop(name, None)
        self.kw, self.rules = kw, vb.LogitsRules(rows, vocab, **kw)

    def want(self, r, t=np.float32):
        k = self.kw
        a, g, b = self.span[r] if "span" in k else (0, 0, 0)
        made = list(self.history[g:b])
        if "tree" in k:
            i = int(np.searchsorted(np.cumsum(self.nq), r, side="right"))
            r0 = sum(self.nq[:i])
            made += [self.drafted[r0 + j] for j in ref.path(self.parents[i], r - r0)]
        bias = list(zip(self.btok[self.bptr[r]:self.bptr[r + 1]].tolist(), self.bval[self.bptr[r]:self.bptr[r + 1]])) if "bias" in k else []
        allowed = self.bits[self.arow[r], :self.vocab] if "allow" in k and self.arow[r] >= 0 else np.ones(self.vocab, bool)
        return ref.logits(self.x[r].float().cpu().numpy(), self.history[a:g], made, self.rep[r] if "repetition" in k else 1, self.freq[r] if "frequency" in k else 0,
                          self.pres[r] if "presence" in k else 0, bias, allowed, t)

    def run(self, x=None, out=True, picked=True):
        x = self.x if x is None else x
        out = torch.full_like(x, 5.0) if out is True else out
        p, st = ints(self.rows) if picked else None, ints(self.rows)
        self.vb.vlac_logits_adjust(x, self.rules, out, p, st)
        return out, p, st

    def check(self, out, picked, st, only=None):
        assert st.tolist() == [0] * self.rows
        for r in range(self.rows) if only is None else only:
            x, at = self.want(r)
            if out is not None:
                w = torch.from_numpy(x).to(self.dtype)
                assert torch.equal(out[r].cpu().nan_to_num(nan=1234.0), w.nan_to_num(nan=1234.0)), r
                y = self.want(r, np.float64)[0]
                fine = np.isfinite(y) & np.isfinite(x)
                half = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[self.dtype]
                # four steps of at most half a step of fp32 each, of magnitudes below |logit| * 1.6 + 0.5 * 80 + 0.6 + 5, and the rounding to the type
                big = np.nan_to_num(np.abs(host(self.x[r])), posinf=0.0) * 1.6 + 50
                assert np.all(np.abs(host(out[r])[fine] - y[fine]) <= 4 * 2.0 ** -24 * big[fine] + half * np.abs(y[fine]) + 2.0 ** -25)
            if picked is not None:
                assert picked[r].item() == at, r


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 7), (2, 33), (5, 1000), (2, 4096), (3, 4097), (2, 32000), (1, 70001), (2, 40008), (33, 64)])
def test_logits(vb, rows, vocab, dtype):
    c = Logits(vb, rows, vocab, dtype, seed=vocab, tree=(rows,))
    c.check(*c.run())
    c.check(c.run(out=None)[0], *c.run(out=None)[1:])
    again = c.x.clone()
    c.check(*c.run(x=again, out=again))
    c.check(*c.run(picked=False))


@pytest.mark.parametrize("drop", [("allow", "allow_row"), ("history", "span"), ("tree", "drafted"), ("bias_ptr", "bias_token", "bias"), ("repetition",), ("frequency", "presence"),
                                  ("history", "span", "tree", "drafted"), ("history", "span", "tree", "drafted", "bias_ptr", "bias_token", "bias", "allow", "allow_row",
                                                                          "repetition", "frequency", "presence")], ids=lambda d: "no_" + d[0] + str(len(d)))
def test_logits_without(vb, drop):
    c = Logits(vb, 9, 5003, seed=len(drop), tree=(4, 5), drop=drop)
    c.check(*c.run())


def test_logits_strides_and_alignment(vb):
    """Rows as columns of a wider buffer at every alignment; what lies beside them is left alone."""
    c = Logits(vb, 4, 4100, torch.bfloat16, seed=1, tree=(4,))
    for shift, width in ((0, 4104), (1, 4101), (8, 4120), (3, 4107)):
        x, out = torch.zeros((4, width), dtype=c.dtype, device="cuda"), torch.full((6, width), 7.0, dtype=c.dtype, device="cuda")
        x[:, shift:shift + 4100] = c.x
        _, p, st = c.run(x=x[:, shift:shift + 4100], out=out[1:-1, shift:shift + 4100])
        c.check(out[1:-1, shift:shift + 4100], p, st)
        out[1:-1, shift:shift + 4100] = 7
        assert torch.all(out == 7)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows", [1, 30, 80, 230, 450])
def test_logits_rows_at_every_alignment(vb, rows, dtype):
    """Odd vocabularies (each row begins elsewhere to 16 bytes), results aligned like the logits and otherwise, in place; tiny vocabularies; nothing beside the rows is
    written."""
    for vocab in (1, 2, 5, 9, 63, 1003, 4097) + ((70007,) if rows < 50 else ()):
        c = Logits(vb, rows, vocab, dtype, seed=vocab + rows, tree=[rows] if rows < 100 else [50] * (rows // 50) + ([rows % 50] if rows % 50 else []), hist=30)
        for shift, width in ((0, vocab), (3, vocab + 4), (1, vocab + 7)):
            only = range(0, rows, max(1, rows // 9))
            x = torch.full((rows, width), 3.0, dtype=dtype, device="cuda")
            x[:, shift:shift + vocab] = c.x
            for out_shift, out_width in ((shift, width), (shift + 1, width + 1), (shift + 8, width + 8)):
                out = torch.full((rows + 2, out_width), 7.0, dtype=dtype, device="cuda")
                cut = out[1:-1, out_shift:out_shift + vocab]
                _, p, st = c.run(x=x[:, shift:shift + vocab], out=cut)
                c.check(cut, p, st, only=only)
                cut.fill_(7.0)
                assert torch.all(out == 7)
            here = x[:, shift:shift + vocab]
            _, p, st = c.run(x=here, out=here)
            c.check(here, p, st, only=only)
            here.fill_(3.0)
            assert torch.all(x == 3)


def test_logits_beyond_32_bits(vb):
    """Element offsets beyond 2^31, results in place."""
    rows, vocab = 17001, 130001
    x = torch.zeros((rows, vocab), dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 2 ** 31
    x[-1, 129999], x[-2, 0], x[5, 77] = 2.0, 1.0, 3.0
    pen = torch.full((rows,), 0.5, device="cuda")
    rules = vb.LogitsRules(rows, vocab, history=dev([129999, 129999, 5]), span=dev([[0, 0, 3]] * rows), frequency=pen)
    p, st = ints(rows), ints(rows)
    vb.vlac_logits_adjust(x, rules, x, p, st)
    assert not torch.any(st) and p[-3:].tolist() == [0, 0, 129999] and p[5].item() == 77
    assert x[-1, [0, 5, 129998, 129999, 130000]].tolist() == [0.0, -0.5, 0.0, 1.0, 0.0] and x[-2, [0, 5, 129999]].tolist() == [1.0, -0.5, -1.0]


def test_logits_special_values(vb):
    """Infinities, NaN, ties, zeros of both signs, rows that the grammar leaves nothing of."""
    c = Logits(vb, 8, 9000, seed=2, tree=(8,), masks=3)
    c.bits[1] = False
    c.kw["allow"].copy_(torch.from_numpy(np.packbits(c.bits, axis=1, bitorder="little").view(np.int32)))
    c.x[0, 5000:] = float("inf")
    c.x[1] = float("-inf")
    c.x[2, 77] = float("nan")
    c.x[3] = -0.0
    c.x[3, 4500:] = 0.0
    c.x[4] = float("nan")
    c.x[5, [8, 4200, 8999]] = 1e30
    c.arow = np.array([0, 0, 2, 2, 1, -1, 1, 2])
    c.kw["allow_row"].copy_(dev(c.arow))
    out, p, st = c.run()
    c.check(out, p, st)
    assert p[4].item() == -1 and p[6].item() == -1 and torch.all(torch.isneginf(out[4])) and torch.all(torch.isneginf(out[6]))


def test_logits_long_history_and_many_rows(vb):
    for rows, vocab, hist, tree in ((300, 3000, 3000, [64] * 4 + [44]), (40, 150000, 5000, [40])):
        c = Logits(vb, rows, vocab, torch.bfloat16, seed=rows, hist=hist, bias=40, tree=tree)
        c.check(*c.run(), only=range(0, rows, 13))


@pytest.mark.parametrize("rows,dtype", [(3, torch.float32), (20, torch.bfloat16), (60, torch.float16), (230, torch.bfloat16), (450, torch.bfloat16)])
def test_logits_more_marks_than_the_table_holds(vb, rows, dtype):
    """Histories of many different tokens, and of one token many times: tables overflow, runs are cut, counts are exact."""
    vocab = 140000 if rows < 100 else 20000
    c = Logits(vb, rows, vocab, dtype, seed=rows, hist=9000, bias=60, tree=[rows] if rows < 100 else [50] * (rows // 50) + ([rows % 50] if rows % 50 else []))
    c.history[:] = np.random.default_rng(rows).integers(0, vocab, len(c.history))
    c.history[5000:9000] = 77
    c.kw["history"].copy_(dev(c.history))
    c.span[:, 2] = np.minimum(c.span[:, 1] + 8000, 18000)
    c.span[:, 0] = np.maximum(c.span[:, 1] - 6000, 0)
    c.kw["span"].copy_(dev(c.span))
    again = c.x.clone()
    c.check(*c.run(x=again, out=again), only=range(0, rows, max(1, rows // 7)))
    c.check(*c.run(), only=range(1, rows, max(1, rows // 5)))


def test_logits_refused_rows(vb):
    """Spans, bias lists and masks out of range: a code each, the row as it was."""
    def fresh():
        return Logits(vb, 6, 3000, seed=3, tree=(6,))
    for name, index, value in (("span", (2, 0), -1), ("span", (2, 2), 81), ("span", (2, 1), 90), ("bias_ptr", (2,), -1), ("bias_ptr", (3,), 10 ** 6), ("allow_row", (2,), 2),
                               ("allow_row", (2,), -2)):
        c = fresh()
        c.kw[name][index] = value
        out, p, st = c.run()
        bad = [r for r in range(6) if st[r].item() != 0]
        assert 2 in bad and set(bad) <= {1, 2, 3} and all(st[r].item() == -1 for r in bad) and torch.all(out[bad] == 5) and all(p[r].item() == 77 for r in bad)
        st[bad] = 0
        c.check(out, p, st, only=[r for r in range(6) if r not in bad])
    c = fresh()                                                                  # rows of no entry have no ancestors
    c.rules.tree.entry[:] = dev([0, -1, 9, -7, 0, 0])
    out, p, st = c.run()
    c.check(out, p, st, only=(0, 4, 5))
    c.kw.pop("tree")
    c.check(out, p, st, only=(1, 2, 3))


# ------------------------------------------------------------------------------------------------ together
def test_a_decoding_step_captured(vb):
    """Candidates of one prompt draft trees, every layer appends and attends, tokens are picked under rules, the confirmed path stays: eager, and captured
    and replayed; the pool, the tokens and the rows are what the definitions say."""
    L, H, KV, D, P, vocab, n = 2, 4, 2, 64, 16, 500, 3
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    rng = np.random.default_rng(3)
    nq, prompt = [9, 1, 33], 70
    parents = [ref.random_tree(x, rng, 3) for x in nq]
    rows, ptr = sum(nq), np.concatenate([[0], np.cumsum(nq)])
    cos, sin = (torch.zeros((400, D // 2), device="cuda") for _ in range(2))
    vb.vlac_rope_tables(cos, sin, 10000.0, factor=2.0, original_len=64.0)
    gain = (1 + 0.1 * torch.empty(D, device="cuda").normal_(generator=gen)).to(torch.bfloat16)
    rope = vb.Rope(cos, sin, False, gain, gain)
    w_head = torch.empty((H * D, vocab), device="cuda").normal_(generator=gen)
    qkv = [torch.empty((rows, H + 2 * KV, D), device="cuda").normal_(generator=gen).to(torch.bfloat16) for _ in range(L)]
    seed_rows = [[torch.empty((prompt, KV, D), device="cuda").normal_(generator=gen).to(torch.bfloat16) for _ in range(2)] for _ in range(L)]

    def fresh():
        p = vb.Pages.empty(L, 60, P, KV, D, n + 1, 12)
        st1 = ints(1)
        vb.vlac_pages_resize(p, dev([0]), dev([prompt]), st1)
        for l in range(L):
            vb.vlac_pages_append(p, l, dev([0]), None, dev([0, prompt]), rope, None, None, None, *seed_rows[l], st1)
            assert st1.item() == 0
        st = ints(n)
        vb.vlac_pages_fork(p, dev([0] * n), dev(range(1, n + 1)), False, st)
        assert st.tolist() == [0] * n
        return p

    drafted = dev(rng.integers(0, vocab, rows))
    allow = torch.from_numpy(np.packbits(rng.random((1, 512)) < 0.5, axis=1, bitorder="little").view(np.int32)).to("cuda")

    def step(p, b):
        vb.vlac_pages_resize(p, b["seqs"], b["lens"], b["st"][0])
        vb.vlac_tree_plan(p, b["tree"], b["seqs"], b["st"][1])
        vb.vlac_prefix_plan(p, b["plan"], b["seqs"], b["tree"].q_ptr, b["st"][2])
        x = 0
        for l in range(L):
            f = qkv[l].clone()
            q, k, v = f[:, :H], f[:, H:H + KV], f[:, H + KV:]
            vb.vlac_pages_append(p, l, b["seqs"], None, b["tree"].q_ptr, rope, b["tree"].pos, q, q, k, v, b["st"][3])
            vb.vlac_tree_attention(p, l, b["plan"], b["tree"], q, D ** -0.5, b["out"][l], None)
            x = x + b["out"][l].float().view(rows, -1)
        b["logits"].copy_(x @ w_head)
        vb.vlac_logits_adjust(b["logits"], b["rules"], b["adjusted"], b["chosen"], b["st"][4])
        vb.vlac_tree_accept(p, b["tree"], b["seqs"], drafted, b["chosen"], b["count"], b["path"], b["tokens"], b["keep_ptr"], b["keep"], b["st"][5])
        vb.vlac_pages_compact(p, b["seqs"], b["seqs"], b["keep_ptr"], b["keep"], b["st"][6])

    def buffers(p):
        tree = vb.Tree(dev(ptr), dev(np.concatenate(parents)), max(nq))
        rules = vb.LogitsRules(rows, vocab, repetition=torch.full((rows,), 1.3, device="cuda"), frequency=torch.full((rows,), 0.2, device="cuda"), tree=tree, drafted=drafted,
                               allow=allow, allow_row=dev([0] * rows))
        return dict(seqs=dev(range(1, n + 1)), lens=dev([prompt + x for x in nq]), tree=tree, plan=vb.PrefixPlan(p, n, rows, H), rules=rules,
                    st=[ints(n) if i != 4 else ints(rows) for i in range(7)], out=torch.zeros((L, rows, H, D), dtype=torch.bfloat16, device="cuda"),
                    logits=torch.zeros((rows, vocab), device="cuda"), adjusted=torch.zeros((rows, vocab), device="cuda"), chosen=ints(rows), count=ints(n), path=ints(rows),
                    tokens=ints(rows), keep_ptr=ints(n + 1), keep=ints(n * prompt + rows))

    # what the decoder chooses does not depend on what was drafted for leaves: draft, along a path, what it chooses
    p = fresh()
    b = buffers(p)
    for _ in range(6):
        p = fresh()
        b["plan"] = vb.PrefixPlan(p, n, rows, H)
        step(p, b)
        for i in range(n):
            at = list(range(nq[i]))
            for j in at[1:]:
                if j % 3:
                    drafted[ptr[i] + j] = b["chosen"][ptr[i] + parents[i][j]]
    p = fresh()
    b = buffers(p)
    step(p, b)
    assert all(set(s.tolist()) == {0} for s in b["st"])
    picked, keep_ptr, keep = b["chosen"].tolist(), b["keep_ptr"].tolist(), b["keep"].tolist()
    paths = [ref.accept(parents[i], drafted.tolist()[ptr[i]:ptr[i + 1]], picked[ptr[i]:ptr[i + 1]]) for i in range(n)]
    assert b["count"].tolist() == [len(x) for x in paths] and max(len(x) for x in paths) > 2
    c, s = (host(t) for t in (cos, sin))
    bits = np.unpackbits(allow.cpu().numpy().view(np.uint8), bitorder="little")[:vocab].astype(bool)
    for r in (0, 8, 9, 20, rows - 1):
        i = int(np.searchsorted(ptr[1:], r, side="right"))
        made = [drafted[ptr[i] + j].item() for j in ref.path(parents[i], r - ptr[i])]
        assert ref.logits(b["logits"][r].cpu().numpy(), [], made, 1.3, 0.2, 0, [], bits)[1] == picked[r]
    for i in range(n):
        assert int(p.len[i + 1]) == prompt + len(paths[i])
        t = p.table[i + 1, :-(-(prompt + len(paths[i])) // P)].long()
        for l in range(L):
            k, v = (x[l, t].reshape(-1, KV, D)[:prompt + len(paths[i])] for x in (p.k, p.v))
            assert torch.equal(v[:prompt], seed_rows[l][1])
            at = [ptr[i] + x for x in paths[i]]
            assert torch.equal(v[prompt:], qkv[l][at][:, H + KV:])
            pos = prompt + np.arange(len(at))                                    # the path's depths
            y, e = ref.turned(host(qkv[l][at][:, H:H + KV]), host(gain), 1e-6, c[pos], s[pos], False, 2.0 ** -8, 1e-38)
            assert np.all(np.abs(host(k[prompt:]) - y) <= e)
    # captured and replayed on a pool in the same state: the same bits
    p2 = fresh()
    state = [x.clone() for x in (p2.table, p2.len, p2.refs, p2.k, p2.v)]
    b2 = buffers(p2)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(p2, b2)
    for _ in range(2):
        for x, y in zip((p2.table, p2.len, p2.refs, p2.k, p2.v), state):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        for name in ("out", "adjusted", "chosen", "count", "path", "tokens", "keep_ptr"):
            assert torch.equal(b[name], b2[name]), name
        assert b2["keep"].tolist()[:keep_ptr[-1]] == keep[:keep_ptr[-1]]
        assert torch.equal(p.len, p2.len) and torch.equal(p.table, p2.table) and torch.equal(p.refs, p2.refs)


def test_two_captured_steps_at_once(vb):
    """Attention, logits and acceptance captured on two streams with buffers of their own over one pool, replayed side by side."""
    c = TreeCase(vb, [(128, [(20, 13), (9, 9), (40, 33)])], 4, 4, 64, seed=7)
    base, base_lse = c.run()
    lg = Logits(vb, 20, 9000, seed=5, tree=(20,))
    want = lg.run()
    work = []
    for s in [torch.cuda.Stream() for _ in range(2)]:
        plan, out, st, g = vb.PrefixPlan(c.pages, 3, c.rows, 4), torch.zeros_like(base), [ints(3), ints(3), ints(20)], torch.cuda.CUDAGraph()
        tree, x, p = tree_of(vb, c.nq, c.parents), torch.zeros_like(lg.x), ints(20)
        seqs = dev(c.seqs)
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=s):
            vb.vlac_tree_plan(c.pages, tree, seqs, st[0])
            vb.vlac_prefix_plan(c.pages, plan, seqs, tree.q_ptr, st[1])
            vb.vlac_tree_attention(c.pages, 0, plan, tree, c.q, c.scale, out, None)
            vb.vlac_logits_adjust(lg.x, lg.rules, x, p, st[2])
        work.append((s, g, out, x, p, (plan, st, tree, seqs)))
    for _ in range(10):
        for s, g, *_ in work:
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for _, _, out, x, p, _ in work:
        assert torch.equal(out, base) and torch.equal(x, want[0]) and torch.equal(p, want[1])


# ------------------------------------------------------------------------------------------------ bounds and expectations of their own
@pytest.mark.parametrize("rot,theta", [(256, 3e-6), (250, 2.5e-6), (254, 1e-4), (128, 10000.0), (256, 1e6), (96, 500000.0), (6, 100.0), (34, 0.5)])
def test_tables_of_far_positions(vb, rot, theta):
    """Every frequency at the last positions there are, against 60 decimal digits: the angle is right to 2^-59 of its own size (frequencies up to 48,000 turns a position
    show it: 10^14 turns), 64-bit arithmetic on a reduced angle adds less than 2^-44, the table's own rounding 2^-24."""
    import decimal
    D = decimal.Decimal
    first, n_pos = 2 ** 31 - 20, 19
    cos, sin = (torch.zeros((n_pos, rot // 2), device="cuda") for _ in range(2))
    vb.vlac_rope_tables(cos, sin, theta, first=first)
    with decimal.localcontext() as ctx:
        ctx.prec = 60
        two_pi = D("6.28318530717958647692528676655900576839433879875021164194988918461563281257")
        per = [D(theta) ** (D(-2 * i) / D(rot)) / two_pi for i in range(rot // 2)]
        turns = [[(first + p) * f for f in per] for p in range(n_pos)]
        angle = np.array([[float((t - t.to_integral_value()) * two_pi) for t in row] for row in turns])
        size = np.array([[float(t * two_pi) for t in row] for row in turns])
    for got, want in ((cos, np.cos(angle)), (sin, np.sin(angle))):
        assert np.all(np.abs(host(got) - want) <= 2.0 ** -59 * size + 2.0 ** -24 * np.abs(want) + 2.0 ** -44)


class ParentsCase(TreeCase):
    """What a row sees comes from the parents alone; `none`: entries that the tree plan refuses, whose rows see only what lies in front of the tree."""
    none = ()

    def want(self, i, layer=0, q=None):
        slot, nq = self.seqs[i], self.nq[i]
        n = int(self.pages.len[slot])
        t = self.pages.table[slot, :-(-n // self.page)].long()
        k, v = (host(x[layer, t].reshape(-1, self.kv_heads, self.d)[:n]) for x in (self.pages.k, self.pages.v))
        r0 = sum(self.nq[:i])
        seen = ref.seen_by(self.parents[i], n)
        if i in self.none:
            seen[:, n - nq:] = False
        return ref.tree_attention(k, v, host((self.q if q is None else q)[r0:r0 + nq]), n, nq, self.heads // self.kv_heads, self.scale, HALF[self.dtype], seen)


@pytest.mark.parametrize("reach", [1, 2, 2000])
@pytest.mark.parametrize("groups", TREES, ids=str)
def test_tree_attention_by_parents(vb, groups, reach):
    for heads, kv_heads, d, dtype, columns in ((4, 1, 128, torch.bfloat16, 0), (2, 2, 64, torch.float16, 30000)):
        c = ParentsCase(vb, TREES[groups], heads, kv_heads, d, dtype=dtype, seed=reach, columns=columns, reach=reach)
        c.check(*c.run())


def test_tree_attention_of_refused_trees_by_parents(vb):
    c = ParentsCase(vb, [(48, [(9, 5), (20, 11), (7, 4)]), (0, [(6, 6)])], seed=4)
    c.tree.parent[6], c.tree.parent[21] = 9, 1                                  # of entry 1, and of entry 3, which sees nothing then
    c.none = (1, 3)
    plan, st, st2 = vb.PrefixPlan(c.pages, 4, c.rows, c.heads), ints(4), ints(4)
    out, lse = torch.full_like(c.q, 5.0), torch.full((c.rows, c.heads), 5.0, device="cuda")
    vb.vlac_tree_plan(c.pages, c.tree, dev(c.seqs), st2)
    vb.vlac_prefix_plan(c.pages, plan, dev(c.seqs), c.tree.q_ptr, st)
    vb.vlac_tree_attention(c.pages, 0, plan, c.tree, c.q, c.scale, out, lse)
    assert st.tolist() == [0] * 4 and st2.tolist() == [0, -1, 0, -1]
    c.check(out, lse, only=(0, 1, 2))
    assert torch.all(out[20:] == 0) and torch.all(torch.isneginf(lse[20:]))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows", [1, 30, 80, 230, 450])
@pytest.mark.parametrize("lie", ["whole", "shifted", "single"])
def test_logits_infinities_as_they_are(vb, lie, rows, dtype):
    """What is not allowed is -infinity itself, not the type's lowest value, and infinities and lowest values among the logits stay what they are."""
    vocab = 4096 if lie == "whole" else 4099
    c = Logits(vb, rows, vocab, dtype, seed=rows, tree=[rows] if rows < 100 else [50] * (rows // 50) + ([rows % 50] if rows % 50 else []), masks=3, allow=0.3)
    low = torch.finfo(dtype).min
    c.x[:, ::7], c.x[:, 3::11], c.x[:, 5::501], c.x[:, 1234::2000] = low, float("-inf"), -low, float("inf")
    c.x[rows // 2, 17::600] = float("nan")
    pad = 1 if lie == "single" else 0
    out = torch.full((rows, vocab + pad), 7.0, dtype=dtype, device="cuda")
    _, p, st = c.run(out=out[:, pad:])
    assert st.tolist() == [0] * rows
    for r in {*range(0, rows, max(1, rows // 9)), rows // 2}:
        x, at = c.want(r)
        got, want = out[r, pad:].cpu(), torch.from_numpy(x).to(dtype)
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got[~got.isnan()], want[~want.isnan()]) and p[r].item() == at
        assert torch.all(torch.isneginf(got[torch.from_numpy(~c.bits[c.arow[r], :vocab])])) if c.arow[r] >= 0 else True
    here = c.x.clone()
    c.run(x=here, out=here)
    assert torch.equal(here.isnan(), out[:, pad:].isnan()) and torch.equal(here.nan_to_num(7.0, float("inf"), float("-inf")), out[:, pad:].nan_to_num(7.0, float("inf"), float("-inf")))
