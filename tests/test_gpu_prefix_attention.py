"""Attention over paged sequences with a shared prefix against its definition in 64 bits.  Bounds: pages_reference.attention."""
import math

import numpy as np
import pytest
import torch

import pages_reference as ref
from paper_2502_02175_b200 import synth

pytestmark = pytest.mark.gpu
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.fixture(scope="module")
def vb():
    from paper_2502_02175_b200 import binding
    return binding


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to("cuda")


class Case:
    """Groups of sequences made with the pool calls: (common rows, [(own rows, query rows), ...]) per group.

    ``columns``: further columns of the tables.  Calls on narrow tables with few rows take a form of their own; wide tables keep them to the
    general one.
    """

    def __init__(self, vb, groups, heads=4, kv_heads=4, d=64, page=16, dtype=torch.bfloat16, seed=0, layers=1, spare=3, q_scale=2.0, fill=float("nan"),
                 columns=30000):
        self.vb, self.heads, self.kv_heads, self.d, self.page, self.dtype = vb, heads, kv_heads, d, page, dtype
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        total = sum(c + sum(o + page for o, _ in m) for c, m in groups) + spare * page
        longest = max([c + o for c, m in groups for o, _ in m] + [1])
        n_slots = sum(len(m) + 1 for _, m in groups) + 1
        self.pages = p = vb.Pages.empty(layers, -(-total // page) + len(groups) + spare, page, kv_heads, d, n_slots, -(-longest // page) + 1 + columns, dtype)
        p.k.fill_(fill)                                                  # rows nobody wrote must never matter
        p.v.fill_(fill)
        self.seqs, self.nq, slot = [], [], 0
        for c, members in groups:
            base = slot
            slot += 1
            self.resize([base], [c])
            self.fill(base, 0, c)
            for o, nq in members:
                st = self.st(1)
                vb.vlac_pages_fork(p, dev([base]), dev([slot]), False, st)
                assert st.item() == 0
                self.resize([slot], [c + o])
                self.fill(slot, c, o)
                self.seqs.append(slot)
                self.nq.append(nq)
                slot += 1
        self.rows = sum(self.nq)
        self.q = (torch.empty((self.rows, heads, d), device="cuda").normal_(generator=self.gen) * q_scale).to(dtype)
        self.scale = 1.0 / math.sqrt(d)

    def st(self, n):
        return torch.full((n,), 9, dtype=torch.int32, device="cuda")

    def resize(self, slots, lens):
        st = self.st(len(slots))
        self.vb.vlac_pages_resize(self.pages, dev(slots), dev(lens), st)
        assert st.tolist() == [0] * len(slots)

    def fill(self, slot, start, n):
        for l in range(self.pages.k.shape[0]):
            x, y = (torch.empty((n, self.kv_heads, self.d), device="cuda").normal_(generator=self.gen).to(self.dtype) for _ in range(2))
            st = self.st(1)
            self.vb.vlac_pages_write(self.pages, l, dev([slot]), dev([start]), dev([0, n]), x, y, st)
            assert st.item() == 0

    def run(self, q=None, layer=0, out=None, lse=True, plan=None):
        n = len(self.seqs)
        q = self.q if q is None else q
        plan = plan or self.vb.PrefixPlan(self.pages, n, self.rows, self.heads)
        out = torch.full((self.rows, self.heads, self.d), 5.0, dtype=self.dtype, device="cuda") if out is None else out
        l = torch.full((self.rows, self.heads), 5.0, device="cuda") if lse else None
        st = self.st(n)
        self.vb.vlac_prefix_plan(self.pages, plan, dev(self.seqs), dev(np.concatenate([[0], np.cumsum(self.nq)])), st)
        self.vb.vlac_prefix_attention(self.pages, layer, plan, q, self.scale, out, l)
        assert st.tolist() == [0] * n
        assert self.vb.vlac_prefix_error(plan) == 0
        return out, l

    def want(self, i, layer=0, q=None):
        """(out, lse, bounds) of sequence i in 64 bits, through its own table."""
        slot, nq = self.seqs[i], self.nq[i]
        n = int(self.pages.len[slot])
        t = self.pages.table[slot, :-(-n // self.page)].long()
        k, v = (x[layer, t].reshape(-1, self.kv_heads, self.d)[:n].double().cpu().numpy() for x in (self.pages.k, self.pages.v))
        r0 = sum(self.nq[:i])
        q = (self.q if q is None else q)[r0:r0 + nq].double().cpu().numpy()
        return ref.attention(k, v, q, n, nq, self.heads // self.kv_heads, self.scale, HALF[self.dtype])

    def check(self, out, lse, layer=0, q=None, only=None):
        for i in range(len(self.seqs)) if only is None else only:
            o, l, eo, el = self.want(i, layer, q)
            r0 = sum(self.nq[:i])
            got = out[r0:r0 + self.nq[i]].double().cpu().numpy()
            bad = np.abs(got - o) > eo
            assert not np.any(bad | ~np.isfinite(got)), (i, np.argwhere(bad)[:3], np.max(np.abs(got - o) / eo))
            if lse is not None:
                gl = lse[r0:r0 + self.nq[i]].double().cpu().numpy()
                inf = np.isneginf(l)
                assert np.array_equal(np.isneginf(gl), inf)
                assert np.all(np.abs(gl[~inf] - l[~inf]) <= el[~inf]), i


# (common rows, [(own rows, query rows)])
GROUPS = {
    "one_row_one_key": [(0, [(1, 1)])],
    "two_candidates": [(32, [(3, 1), (5, 1)])],
    "unshared_tail": [(37, [(1, 1), (20, 1), (64, 1)])],                        # the partly filled page is each one's own
    "page_ends": [(16, [(15, 1), (16, 1), (17, 1)]), (64, [(64, 1), (1, 1)])],
    "chunks_of_7": [(100, [(7, 7), (9, 7), (30, 7)])],
    "prefill": [(0, [(33, 33)]), (48, [(130, 70)]), (0, [(65, 2)])],
    "more_queries_than_rows": [(0, [(3, 5), (1, 4), (0, 2)])],
    "nothing_to_do": [(48, [(2, 0), (2, 1), (2, 0), (3, 1)])],
    "many_single": [(0, [(n, 1)]) for n in (1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300)],
    "ragged_groups": [(160, [(n % 23 + 1, 1) for n in range(19)]), (0, [(700, 3)]), (320, [(n + 2, 2) for n in range(9)])],
    "long": [(4100, [(n + 1, 1) for n in range(5)])],
    "tiles": [(257, [(3, 3)] * 50), (130, [(2, 1)] * 33), (640, [(200, 150)])],
    "crowd": [(200, [(n % 7 + 1, 1) for n in range(70)])],
}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("heads,kv_heads,d", [(4, 4, 64), (4, 1, 128), (6, 2, 64), (2, 2, 128), (15, 3, 64), (17, 1, 64)])
@pytest.mark.parametrize("groups", GROUPS, ids=str)
@pytest.mark.parametrize("columns", [0, 30000], ids=["narrow_tables", "wide_tables"])
def test_against_the_definition(vb, columns, groups, heads, kv_heads, d, dtype):
    c = Case(vb, GROUPS[groups], heads, kv_heads, d, dtype=dtype, seed=len(groups), columns=columns)
    first = c.run()
    c.check(*first)
    again = c.run()                                                          # and once more: nothing is left over
    assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


@pytest.mark.parametrize("page", [8, 32, 64, 128, 256])
def test_page_sizes(vb, page):
    c = Case(vb, [(page * 3 + 5, [(1, 1), (page, 1), (page + 3, 2)]), (page, [(2, 2)] * 18)], 8, 2, 128, page=page, seed=page)
    c.check(*c.run())


@pytest.mark.parametrize("columns", [0, 30000], ids=["narrow_tables", "wide_tables"])
def test_layers_strides_and_no_lse(vb, columns):
    """A layer of several; q and out as slices of wider buffers (a fused projection's rows); lse left out."""
    c = Case(vb, [(50, [(3, 1), (4, 2)])], 4, 2, 64, layers=3, seed=2, columns=columns)
    wide = torch.full((c.rows, 3, c.heads, c.d), 3.0, dtype=c.dtype, device="cuda")
    wide[:, 1] = c.q
    for layer in (2, 0):
        out = torch.full((c.rows + 2, 2 * c.heads, c.d), 7.0, dtype=c.dtype, device="cuda")
        c.run(q=wide[:, 1], layer=layer, out=out[1:-1, :c.heads], lse=False)
        c.check(out[1:-1, :c.heads], None, layer)
        assert torch.all(out[0] == 7) and torch.all(out[-1] == 7) and torch.all(out[:, c.heads:] == 7)


@pytest.mark.parametrize("columns", [0, 30000], ids=["narrow_tables", "wide_tables"])
def test_refused_entries_leave_their_rows(vb, columns):
    """Slots and pages out of range: a code each, their rows untouched, the others right; rows behind the last untouched."""
    c = Case(vb, [(48, [(3, 1), (5, 2), (2, 1), (4, 1)])], seed=4, columns=columns)
    n, rows = 4, c.rows + 3
    q = torch.cat([c.q, c.q[:3]])
    plan = vb.PrefixPlan(c.pages, n, rows, c.heads)
    ptr = dev([0, 1, 3, 4, 5])
    keep_table = c.pages.table.clone()
    for kind, code in (("slot", -1), ("slot_low", -1), ("page", -2), ("page_low", -2), ("len", -2)):
        seqs = list(c.seqs)
        keep_len = c.pages.len.clone()
        if kind == "slot":
            seqs[1] = 10 ** 6
        elif kind == "slot_low":
            seqs[1] = -1
        elif kind == "page":
            c.pages.table[seqs[1], 1] = 10 ** 6
        elif kind == "page_low":
            c.pages.table[seqs[1], 3] = -7
        else:
            c.pages.len[seqs[1]] = 10 ** 7
        out, lse, st = torch.full((rows, c.heads, c.d), 5.0, dtype=c.dtype, device="cuda"), torch.full((rows, c.heads), 5.0, device="cuda"), c.st(n)
        vb.vlac_prefix_plan(c.pages, plan, dev(seqs), ptr, st)
        vb.vlac_prefix_attention(c.pages, 0, plan, q, c.scale, out, lse)
        assert st.tolist() == [0, code, 0, 0]
        assert torch.all(out[1:3] == 5) and torch.all(lse[1:3] == 5) and torch.all(out[5:] == 5) and torch.all(lse[5:] == 5)
        c.pages.table.copy_(keep_table)
        c.pages.len.copy_(keep_len)
        c.check(out, lse, only=(0, 2, 3))
    # pointers: one too large refuses its entry, one that falls refuses all (rows would overlap)
    for bad, want in (([0, 1, 3, 4, 99], [0, 0, 0, -1]), ([0, 3, 1, 4, 5], [-1] * 4), ([-1, 1, 3, 4, 5], [-1, 0, 0, 0])):
        out = torch.full((rows, c.heads, c.d), 5.0, dtype=c.dtype, device="cuda")
        vb.vlac_prefix_plan(c.pages, plan, dev(c.seqs), dev(bad), st)
        vb.vlac_prefix_attention(c.pages, 0, plan, q, c.scale, out)
        assert st.tolist() == want
        r0 = 0 if want[0] else 1
        assert (torch.all(out == 5) if min(want) == max(want) else torch.all(out[(4 if want[3] else 0):(99 if want[3] else 1)] == 5))


@pytest.mark.parametrize("columns", [0, 30000], ids=["narrow_tables", "wide_tables"])
def test_values_a_row_does_not_see_never_reach_it(vb, columns):
    """NaN and infinities in the K and V rows of later queries of the same chunk: earlier rows stay exact, the rows that see them do not."""
    for d, heads in ((64, 1), (128, 3)):
        c = Case(vb, [(40, [(12, 7), (9, 9)])], heads, 1, d, seed=d, columns=columns)
        clean, clean_lse = c.run()
        slot = c.seqs[0]
        n = int(c.pages.len[slot])
        at = lambda pos: (int(c.pages.table[slot, pos // 16]), pos % 16)
        for pos, what in ((n - 1, float("nan")), (n - 2, float("inf"))):
            pg, r = at(pos)
            c.pages.v[0, pg, r, 0, 5] = what
        pg, r = at(n - 1)
        c.pages.k[0, pg, r, 0, 3] = float("nan")
        out, lse = c.run()
        assert torch.equal(out[:5], clean[:5]) and torch.equal(lse[:6], clean_lse[:6])
        assert torch.equal(out[7:], clean[7:]) and torch.equal(lse[7:], clean_lse[7:])
        assert torch.all(torch.isposinf(out[5, :, 5])) and torch.equal(out[5, :, 6:], clean[5, :, 6:]) and torch.equal(out[5, :, :5], clean[5, :, :5])
        assert torch.all(torch.isnan(out[6])) and torch.all(torch.isnan(lse[6]))


@pytest.mark.parametrize("columns", [0, 30000], ids=["narrow_tables", "wide_tables"])
def test_extreme_scores(vb, columns):
    """Scores of some hundreds (one key takes all), and equal ones of zero."""
    for q_scale in (200.0, 0.0):
        c = Case(vb, [(70, [(5, 1), (3, 2), (66, 1)]), (0, [(90, 40)])], 4, 2, 64, seed=11, q_scale=q_scale, columns=columns)
        c.check(*c.run())


def test_more_work_than_warps(vb):
    """Runs of many units that cut tiles and span pieces: the same bits every time, one plan for several layers."""
    c = Case(vb, [(390, [(n % 5 + 1, 1) for n in range(3)])] + [(0, [(380 + n, 1)]) for n in range(60)], 32, 32, 64, layers=2, seed=14)
    plan = vb.PrefixPlan(c.pages, len(c.seqs), c.rows, c.heads)
    first = c.run(plan=plan)
    c.check(*first, only=(0, 2, 3, 40, 62))
    for layer in (1, 0, 1):
        out, lse = torch.zeros_like(first[0]), torch.zeros_like(first[1])
        vb.vlac_prefix_attention(c.pages, layer, plan, c.q, c.scale, out, lse)
        c.check(out, lse, layer, only=(1, 20, 62))
        assert layer == 1 or (torch.equal(out, first[0]) and torch.equal(lse, first[1]))


@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
def test_scales(vb, scale):
    """Any finite scale, negative ones and zero included, on narrow and wide segments."""
    c = Case(vb, [(300, [(5, 1), (3, 2), (66, 1)]), (400, [(9, 8)] * 12)], 4, 2, 128, seed=12, q_scale=0.5)
    c.scale = scale
    c.check(*c.run())


@pytest.mark.parametrize("prefix", [128, 129 * 8, 8 * 1000 + 8])
def test_wide_prefixes_in_small_and_large_pages(vb, prefix):
    """Common pages that end inside a block of keys, in pages smaller and larger than it; scattered pages."""
    for page in (8, 256):
        c = Case(vb, [(prefix, [(n + 1, 1) for n in range(20)])], 2, 1, 64 if page == 8 else 128, page=page, seed=prefix)
        c.check(*c.run(), only=(0, 7, 19))


def test_infinities_in_a_common_page(vb):
    """What every row sees reaches every row: an infinite V in the prefix gives infinite outputs in that column and no other."""
    c = Case(vb, [(200, [(n + 1, 1) for n in range(24)])], 4, 4, 64, seed=13)
    clean, clean_lse = c.run()
    pg = int(c.pages.table[c.seqs[0], 2])
    c.pages.v[0, pg, 3, 1, 7] = float("-inf")
    out, lse = c.run()
    assert torch.all(torch.isneginf(out[:, 1, 7])) and torch.equal(lse, clean_lse)
    out[:, 1, 7] = clean[:, 1, 7]
    assert torch.equal(out, clean)


@pytest.mark.parametrize("columns", [0, 30000], ids=["narrow_tables", "wide_tables"])
def test_same_slot_twice_and_any_order(vb, columns):
    """A slot may be listed twice, and the order of the list decides nothing but the division of the work."""
    c = Case(vb, [(96, [(3, 1), (20, 1), (1, 1)]), (64, [(2, 1), (9, 1)])], 8, 2, 64, seed=5, columns=columns)
    c.check(*c.run())
    order = [4, 0, 2, 1, 3, 0, 4]
    c.seqs, c.nq, c.q, c.rows = [c.seqs[i] for i in order], [1] * 7, c.q[order].contiguous(), 7
    c.check(*c.run())


@pytest.mark.parametrize("columns", [0, 30000], ids=["narrow_tables", "wide_tables"])
def test_repeatable_bits_and_plan_for_all_layers(vb, columns):
    """The same bits every time; one plan serves several layers and several calls."""
    c = Case(vb, [(500, [(n + 1, 1) for n in range(12)])], 8, 8, 128, layers=2, seed=6, columns=columns)
    plan = vb.PrefixPlan(c.pages, len(c.seqs), c.rows, c.heads)
    first = c.run(plan=plan)
    for layer in (1, 0, 1):
        out, lse = torch.zeros_like(first[0]), torch.zeros_like(first[1])
        vb.vlac_prefix_attention(c.pages, layer, plan, c.q, c.scale, out, lse)
        c.check(out, lse, layer)
        if layer == 0:
            assert torch.equal(out, first[0]) and torch.equal(lse, first[1])


@pytest.mark.parametrize("columns", [0, 30000], ids=["narrow_tables", "wide_tables"])
def test_two_graphs_on_two_streams(vb, columns):
    """Two captured token passes with plans of their own, replayed at the same time, and again after the sequences grew."""
    c = Case(vb, [(128, [(3, 1), (4, 1), (9, 1)])], 4, 4, 64, seed=7, spare=12, columns=columns + 4)
    ptr, streams, work = dev([0, 1, 2, 3]), [torch.cuda.Stream() for _ in range(2)], []
    seqs = dev(c.seqs)
    torch.cuda.synchronize()
    for s in streams:
        plan, out, st = vb.PrefixPlan(c.pages, 3, 3, 4), torch.zeros((3, 4, 64), dtype=c.dtype, device="cuda"), c.st(3)
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=s):
            vb.vlac_prefix_plan(c.pages, plan, seqs, ptr, st)
            vb.vlac_prefix_attention(c.pages, 0, plan, c.q, c.scale, out)
        work.append((g, plan, out, st))
    for grow in range(3):
        torch.cuda.synchronize()
        for _ in range(5):
            for s, (g, *_rest) in zip(streams, work):
                with torch.cuda.stream(s):
                    g.replay()
        torch.cuda.synchronize()
        for _, _, out, st in work:
            assert st.tolist() == [0, 0, 0]
            c.check(out, None)
        lens = [int(c.pages.len[s]) + 7 for s in c.seqs]
        c.resize(c.seqs, lens)
        for s, n in zip(c.seqs, lens):
            c.fill(s, n - 7, 7)


def test_far_pages(vb):
    """Element offsets beyond 2^31 in K and V: the last pages of a pool of 5 GB a side."""
    n_pages, page, kv, d = 10000, 256, 16, 64
    k = torch.zeros((1, n_pages, page, kv, d), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    assert k.numel() > 2 ** 31
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    ids = [n_pages - 1, 3, n_pages - 2, n_pages // 2]
    for i in ids:
        k[0, i].normal_(generator=g)
        v[0, i].normal_(generator=g)
    pages = vb.Pages(k, v, dev([ids, [ids[0], ids[2], -1, -1]]), dev([4 * 256 - 3, 300]), torch.zeros(n_pages, dtype=torch.int32, device="cuda"))
    q = (torch.empty((2, 32, d), device="cuda").normal_(generator=g) * 2).to(torch.bfloat16)
    plan, out, st = vb.PrefixPlan(pages, 2, 2, 32), torch.zeros_like(q), torch.zeros(2, dtype=torch.int32, device="cuda")
    vb.vlac_prefix_plan(pages, plan, dev([0, 1]), dev([0, 1, 2]), st)
    vb.vlac_prefix_attention(pages, 0, plan, q, 0.125, out)
    assert st.tolist() == [0, 0]
    for i, n in ((0, 4 * 256 - 3), (1, 300)):
        t = pages.table[i, :-(-n // page)].long()
        kh, vh = (x[0, t].reshape(-1, kv, d)[:n].double().cpu().numpy() for x in (k, v))
        o, _, eo, _ = ref.attention(kh, vh, q[i:i + 1].double().cpu().numpy(), n, 1, 2, 0.125, HALF[torch.bfloat16])
        assert np.all(np.abs(out[i:i + 1].double().cpu().numpy() - o) <= eo)


def test_far_pages_of_the_last_layer(vb):
    """The same offsets through writes, forks, copies and a wide segment: only the last pages of a two-layer pool are free."""
    n_pages, page, kv, d, L = 5000, 256, 16, 64, 2
    pages = vb.Pages.empty(L, n_pages, page, kv, d, 24, 6)
    assert pages.k.numel() > 2 ** 31
    free = 32
    pages.refs[:n_pages - free] = 1
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    st1, n = torch.zeros(1, dtype=torch.int32, device="cuda"), 1000
    vb.vlac_pages_resize(pages, dev([0]), dev([n]), st1)
    rows = [torch.empty((n, kv, d), device="cuda").normal_(generator=g).to(torch.bfloat16) for _ in range(2)]
    vb.vlac_pages_write(pages, 1, dev([0]), dev([0]), dev([0, n]), *rows, st1)
    assert st1.item() == 0 and int(pages.table[0, 0]) == n_pages - free
    vb.vlac_pages_fork(pages, dev([0]), dev([1]), True, st1)
    kids = dev(range(2, 22))
    st = torch.zeros(20, dtype=torch.int32, device="cuda")
    vb.vlac_pages_fork(pages, dev([1] * 20), kids, False, st)
    assert st.tolist() == [0] * 20 and int(pages.refs[n_pages - 1]) in (0, 1)
    t = pages.table[1, :4].long()
    assert torch.equal(pages.k[1, t].reshape(-1, kv, d)[:n], rows[0]) and torch.equal(pages.v[1, t].reshape(-1, kv, d)[:n], rows[1])
    q = (torch.empty((20, 32, d), device="cuda").normal_(generator=g) * 2).to(torch.bfloat16)
    plan, out = vb.PrefixPlan(pages, 20, 20, 32), torch.zeros_like(q)
    vb.vlac_prefix_plan(pages, plan, kids, dev(range(21)), st)
    vb.vlac_prefix_attention(pages, 1, plan, q, 0.125, out)
    assert st.tolist() == [0] * 20 and vb.vlac_prefix_error(plan) == 0
    kh, vh = (x.double().cpu().numpy() for x in rows)
    for i in (0, 19):
        o, _, eo, _ = ref.attention(kh, vh, q[i:i + 1].double().cpu().numpy(), n, 1, 2, 0.125, HALF[torch.bfloat16])
        assert np.all(np.abs(out[i:i + 1].double().cpu().numpy() - o) <= eo)


def test_candidates_of_a_control_step(vb):
    """The whole use: a control step's prompt becomes a prefix, candidates are forked from it, grow token by token, attend in
    every layer, are pruned and given back."""
    cfg = synth.tiny_config()
    model = synth.make_model(cfg, 1)
    devm = vb.DeviceModel(model)
    ctx = vb.vlac_create(vb.make_config(cfg, 1), devm.weights)
    cache = vb.vlac_cache_alloc(ctx, 1)
    try:
        rng = np.random.default_rng(1)
        feats = vb.upload_bf16(synth.f32_to_bf16(rng.standard_normal((1, cfg.n_vision, cfg.hidden), dtype=np.float32)))
        frames = torch.from_numpy(synth.rerandomised_pair(cfg, 1, 13)[0][None]).to("cuda").contiguous()
        ids = torch.from_numpy(synth.make_prompt_ids(cfg, 1)).to("cuda")
        tokens = torch.zeros((1, cfg.n_action), dtype=torch.int32, device="cuda")
        vb.vlac_step(ctx, cache, frames, feats, ids, vb.make_params()[0], False, tokens)
        n, L, H, d = 6, cfg.seq_len, cfg.n_heads, cfg.head_dim
        pages = vb.Pages.empty(cfg.n_layers, 40, 16, H, d, n + 1, 8)
        st1, st = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
        root, kids = dev([0]), dev(np.arange(1, n + 1))
        vb.vlac_pages_resize(pages, root, dev([L]), st1)
        vb.vlac_pages_from_cache(pages, cache, 0, 0, L, st1)
        vb.vlac_pages_fork(pages, dev([0] * n), kids, False, st)
        assert int(pages.refs.max()) == n + 1
        plan, ptr = vb.PrefixPlan(pages, n, n, H), dev(np.arange(n + 1))
        rows = {}
        for t in range(4):
            vb.vlac_pages_resize(pages, kids, dev([L + t + 1] * n), st)
            vb.vlac_prefix_plan(pages, plan, kids, ptr, st)
            assert st.tolist() == [0] * n
            for l in range(cfg.n_layers):
                q, k, v = (torch.randn((n, H, d), device="cuda").to(torch.bfloat16) for _ in range(3))
                rows[t, l] = (k, v)
                out = torch.zeros_like(q)
                vb.vlac_pages_write(pages, l, kids, None, ptr, k, v, st)
                vb.vlac_prefix_attention(pages, l, plan, q, d ** -0.5, out)
                kc, vc = (torch.empty((cfg.max_seq, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
                vb.vlac_cache_read(cache, vb.PART_K, 0, l, kc)
                vb.vlac_cache_read(cache, vb.PART_V, 0, l, vc)
                for i in range(n):
                    kk = torch.cat([kc[:L]] + [rows[x, l][0][i:i + 1] for x in range(t + 1)]).double().cpu().numpy()
                    vv = torch.cat([vc[:L]] + [rows[x, l][1][i:i + 1] for x in range(t + 1)]).double().cpu().numpy()
                    o, _, eo, _ = ref.attention(kk, vv, q[i:i + 1].double().cpu().numpy(), L + t + 1, 1, 1, d ** -0.5, HALF[torch.bfloat16])
                    assert np.all(np.abs(out[i:i + 1].double().cpu().numpy() - o) <= eo), (t, l, i)
        # prune vision tokens of one candidate, attend again, then give everything back
        keep = np.concatenate([[0], np.arange(1, 65, 2), np.arange(65, L + 4)])
        vb.vlac_pages_compact(pages, dev([2]), dev([2]), dev([0, len(keep)]), dev(keep), st1)
        assert st1.item() == 0 and int(pages.len[2]) == len(keep)
        plan1, q, out = vb.PrefixPlan(pages, 1, 1, H), torch.randn((1, H, d), device="cuda").to(torch.bfloat16), torch.zeros((1, H, d), dtype=torch.bfloat16, device="cuda")
        vb.vlac_prefix_plan(pages, plan1, dev([2]), dev([0, 1]), st1)
        vb.vlac_prefix_attention(pages, 1, plan1, q, d ** -0.5, out)
        kk = torch.cat([kc[:L]] + [rows[x, 1][0][1:2] for x in range(4)])[keep].double().cpu().numpy()
        vv = torch.cat([vc[:L]] + [rows[x, 1][1][1:2] for x in range(4)])[keep].double().cpu().numpy()
        o, _, eo, _ = ref.attention(kk, vv, q.double().cpu().numpy(), len(keep), 1, 1, d ** -0.5, HALF[torch.bfloat16])
        assert np.all(np.abs(out.double().cpu().numpy() - o) <= eo)
        vb.vlac_pages_free(pages, dev(np.arange(n + 1)), torch.zeros(n + 1, dtype=torch.int32, device="cuda"))
        assert int(pages.refs.abs().max()) == 0 and int(pages.len.max()) == 0 and int(pages.table.max()) == -1
    finally:
        vb.vlac_cache_free(cache)
        vb.vlac_destroy(ctx)


def test_without_a_plan_nothing_is_computed(vb):
    c = Case(vb, [(400, [(n + 1, 1) for n in range(20)])], 4, 4, 64, seed=15)
    plan, out = vb.PrefixPlan(c.pages, 20, 20, 4), torch.full_like(c.q, 5.0)
    vb.vlac_prefix_attention(c.pages, 0, plan, c.q, c.scale, out)
    assert torch.all(out == 5.0) and vb.vlac_prefix_error(plan) == 0
    vb.vlac_prefix_attention(c.pages, 0, vb.PrefixPlan(c.pages, 0, 0, 4), c.q[:0], c.scale, out[:0])
    vb.vlac_prefix_plan(c.pages, vb.PrefixPlan(c.pages, 2, 0, 4), dev(c.seqs[:2]), dev([0, 0, 0]), c.st(2))


@pytest.mark.parametrize("heads,kv_heads", [(64, 1), (24, 1), (128, 1), (192, 1), (66, 33), (64, 64)])
def test_many_heads_a_group_and_many_groups(vb, heads, kv_heads):
    """Query heads per K/V head that divide a tile, do not, and are more than one; K/V heads that are no power of two."""
    c = Case(vb, [(270, [(3, 2), (1, 1), (40, 3)]), (0, [(70, 1)])], heads, kv_heads, 64, seed=heads)
    c.check(*c.run())


def test_wrong_tensors_are_refused(vb):
    c = Case(vb, [(16, [(2, 1), (3, 1)])])
    plan, st, ptr, out = vb.PrefixPlan(c.pages, 2, 2, 4), c.st(2), dev([0, 1, 2]), torch.zeros_like(c.q)
    seqs = dev(c.seqs)
    with pytest.raises(AssertionError):
        vb.vlac_prefix_plan(c.pages, plan, seqs.long(), ptr, st)
    with pytest.raises(AssertionError):
        vb.vlac_prefix_plan(c.pages, plan, seqs[:1], ptr, st)
    vb.vlac_prefix_plan(c.pages, plan, seqs, ptr, st)
    for q in (c.q.float(), c.q[:1], c.q[:, :2], c.q.half(), c.q.cpu(), c.q.transpose(1, 2)):
        with pytest.raises(AssertionError):
            vb.vlac_prefix_attention(c.pages, 0, plan, q, 1.0, out)
    with pytest.raises(AssertionError):
        vb.vlac_prefix_attention(c.pages, 0, plan, c.q, 1.0, out, torch.zeros((2, 3), device="cuda"))
    with pytest.raises(vb.VlacError):
        vb.vlac_prefix_attention(c.pages, 1, plan, c.q, 1.0, out)
    with pytest.raises(vb.VlacError):
        vb.PrefixPlan(vb.Pages.empty(1, 4, 16, 3, 64, 2, 2), 2, 2, 4)


def test_a_plan_of_another_pool_is_refused(vb):
    """A plan's slots and page counts are those of its pool's tables."""
    c, other = Case(vb, [(16, [(2, 1), (3, 1)])]), Case(vb, [(16, [(2, 1), (3, 1)])])
    plan, st, ptr, out = vb.PrefixPlan(other.pages, 2, 2, 4), c.st(2), dev([0, 1, 2]), torch.zeros_like(c.q)
    with pytest.raises(AssertionError):
        vb.vlac_prefix_plan(c.pages, plan, dev(c.seqs), ptr, st)
    with pytest.raises(AssertionError):
        vb.vlac_prefix_attention(c.pages, 0, plan, c.q, 1.0, out)


@pytest.mark.parametrize("n", [17, 200, 1024])
def test_findings_of_every_cta_reach_the_plan(vb, n):
    """Many sequences of two pages in wide tables, none with a neighbour's pages, some with a page out of range: hardly anything to read, so
    the plan's CTAs report to the first as early as they can.  A sequence that joined its neighbour would see the neighbour's first page."""
    page, d, heads = 8, 64, 2
    pages = vb.Pages.empty(1, n + 1, page, heads, d, n, 5000)
    pages.v[0] = (torch.arange(n + 1, device="cuda") % 251).to(torch.bfloat16)[:, None, None, None]        # (whole numbers up to 256 are exact)
    order = torch.randperm(n, generator=torch.Generator().manual_seed(n)).to(torch.int32)
    bad = torch.arange(n) % 7 == 3
    pages.table[:, :2] = torch.where(bad, n + 1, order).cuda()[:, None]                                     # one page, twice
    pages.len.fill_(2 * page)
    q = torch.ones((n, heads, d), dtype=torch.bfloat16, device="cuda")
    plan, seqs, ptr, st = vb.PrefixPlan(pages, n, n, heads), dev(np.arange(n)), dev(np.arange(n + 1)), torch.full((n,), 9, dtype=torch.int32, device="cuda")
    want = torch.where(bad, 5, order % 251).to(torch.bfloat16).cuda()[:, None, None].expand(n, heads, d)    # (scores of zero: weights of one)
    codes = torch.where(bad, -2, 0).cuda()
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(200):
        out = torch.full_like(q, 5.0)
        vb.vlac_prefix_plan(pages, plan, seqs, ptr, st)
        vb.vlac_prefix_attention(pages, 0, plan, q, 0.125, out)
        wrong += (out != want).sum() + (st != codes).sum()
    assert wrong.item() == 0 and vb.vlac_prefix_error(plan) == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("gap", [10.0, 14.0, 16.0, 17.4, 19.0])
@pytest.mark.parametrize("kv_heads,n,members", [(1024, 4096, 12), (160, 16384, 20)], ids=["narrow", "wide"])
def test_many_keys_far_behind_one(vb, kv_heads, n, members, gap, dtype):
    """One key takes nearly all of the sum, and thousands of equal ones make the whole output (its V row is zero): weights far below the largest
    are not lost to the range of fp16.  So many heads that a piece holds most of a head's keys; the one lies early in some, late in others.
    Bound: that of the definition, and below fp16's normal numbers half a step of them (2^-25): for the output, and for every weight, in units of the
    largest (2^14 narrow, at least 2^9 wide)."""
    c = Case(vb, [(n, [(1, 1)] * members)], kv_heads, kv_heads, 64, page=64, dtype=dtype, seed=int(gap), fill=0.0)
    p, t = c.pages, c.pages.table[c.seqs[0], :-(-n // c.page)].long()
    p.k.zero_()
    p.v[0].uniform_(0.5, 1.0, generator=c.gen)
    heads = torch.arange(kv_heads, device="cuda")
    at = (heads * 37) % n                                                     # position of the head's one key
    p.k[0, t[at // c.page], at % c.page, heads, 0] = gap / 2
    p.v[0, t[at // c.page], at % c.page, heads] = 0
    c.q.zero_()
    c.q[:, :, 0] = 16.0                                                       # times the scale of 1/8: the gap
    out, lse = c.run()
    some = [0, 1, kv_heads // 3, kv_heads - 1]
    t = torch.cat([t, c.pages.table[c.seqs[-1], n // c.page:n // c.page + 1].long()])
    k, v = (x[0, t][:, :, some].reshape(-1, 4, 64)[:n + 1].double().cpu().numpy() for x in (p.k, p.v))
    o, l, eo, el = ref.attention(k, v, c.q[-1:, some].double().cpu().numpy(), n + 1, 1, 1, c.scale, HALF[dtype])
    if dtype is torch.float16:
        eo = eo + 2.0 ** -25 + n * 2.0 ** -25 * 2.0 ** (-14 if members <= 16 else -9)
    assert np.all(o > 3 * eo)                                                 # (the bound tells a lost sum from a kept one)
    assert np.all(np.abs(out[-1:, some].double().cpu().numpy() - o) <= eo)
    assert np.all(np.abs(lse[-1:, some].double().cpu().numpy() - l) <= el)


@pytest.mark.parametrize("members", [2, 20], ids=["narrow", "wide"])
def test_a_plan_for_something_else_computes_nothing(vb, members):
    """Through the C interface: a plan's memory used with another pool, or with other numbers of sequences, rows or heads, leaves the output as it
    was and says so; its own pool's calls are right before and behind."""
    c = Case(vb, [(400, [(n + 1, 1) for n in range(members)])], 4, 4, 64, seed=16)
    first = c.run(plan=(plan := vb.PrefixPlan(c.pages, members, c.rows, 4)))
    c.check(*first)
    p = c.pages
    others = [vb.Pages.empty(1, 4, 16, 4, 64, 3, 2), vb.Pages(p.k, p.v, p.table.clone(), p.len, p.refs),
              vb.Pages(p.k, p.v, p.table[:, :30].contiguous(), p.len, p.refs), vb.Pages(p.k[:, :5].contiguous(), p.v[:, :5].contiguous(), p.table, p.len, p.refs[:5])]
    out, q = torch.full((64, 4, 64), 5.0, dtype=c.dtype, device="cuda"), torch.zeros((64, 4, 64), dtype=c.dtype, device="cuda")
    big = torch.zeros((1 << 24,), dtype=torch.uint8, device="cuda")      # room for every form of the struct
    big[:plan.mem.numel()] = plan.mem
    st, seqs, ptr = c.st(members), dev(c.seqs), dev(np.concatenate([[0], np.cumsum(c.nq)]))

    def call(pool, n=members, rows=c.rows, heads=4):
        x = vb.vlac_prefix(n, rows, heads, big.data_ptr(), big.numel())
        rc = vb.lib.vlac_prefix_attention(pool.ref, 0, vb.C.byref(x), q.data_ptr(), heads * 64, 0.125, out.data_ptr(), heads * 64, None, torch.cuda.current_stream().cuda_stream)
        return rc, vb.lib.vlac_prefix_error(vb.C.byref(x), torch.cuda.current_stream().cuda_stream)

    mine = vb.vlac_prefix(members, c.rows, 4, big.data_ptr(), big.numel())
    for pool, other in [(o, {}) for o in others] + [(p, dict(n=members + 1)), (p, dict(n=members - 1)), (p, dict(rows=c.rows + 1)), (p, dict(heads=8))]:
        vb.lib.vlac_prefix_plan(p.ref, vb.C.byref(mine), seqs.data_ptr(), ptr.data_ptr(), st.data_ptr(), torch.cuda.current_stream().cuda_stream)
        assert vb.lib.vlac_prefix_error(vb.C.byref(mine), torch.cuda.current_stream().cuda_stream) == 0
        assert call(pool, **other) == (0, -1)
        assert torch.all(out == 5.0)
    vb.lib.vlac_prefix_plan(p.ref, vb.C.byref(mine), seqs.data_ptr(), ptr.data_ptr(), st.data_ptr(), torch.cuda.current_stream().cuda_stream)
    q[:c.rows] = c.q
    assert call(p) == (0, 0) and torch.equal(out[:c.rows], first[0]) and torch.all(out[c.rows:] == 5.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("heads,kv_heads,d", [(4, 4, 128), (4, 4, 64), (6, 2, 64), (8, 1, 128)])
@pytest.mark.parametrize("members", [20, 150])
def test_loads_that_come_late(vb, members, heads, kv_heads, d, dtype):
    """Common pages that arrive a millisecond late: every wait takes its slow path, and the bits are the same."""
    c = Case(vb, [(1500, [(2, 1)] * members)], heads, kv_heads, d, dtype=dtype, seed=17)
    plan = vb.PrefixPlan(c.pages, members, c.rows, heads)
    first = c.run(plan=plan)
    c.check(*first, only=(0, members - 1))
    out, lse = torch.zeros_like(first[0]), torch.zeros_like(first[1])
    vb.vlac_selftest_prefix_wait(c.pages, 0, plan, c.q, c.scale, out, lse, 1000, 100000)
    assert vb.vlac_prefix_error(plan) == 0
    assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    for delay, limit in ((100001, 10), (0, 0), (0, 100001)):
        with pytest.raises(vb.VlacError):
            vb.vlac_selftest_prefix_wait(c.pages, 0, plan, c.q, c.scale, out, lse, delay, limit)


@pytest.mark.parametrize("heads,kv_heads,d,dtype", [(4, 4, 128, torch.bfloat16), (4, 4, 64, torch.float16), (6, 2, 64, torch.bfloat16), (8, 1, 128, torch.float16)])
@pytest.mark.parametrize("prefix,members", [(64, 20), (1500, 20), (3000, 150)])
def test_waits_that_give_up(vb, prefix, members, heads, kv_heads, d, dtype):
    """Loads that begin behind the waits' limit: the call ends, the plan says so, and the next plan and call are right (products, copies and
    tensor memory of the one that gave up are done with).  With few and many tiles for the ring, Q by TMA and by hand."""
    c = Case(vb, [(prefix, [(2, 1)] * members)], heads, kv_heads, d, dtype=dtype, seed=18)
    plan = vb.PrefixPlan(c.pages, members, c.rows, heads)
    first = c.run(plan=plan)
    c.check(*first, only=(0, members - 1))
    out, lse = torch.zeros_like(first[0]), torch.zeros_like(first[1])
    vb.vlac_selftest_prefix_wait(c.pages, 0, plan, c.q, c.scale, out, lse, 5000, 500)
    assert vb.vlac_prefix_error(plan) == -5
    vb.vlac_prefix_attention(c.pages, 0, plan, c.q, c.scale, out, lse)
    assert vb.vlac_prefix_error(plan) == -5                              # until the next plan
    assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    for _ in range(3):
        again = c.run(plan=plan)                                         # (asserts that the error is gone)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


def test_a_plan_without_rows_judges_its_entries(vb):
    """No query rows at all: slots, lengths and pointers are looked at as ever; what a plan with rows says of the same entries without rows."""
    c = Case(vb, [(16, [(2, 1), (3, 1), (4, 1)])])
    c.pages.len[c.seqs[2]] = 10 ** 7
    seqs = dev([c.seqs[0], -1, c.seqs[2], 10 ** 6, c.seqs[1]])
    for rows, plan in ((0, vb.PrefixPlan(c.pages, 5, 0, 4)), (1, vb.PrefixPlan(c.pages, 5, 1, 4))):
        for ptr, want in (([0, 0, 0, 0, 0, 0], [0, -1, -2, -1, 0]), ([0, 0, 0, 0, 0, 9], [0, -1, -2, -1, -1]), ([-1, 0, 0, 0, 0, 0], [-1, -1, -2, -1, 0]),
                          ([0, -1, 0, 0, 0, 0], [-1] * 5)):
            st = c.st(5)
            vb.vlac_prefix_plan(c.pages, plan, seqs, dev(ptr), st)
            assert st.tolist() == want, (rows, ptr)


def test_queries_and_results_in_one_buffer(vb):
    """Rows of q and of out side by side, interleaved or with strides of their own in one buffer are right; where any two share an element the call
    is refused and nothing is written."""
    c = Case(vb, [(20, [(n + 1, 1) for n in range(5)])], 1, 1, 64, seed=19)
    plan = vb.PrefixPlan(c.pages, 5, 5, 1)
    first, _ = c.run(plan=plan)
    rng, seen = np.random.default_rng(20), set()
    for _ in range(400):
        qs, os = (int(x) * 8 for x in rng.choice([8, 9, 16, 17, 24, 40], 2))
        if rng.random() < 0.5:
            os = qs
        at_q, at_o = (int(x) * 8 for x in rng.integers(0, 100, 2))
        buf = torch.full((2600,), 7.0, dtype=c.dtype, device="cuda")
        q, out = (torch.as_strided(buf, (5, 1, 64), (s, 64, 1), at) for s, at in ((qs, at_q), (os, at_o)))
        q.copy_(c.q)
        used_q, used_o = (np.concatenate([np.arange(64) + at + r * s for r in range(5)]) for s, at in ((qs, at_q), (os, at_o)))
        shared = len(np.intersect1d(used_q, used_o)) > 0
        before, want = buf.clone(), buf.clone()
        seen.add((shared, qs == os))
        if shared:
            with pytest.raises(vb.VlacError) as e:
                vb.vlac_prefix_attention(c.pages, 0, plan, q, c.scale, out)
            assert e.value.status == -1
        else:
            torch.as_strided(want, (5, 1, 64), (os, 64, 1), at_o).copy_(first)
            vb.vlac_prefix_attention(c.pages, 0, plan, q, c.scale, out)
        assert torch.equal(buf, before if shared else want), (qs, os, at_q, at_o)
    assert len(seen) == 4
