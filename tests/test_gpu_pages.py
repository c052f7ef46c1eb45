"""The paged-pool calls on the GPU against the host mirror: tables, lengths, reference counts, codes and rows, bit for bit."""
import numpy as np
import pytest
import torch

import pages_reference as ref
from paper_2502_02175_b200 import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vb():
    from paper_2502_02175_b200 import binding
    return binding


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to("cuda")


class Pair:
    """The same pool on the device and as a host mirror."""

    def __init__(self, vb, seed, layers=2, n_pages=60, page=16, heads=2, d=64, slots=9, max_pages=7, dtype=torch.bfloat16, cap=None):
        self.cap = cap or max_pages * page                               # lengths that are drawn
        self.vb, self.rng = vb, np.random.default_rng(seed)
        self.pages = vb.Pages.empty(layers, n_pages, page, heads, d, slots, max_pages, dtype)
        for t in (self.pages.k, self.pages.v):
            t.view(torch.int16).copy_(torch.from_numpy(self.rng.integers(-32768, 32768, tuple(t.shape)).astype(np.int16)))
        self.host = ref.HostPool(self.bits(self.pages.k), self.bits(self.pages.v), *(t.cpu().numpy() for t in (self.pages.table, self.pages.len, self.pages.refs)))

    @staticmethod
    def bits(t):
        return t.view(torch.int16).cpu().numpy()

    def same(self, status, want):
        assert status.tolist() == want
        h, p = self.host, self.pages
        assert np.array_equal(p.len.cpu().numpy(), h.len)
        assert np.array_equal(p.table.cpu().numpy(), h.table)
        assert np.array_equal(p.refs.cpu().numpy(), h.refs)
        assert np.array_equal(self.bits(p.k).reshape(h.k.shape), h.k)
        assert np.array_equal(self.bits(p.v).reshape(h.v.shape), h.v)

    def status(self, n):
        return torch.full((n,), 77, dtype=torch.int32, device="cuda")

    def resize(self, seqs, lens, check=True):
        st = self.status(len(seqs))
        self.vb.vlac_pages_resize(self.pages, dev(seqs), dev(lens), st)
        want = self.host.resize(list(seqs), list(lens))
        if check:
            self.same(st, want)
        return want

    def free(self, seqs):
        st = self.status(len(seqs))
        self.vb.vlac_pages_free(self.pages, dev(seqs), st)
        self.same(st, self.host.resize(list(seqs), [0] * len(seqs)))

    def fork(self, src, dst, deep):
        st = self.status(len(src))
        self.vb.vlac_pages_fork(self.pages, dev(src), dev(dst), deep, st)
        want = self.host.fork(list(src), list(dst), deep)
        self.same(st, want)
        return want

    def compact(self, src, dst, keeps):
        st = self.status(len(src))
        ptr = np.concatenate([[0], np.cumsum([len(x) for x in keeps])])
        self.vb.vlac_pages_compact(self.pages, dev(src), dev(dst), dev(ptr), dev([y for x in keeps for y in x]), st)
        want = self.host.compact(list(src), list(dst), keeps)
        self.same(st, want)
        return want

    def write(self, layer, seqs, start, counts, stride=None):
        n, w = int(sum(counts)), self.host.k.shape[-1]
        s = self.pages.struct
        ptr = np.concatenate([[0], np.cumsum(counts)])
        rows = []
        for _ in range(2):
            x = torch.from_numpy(self.rng.integers(-32768, 32768, (n, stride or w)).astype(np.int16)).to("cuda").view(self.pages.dtype)
            rows.append(x[:, :w].view(n, s.n_kv_heads, s.head_dim) if n else torch.empty((0, s.n_kv_heads, s.head_dim), dtype=self.pages.dtype, device="cuda"))
        st = self.status(len(seqs))
        self.vb.vlac_pages_write(self.pages, layer, dev(seqs), None if start is None else dev(start), dev(ptr), rows[0], rows[1], st)
        host = [self.bits(x.contiguous()).reshape(n, w) for x in rows]
        want = self.host.write(layer, list(seqs), start, ptr.tolist(), host[0], host[1])
        self.same(st, want)
        return want


SHAPES = [dict(), dict(page=8, n_pages=37, max_pages=11, d=128, heads=1), dict(page=32, n_pages=19, max_pages=4, layers=3, dtype=torch.float16),
          dict(page=256, n_pages=11, max_pages=2, layers=1, heads=3), dict(page=64, n_pages=5, max_pages=2, slots=5),
          dict(max_pages=9000, cap=112)]              # tables too long for one CTA


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("seed", range(3))
def test_random_calls(vb, shape, seed):
    """Whatever the order of calls -- pages running out, repeated and foreign slots, positions out of order, lengths out of range -- the
    device holds what the mirror holds after each."""
    p = Pair(vb, seed, **shape)
    rng, slots, cap = p.rng, len(p.host.len), p.cap
    codes = set()
    for i in range(40):
        n = int(rng.integers(1, 5))
        op = rng.choice(["resize", "fork", "compact", "write", "free"], p=[0.3, 0.25, 0.25, 0.15, 0.05])
        pick = lambda: [int(x) for x in rng.integers(-1 if rng.random() < 0.1 else 0, slots + (rng.random() < 0.1), n)]
        a = pick()
        b = [int(x) for x in rng.permutation(slots)[:n]] if n <= slots else pick()
        if op == "resize":
            codes.update(p.resize(a if rng.random() < 0.3 else b, [int(x) for x in rng.integers(-1 if rng.random() < 0.1 else 0, cap + 2, n)]))
        elif op == "fork":
            codes.update(p.fork(a, b, bool(rng.integers(2))))
        elif op == "compact":
            keeps = []
            for s in a:
                have = int(p.host.len[s]) if 0 <= s < slots else 5
                kind = rng.random()
                keep = sorted(rng.choice(have, rng.integers(0, have + 1), replace=False).tolist()) if kind < 0.7 else list(range(rng.integers(0, have + 1)))
                if kind > 0.95:
                    keep = keep[::-1] + [0, 0]
                keeps.append(keep)
            dst = [s if rng.random() < 0.4 else d for s, d in zip(a, b)]
            codes.update(p.compact(a, dst, keeps))
        elif op == "write":
            counts = [int(x) for x in rng.integers(0, 40, n)]
            start = None if rng.random() < 0.5 else [int(x) for x in rng.integers(-1 if rng.random() < 0.1 else 0, cap, n)]
            codes.update(p.write(int(rng.integers(p.pages.k.shape[0])), b, start, counts, None if rng.random() < 0.5 else p.host.k.shape[-1] + 24))
        else:
            p.free(b)
    assert ref.OK in codes and ref.INVALID in codes


def test_lists_of_the_largest_size(vb):
    """1024 entries: taken, forked, pruned and given back in one call each; an entry too many is refused on the host."""
    p = Pair(vb, 5, layers=1, n_pages=2600, page=8, heads=1, slots=2048, max_pages=3)
    lens = p.rng.integers(0, 17, 1024).tolist()
    assert p.resize(list(range(1024)), lens) == [0] * 1024
    assert set(p.fork(list(range(1024)), list(range(2047, 1023, -1)), False)) == {0}
    p.compact(list(range(1024)), list(range(1024)), [list(range(n // 2, n)) for n in lens])
    p.free(list(range(1024, 2048)))
    with pytest.raises(vb.VlacError) as e:
        vb.vlac_pages_free(p.pages, dev(np.arange(1025)), p.status(1025))
    assert e.value.status == -6
    vb.vlac_pages_free(p.pages, dev([]), p.status(0))


@pytest.mark.parametrize("n_pages", [1, 3, 4096 * 8 + 5, 100003])
def test_pools_of_any_size_hand_out_the_lowest_pages(vb, n_pages):
    """Free pages scattered over small and large pools (numbers beyond what one CTA's scan holds at once)."""
    p = Pair(vb, 6, layers=1, n_pages=n_pages, page=8, heads=1, slots=6, max_pages=max(1, n_pages // 3))
    taken = p.rng.random(n_pages) < 0.5
    p.host.refs[taken] = 1
    p.pages.refs.copy_(dev(p.host.refs))
    mp = p.host.max_pages
    p.resize([4, 1, 3], [mp * 8 // 2 + 1, 8 * mp, min(5, 8 * mp)])
    p.resize([1, 0, 4], [8 * mp // 3, 8 * mp, 0])
    p.resize([2, 5], [8 * mp, 1])


def test_running_out_refuses_in_order(vb):
    p = Pair(vb, 7, n_pages=10, slots=6)
    assert p.resize([0, 1, 2, 3], [16 * 4, 16 * 7, 5, 0]) == [0, -3, -3, 0]
    assert p.resize([1, 2], [16 * 2, 5]) == [0, 0]
    assert p.fork([0, 1], [4, 5], True) == [-3, -3]                      # 3 pages left; the second would fit, but comes behind
    assert p.fork([0, 1], [4, 5], False) == [0, 0]                      # shared: no page needed
    assert p.compact([0], [0], [list(range(1, 64))]) == [-3]             # in place: unchanged
    assert p.compact([1], [1], [list(range(1, 32))]) == [0]


def test_cut_inside_a_shared_page_is_refused(vb):
    p = Pair(vb, 8)
    p.resize([0], [40])
    p.fork([0], [1], False)
    assert p.resize([0, 1], [20, 40]) == [-2, 0]
    assert p.resize([0, 1], [16, 24]) == [0, -2]                        # at a page's end it stays whole; refs count as the call found them
    assert p.compact([1], [1], [list(range(20))]) == [0]                 # this way its rows get a page of their own
    assert p.write(0, [1], [16], [4]) == [0]
    assert p.write(0, [1], [15], [2]) == [-2]                            # page 0 is still slot 0's too


def test_bad_tables_are_refused_and_never_followed(vb):
    """Page numbers and lengths out of range in the tables themselves: a code, and no other slot changes."""
    p = Pair(vb, 9)
    p.resize([0, 1, 2], [40, 40, 40])
    for t, x in (("table", 1000), ("table", -1), ("table", -2 ** 31), ("table", 2 ** 31 - 1), ("len", -1), ("len", 10 ** 6)):
        old_table, old_len = p.host.table.copy(), p.host.len.copy()
        if t == "table":
            p.host.table[1, 1] = x
        else:
            p.host.len[1] = x
        p.pages.table.copy_(dev(p.host.table))
        p.pages.len.copy_(dev(p.host.len))
        assert p.fork([1, 0], [3, 4], False) == [-2, 0]
        assert p.fork([0, 2], [1, 5], True)[0] == -2
        if p.host.len[1] > 0 and p.host.len[1] < 1000:
            assert p.compact([1, 2], [1, 2], [list(range(30)), list(range(2, 30))])[0] == -2
            p.host.compact([2], [2], [list(range(28))])
            vb.vlac_pages_compact(p.pages, dev([2]), dev([2]), dev([0, 28]), dev(range(28)), p.status(1))
            assert p.write(1, [1, 0], [10, 36], [20, 4])[0] == -2
        assert p.resize([1], [3]) == [-2]
        p.host.table[1], p.host.len[1] = old_table[1], old_len[1]
        p.pages.table.copy_(dev(p.host.table))
        p.pages.len.copy_(dev(p.host.len))
        p.free([3, 4, 5])
        p.resize([2], [40])


def test_keep_and_row_pointers_out_of_range(vb):
    p = Pair(vb, 10)
    p.resize([0, 1, 2], [40, 40, 40])
    st = p.status(3)
    vb.vlac_pages_compact(p.pages, dev([0, 1, 2]), dev([3, 4, 5]), dev([0, 50, 2, 2]), dev([1, 2]), st)
    assert st.tolist() == [-1, -1, 0]
    p.host.compact([2], [5], [[]])
    p.same(torch.zeros(0), [])
    x = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    vb.vlac_pages_write(p.pages, 0, dev([0, 1, 2]), None, dev([0, 3, 2, 2]), x, x, st)
    assert st.tolist() == [-1, -1, 0]
    vb.vlac_pages_write(p.pages, 0, dev([0, 1, 2]), None, dev([-1, 0, 0, 9]), x, x, st)
    assert st.tolist() == [-1, 0, -1]
    p.same(torch.zeros(0), [])


def test_captured_and_replayed_on_another_stream(vb):
    """Fork and append captured once: the replay does the same on whatever the tables hold then."""
    p = Pair(vb, 11)
    p.resize([0], [35])
    src, dst, ptr = dev([0, 0, 0]), dev([1, 2, 3]), dev([0, 1, 2, 3])
    lens, st = dev([36, 36, 36]), p.status(3)
    x = torch.from_numpy(p.rng.integers(-32768, 32768, (3, 2, 64)).astype(np.int16)).to("cuda").view(torch.bfloat16)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        vb.vlac_pages_fork(p.pages, src, dst, False, st)
        vb.vlac_pages_resize(p.pages, dst, lens, st)
        vb.vlac_pages_write(p.pages, 1, dst, None, ptr, x, x, st)
    rows = p.bits(x).reshape(3, -1)
    for n in (35, 17, 64):
        p.resize([0], [n])
        lens.fill_(n + 1)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            g.replay()
        torch.cuda.synchronize()
        p.host.fork([0, 0, 0], [1, 2, 3], False)
        p.host.resize([1, 2, 3], [n + 1] * 3)
        p.same(st, p.host.write(1, [1, 2, 3], None, [0, 1, 2, 3], rows, rows))


def test_from_cache_takes_a_steps_prompt(vb):
    """The K/V rows a control step left become the pages of a slot, all layers; what does not fit is refused."""
    cfg = synth.tiny_config()
    model = synth.make_model(cfg, 0)
    devm = vb.DeviceModel(model)
    ctx = vb.vlac_create(vb.make_config(cfg, 2), devm.weights)
    cache = vb.vlac_cache_alloc(ctx, 2)
    try:
        rng = np.random.default_rng(3)
        kv = {}
        for seq in range(2):
            for part in (vb.PART_K, vb.PART_V):
                for l in range(cfg.n_layers):
                    t = torch.from_numpy(rng.standard_normal((cfg.max_seq, cfg.n_heads, cfg.head_dim)).astype(np.float32)).to("cuda").to(torch.bfloat16)
                    vb.vlac_cache_write(cache, part, seq, l, t)
                    kv[seq, part, l] = t
        pages = vb.Pages.empty(cfg.n_layers, 30, 16, cfg.n_heads, cfg.head_dim, 4, 8)
        st, st2 = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
        vb.vlac_pages_resize(pages, dev([1, 2]), dev([cfg.seq_len, cfg.max_seq]), st2)
        for seq, slot, n in ((0, 1, cfg.seq_len), (1, 2, cfg.max_seq)):
            vb.vlac_pages_from_cache(pages, cache, seq, slot, n, st)
            assert st.item() == 0
            t = pages.table[slot, :-(-n // 16)].long()
            for l in range(cfg.n_layers):
                assert torch.equal(pages.k[l, t].reshape(-1, cfg.n_heads, cfg.head_dim)[:n], kv[seq, vb.PART_K, l][:n])
                assert torch.equal(pages.v[l, t].reshape(-1, cfg.n_heads, cfg.head_dim)[:n], kv[seq, vb.PART_V, l][:n])
        vb.vlac_pages_from_cache(pages, cache, 0, 1, cfg.seq_len + 1, st)
        assert st.item() == -1                                            # longer than the slot
        vb.vlac_pages_fork(pages, dev([1]), dev([3]), False, st)
        vb.vlac_pages_from_cache(pages, cache, 0, 1, cfg.seq_len, st)
        assert st.item() == -2                                            # its pages are slot 3's too now
        for bad in (dict(seq=2), dict(seq=-1), dict(slot=4), dict(slot=-1), dict(n_rows=cfg.max_seq + 1), dict(n_rows=-1)):
            a = dict(seq=0, slot=2, n_rows=4)
            a.update(bad)
            with pytest.raises(vb.VlacError) as e:
                vb.vlac_pages_from_cache(pages, cache, a["seq"], a["slot"], a["n_rows"], st)
            assert e.value.status == -1
        for other in (vb.Pages.empty(1, 4, 16, cfg.n_heads, 64, 4, 8), vb.Pages.empty(2, 4, 16, 2, 64, 4, 8), vb.Pages.empty(2, 4, 16, 4, 128, 4, 8),
                      vb.Pages.empty(2, 4, 16, 4, 64, 4, 8, torch.float16)):
            with pytest.raises(vb.VlacError):
                vb.vlac_pages_from_cache(other, cache, 0, 0, 4, st)
    finally:
        vb.vlac_cache_free(cache)
        vb.vlac_destroy(ctx)


@pytest.mark.parametrize("shape", [dict(), dict(max_pages=9000, cap=112)], ids=["short_tables", "long_tables"])
def test_refused_entries_with_keep_pointers_out_of_range(vb, shape):
    """Both forms of the bookkeeping: a padded, repeated, read or broken entry is refused for what it is, its pointers are never followed, and
    the others stand.  (The keep list lies inside a larger buffer.)"""
    p = Pair(vb, 12, slots=12, **shape)
    p.resize([0, 1, 2, 3, 4], [40, 40, 40, 40, 40])
    p.host.len[3] = 10 ** 6
    p.pages.len.copy_(dev(p.host.len))
    room = torch.full((20000,), 10 ** 9, dtype=torch.int32, device="cuda")
    keep = room[10000:10004]
    keep.copy_(dev([0, 1, 5, 30]))
    far, low = 9000, -9000
    src = [0, -1, 12, 1, 1, 3, 2, 4, 2, 0]
    dst = [5, 6, 7, 5, -7, 8, 2, 12, 9, 10]
    ptr = [0, 4, far, far, low, low + 1, far, 4, far, 2, 4]
    want = [0, -1, -1, -1, -1, -2, -1, -1, -1, 0]
    st = p.status(10)
    vb.vlac_pages_compact(p.pages, dev(src), dev(dst), dev(ptr), keep, st)
    assert st.tolist() == want
    kept = {0: [0, 1, 5, 30], 9: [5, 30]}
    for i, (a, b) in {i: (src[i], dst[i]) for i in kept}.items():
        assert p.host.compact([a], [b], [kept[i]]) == [0]
    p.same(st, want)


def test_one_wrong_position_anywhere_in_a_long_keep_list(vb):
    """One entry, all warps of the bookkeeping on its list: whichever of them meets the wrong position, the code is the same, and a list without
    one stands."""
    p = Pair(vb, 13, layers=1, n_pages=600, page=8, heads=1, slots=3, max_pages=300)
    p.resize([0], [2400])
    rng, st = p.rng, p.status(1)
    for at in [1, 31, 32, 511, 512, 513, 1999] + rng.integers(1, 2000, 40).tolist():
        keep = sorted(rng.choice(2400, 2000, replace=False).tolist())
        keep[at] = keep[at - 1] if at % 2 else 2400 if at == 1999 else -1
        vb.vlac_pages_compact(p.pages, dev([0]), dev([1]), dev([0, 2000]), dev(keep), st)
        assert st.item() == -1, at
    p.same(st, [-1])
    assert p.compact([0], [1], [sorted(rng.choice(2400, 2000, replace=False).tolist())]) == [0]
    assert p.compact([0], [0], [list(range(2000))]) == [0]


def test_from_cache_refuses_what_a_pruned_step_left(vb):
    """A step that drops vision tokens leaves holes in the later layers: refused, also behind a step that reuses rows, until a sequence is
    recomputed whole; rows in front of the first hole are taken."""
    cfg = synth.tiny_config()
    devm = vb.DeviceModel(synth.make_model(cfg, 2))
    ctx = vb.vlac_create(vb.make_config(cfg, 2), devm.weights)
    cache = vb.vlac_cache_alloc(ctx, 2)
    try:
        rng = np.random.default_rng(4)
        feats = vb.upload_bf16(synth.f32_to_bf16(rng.standard_normal((2, cfg.n_vision, cfg.hidden), dtype=np.float32)))
        frames = torch.from_numpy(np.repeat(synth.rerandomised_pair(cfg, 2, 13)[0][None], 2, 0)).to("cuda").contiguous()
        ids = torch.from_numpy(np.concatenate([synth.make_prompt_ids(cfg, 1)] * 2)).to("cuda")
        tokens = torch.zeros((2, cfg.n_action), dtype=torch.int32, device="cuda")
        pages = vb.Pages.empty(cfg.n_layers, 40, 16, cfg.n_heads, cfg.head_dim, 2, 8)
        st, st2, L = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), cfg.seq_len
        vb.vlac_pages_resize(pages, dev([0, 1]), dev([L, L]), st2)

        def codes(n=L):
            out = []
            for seq in range(2):
                vb.vlac_pages_from_cache(pages, cache, seq, seq, n, st)
                out.append(st.item())
            return out

        step = lambda full, params=None: vb.vlac_step(ctx, cache, frames, feats, ids, params, full, tokens)
        pruned = lambda keep: vb.vlac_step_pruned(ctx, cache, frames, feats, ids, 1, keep, tokens)
        reuse, _keep = vb.make_params(top_k=32, alpha_override=[0.5, 1.0])
        step(False, reuse)
        assert codes() == [0, 0]
        pruned(24)
        assert codes() == [-2, -2] and codes(cfg.n_text_pre) == [0, 0]
        before = pages.k.clone()
        assert codes() == [-2, -2] and torch.equal(pages.k, before)
        step(False, reuse)                                                # (rows of dropped positions may be reused: still not there)
        assert codes() == [-2, -2]
        vb.vlac_cache_reset(cache, 1)
        step(False, reuse)
        assert codes() == [-2, 0]
        step(True)
        assert codes() == [0, 0]
        pruned(24)
        assert codes() == [-2, -2]
        pruned(cfg.n_vision)                                              # nothing dropped: a plain step
        assert codes() == [0, 0]
        pruned(24)
        g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=s):
            step(True)
        assert codes() == [-2, -2]                                        # captured, not run
        g.replay()
        assert codes() == [0, 0]
    finally:
        vb.vlac_cache_free(cache)
        vb.vlac_destroy(ctx)
