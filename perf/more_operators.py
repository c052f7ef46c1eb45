"""A step of speculative decoding over the paged K/V pool, as measured: inputs, plain forms and calls.

A small drafter proposes a tree of tokens behind what a sequence holds; the decoder runs all of them in one pass.  Their K/V rows
are appended to the pool with the rotation applied on the way (`append`, its tables from `tables`), every row attends to the
sequence and to its own ancestors in the tree (`tree`), the logits of every row are adjusted by penalties, biases and the grammar of the
action tokens (`logits`), and the path whose tokens the decoder would have chosen itself is accepted, with lists of the rows that
stay in the cache (`accept`).

Layout of the pool: k, v [n_layers][n_pages][page][kv_heads][head_dim]; table int32 [slots][max_pages] (-1 behind the last
page of a sequence); len int32 [slots]; refs int32 [n_pages].  The drafted rows of a sequence are its newest; the parent of a row is
a row of the same tree in front of it, -1 for the first.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one control loop at the 7B shape, 25 drafted rows behind a 290-position prompt: one layer of a decoded pass (latency)
        dict(name="tree_7b_25_rows", kind="tree", dtype="bf16", heads=32, kv_heads=32, head_dim=128, page=16, groups=1, members=1,
             prefix=288, depth=7, suffix=3, rows=25, ragged=1),
        # eight candidates of one two-camera prompt, each with a small tree of its own; head width 64, shared K/V heads, fp16
        dict(name="tree_8_candidates_fp16", kind="tree", dtype="fp16", heads=32, kv_heads=8, head_dim=64, page=16, groups=1, members=8,
             prefix=544, depth=5, suffix=21, rows=13, ragged=2),
        # four loops with histories of 65,600 positions (many past frames kept), trees of up to 64 rows, 8 K/V heads
        dict(name="tree_long_history", kind="tree", dtype="bf16", heads=32, kv_heads=8, head_dim=128, page=16, groups=4, members=1,
             prefix=65600, depth=9, suffix=37, rows=64, ragged=3),
        # sixteen loops behind 8,208 positions each at the 7B shape, trees of up to 61 rows: 2 GB of K and V
        dict(name="tree_16_loops", kind="tree", dtype="bf16", heads=32, kv_heads=32, head_dim=128, page=16, groups=16, members=1,
             prefix=8208, depth=8, suffix=50, rows=61, ragged=4),
        # the new token of each of 64 candidates at the 7B shape: whole heads rotated, no norms
        dict(name="append_64_tokens", kind="append", dtype="bf16", heads=32, kv_heads=32, head_dim=128, page=16, pool=2048, seqs=64,
             rows=300, new=1, rot=128, interleaved=0, norm=0, tree=0, ragged=5),
        # eight prompts of up to 4099 rows behind their projections, heads normalised, a quarter of each rotated in pairs
        dict(name="append_8_prompts", kind="append", dtype="fp16", heads=32, kv_heads=8, head_dim=128, page=16, pool=4096, seqs=8,
             rows=4100, new=4099, rot=32, interleaved=1, norm=1, tree=0, ragged=6),
        # a tree's 25 rows of logits at the 7B vocabulary: 256 action tokens allowed in some rows, penalties over the generated tokens
        dict(name="logits_25_rows", kind="logits", dtype="fp32", rows=25, vocab=32000, history=300, bias=16, masks=3, allow=0.008, tree=25, depth=7, ragged=7),
        # 512 rows of a batch of candidates over a large vocabulary, bf16
        dict(name="logits_512_rows", kind="logits", dtype="bf16", rows=512, vocab=128000, history=2048, bias=300, masks=5, allow=0.5, tree=64, depth=9, ragged=8),
        # what one loop's tree comes to
        dict(name="accept_one_tree", kind="accept", dtype="bf16", kv_heads=1, head_dim=64, page=16, seqs=1, rows=25, depth=7, len=315, ragged=9),
        # and what 64 trees of up to 61 rows behind up to 4100 positions come to
        dict(name="accept_64_trees", kind="accept", dtype="bf16", kv_heads=1, head_dim=64, page=16, seqs=64, rows=61, depth=8, len=4100, ragged=10),
        # tables of the library's own decoder with room for some frames more
        dict(name="tables_2048", kind="tables", positions=2048, rot=128, theta=10000.0, factor=1.0, original=0, first=0, amplitude=1.0),
        # tables for 262,144 positions, stretched eight times from 32,768
        dict(name="tables_long", kind="tables", positions=262144, rot=128, theta=500000.0, factor=8.0, original=32768, first=0, amplitude=1.2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tree", "tree", "tree", "append", "append", "logits", "logits", "accept", "tables"])
    c = dict(kind=kind, ragged=rng.randrange(1 << 20))
    if kind == "tables":
        return dict(kind=kind, positions=_log(rng, 1, 262144), rot=rng.choice([16, 32, 64, 96, 128]), theta=rng.choice([10000.0, 500000.0, 1000000.0]),
                    factor=rng.choice([1.0, 2.0, 4.0, 8.0, 40.0]), original=rng.choice([0, 4096, 8192, 32768]), first=rng.choice([0, 0, _log(rng, 1, 1000000)]),
                    amplitude=rng.choice([1.0, 1.0, 1.14, 1.37]))
    if kind == "logits":
        c.update(dtype=rng.choice(["fp32", "bf16", "fp16"]), rows=_log(rng, 1, 512))
        c["vocab"] = _log(rng, 1000, min(260000, 6.5e7 / c["rows"]))
        c.update(history=_log(rng, 1, 4096), bias=rng.choice([0, 1, 40, 300]), masks=rng.choice([0, 1, 4, 30]), allow=rng.choice([0.002, 0.1, 0.9]),
                 tree=rng.choice([0, 0, 1, 17, 64, 200]), depth=rng.choice([1, 4, 9, 30]))
        return c
    c.update(head_dim=rng.choice([64, 128]), page=rng.choice([8, 16, 16, 32, 64, 128]), dtype=rng.choice(["bf16", "fp16"]), depth=rng.choice([1, 3, 6, 12, 40]))
    if kind == "accept":
        c.update(kv_heads=1, seqs=_log(rng, 1, 64), rows=_log(rng, 1, 256))
        c["len"] = c["rows"] + _log(rng, 1, 4100)
        return c
    kv = rng.choice([1, 2, 4, 8, 16, 32])
    c["kv_heads"], c["heads"] = kv, kv * rng.choice([r for r in (1, 2, 3, 4, 5, 7, 8) if kv * r <= 40])
    d = c["head_dim"]
    if kind == "tree":
        c["groups"] = rng.choice([1, 1, 2, 3, 6, 16])
        c["members"] = _log(rng, 1, max(1, 24 // c["groups"]))
        n = c["groups"] * c["members"]
        c["rows"] = rng.choice([1, 2, 5, 9, 16, 25, 33, 64, 128])
        # no more K and V, and no more scores, than the largest listed cases
        most = min(65600, 2.5e8 / (n * kv * d), 4.0e8 / (n * c["heads"] * c["rows"]))
        c["prefix"] = _log(rng, 1, max(16, most))
        c["suffix"] = rng.randrange(0, 100)
        return c
    c.update(seqs=_log(rng, 1, 64), rot=rng.choice([r for r in (0, 16, 32, 48, 64, 96, 128) if r <= d]), interleaved=rng.choice([0, 1]), norm=rng.choice([0, 1]),
             tree=rng.choice([0, 0, 1]))
    c["rows"] = _log(rng, 1, max(2, min(4100, 1.2e8 / ((kv + c["heads"] / 2) * d * c["seqs"]))))
    c["new"] = min(c["rows"], 64) if c["tree"] else rng.randrange(1, c["rows"] + 1)
    c["pool"] = c["seqs"] * -(-c["rows"] // c["page"]) + rng.randrange(1, 40)
    return c


# ------------------------------------------------------------------------------------------------ shapes of a case
def _trees(sizes, depth, r):
    """A tree of each size, no row deeper than `depth`: parents within the tree, and how deep the rows are."""
    parents, depths = [], []
    for n in sizes:
        p, d = np.full(n, -1), np.zeros(n, np.int64)
        for j in range(1, n):
            at = np.nonzero(d[:j] < depth)[0]
            p[j] = at[-1 - min(len(at) - 1, int(r.geometric(0.25)) - 1)]       # (drafters extend what they drafted last)
            d[j] = d[p[j]] + 1
        parents.append(p)
        depths.append(d)
    return parents, depths


def _lengths(case):
    """Lengths that the case stands for (they belong to the case, not to the seed): host lists."""
    r = np.random.RandomState(case["ragged"])
    if case["kind"] == "tree":
        n = case["groups"] * case["members"]
        pre = [max(0, (case["prefix"] if g == 0 else int(r.randint(case["prefix"] // 2, case["prefix"] + 1))) // case["page"]) * case["page"]
               for g in range(case["groups"])]
        nq = [case["rows"] if i == 0 else int(r.randint((case["rows"] + 1) // 2, case["rows"] + 1)) for i in range(n)]
        return pre, [nq[i] + int(r.randint(0, case["suffix"] + 1)) for i in range(n)], nq
    if case["kind"] == "append":
        lens = [case["rows"] - (int(r.randint(0, (case["rows"] - case["new"]) // 2 + 1)) if i else 0) for i in range(case["seqs"])]
        return lens, [case["new"] if i == 0 or case["new"] == 1 else int(r.randint((case["new"] + 1) // 2, case["new"] + 1)) for i in range(case["seqs"])]
    if case["kind"] == "accept":
        nq = [case["rows"] if i == 0 else int(r.randint((case["rows"] + 1) // 2, case["rows"] + 1)) for i in range(case["seqs"])]
        return [case["len"] if i == 0 else int(r.randint(nq[i], case["len"] + 1)) for i in range(case["seqs"])], nq
    hist = [case["history"] if i == 0 else int(r.randint(0, case["history"] + 1)) for i in range(case["rows"])]
    return hist, [case["bias"] if i == 0 else int(r.randint(0, case["bias"] + 1)) for i in range(case["rows"])]


def _pages(rows, page):
    return -(-rows // page)


def work(case):
    if case["kind"] == "tables":
        return {"bytes": 8 * case["positions"] * (case["rot"] // 2), "flops": 0}
    if case["kind"] == "logits":
        size = 4 if case["dtype"] == "fp32" else 2
        hist, bias = _lengths(case)
        return {"bytes": 2 * size * case["rows"] * case["vocab"] + 4 * case["masks"] * _pages(case["vocab"], 32) + 4 * sum(hist) + 8 * sum(bias) + 4 * case["rows"], "flops": 0}
    if case["kind"] == "accept":
        lens, nq = _lengths(case)
        return {"bytes": 4 * sum(n - q + 1 for n, q in zip(lens, nq)) + 4 * 5 * sum(nq), "flops": 0}
    d = case["head_dim"]
    if case["kind"] == "append":
        new = sum(_lengths(case)[1])
        return {"bytes": 2 * 2 * d * new * (case["heads"] + 2 * case["kv_heads"]) + 4 * case["rot"] * new, "flops": 0}
    pre, suf, nq = _lengths(case)
    m, keys, pairs = case["members"], 0, 0
    r = np.random.RandomState(case["ragged"] + 1)
    depths = _trees(nq, case["depth"], r)[1]
    for i, (s, q) in enumerate(zip(suf, nq)):
        keys += s + (pre[i // m] if i % m == 0 else 0)
        pairs += q * (pre[i // m] + s - q) + int(depths[i].sum()) + q
    return {"bytes": keys * 4 * case["kv_heads"] * d + sum(nq) * case["heads"] * (2 * 2 * d + 4), "flops": 4.0 * pairs * case["heads"] * d}


# ------------------------------------------------------------------------------------------------ inputs
def _dev(x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(x, dtype)).to("cuda")


def _ptr(counts):
    return _dev(np.concatenate([[0], np.cumsum(counts)]))


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _pool(case, seed, lens, max_pages, n_pages):
    """A pool in use: sequence i of `lens` rows holds pages scattered over the pool."""
    r, g = np.random.RandomState(seed % (1 << 31)), _gen(seed)
    shape = (1, n_pages, case["page"], case["kv_heads"], case["head_dim"])
    k, v = (torch.empty(shape, dtype=TYPES[case["dtype"]], device="cuda").normal_(generator=g) for _ in range(2))
    table = np.full((len(lens), max_pages), -1, np.int32)
    refs = np.zeros(n_pages, np.int32)
    order, at = r.permutation(n_pages).astype(np.int32), 0
    for i, n in enumerate(lens):
        c = _pages(n, case["page"])
        table[i, :c] = order[at:at + c]
        at += c
    refs[order[:at]] = 1
    return dict(case=case, k=k, v=v, table=_dev(table), len=_dev(lens), refs=_dev(refs)), r, g


def prepare(case, seed):
    kind = case["kind"]
    if kind == "tables":
        # another seed begins elsewhere: tables of a window that moves with the history
        half = (case["positions"], case["rot"] // 2)
        st = dict(case=case, first=case["first"] + seed % 4096, cos=torch.zeros(half, device="cuda"), sin=torch.zeros(half, device="cuda"))
        if own:
            from paper_2502_02175_b200 import binding as vb
            st["vb"] = vb
        return st
    if kind == "logits":
        return _prepare_logits(case, seed)
    if kind == "tree":
        pre, suf, nq = _lengths(case)
        n, m = len(suf), case["members"]
        # the groups' common pages belong to the first member; the others point at them
        lens = [pre[i // m] + suf[i] if i % m == 0 else suf[i] for i in range(n)]
        st, r, g = _pool(case, seed, lens, max(_pages(pre[i // m] + suf[i], case["page"]) for i in range(n)) + 3, sum(_pages(x, case["page"]) for x in lens) + 5)
        t, refs = st["table"].cpu().numpy(), st["refs"].cpu().numpy()
        for i in range(n):
            c, s = pre[i // m] // case["page"], i // m * m
            if i % m and c:
                t[i, c:c + _pages(suf[i], case["page"])] = t[i, :_pages(suf[i], case["page"])].copy()
                t[i, :c] = t[s, :c]
                refs[t[s, :c]] += 1
        lens = [pre[i // m] + suf[i] for i in range(n)]
        parents, _ = _trees(nq, case["depth"], np.random.RandomState(case["ragged"] + 1))
        st.update(table=_dev(t), len=_dev(lens), refs=_dev(refs), seqs=_dev(np.arange(n)), q_ptr=_ptr(nq), parent=_dev(np.concatenate(parents)),
                  rows=sum(nq), most=max(lens), most_rows=max(nq), scale=1.0 / math.sqrt(case["head_dim"]))
        st["q"] = (torch.empty((st["rows"], case["heads"], case["head_dim"]), device="cuda").normal_(generator=g) * 2.0).to(st["k"].dtype)
        st["out"] = torch.zeros_like(st["q"])
        st["lse"] = torch.zeros((st["rows"], case["heads"]), dtype=torch.float32, device="cuda")
        st["status"] = torch.zeros(n, dtype=torch.int32, device="cuda")
    elif kind == "append":
        lens, new = _lengths(case)
        n = case["seqs"]
        st, r, g = _pool(case, seed, lens, max(_pages(x, case["page"]) for x in lens) + 1, case["pool"])
        slots = r.permutation(n).astype(np.int32)
        count = [new[s] for s in slots]
        start = [lens[s] - new[s] for s in slots]
        rows = sum(count)
        at = np.concatenate([np.arange(c) for c in count])
        if case["tree"]:                                                         # drafted rows: their depth, not their place, is their position
            at = np.concatenate(_trees(count, case["depth"], np.random.RandomState(case["ragged"] + 1))[1])
        pos = np.repeat(start, count) + at
        far = 1 + max(lens)
        freq = 10000.0 ** (-torch.arange(case["rot"] // 2, dtype=torch.float64, device="cuda") * 2.0 / max(1, case["rot"]))
        angle = torch.arange(far, dtype=torch.float64, device="cuda")[:, None] * freq
        dt = TYPES[case["dtype"]]
        make = lambda h: torch.empty((rows, h, case["head_dim"]), dtype=dt, device="cuda").normal_(generator=g)  # noqa: E731
        st.update(seqs=_dev(slots), start=_dev(start), row_ptr=_ptr(count), rows=rows, pos=_dev(pos), cos=angle.cos().float(), sin=angle.sin().float(),
                  q=make(case["heads"]), k_new=make(case["kv_heads"]), v_new=make(case["kv_heads"]), eps=1e-6,
                  status=torch.zeros(n, dtype=torch.int32, device="cuda"))
        st["q_out"] = torch.zeros_like(st["q"])
        gain = lambda: (1.0 + 0.1 * torch.empty(case["head_dim"], device="cuda").normal_(generator=g)).to(dt)  # noqa: E731
        st["q_gain"], st["k_gain"] = (gain(), gain()) if case["norm"] else (None, None)
    else:
        lens, nq = _lengths(case)
        n = case["seqs"]
        st, r, g = _pool(case, seed, lens, max(_pages(x, case["page"]) for x in lens) + 1, sum(_pages(x, case["page"]) for x in lens) + 5)
        parents, _ = _trees(nq, case["depth"], np.random.RandomState(case["ragged"] + 1))
        slots = r.permutation(n).astype(np.int32)
        ln = np.zeros(n, np.int32)
        ln[slots] = lens
        t = st["table"].cpu().numpy()
        tt = np.empty_like(t)
        tt[slots] = t                                                            # sequence i lives in slot slots[i]
        rows, keep = sum(nq), sum(lens)
        # a drafter of four likely tokens: about every third drafted row is what the decoder chooses
        st.update(seqs=_dev(slots), len=_dev(ln), table=_dev(tt), q_ptr=_ptr(nq), parent=_dev(np.concatenate(parents)), rows=rows, most_rows=max(nq),
                  drafted=_dev(r.randint(100, 104, rows)), chosen=_dev(r.randint(100, 104, rows)), n_keep=keep)
        new = lambda k, v=0: torch.full((k,), v, dtype=torch.int32, device="cuda")  # noqa: E731
        st.update(count=new(n), path=new(rows, -1), tokens=new(rows, -1), keep_ptr=new(n + 1), keep=new(keep), status=new(n))
    if own:                                                                      # the handles that a program keeps
        from paper_2502_02175_b200 import binding as vb
        st["vb"] = vb
        st["pages"] = vb.Pages(st["k"], st["v"], st["table"], st["len"], st["refs"])
        if kind == "tree":
            st["plan"] = vb.PrefixPlan(st["pages"], st["seqs"].numel(), st["rows"], case["heads"])
        if kind in ("tree", "accept"):
            st["tree"] = vb.Tree(st["q_ptr"], st["parent"], st["most_rows"])
            st["tree_status"] = torch.zeros_like(st["status"])
        if kind == "append":
            st["rope"] = vb.Rope(st["cos"], st["sin"], bool(case["interleaved"]), st["q_gain"], st["k_gain"], st["eps"])
    return st


def _prepare_logits(case, seed):
    r, g = np.random.RandomState(seed % (1 << 31)), _gen(seed)
    rows, vocab = case["rows"], case["vocab"]
    hist, bias = _lengths(case)
    # tokens come back: a few hundred of the vocabulary make up most of a history
    common = r.randint(0, vocab, 200)
    tokens = np.where(r.rand(sum(hist)) < 0.7, common[r.randint(0, 200, sum(hist))], r.randint(0, vocab, sum(hist)))
    begin = np.concatenate([[0], np.cumsum(hist)[:-1]])
    span = np.stack([begin, begin + (np.array(hist) * r.rand(rows)).astype(np.int64), begin + hist], 1)      # prompt, generated
    drafted = common[r.randint(0, 200, rows)]
    sizes = [min(case["tree"], rows - i) for i in range(0, rows, case["tree"])] if case["tree"] else [1] * rows
    parents, _ = _trees(sizes, case["depth"], np.random.RandomState(case["ragged"] + 1))
    st = dict(case=case, rows=rows, vocab=vocab, span=_dev(span), history=_dev(tokens), drafted=_dev(drafted), q_ptr=_ptr(sizes), parent=_dev(np.concatenate(parents)),
              most_rows=max(sizes), n_hist=sum(hist), n_bias=sum(bias))
    st["logits"] = (torch.empty((rows, vocab), device="cuda").normal_(generator=g) * 3.0).to(TYPES[case["dtype"]])
    one = lambda lo, hi: _dev(r.uniform(lo, hi, rows), np.float32)  # noqa: E731
    st.update(repetition=one(1.0, 1.5), frequency=one(0.0, 0.3), presence=one(0.0, 0.5))
    st["bias_ptr"] = _ptr(bias)
    st["bias_token"] = _dev(np.concatenate([r.choice(vocab, b, replace=False) for b in bias] + [np.zeros(0)]))
    st["bias"] = _dev(r.uniform(-4.0, 4.0, sum(bias)), np.float32)
    words = _pages(vocab, 32)
    bits = r.rand(case["masks"], words * 32) < case["allow"]
    bits[:, 7] = True
    st["allow"] = _dev(np.packbits(bits.reshape(-1, 32), axis=1, bitorder="little").view(np.int32).reshape(case["masks"], words)) if case["masks"] else None
    st["allow_row"] = _dev(r.randint(-1, case["masks"], rows)) if case["masks"] else None                    # -1: this row is free
    st.update(out=torch.zeros_like(st["logits"]), tokens=torch.zeros(rows, dtype=torch.int32, device="cuda"), status=torch.zeros(rows, dtype=torch.int32, device="cuda"))
    if own:
        from paper_2502_02175_b200 import binding as vb
        st["vb"] = vb
        st["tree"] = vb.Tree(st["q_ptr"], st["parent"], st["most_rows"]) if case["tree"] else None
        st["tree_status"] = torch.zeros(len(sizes), dtype=torch.int32, device="cuda")
        st["rules"] = vb.LogitsRules(rows, vocab, history=st["history"], span=st["span"], repetition=st["repetition"], frequency=st["frequency"],
                                     presence=st["presence"], bias_ptr=st["bias_ptr"], bias_token=st["bias_token"], bias=st["bias"], allow=st["allow"],
                                     allow_row=st["allow_row"], tree=st["tree"], drafted=st["drafted"] if case["tree"] else None)
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        return PLAIN[kind](st)
    vb = st["vb"]
    if kind == "tree":
        vb.vlac_tree_plan(st["pages"], st["tree"], st["seqs"], st["tree_status"])
        vb.vlac_prefix_plan(st["pages"], st["plan"], st["seqs"], st["q_ptr"], st["status"])
        vb.vlac_tree_attention(st["pages"], 0, st["plan"], st["tree"], st["q"], st["scale"], st["out"], st["lse"])
        return {"out": st["out"], "lse": st["lse"], "status": st["status"]}
    if kind == "append":
        vb.vlac_pages_append(st["pages"], 0, st["seqs"], st["start"], st["row_ptr"], st["rope"], st["pos"] if case["tree"] else None, st["q"], st["q_out"],
                             st["k_new"], st["v_new"], st["status"])
        return {"q": st["q_out"], "k": st["k"], "v": st["v"], "status": st["status"]}
    if kind == "logits":
        if st["tree"] is not None:
            vb.vlac_tree_plan(None, st["tree"], None, st["tree_status"])
        vb.vlac_logits_adjust(st["logits"], st["rules"], st["out"], st["tokens"], st["status"])
        return {"out": st["out"], "tokens": st["tokens"], "status": st["status"]}
    if kind == "accept":
        vb.vlac_tree_accept(st["pages"], st["tree"], st["seqs"], st["drafted"], st["chosen"], st["count"], st["path"], st["tokens"], st["keep_ptr"], st["keep"],
                            st["status"])
        return _accepted(st, st["count"], st["path"], st["tokens"], st["keep_ptr"], st["keep"])
    vb.vlac_rope_tables(st["cos"], st["sin"], case["theta"], first=st["first"], factor=case["factor"], original_len=case["original"], turns=(1.0, 32.0),
                        amplitude=case["amplitude"])
    return {"cos": st["cos"], "sin": st["sin"]}


def _accepted(st, count, path, tokens, keep_ptr, keep):
    # (behind keep_ptr's last the list has no meaning: the buffer is as the call left it, zeros)
    return {"count": count, "path": path, "tokens": tokens, "keep_ptr": keep_ptr, "keep": keep, "status": st["status"]}


# ---- plain forms
def _ancestors(st):
    """[n, Q, Q]: whether row a of a tree is row j or in front of it on its path, padded; which rows are there; and their places among all rows."""
    ptr, Q = st["q_ptr"].long(), st["most_rows"]
    nq = ptr[1:] - ptr[:-1]
    j = torch.arange(Q, device="cuda")
    real = j[None, :] < nq[:, None]
    at = (ptr[:-1, None] + j).clamp(max=st["rows"] - 1)
    parent = torch.where(real, st["parent"][at].long(), -1)
    step = (parent[:, :, None] == j).float() + torch.eye(Q, device="cuda")
    return torch.linalg.matrix_power(step, st["case"]["depth"]) > 0, real, at, parent


def _plain_tree(st):
    case = st["case"]
    H, KV, D, P, n, Q = case["heads"], case["kv_heads"], case["head_dim"], case["page"], st["seqs"].numel(), st["most_rows"]
    seen, real, rows, _ = _ancestors(st)
    slots = st["seqs"].long()
    table, ln = st["table"][slots].long(), st["len"][slots].long()
    nq = real.sum(-1)
    at = torch.arange(st["most"], device="cuda")
    page = torch.gather(table, 1, (at // P)[None, :].expand(n, -1)).clamp(min=0)
    pool = page * P + at % P                                                       # pool row of each position, [n, most]
    k, v = st["k"][0].view(-1, KV, D)[pool].float(), st["v"][0].view(-1, KV, D)[pool].float()
    q = (st["q"][rows].float() * st["scale"]).view(n, Q, KV, H // KV, D)
    s = torch.einsum("nqkrd,nskd->nkqrs", q, k)
    behind = at[None, :] - (ln - nq)[:, None]                                      # row of the tree at each position; negative in front of it
    mask = torch.gather(seen, 2, behind.clamp(0, Q - 1)[:, None, :].expand(-1, Q, -1))
    mask = (mask | (behind < 0)[:, None, :]) & (at[None, :] < ln[:, None])[:, None, :]
    s.masked_fill_(~mask[:, None, :, None, :], -math.inf)
    m = s.amax(-1, keepdim=True).clamp(min=-3.0e38)
    s.sub_(m).exp_()
    l = s.sum(-1, keepdim=True)
    o = torch.einsum("nkqrs,nskd->nqkrd", s.div_(l), v).reshape(n * Q, H, D)
    lse = (m + torch.log(l)).squeeze(-1).permute(0, 2, 1, 3).reshape(n * Q, H)
    to = torch.where(real, rows, st["rows"]).view(-1)                              # padded rows all land in one row behind the last
    out = torch.zeros((st["rows"] + 1, H, D), device="cuda").index_copy_(0, to, o)[:-1]
    lse = torch.zeros((st["rows"] + 1, H), device="cuda").index_copy_(0, to, lse)[:-1]
    return {"out": out.to(st["q"].dtype), "lse": lse, "status": torch.zeros_like(st["status"])}


def _turned(x, gain, st, at):
    """Heads normalised and rotated, 32 bits."""
    r = st["case"]["rot"]
    x = x.float()
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + st["eps"]) * gain.float()
    if r == 0:
        return x
    c, s = st["cos"][at][:, None, :], st["sin"][at][:, None, :]
    if st["case"]["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * c - b * s, a * s + b * c], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _plain_append(st):
    P = st["case"]["page"]
    ptr, slots = st["row_ptr"].long(), st["seqs"].long()
    i = torch.repeat_interleave(torch.arange(slots.numel(), device="cuda"), ptr[1:] - ptr[:-1], output_size=st["rows"])
    place = st["start"].long()[i] + torch.arange(st["rows"], device="cuda") - ptr[:-1][i]
    at = st["pos"].long() if st["case"]["tree"] else place
    to = st["table"].long()[slots[i], place // P] * P + place % P
    q = _turned(st["q"], st["q_gain"], st, at).to(st["q"].dtype)
    k = _turned(st["k_new"], st["k_gain"], st, at).to(st["k"].dtype)
    for x, y in ((st["k"], k), (st["v"], st["v_new"])):
        x[0].view(-1, *y.shape[1:]).index_copy_(0, to, y)
    return {"q": q, "k": st["k"], "v": st["v"], "status": st["status"].zero_()}


def _plain_logits(st):
    rows, vocab = st["rows"], st["vocab"]
    x = st["logits"].float()
    span = st["span"].long()
    r = torch.arange(rows, device="cuda")
    i = torch.repeat_interleave(r, span[:, 2] - span[:, 0], output_size=st["n_hist"])
    generated = torch.arange(st["n_hist"], device="cuda") >= span[i, 1]
    cell = i * vocab + st["history"].long()
    made = torch.zeros(rows * vocab, device="cuda").index_add_(0, cell, generated.float())
    seen = torch.zeros(rows * vocab, device="cuda").index_add_(0, cell, torch.ones(st["n_hist"], device="cuda"))
    if st["case"]["tree"]:                                                         # the drafted tokens on a row's path are generated ones
        path, real, at, _ = _ancestors(st)
        on = path & real[:, :, None] & real[:, None, :]
        cell = (at[:, :, None] * vocab + st["drafted"].long()[at][:, None, :]).view(-1)
        made.index_add_(0, cell, on.float().view(-1))
        seen.index_add_(0, cell, on.float().view(-1))
    made, seen = made.view(rows, vocab), seen.view(rows, vocab) > 0
    rep, freq, pres = (st[n][:, None] for n in ("repetition", "frequency", "presence"))
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    x = x - freq * made
    x = x - pres * (made > 0)
    count = (st["bias_ptr"][1:] - st["bias_ptr"][:-1]).long()
    x[torch.repeat_interleave(r, count, output_size=st["n_bias"]), st["bias_token"].long()] += st["bias"]
    if st["allow"] is not None:
        bit = (st["allow"][..., None] >> torch.arange(32, dtype=torch.int32, device="cuda")) & 1
        of = st["allow_row"].long()
        allowed = (bit.view(bit.shape[0], -1)[of.clamp(min=0), :vocab] != 0) | (of < 0)[:, None]
        x = x.masked_fill(~allowed, -math.inf)
    best = torch.where(x == x.amax(-1, keepdim=True), torch.arange(vocab, device="cuda"), vocab).amin(-1)
    return {"out": x.to(st["logits"].dtype), "tokens": best.to(torch.int32), "status": torch.zeros_like(st["status"])}


def _plain_accept(st):
    n, Q = st["seqs"].numel(), st["most_rows"]
    path, real, at, parent = _ancestors(st)
    j = torch.arange(Q, device="cuda")
    drafted, chosen = st["drafted"][at], st["chosen"][at]
    fits = (parent >= 0) & (drafted == torch.gather(chosen, 1, parent.clamp(min=0)))
    # of several children that fit the first is taken
    first = torch.full((n, Q + 1), Q, device="cuda").scatter_reduce_(1, torch.where(fits, parent, Q), j[None, :].expand(n, -1), "amin")[:, :Q]
    fits = (fits & (torch.gather(first, 1, parent.clamp(min=0)) == j)) | (j == 0)
    taken = real & (fits[:, None, :] | ~path).all(-1)
    count = taken.sum(-1)
    place = torch.cumsum(taken, 1) - 1                                             # a path's rows ascend
    to = torch.where(taken, torch.gather(at, 1, place.clamp(min=0)), st["rows"]).view(-1)
    blank = torch.full((st["rows"] + 1,), -1, dtype=torch.int32, device="cuda")
    paths = blank.clone().scatter_(0, to, j.to(torch.int32).repeat(n))[:-1]
    tokens = blank.clone().scatter_(0, to, chosen.reshape(-1))[:-1]
    # rows that stay: all in front of the tree, then the path
    ln = st["len"][st["seqs"].long()].long()
    before = ln - real.sum(-1)
    kept = before + count
    keep_ptr = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), torch.cumsum(kept, 0)])
    x = torch.arange(st["n_keep"], device="cuda")
    i = torch.searchsorted(keep_ptr, x, right=True) - 1
    inside = i < n
    i = i.clamp(max=n - 1)
    off = x - keep_ptr[i]
    of = paths.long()[(st["q_ptr"].long()[i] + off - before[i]).clamp(0, st["rows"] - 1)]
    keep = torch.where(inside, torch.where(off < before[i], off, before[i] + of), 0)
    return _accepted(st, count.to(torch.int32), paths, tokens, keep_ptr.to(torch.int32), keep.to(torch.int32))


def _plain_tables(st):
    case = st["case"]
    half = case["rot"] // 2
    f = case["theta"] ** (-torch.arange(half, dtype=torch.float64, device="cuda") * 2.0 / case["rot"])
    turns = case["original"] * f / (2.0 * math.pi)
    keep = ((turns - 1.0) / 31.0).clamp(0.0, 1.0) if case["original"] else torch.zeros_like(f)
    f = f * (keep + (1.0 - keep) / case["factor"])
    angle = torch.arange(st["first"], st["first"] + case["positions"], dtype=torch.float64, device="cuda")[:, None] * f
    return {"cos": (case["amplitude"] * torch.cos(angle)).float(), "sin": (case["amplitude"] * torch.sin(angle)).float()}


PLAIN = {"tree": _plain_tree, "append": _plain_append, "logits": _plain_logits, "accept": _plain_accept, "tables": _plain_tables}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    if case["kind"] == "accept":                                                   # whole numbers only
        return None
    st = prepare(case, seed)
    return {"tree": _exact_tree, "append": _exact_append, "logits": _exact_logits, "tables": _exact_tables}[case["kind"]](case, st)


def _path(parent, j):
    found = []
    while j >= 0:
        found.append(j)
        j = int(parent[j])
    return found


def _exact_tree(case, st):
    """One sequence after the other over its own table, the rows that a row of the tree sees found by walking up."""
    H, KV, D, P = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    ptr, parents = st["q_ptr"].tolist(), st["parent"].cpu().numpy()
    out = torch.zeros((st["rows"], H, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((st["rows"], H), dtype=torch.float64, device="cuda")
    for i, slot in enumerate(st["seqs"].tolist()):
        n, nq = int(st["len"][slot]), ptr[i + 1] - ptr[i]
        pages = st["table"][slot, :-(-n // P)].long()
        seen = np.zeros((nq, n), bool)
        seen[:, :n - nq] = True
        for j in range(nq):
            seen[j, [n - nq + a for a in _path(parents[ptr[i]:], j)]] = True
        seen = torch.from_numpy(seen).to("cuda")
        for h in range(KV):
            k, v = (x[0, pages, :, h].reshape(-1, D)[:n].double() for x in (st["k"], st["v"]))
            for e in range(h * (H // KV), (h + 1) * (H // KV)):
                s = (st["q"][ptr[i]:ptr[i + 1], e].double() @ k.T / math.sqrt(D)).masked_fill(~seen, -math.inf)
                lse[ptr[i]:ptr[i + 1], e] = torch.logsumexp(s, -1)
                out[ptr[i]:ptr[i + 1], e] = torch.softmax(s, -1) @ v
    return {"out": out, "lse": lse, "status": None}


def _exact_append(case, st):
    P, D, r = case["page"], case["head_dim"], case["rot"]
    h = torch.arange(D, device="cuda")
    # dimension e of the rotated part is x_e cos +- (its partner) sin
    if case["interleaved"]:
        partner, angle, sign = h ^ 1, h // 2, torch.where(h % 2 == 0, -1.0, 1.0)
    else:
        partner, angle, sign = (h + r // 2) % max(1, r), h % max(1, r // 2), torch.where(h < r // 2, -1.0, 1.0)
    inside = h < r
    partner = torch.where(inside, partner, h)
    angle = torch.where(inside, angle, 0)

    def turned(x, gain, pos):
        x = x.double()
        if gain is not None:
            x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / D + st["eps"]) * gain.double()
        if not r:
            return x
        c, s = st["cos"].double()[pos][:, angle], st["sin"].double()[pos][:, angle]
        y = x * c[:, None, :] + sign.double() * x[..., partner] * s[:, None, :]
        return torch.where(inside, y, x)

    k, v = st["k"].double(), st["v"].double()
    q = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    ptr, start = st["row_ptr"].tolist(), st["start"].tolist()
    for i, slot in enumerate(st["seqs"].tolist()):
        a, b = ptr[i], ptr[i + 1]
        place = torch.arange(start[i], start[i] + b - a, device="cuda")
        pos = st["pos"][a:b].long() if case["tree"] else place
        pages = st["table"][slot, place // P].long()
        k[0, pages, place % P] = turned(st["k_new"][a:b], st["k_gain"], pos)
        v[0, pages, place % P] = st["v_new"][a:b].double()
        q[a:b] = turned(st["q"][a:b], st["q_gain"], pos)
    return {"q": q, "k": k, "v": v, "status": None}


def _exact_logits(case, st):
    rows, vocab = st["rows"], st["vocab"]
    span, hist, ptr = st["span"].tolist(), st["history"].cpu().numpy(), st["bias_ptr"].tolist()
    drafted, parents, starts = st["drafted"].cpu().numpy(), st["parent"].cpu().numpy(), st["q_ptr"].tolist()
    first = {r: a for a, b in zip(starts, starts[1:]) for r in range(a, b)}
    out = torch.empty((rows, vocab), dtype=torch.float64, device="cuda")
    words = None if st["allow"] is None else st["allow"].cpu().numpy().view(np.uint8)
    for r in range(rows):
        a, g, b = span[r]
        prompt, made = hist[a:g], hist[g:b]
        if case["tree"]:
            made = np.concatenate([made, drafted[[first[r] + j for j in _path(parents[first[r]:], r - first[r])]]])
        c = torch.from_numpy(np.bincount(made, minlength=vocab)).to("cuda").double()
        seen = torch.from_numpy(np.bincount(np.concatenate([prompt, made]), minlength=vocab) > 0).to("cuda")
        rep, freq, pres = (float(st[n][r]) for n in ("repetition", "frequency", "presence"))
        x = st["logits"][r].double()
        x = torch.where(seen & (x > 0), x / rep, torch.where(seen, x * rep, x)) - freq * c - pres * (c > 0)
        x[st["bias_token"][ptr[r]:ptr[r + 1]].long()] += st["bias"][ptr[r]:ptr[r + 1]].double()
        if words is not None and int(st["allow_row"][r]) >= 0:
            bits = np.unpackbits(words[int(st["allow_row"][r])], bitorder="little")[:vocab]
            x[torch.from_numpy(bits == 0).to("cuda")] = -math.inf
        out[r] = x
    return {"out": out, "tokens": None, "status": None}


def _exact_tables(case, st):
    """Angles as turns, reduced before the functions are taken (numpy's extended type on the host where it has one)."""
    r = np.longdouble(case["rot"])
    i = np.arange(case["rot"] // 2).astype(np.longdouble)
    f = np.exp(-(2 * i / r) * np.log(np.longdouble(case["theta"])))
    pi = np.longdouble("3.14159265358979323846264338327950288")
    turns = case["original"] * f / (2 * pi)
    keep = np.clip((turns - 1) / 31, 0, 1) if case["original"] else np.zeros_like(f)
    per = f * (keep + (1 - keep) / np.longdouble(case["factor"])) / (2 * pi)
    p = np.arange(st["first"], st["first"] + case["positions"]).astype(np.longdouble)[:, None]
    turn = p * per
    angle = torch.from_numpy(((turn - np.rint(turn)) * (2 * pi)).astype(np.float64)).to("cuda")
    return {"cos": case["amplitude"] * torch.cos(angle), "sin": case["amplitude"] * torch.sin(angle)}
