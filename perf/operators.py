"""The paged K/V pool and the attention over a shared prefix, as measured: inputs, plain forms and calls.

One prompt (about 290 positions for one camera, 552 for two) is the common beginning of several candidate action
sequences, or of the control loops of several robots with one instruction.  Its K/V rows live once in a pool of pages;
candidates are forked from it, grown, pruned and given back, and one attention call per layer reads the common pages once
for all of them.

Layout of the pool: k, v [n_layers][n_pages][page][kv_heads][head_dim]; table int32 [slots][max_pages] (-1 behind the last
page of a sequence); len int32 [slots]; refs int32 [n_pages] (0: the page is free).  Pages are taken lowest number first.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # best-of-8 action decoding from one 290-position prompt at the 7B shape: one layer, one new token per candidate
        # (the smallest call a control loop makes at every layer of every token: latency)
        dict(name="attn_7b_8_candidates", kind="attention", dtype="bf16", heads=32, kv_heads=32, head_dim=128, page=16,
             groups=1, members=8, prefix=288, suffix=9, q=1, ragged=1),
        # five instructions being served at once, each with its own prompt history of two to four thousand positions (several
        # past frames kept), 13 candidates each at different depths; head width 64, fp16
        dict(name="attn_5_prompts_fp16", kind="attention", dtype="fp16", heads=32, kv_heads=32, head_dim=64, page=64,
             groups=5, members=13, prefix=4096, suffix=300, q=1, ragged=2),
        # 32 candidates behind a 65,600-position history in a decoder with 8 K/V heads (the cache decides: HBM)
        dict(name="attn_gqa_long_history", kind="attention", dtype="bf16", heads=32, kv_heads=8, head_dim=128, page=16,
             groups=1, members=32, prefix=65600, suffix=515, q=1, ragged=3),
        # 64 action chunks of 7 rows decoded in parallel behind a shared 8,208-position history, 7B shape: 448 query rows a
        # head (the matrix products decide)
        dict(name="attn_chunks_of_7", kind="attention", dtype="bf16", heads=32, kv_heads=32, head_dim=128, page=16,
             groups=1, members=64, prefix=8208, suffix=40, q=7, ragged=4),
        # one prompt of the 7B shape forked into 8 candidates: shared pages, a tail of 2 rows copied in 32 layers
        dict(name="fork_8_candidates", kind="fork", dtype="bf16", layers=32, kv_heads=32, head_dim=128, page=16, pool=256,
             parents=1, children=8, rows=290, deep=0, ragged=5),
        # the eight sequences of a served batch copied whole (a next step overwrites their rows in place)
        dict(name="copy_batch_of_8", kind="fork", dtype="bf16", layers=32, kv_heads=32, head_dim=128, page=16, pool=512,
             parents=8, children=1, rows=297, deep=1, ragged=6),
        # attention-based pruning of one frame: 128 of 256 vision tokens of a 290-position prompt stay
        dict(name="compact_one_frame", kind="compact", dtype="bf16", layers=32, kv_heads=32, head_dim=128, page=16, pool=128,
             seqs=1, rows=290, keep=162, ragged=7),
        # the same for a batch of 8 two-camera prompts
        dict(name="compact_batch_of_8", kind="compact", dtype="bf16", layers=32, kv_heads=32, head_dim=128, page=16, pool=512,
             seqs=8, rows=552, keep=300, ragged=8),
        # eight episodes end and eight begin: their pages are given back and taken anew
        dict(name="admit_8_episodes", kind="admit", dtype="bf16", layers=2, kv_heads=4, head_dim=64, page=16, pool=4096,
             seqs=8, rows=552, ragged=9),
        # 512 sequences of up to 4096 rows change hands in a pool of 131,072 pages
        dict(name="admit_512_sequences", kind="admit", dtype="bf16", layers=1, kv_heads=1, head_dim=64, page=16, pool=131072,
             seqs=512, rows=4096, ragged=10),
        # one new row for each of 64 candidates in one layer: the write of every decoded token
        dict(name="write_64_tokens", kind="write", dtype="bf16", layers=1, kv_heads=32, head_dim=128, page=16, pool=2048,
             seqs=64, rows=300, new=1, ragged=11),
        # 8 prompts of up to 4096 positions written after their prefill, one layer of the 7B shape
        dict(name="write_8_prompts", kind="write", dtype="bf16", layers=1, kv_heads=32, head_dim=128, page=16, pool=4096,
             seqs=8, rows=4100, new=4099, ragged=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "attention", "fork", "compact", "admit", "write"])
    d = rng.choice([64, 128])
    page = rng.choice([8, 16, 16, 32, 64, 128])
    c = dict(kind=kind, dtype=rng.choice(["bf16", "fp16"]), head_dim=d, page=page, ragged=rng.randrange(1 << 20))
    if kind == "attention":
        kv = rng.choice([1, 2, 4, 8, 16, 32])
        c["kv_heads"], c["heads"] = kv, kv * rng.choice([r for r in (1, 2, 3, 4, 5, 7, 8) if kv * r <= 40])
        c["groups"] = rng.choice([1, 1, 2, 3, 6])
        c["members"] = _log(rng, 1, 48 // c["groups"])
        c["q"] = rng.choice([1, 1, 1, 2, 7, 8, 33])
        most = 3.0e10 / (c["groups"] * c["members"] * c["q"] * c["heads"] * d * 4)      # no more products than the largest listed case
        c["prefix"] = _log(rng, 1, max(16, min(65600, most / 2, 5e8 / (c["groups"] * kv * d))))
        c["suffix"] = c["q"] + _log(rng, 1, max(2, min(600, most / 2)))
        return c
    c["kv_heads"] = rng.choice([1, 4, 8, 32])
    row = c["kv_heads"] * d * 4                                            # bytes of one row of K and V
    if kind == "admit":
        c.update(layers=1, kv_heads=1, seqs=_log(rng, 1, 512), rows=_log(rng, 1, 4096))
        c["pool"] = c["seqs"] * -(-c["rows"] // page) + _log(rng, 1, 30000)
        return c
    c["layers"] = rng.choice([1, 2, 7, 32])
    most = 1.2e9 / (row * c["layers"])                                      # rows that may move
    if kind == "fork":
        c["deep"] = rng.choice([0, 1])
        c["parents"] = _log(rng, 1, 8)
        c["children"] = _log(rng, 1, 64 // c["parents"])
        c["rows"] = _log(rng, 1, max(2, min(4096, most / (c["parents"] * (c["children"] + 1)))))
        c["pool"] = c["parents"] * (c["children"] + 1) * -(-c["rows"] // page) + rng.randrange(1, 40)
    elif kind == "compact":
        c["seqs"] = _log(rng, 1, 16)
        c["rows"] = _log(rng, 1, max(2, min(4096, most / (2 * c["seqs"]))))
        c["keep"] = rng.randrange(0, c["rows"] + 1)
        c["pool"] = c["seqs"] * (-(-c["rows"] // page) + -(-c["keep"] // page)) + rng.randrange(1, 40)
    else:
        c["layers"] = 1
        c["seqs"] = _log(rng, 1, 64)
        c["rows"] = _log(rng, 1, max(2, min(4100, 1.0e9 / (row * c["seqs"]))))
        c["new"] = rng.randrange(1, c["rows"] + 1)
        c["pool"] = c["seqs"] * -(-c["rows"] // page) + rng.randrange(1, 40)
    return c


# ------------------------------------------------------------------------------------------------ shapes of a case
def _lengths(case):
    """Lengths that the case stands for (they belong to the case, not to the seed): host lists."""
    r = np.random.RandomState(case["ragged"])
    if case["kind"] == "attention":
        n = case["groups"] * case["members"]
        pre = [max(0, (case["prefix"] if g == 0 else int(r.randint(case["prefix"] // 2, case["prefix"] + 1))) // case["page"]) * case["page"]
               for g in range(case["groups"])]
        nq = [case["q"] if i == 0 or case["q"] == 1 else int(r.randint(1, case["q"] + 1)) if case["q"] > 8 else case["q"] for i in range(n)]
        suf = [int(r.randint(nq[i], case["suffix"] + 1)) for i in range(n)]
        return pre, suf, nq
    if case["kind"] == "fork":
        return [case["rows"] - (int(r.randint(0, case["rows"] // 4 + 1)) if p else 0) for p in range(case["parents"])]
    if case["kind"] == "compact":
        return [case["rows"]] * case["seqs"], [max(0, case["keep"] - (int(r.randint(0, case["keep"] // 4 + 1)) if i else 0)) for i in range(case["seqs"])]
    if case["kind"] == "admit":
        return [int(r.randint(1, case["rows"] + 1)) for _ in range(case["seqs"])], [int(r.randint(1, case["rows"] + 1)) for _ in range(case["seqs"])]
    lens = [case["rows"] - (int(r.randint(0, (case["rows"] - case["new"]) // 2 + 1)) if i else 0) for i in range(case["seqs"])]
    new = [case["new"] if i == 0 or case["new"] == 1 else int(r.randint((case["new"] + 1) // 2, case["new"] + 1)) for i in range(case["seqs"])]
    return lens, new


def _pages(rows, page):
    return -(-rows // page)


def work(case):
    page, d = case["page"], case["head_dim"]
    if case["kind"] == "attention":
        pre, suf, nq = _lengths(case)
        m, row = case["members"], 2 * 2 * case["kv_heads"] * d                # bytes of a K and a V row
        keys, pairs = 0, 0
        for i, (s, q) in enumerate(zip(suf, nq)):
            keys += s + (pre[i // m] if i % m == 0 else 0)
            pairs += q * (pre[i // m] + s) - q * (q - 1) // 2
        return {"bytes": keys * row + sum(nq) * case["heads"] * (2 * 2 * d + 4), "flops": 4.0 * pairs * case["heads"] * d}
    row = 2 * 2 * case["kv_heads"] * d * case["layers"]
    if case["kind"] == "fork":
        rows = [n if case["deep"] else n % page for n in _lengths(case)]
        return {"bytes": sum(rows) * row * (1 + case["children"]) + 8 * sum(_pages(n, page) for n in _lengths(case)) * (1 + case["children"]), "flops": 0}
    if case["kind"] == "compact":
        return {"bytes": sum(_lengths(case)[1]) * row * 2 + 8 * sum(_pages(n, page) for n in _lengths(case)[0]), "flops": 0}
    if case["kind"] == "admit":
        old, new = _lengths(case)
        return {"bytes": 4 * 3 * (sum(_pages(n, page) for n in old) + sum(_pages(n, page) for n in new)), "flops": 0}
    return {"bytes": sum(_lengths(case)[1]) * row * 2, "flops": 0}


# ------------------------------------------------------------------------------------------------ inputs
def _pool(case, seed, lens, max_pages, spare_slots, n_pages, layers):
    """A pool in use: sequence i of `lens` rows holds pages scattered over the pool; `spare_slots` slots are empty."""
    r = np.random.RandomState(seed % (1 << 31))
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    shape = (layers, n_pages, case["page"], case["kv_heads"], case["head_dim"])
    dt = TYPES[case["dtype"]]
    k = torch.empty(shape, dtype=dt, device="cuda").normal_(generator=g)
    v = torch.empty(shape, dtype=dt, device="cuda").normal_(generator=g)
    table = np.full((len(lens) + spare_slots, max_pages), -1, np.int32)
    refs = np.zeros(n_pages, np.int32)
    order, at = r.permutation(n_pages).astype(np.int32), 0
    for i, n in enumerate(lens):
        c = _pages(n, case["page"])
        table[i, :c] = order[at:at + c]
        at += c
    refs[order[:at]] = 1
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to("cuda")
    st = dict(case=case, k=k, v=v, table=dev(table), len=dev(np.array(list(lens) + [0] * spare_slots, np.int32)), refs=dev(refs))
    return st, r, g, dev


def prepare(case, seed):
    kind, page = case["kind"], case["page"]
    if kind == "attention":
        pre, suf, nq = _lengths(case)
        n, m = len(suf), case["members"]
        # the groups' common pages belong to the first member; the others point at them
        lens = [pre[i // m] + suf[i] if i % m == 0 else suf[i] for i in range(n)]
        maxp = max(_pages(pre[i // m] + suf[i], page) for i in range(n)) + 3
        st, r, g, dev = _pool(case, seed, lens, maxp, 0, sum(_pages(x, page) for x in lens) + 5, 1)
        t = st["table"].cpu().numpy()
        refs = st["refs"].cpu().numpy()
        for i in range(n):
            c, s = pre[i // m] // page, i // m * m
            if i % m and c:
                t[i, c:c + _pages(suf[i], page)] = t[i, :_pages(suf[i], page)].copy()
                t[i, :c] = t[s, :c]
                refs[t[s, :c]] += 1
        rows = sum(nq)
        slots = r.permutation(n).astype(np.int32) if case["groups"] == 1 else np.arange(n, dtype=np.int32)
        tt = np.empty_like(t)
        tt[slots] = t                                                            # sequence i lives in slot slots[i]
        ln = np.zeros(n, np.int32)
        ln[slots] = [pre[i // m] + suf[i] for i in range(n)]
        st.update(table=dev(tt), len=dev(ln), refs=dev(refs), seqs=dev(slots), rows=rows, prefix=dev(np.array(pre, np.int64)),
                  most_prefix=max(pre), most_suffix=max(suf), q_ptr=dev(np.concatenate([[0], np.cumsum(nq)]).astype(np.int32)),
                  scale=1.0 / math.sqrt(case["head_dim"]))
        st["q"] = (torch.empty((rows, case["heads"], case["head_dim"]), device="cuda").normal_(generator=g) * 2.0).to(st["k"].dtype)
        st["out"] = torch.zeros_like(st["q"])
        st["lse"] = torch.zeros((rows, case["heads"]), dtype=torch.float32, device="cuda")
        st["status"] = torch.zeros(n, dtype=torch.int32, device="cuda")
    elif kind == "fork":
        lens = _lengths(case)
        n = case["parents"] * case["children"]
        st, r, g, dev = _pool(case, seed, lens, max(_pages(x, page) for x in lens) + 2, n, case["pool"], case["layers"])
        par = np.repeat(np.arange(case["parents"], dtype=np.int32), case["children"])
        st.update(src=dev(par), dst=dev((case["parents"] + np.arange(n)).astype(np.int32)),
                  moved=sum((lens[p] if case["deep"] else lens[p] % page) for p in par))
        st["status"] = torch.zeros(n, dtype=torch.int32, device="cuda")
    elif kind == "compact":
        lens, keep = _lengths(case)
        n = case["seqs"]
        st, r, g, dev = _pool(case, seed, lens, max(_pages(x, page) for x in lens) + 2, n, case["pool"], case["layers"])
        # the leading text position always stays; the others are what attention left
        rows = [np.sort(np.concatenate([[0], 1 + r.choice(lens[i] - 1, keep[i] - 1, replace=False)]))[:keep[i]] if keep[i] else np.zeros(0) for i in range(n)]
        st.update(src=dev(np.arange(n, dtype=np.int32)), dst=dev((n + np.arange(n)).astype(np.int32)), keep=dev(np.concatenate(rows).astype(np.int32)),
                  keep_ptr=dev(np.concatenate([[0], np.cumsum(keep)]).astype(np.int32)), most_keep=max(keep))
        st["status"] = torch.zeros(n, dtype=torch.int32, device="cuda")
    elif kind == "admit":
        old, new = _lengths(case)
        n = case["seqs"]
        st, r, g, dev = _pool(case, seed, old, max(_pages(x, page) for x in old + new) + 1, 0, case["pool"], case["layers"])
        st.update(seqs=dev(r.permutation(n).astype(np.int32)), lens=dev(np.array(new, np.int32)))
        st["status"] = torch.zeros(n, dtype=torch.int32, device="cuda")
    else:
        lens, new = _lengths(case)
        n = case["seqs"]
        st, r, g, dev = _pool(case, seed, lens, max(_pages(x, page) for x in lens) + 1, 0, case["pool"], 1)
        slots = r.permutation(n).astype(np.int32)
        rows = [new[s] for s in slots]
        st.update(seqs=dev(slots), start=dev(np.array([lens[s] - new[s] for s in slots], np.int32)), rows=sum(rows),
                  row_ptr=dev(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)))
        w = (sum(rows), case["kv_heads"], case["head_dim"])
        st["k_new"] = torch.empty(w, dtype=st["k"].dtype, device="cuda").normal_(generator=g)
        st["v_new"] = torch.empty(w, dtype=st["k"].dtype, device="cuda").normal_(generator=g)
        st["status"] = torch.zeros(n, dtype=torch.int32, device="cuda")
    if own:                                                                      # the handles that a program keeps
        from paper_2502_02175_b200 import binding as vb
        st["vb"] = vb
        st["pages"] = vb.Pages(st["k"], st["v"], st["table"], st["len"], st["refs"])
        if kind == "attention":
            st["plan"] = vb.PrefixPlan(st["pages"], st["seqs"].numel(), st["rows"], case["heads"])
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    case = st["case"]
    kind = case["kind"]
    if kind == "attention":
        if own:
            vb = st["vb"]
            vb.vlac_prefix_plan(st["pages"], st["plan"], st["seqs"], st["q_ptr"], st["status"])
            vb.vlac_prefix_attention(st["pages"], 0, st["plan"], st["q"], st["scale"], st["out"], st["lse"])
            return {"out": st["out"], "lse": st["lse"], "status": st["status"]}
        return _plain_attention(st)
    if own:
        vb = st["vb"]
        if kind == "fork":
            vb.vlac_pages_fork(st["pages"], st["src"], st["dst"], bool(case["deep"]), st["status"])
        elif kind == "compact":
            vb.vlac_pages_compact(st["pages"], st["src"], st["dst"], st["keep_ptr"], st["keep"], st["status"])
        elif kind == "admit":
            vb.vlac_pages_free(st["pages"], st["seqs"], st["status"])
            vb.vlac_pages_resize(st["pages"], st["seqs"], st["lens"], st["status"])
        else:
            vb.vlac_pages_write(st["pages"], 0, st["seqs"], st["start"], st["row_ptr"], st["k_new"], st["v_new"], st["status"])
    elif kind == "fork":
        _plain_fork(st)
    elif kind == "compact":
        _plain_compact(st)
    elif kind == "admit":
        _plain_release(st, st["seqs"].long())
        _plain_resize(st, st["seqs"].long(), st["lens"].long())
        st["status"].zero_()
    else:
        _plain_write(st)
    return {"k": st["k"], "v": st["v"], "table": st["table"], "len": st["len"], "refs": st["refs"], "status": st["status"]}


# ---- plain forms
def _plain_attention(st):
    case = st["case"]
    G, M, H, KV, D, P = case["groups"], case["members"], case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    n, Q = G * M, case["q"]
    kf, vf = st["k"][0].view(-1, KV, D), st["v"][0].view(-1, KV, D)
    slots = st["seqs"].long()
    table, ln = st["table"][slots].long(), st["len"][slots].long()
    ptr = st["q_ptr"].long()
    nq = ptr[1:] - ptr[:-1]
    j = torch.arange(Q, device="cuda")
    real = j[None, :] < nq[:, None]                                                # [n, Q]
    q = st["q"][(ptr[:-1, None] + j).clamp(max=st["rows"] - 1)].float()            # [n, Q, H, D]
    q = q.view(n, Q, KV, H // KV, D) * st["scale"]
    pos = ln[:, None] - nq[:, None] + j                                            # position of each query

    def rows(tab, at):                                                             # pool rows of positions `at` of sequences with tables `tab`
        page = torch.gather(tab, 1, (at // P).clamp(max=tab.shape[1] - 1)).clamp(min=0)
        return page * P + at % P

    # scores over the common pages: read once for a group
    ap = torch.arange(st["most_prefix"], device="cuda")[None, :].expand(G, -1)
    rp = rows(table.view(G, M, -1)[:, 0], ap)
    kp, vp = kf[rp].float(), vf[rp].float()                                        # [G, p, KV, D]
    sp = torch.einsum("gmkrd,gpkd->gkmrp", q.view(G, M * Q, KV, H // KV, D), kp)   # [G, KV, M*Q, r, p]
    sp = sp.masked_fill((ap >= st["prefix"][:, None])[:, None, None, None, :], -math.inf)
    sp = sp.reshape(G, KV, M, Q, H // KV, -1).permute(0, 2, 1, 3, 4, 5).reshape(n, KV, Q, H // KV, -1)
    # and over each sequence's own rows
    own_at = st["prefix"].repeat_interleave(M, output_size=n)[:, None] + torch.arange(st["most_suffix"], device="cuda")
    rs = rows(table, own_at)
    ks, vs = kf[rs].float(), vf[rs].float()                                        # [n, s, KV, D]
    ss = torch.einsum("nqkrd,nskd->nkqrs", q, ks)
    ss = ss.masked_fill((own_at[:, None, :] > pos[:, :, None])[:, None, :, None, :], -math.inf)
    s = torch.cat([sp, ss], -1)
    m = s.amax(-1, keepdim=True).clamp(min=-3.0e38)
    e = torch.exp(s - m)
    l = e.sum(-1, keepdim=True)
    e = e / l
    p0 = sp.shape[-1]
    ep = e[..., :p0].reshape(G, M, KV, Q, H // KV, p0).permute(0, 2, 1, 3, 4, 5).reshape(G, KV, M * Q, H // KV, p0)
    o = torch.einsum("gkmrp,gpkd->gmkrd", ep, vp).reshape(n, Q, H, D)
    o = o + torch.einsum("nkqrs,nskd->nqkrd", e[..., p0:], vs).reshape(n, Q, H, D)
    lse = (m + torch.log(l)).squeeze(-1).permute(0, 2, 1, 3).reshape(n, Q, H)
    # padded rows all land in one row behind the last
    to = torch.where(real, ptr[:-1, None] + j, st["rows"]).view(-1)
    out = torch.zeros((st["rows"] + 1, H, D), device="cuda").index_copy_(0, to, o.reshape(n * Q, H, D))[:-1]
    lse = torch.zeros((st["rows"] + 1, H), device="cuda").index_copy_(0, to, lse.reshape(n * Q, H))[:-1]
    return {"out": out.to(st["q"].dtype), "lse": lse, "status": torch.zeros_like(st["status"])}


def _plain_release(st, slots):
    """The pages of these slots are given back, the slots are empty."""
    t = st["table"][slots].long()
    st["refs"].index_add_(0, t.clamp(min=0).view(-1), -(t >= 0).to(torch.int32).view(-1))
    st["table"][slots] = -1
    st["len"][slots] = 0


def _plain_take(st, need):
    """Free pages in ascending order, and where in that order each request's begin."""
    free = st["refs"] == 0
    rank = torch.cumsum(free, 0) - 1
    n = free.numel()
    order = torch.zeros(n + 1, dtype=torch.long, device="cuda")
    order.scatter_(0, torch.where(free, rank, n), torch.arange(n, device="cuda"))
    return order, torch.cumsum(need, 0) - need


def _plain_place(st, shared_of, slots, shared, total, length):
    """Tables of `slots`: `shared` leading pages of the tables `shared_of`, then new pages up to `total`."""
    P = st["table"].shape[1]
    j = torch.arange(P, device="cuda")[None, :]
    order, start = _plain_take(st, total - shared)
    new = order[(start[:, None] + j - shared[:, None]).clamp(0, order.numel() - 1)]
    t = torch.where(j < shared[:, None], shared_of, torch.where(j < total[:, None], new, -1))
    st["refs"].index_add_(0, t.clamp(min=0).view(-1), (t >= 0).to(torch.int32).view(-1))
    st["table"][slots] = t.to(torch.int32)
    st["len"][slots] = length.to(torch.int32)
    return t


def _plain_copy(st, from_row, to_row):
    for x in (st["k"], st["v"]):
        f = x.view(x.shape[0], x.shape[1] * x.shape[2], -1)
        f[:, to_row] = f[:, from_row]


def _plain_fork(st):
    P = st["case"]["page"]
    src, dst = st["src"].long(), st["dst"].long()
    _plain_release(st, dst)
    length, old = st["len"][src].long(), st["table"][src].long()
    total = (length + P - 1) // P
    shared = torch.zeros_like(total) if st["case"]["deep"] else length // P
    new = _plain_place(st, old, dst, shared, total, length)
    if st["moved"]:
        count = length - shared * P
        i = torch.repeat_interleave(torch.arange(src.numel(), device="cuda"), count, output_size=st["moved"])
        at = torch.arange(st["moved"], device="cuda") - (torch.cumsum(count, 0) - count)[i] + shared[i] * P
        _plain_copy(st, old[i, at // P] * P + at % P, new[i, at // P] * P + at % P)
    st["status"].zero_()


def _plain_compact(st):
    P = st["case"]["page"]
    src, dst, ptr, keep = st["src"].long(), st["dst"].long(), st["keep_ptr"].long(), st["keep"].long()
    _plain_release(st, dst)
    old = st["table"][src].long()
    count = ptr[1:] - ptr[:-1]
    i = torch.repeat_interleave(torch.arange(src.numel(), device="cuda"), count, output_size=keep.numel())
    at = torch.arange(keep.numel(), device="cuda") - ptr[:-1][i]
    moves = torch.where(keep != at, at, count[i])                                  # leading rows that stay where they are
    shared = count.scatter_reduce(0, i, moves, "amin") // P
    total = (count + P - 1) // P
    new = _plain_place(st, old, dst, shared, total, count)
    if keep.numel():                                                               # (a row of a shared page is copied onto itself)
        _plain_copy(st, old[i, keep // P] * P + keep % P, new[i, at // P] * P + at % P)
    st["status"].zero_()


def _plain_resize(st, slots, lens):
    P = st["case"]["page"]
    total = (lens + P - 1) // P
    _plain_place(st, st["table"][slots].long(), slots, torch.zeros_like(total), total, lens)


def _plain_write(st):
    P = st["case"]["page"]
    ptr, slots = st["row_ptr"].long(), st["seqs"].long()
    i = torch.repeat_interleave(torch.arange(slots.numel(), device="cuda"), ptr[1:] - ptr[:-1], output_size=st["rows"])
    at = st["start"].long()[i] + torch.arange(st["rows"], device="cuda") - ptr[:-1][i]
    to = st["table"].long()[slots[i], at // P] * P + at % P
    for x, y in ((st["k"], st["k_new"]), (st["v"], st["v_new"])):
        x[0].view(-1, *y.shape[1:]).index_copy_(0, to, y)
    st["status"].zero_()


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    """Attention by its definition, one sequence after the other over its own table; the other operators copy and count."""
    if case["kind"] != "attention":
        return None
    st = prepare(case, seed)
    H, KV, D, P = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    slots, ptr = st["seqs"].tolist(), st["q_ptr"].tolist()
    out = torch.zeros((st["rows"], H, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((st["rows"], H), dtype=torch.float64, device="cuda")
    for i, slot in enumerate(slots):
        n = int(st["len"][slot])
        pages = st["table"][slot, :-(-n // P)].long()
        k = st["k"][0, pages].reshape(-1, KV, D)[:n].double().repeat_interleave(H // KV, 1)
        v = st["v"][0, pages].reshape(-1, KV, D)[:n].double().repeat_interleave(H // KV, 1)
        q = st["q"][ptr[i]:ptr[i + 1]].double()
        s = torch.matmul(q.transpose(0, 1), k.permute(1, 2, 0)) / math.sqrt(D)       # [H, nq, n]
        nq = ptr[i + 1] - ptr[i]
        seen = torch.arange(n, device="cuda")[None, :] <= n - nq + torch.arange(nq, device="cuda")[:, None]
        s = s.masked_fill(~seen, -math.inf)
        lse[ptr[i]:ptr[i + 1]] = torch.logsumexp(s, -1).transpose(0, 1)
        out[ptr[i]:ptr[i + 1]] = torch.matmul(torch.softmax(s, -1), v.transpose(0, 1)).transpose(0, 1)
    return {"out": out, "lse": lse, "status": None}
