"""Measured cases of the chunk attention and of the page operators, with their plain forms.

``chunk``    attention of a few or many new tokens per sequence over the paged cache, causal, with or without ALiBi and a
             local window: drafts to verify, decode rows and prompt chunks in one call
``copy``     whole pages copied inside the pools of all layers
``fork``     sequences continued from others': their pages shared, the part-full last page copied
``resize``   sequences to new lengths: pages dropped, pages given, a shared part-full page copied before it is written
``compact``  the pages in use moved to the front of the pools, tables rewritten

``own`` False computes them from elementary torch operations (scores and sums in 32 bits), True through
``paper_2505_02351_b200.binding``.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    """The cases.  Head shapes, page sizes and lengths are those of the named workloads (32/8 and 64/8 heads of the short and
    the large decode batch, 32/4 of the long-sequence batch, contexts of 16 to 32768 tokens, chunks of up to 2048)."""
    att = dict(op="chunk", Hq=32, Hkv=8, D=128, bs=16, ones=0, q_lo=1, q_hi=1, window=0, alibi=False, fused=False, lens_seed=0)
    pg = dict(layers=32, Hkv=8, D=128, bs=16, dtype="bf16", lens_seed=0)
    return [
        # four short chats, four drafted tokens each: the time of a call
        dict(att, name="chunk_4_drafts", B=4, q_lo=4, q_hi=4, n_lo=60, n_hi=600),
        # the decode batch of 32, up to six tokens to verify per sequence, q as it comes out of the fused projection
        dict(att, name="chunk_32_verify", B=32, q_lo=3, q_hi=6, n_lo=512, n_hi=2048, fused=True, lens_seed=1),
        # long contexts, eight drafts each, ALiBi: the cache has to be read once
        dict(att, name="chunk_8_long", B=8, Hkv=4, q_lo=8, q_hi=8, n_lo=16384, n_hi=32768, alibi=True, lens_seed=2),
        # a step that serves 60 decoding sequences and four prompts' chunks
        dict(att, name="chunk_mixed_64", B=64, Hq=64, bs=32, ones=60, q_lo=300, q_hi=512, n_lo=16, n_hi=8192, lens_seed=3),
        # the last chunk of one long prompt: the products bound it
        dict(att, name="chunk_prompt_end", B=1, q_lo=511, q_hi=511, n_lo=32768, n_hi=32768, alibi=True, lens_seed=4),
        # a local window, heads of 64, an odd number of new tokens
        dict(att, name="chunk_16_window", B=16, Hq=16, D=64, q_lo=33, q_hi=33, n_lo=4096, n_hi=16384, window=1024, lens_seed=5),
        # pages written to another place in the pools of all layers (32 layers, K and V)
        dict(pg, op="copy", name="copy_64_pages", blocks=512, pages=64),
        # one chat continued four ways in a small model
        dict(pg, op="fork", name="fork_4_ways", layers=4, blocks=512, parents=1, children=4, n_lo=541, n_hi=541),
        # many samples of one long prompt in a model of 32 layers
        dict(pg, op="fork", name="fork_128_samples", blocks=1536, parents=1, children=128, n_lo=16383, n_hi=16383),
        # a step of the decode batch: some sequences grow by a token or a few, some end, some begin
        dict(pg, op="resize", name="resize_32_step", layers=4, blocks=4096, S=40, n=32, n_lo=1, n_hi=2048, shared=2, lens_seed=6),
        # the large ragged batch
        dict(pg, op="resize", name="resize_256_step", layers=2, Hkv=2, blocks=32768, S=300, n=256, n_lo=16, n_hi=8192, shared=9, lens_seed=7),
        # pools of which a part is in use, scattered
        dict(pg, op="compact", name="compact_512", blocks=512, S=24, n_lo=16, n_hi=512, lens_seed=8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["chunk"] * 5 + ["copy", "fork", "resize", "compact"])
    if op == "chunk":
        while True:
            Hq, Hkv = rng.choice([(32, 8), (32, 4), (64, 8), (16, 8), (8, 8), (16, 4)])
            B = _log_int(rng, 1, 64)
            q_lo, n_lo = _log_int(rng, 1, 512), _log_int(rng, 1, 16384)
            q_lo = min(q_lo, n_lo)
            c = dict(op=op, Hq=Hq, Hkv=Hkv, D=rng.choice([64, 128, 128]), bs=rng.choice([16, 32]), B=B,
                     ones=rng.choice([0, 0, rng.randrange(B)]), q_lo=q_lo, q_hi=q_lo + rng.choice([0, rng.randrange(q_lo + 1)]),
                     n_lo=n_lo, n_hi=n_lo + rng.choice([0, rng.randrange(n_lo + 1)]), window=rng.choice([0, 0, 0, _log_int(rng, 16, 4096)]),
                     alibi=rng.random() < 0.5, fused=rng.random() < 0.3, lens_seed=rng.randrange(1 << 20))
            w = work(c)
            if w["bytes"] <= 4e8 and w["flops"] <= 2.5e11:
                return c
    c = dict(op=op, D=rng.choice([64, 128]), bs=rng.choice([16, 32]), dtype=rng.choice(["fp32", "bf16", "bf16"]),
             Hkv=rng.choice([1, 2, 4, 8]), layers=_log_int(rng, 1, 32), lens_seed=rng.randrange(1 << 20))
    page = c["Hkv"] * c["bs"] * c["D"] * (4 if c["dtype"] == "fp32" else 2) * 2 * c["layers"]
    blocks = min(32768, int(1.07e9 / page))                     # pools of a gigabyte at most
    if op == "copy":
        c |= dict(blocks=max(2, _log_int(rng, 2, blocks)))
        return c | dict(pages=rng.randrange(1, min(c["blocks"] // 2, int(1.4e8 / page) + 1) + 1))
    if op == "compact":
        n = _log_int(rng, 1, 2048)
        return c | dict(blocks=max(4, min(blocks, int(5e8 / page))), S=_log_int(rng, 1, 256), n_lo=n, n_hi=rng.randrange(n, 2 * n + 1))
    if op == "fork":
        n = _log_int(rng, 1, 16384)
        parents = rng.choice([1, 1, 2, 5])
        children = _log_int(rng, 1, max(1, min(128, int(1.2e8 / page))))
        need = parents * (2 * n // c["bs"] + 1)
        # now and then fewer free pages than children
        return c | dict(blocks=need + max(1, children - rng.choice([0, 0, 0, 2])), parents=parents, children=children, n_lo=n,
                        n_hi=rng.randrange(n, 2 * n + 1)) if (need + children) * page <= 1.5e9 else draw(rng)
    S = _log_int(rng, 2, 300)
    n = _log_int(rng, 1, 8192)
    return c | dict(blocks=max(16, blocks // rng.choice([1, 1, 8])), S=S, n=rng.randrange(1, S + 1), n_lo=n, n_hi=2 * n, shared=rng.choice([0, 1, 5]))


# ------------------------------------------------------------------------------------------------- lengths, sizes
def _spread(rng, lo, hi, k):
    return np.rint(np.exp(rng.uniform(np.log(lo), np.log(hi), size=k))).astype(np.int64)


def _chunk_lens(c):
    """(new tokens, context length) of every sequence: part of the case, not of the seed."""
    rng = np.random.default_rng(c["lens_seed"])
    q = rng.integers(c["q_lo"], c["q_hi"] + 1, size=c["B"])
    q[:c["ones"]] = 1
    return q, np.maximum(_spread(rng, c["n_lo"], c["n_hi"], c["B"]), q)


def _visible(c, q, n):
    """(keys that some row of a sequence sees, pairs of row and key) of a sequence of n tokens, the last q new."""
    pos = np.arange(n - q, n)
    seen = pos + 1 if not c["window"] else np.minimum(pos + 1, c["window"])
    return n - max(0, n - q - c["window"] + 1 if c["window"] else 0), int(seen.sum())


def _es(c):
    return 4 if c["dtype"] == "fp32" else 2


def _pages_plan(c):
    """What the scheduler's side of the page cases holds: tables, lengths, counts and what is asked, on the host."""
    rng = np.random.default_rng(c["lens_seed"])
    nb, bs = c["blocks"], c["bs"]
    if c["op"] == "copy":
        perm = rng.permutation(nb).astype(np.int32)
        k = c["pages"]
        src, dst = perm[:k], perm[k:2 * k]
        if k > 2:
            src[k // 2] = -1                                    # a pair of a captured list that is not in use
        return dict(src=src, dst=dst)
    free = list(rng.permutation(nb).astype(np.int32))
    if c["op"] == "fork":
        P, C = c["parents"], c["children"]
        S = P + C + 1
        lens = np.zeros(S, dtype=np.int32)
        lens[:P] = _spread(rng, c["n_lo"], c["n_hi"], P)
        asked = dict(parents=rng.integers(0, P, size=C).astype(np.int32), children=(P + rng.permutation(C)).astype(np.int32))
        asked["parents"].sort()
        wide = int(-(-lens.max() // bs)) + 1
    else:
        S = c["S"]
        lens = np.zeros(S, dtype=np.int32)
        room = nb
        for s in range(S):                                      # as many as fit into three quarters of the pool
            n = int(_spread(rng, c["n_lo"], c["n_hi"], 1)[0])
            if room - -(-n // bs) < nb // 4:
                continue
            lens[s] = n
            room -= -(-n // bs)
        if c["op"] == "resize":
            seqs = rng.permutation(S)[:c["n"]].astype(np.int32)
            kind, old = rng.random(c["n"]), lens[seqs]
            new = np.where(kind < 0.6, old + rng.integers(1, 7, size=c["n"]), np.where(kind < 0.75, 0, np.where(
                kind < 0.85, old // 2, old + _spread(rng, 1, max(2, c["n_lo"]), c["n"]))))
            wide = int(-(-max(lens.max(), new.max()) // bs)) + 1
            asked = dict(seqs=seqs, new=new.astype(np.int32), old=old.astype(np.int32))
        else:
            wide = int(-(-lens.max() // bs)) + 1
            asked = {}
    table, ref = np.full((S, wide), -1, dtype=np.int32), np.zeros(nb, dtype=np.int32)
    for s in range(S):
        for i in range(-(-int(lens[s]) // bs)):
            table[s, i] = free.pop()
            ref[table[s, i]] += 1
    if c["op"] == "resize":                                     # a few sequences share their pages with another, the last one part full
        for a in range(min(c["shared"], S // 2)):
            s, t = a, S - 1 - a
            if lens[s]:
                k = -(-int(lens[s]) // bs)
                drop = table[t, :-(-int(lens[t]) // bs)]
                ref[drop] -= 1
                table[t] = -1
                table[t, :k], lens[t] = table[s, :k], lens[s]
                ref[table[s, :k]] += 1
        at = {int(s): i for i, s in enumerate(asked["seqs"])}
        for a in range(min(c["shared"], S // 2)):
            if S - 1 - a in at:
                asked["old"][at[S - 1 - a]] = lens[S - 1 - a]
    return dict(asked, table=table, lens=lens, ref=ref)


def work(case):
    c = case
    if c["op"] == "chunk":
        q, n = _chunk_lens(c)
        keys, pairs = (sum(x) for x in zip(*(_visible(c, int(a), int(b)) for a, b in zip(q, n))))
        return {"bytes": keys * 2 * c["Hkv"] * c["D"] * 2 + 2 * int(q.sum()) * c["Hq"] * c["D"] * 2 + 4 * (keys // c["bs"] + 2 * c["B"]),
                "flops": 4 * pairs * c["Hq"] * c["D"]}
    p = _pages_plan(c)
    row = c["Hkv"] * c["D"] * _es(c) * 2 * c["layers"]          # a token's rows in all pools
    if c["op"] == "copy":
        k = int((p["src"] >= 0).sum())
        return {"bytes": 2 * k * row * c["bs"] + 8 * len(p["src"]), "flops": 0}
    if c["op"] == "fork":
        n = p["lens"][p["parents"]]
        pages = -(-n // c["bs"])
        # the children's entries written, the parents' read, a count read and written for each page
        return {"bytes": int((2 * (n % c["bs"]) * row).sum() + 4 * pages.sum() + 12 * (-(-p["lens"] // c["bs"])).sum() + 4 * c["blocks"]), "flops": 0}
    if c["op"] == "resize":
        moved = np.abs(-(-p["new"] // c["bs"]) - -(-p["old"] // c["bs"]))
        return {"bytes": int(16 * moved.sum() + 20 * c["n"] + 4 * c["blocks"]), "flops": 0}
    used = int((p["ref"] > 0).sum())
    moves = int((p["ref"][used:] > 0).sum())
    return {"bytes": 2 * moves * row * c["bs"] + 8 * int((-(-p["lens"] // c["bs"])).sum()) + 12 * c["blocks"], "flops": 0}


# ------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    c = dict(case)
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(dev)  # noqa: E731
    if c["op"] == "chunk":
        return _prepare_chunk(c, gen, np.random.default_rng(int(seed)), dev, i32)
    plan = _pages_plan(c)
    st = {"case": c, "pools": torch.randn(2 * c["layers"], c["blocks"], c["Hkv"], c["bs"], c["D"], generator=gen, device=dev,
                                          dtype=DTYPES[c["dtype"]])}
    for k, a in plan.items():
        st[k] = i32(a)
    if c["op"] != "copy":
        n = len(plan.get("seqs", plan.get("children", ())))
        st["done"] = torch.zeros(n, device=dev, dtype=torch.int32)
        st["turn"] = 0
    if c["op"] == "compact":
        used = int((plan["ref"] > 0).sum())
        st["moves"] = int((plan["ref"][used:] > 0).sum())       # for the plain form
        st["table_out"], st["ref_out"] = torch.empty_like(st["table"]), torch.empty_like(st["ref"])
        st["map"], st["used"] = torch.empty_like(st["ref"]), torch.zeros(1, device=dev, dtype=torch.int32)
    if own:
        from paper_2505_02351_b200 import binding
        st["handle"] = binding.page_pools(list(st["pools"]))
        if c["op"] != "copy":
            need = binding.pages_workspace_bytes(max(1, st["done"].numel()), c["blocks"])
            st["workspace"] = torch.empty(need, device=dev, dtype=torch.uint8)
    return st


def _prepare_chunk(c, gen, rng, dev, i32):
    q, n = _chunk_lens(c)
    B, Hq, Hkv, D, bs = c["B"], c["Hq"], c["Hkv"], c["D"], c["bs"]
    pages = -(-n // bs)
    pool = int(pages.sum()) + int(pages.sum()) // 8 + 1
    perm = rng.permutation(pool).astype(np.int32)
    table = np.full((B, int(pages.max())), -1, dtype=np.int32)
    cur = 0
    for s in range(B):
        table[s, :pages[s]] = perm[cur:cur + pages[s]]
        cur += int(pages[s])
    T = int(q.sum())
    randn = lambda *s: torch.randn(*s, generator=gen, device=dev).to(torch.bfloat16)  # noqa: E731
    rows = randn(T, (Hq + 2 * Hkv) * D if c["fused"] else Hq * D)
    st = {"case": c, "q": rows[:, :Hq * D].unflatten(1, (Hq, D)), "k_cache": randn(pool, Hkv, bs, D), "v_cache": randn(pool, Hkv, bs, D),
          "table": i32(table), "lens": i32(n), "start": i32(np.concatenate([[0], np.cumsum(q)])), "scale": 1.0 / math.sqrt(D),
          "slopes": torch.exp2(-8.0 * torch.arange(1, Hq + 1, device=dev, dtype=torch.float32) / Hq) if c["alibi"] else None,
          "q_lens": [int(x) for x in q], "n": [int(x) for x in n],             # known to the program that plans the batch
          "out": torch.empty(T, Hq, D, device=dev, dtype=torch.bfloat16)}
    if own:
        from paper_2505_02351_b200 import binding
        st["workspace"] = torch.empty(binding.chunk_workspace_bytes(Hq, Hkv, D, int(q.max())), device=dev, dtype=torch.uint8)
    return st


# ------------------------------------------------------------------------------------------------- one pass
def run(state):
    op = state["case"]["op"]
    if own:
        return _run_own(state)
    return {"chunk": _plain_chunk, "copy": _plain_copy, "fork": _plain_fork, "resize": _plain_resize, "compact": _plain_compact}[op](state)


def _run_own(st):
    from paper_2505_02351_b200 import binding
    op = st["case"]["op"]
    if op == "chunk":
        binding.paged_attention_chunk(st["out"], st["q"], st["start"], max(st["q_lens"]), st["k_cache"], st["v_cache"], st["table"],
                                      st["lens"], st["slopes"], st["scale"], st["workspace"], window=st["case"]["window"])
        return st["out"]
    if op == "copy":
        binding.cache_copy_pages(st["handle"], st["src"], st["dst"])
        return st["pools"]
    if op == "fork":
        binding.cache_fork(st["handle"], st["table"], st["lens"], st["ref"], st["parents"], st["children"], st["done"], st["workspace"])
        return [st["pools"], st["table"], st["lens"], st["ref"], st["done"]]
    if op == "resize":
        binding.cache_resize(st["handle"], st["table"], st["lens"], st["ref"], st["seqs"], _asked(st), st["done"], st["workspace"])
        return [st["pools"], st["table"], st["lens"], st["ref"], st["done"]]
    binding.cache_compact(st["handle"], st["table"], st["lens"], st["ref"], st["table_out"], st["ref_out"], st["map"], st["used"],
                          st["workspace"])
    return [st["pools"], st["table_out"], st["ref_out"], st["map"], st["used"]]


def _asked(st):
    """The lengths of this step: there, and in the next step back."""
    st["turn"] += 1
    return st["new"] if st["turn"] % 2 else st["old"]


def _plain_chunk(st):
    c = st["case"]
    Hkv, D, bs = c["Hkv"], c["D"], c["bs"]
    G, out, t0 = c["Hq"] // Hkv, [], 0
    for s, (q, n) in enumerate(zip(st["q_lens"], st["n"])):
        lo = max(0, n - q - c["window"] + 1) // bs * bs if c["window"] else 0
        ids = st["table"][s, lo // bs:-(-n // bs)].long()
        k, v = (x[ids].float().permute(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :n - lo] for x in (st["k_cache"], st["v_cache"]))
        x = st["q"][t0:t0 + q].float().view(q, Hkv, G, D).permute(1, 2, 0, 3).reshape(Hkv, G * q, D)
        z = (x @ k.transpose(1, 2)).view(Hkv, G, q, n - lo) * st["scale"]
        back = torch.arange(n - q, n, device=z.device)[:, None] - torch.arange(lo, n, device=z.device)
        if st["slopes"] is not None:
            z -= st["slopes"].view(Hkv, G, 1, 1) * back
        seen = back >= 0 if not c["window"] else (back >= 0) & (back < c["window"])
        z.masked_fill_(~seen, -math.inf)
        p = torch.exp(z - z.amax(-1, keepdim=True))
        del z
        o = (p.view(Hkv, G * q, -1) @ v) / p.sum(-1).view(Hkv, G * q, 1)
        out.append(o.view(Hkv, G, q, D).permute(2, 0, 1, 3).reshape(q, Hkv * G, D))
        t0 += q
    return torch.cat(out).to(torch.bfloat16)


def _plain_copy(st):
    src, dst = st["src"].long(), st["dst"].long()
    live = (src >= 0) & (dst >= 0)
    t = torch.where(live, torch.arange(len(src), device=src.device), live.long().argmax())      # the others repeat a live pair
    st["pools"][:, dst[t]] = st["pools"][:, src[t]]
    return st["pools"]


def _copy_rows(pools, src, dst, rows):
    """The first `rows` tokens of page src to page dst in every pool (rows 0: nothing)."""
    bs = pools.shape[3]
    live = rows > 0
    t = torch.where(live, torch.arange(len(src), device=src.device), live.long().argmax())
    rows = rows[t]                                              # (all 0 where no pair is live)
    first = (torch.arange(bs, device=src.device) < rows[:, None])[None, :, None, :, None]
    d = torch.where(rows > 0, dst[t], 0)
    pools[:, d] = torch.where(first, pools[:, torch.where(rows > 0, src[t], 0)], pools[:, d])


def _free_pages(ref):
    return torch.sort((ref != 0).to(torch.int8), stable=True).indices, (ref == 0).sum()


def _plain_fork(st):
    c, table, lens, ref = st["case"], st["table"], st["lens"], st["ref"]
    bs, S, W = c["bs"], table.shape[0], table.shape[1]
    p, ch = st["parents"].long(), st["children"].long()
    valid = (p >= 0) & (ch >= 0)
    idx = torch.arange(W, device=ref.device)
    row = torch.where(valid, ch, S)                             # row S is nobody's
    big = torch.cat([table, table.new_full((1, W), -1)])
    n0 = torch.cat([lens, lens.new_zeros(1)])
    held = idx < ((n0[row] + bs - 1) // bs)[:, None]
    ref.index_add_(0, big[row].clamp_min(0).view(-1).long(), -held.view(-1).to(ref.dtype))
    big[row] = torch.where(held, -1, big[row])
    n = torch.where(valid, lens[p.clamp_min(0)], 0)
    need = valid & (n % bs != 0)
    order, there = _free_pages(ref)
    upto = torch.cumsum(need.long(), 0)
    done = valid & (~need | (upto <= there))
    fresh = order[(upto - 1).clamp(0, ref.numel() - 1)]
    whole = (n // bs).long()
    shared = (idx < whole[:, None]) & done[:, None]
    of = table[p.clamp_min(0)]
    ref.index_add_(0, of.clamp_min(0).view(-1).long(), shared.view(-1).to(ref.dtype))
    own_page = done & need
    new = torch.where(shared, of, big[row])
    new = torch.where((idx == whole[:, None]) & own_page[:, None], fresh[:, None].to(new.dtype), new)
    big[row] = new
    ref.index_add_(0, fresh, own_page.to(ref.dtype))
    last = of.gather(1, whole.clamp_max(W - 1)[:, None])[:, 0].long()
    _copy_rows(st["pools"], last, fresh, torch.where(own_page, n % bs, 0).long())
    n0[row] = torch.where(done, n, 0).to(n0.dtype)
    table.copy_(big[:S])
    lens.copy_(n0[:S])
    st["done"].copy_(done)
    return [st["pools"], table, lens, ref, st["done"]]


def _plain_resize(st):
    c, table, lens, ref = st["case"], st["table"], st["lens"], st["ref"]
    bs, S, W, nb = c["bs"], table.shape[0], table.shape[1], ref.numel()
    s, new = st["seqs"].long(), _asked(st).long()
    valid = (s >= 0) & (new >= 0) & (new <= W * bs)
    idx = torch.arange(W, device=ref.device)
    row = torch.where(valid, s, S)
    big = torch.cat([table, table.new_full((1, W), -1)])
    n0 = torch.cat([lens, lens.new_zeros(1)])
    old = n0[row].long()
    have, want = (old + bs - 1) // bs, (new + bs - 1) // bs
    dropped = (idx >= want[:, None]) & (idx < have[:, None]) & valid[:, None]
    mine = big[row]
    ref.index_add_(0, mine.clamp_min(0).view(-1).long(), -dropped.view(-1).to(ref.dtype))
    mine = torch.where(dropped, -1, mine)
    last = mine.gather(1, (have - 1).clamp(0, W - 1)[:, None])[:, 0].long()
    grows = valid & (new > old)
    split = grows & (old % bs != 0) & (ref[last.clamp_min(0)] > 1)
    need = torch.where(grows, want - have + split, 0)
    order, there = _free_pages(ref)
    upto = torch.cumsum(need, 0)
    done = valid & ((need == 0) | (upto <= there))
    given, split = torch.where(done, need, 0), split & done
    first = have - split.long()                                 # the first entry that gets a page
    k = idx - first[:, None]
    gets = (k >= 0) & (k < given[:, None])
    page = order[(upto - need)[:, None].add(k).clamp(0, nb - 1)]
    fresh = order[(upto - need).clamp(0, nb - 1)]
    big[row] = torch.where(gets, page.to(mine.dtype), mine)
    ref.index_add_(0, page.view(-1), gets.view(-1).to(ref.dtype))
    ref.index_add_(0, last.clamp_min(0), -split.to(ref.dtype))
    _copy_rows(st["pools"], last, fresh, torch.where(split, old % bs, 0))
    n0[row] = torch.where(done, new, old).to(n0.dtype)
    table.copy_(big[:S])
    lens.copy_(n0[:S])
    st["done"].copy_(done)
    return [st["pools"], table, lens, ref, st["done"]]


def _plain_compact(st):
    c, table, lens, ref = st["case"], st["table"], st["lens"], st["ref"]
    ids = torch.arange(ref.numel(), device=ref.device)
    used = ref > 0
    U = used.sum()
    mover, hole = used & (ids >= U), ~used & (ids < U)
    holes = torch.sort((~hole).to(torch.int8), stable=True).indices
    page_map = torch.where(mover, holes[(torch.cumsum(mover.long(), 0) - 1).clamp_min(0)], torch.where(used, ids, -1)).to(torch.int32)
    held = torch.arange(table.shape[1], device=ref.device) < ((lens + c["bs"] - 1) // c["bs"])[:, None]
    st["table_out"].copy_(torch.where(held, page_map[table.clamp_min(0).long()], table))
    st["ref_out"].zero_().index_add_(0, page_map.clamp_min(0).long(), torch.where(used, ref, 0))
    m = st["moves"]
    movers = torch.sort((~mover).to(torch.int8), stable=True).indices
    st["pools"][:, holes[:m]] = st["pools"][:, movers[:m]]
    st["map"].copy_(page_map)
    st["used"].copy_(U.view(1))
    return [st["pools"], st["table_out"], st["ref_out"], st["map"], st["used"]]


# ------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    c = case
    if c["op"] != "chunk":
        return None                                             # whole numbers, and values that are copied as they are
    st = prepare(case, seed)
    G, bs, t0, out = c["Hq"] // c["Hkv"], c["bs"], 0, torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    for s, (q, n) in enumerate(zip(st["q_lens"], st["n"])):     # every sequence and head alone, over its whole context
        ids = st["table"][s, :-(-n // bs)].long()
        pos, key = torch.arange(n - q, n, device="cuda"), torch.arange(n, device="cuda")
        unseen = key > pos[:, None]
        if c["window"]:
            unseen |= key <= pos[:, None] - c["window"]
        for h in range(c["Hq"]):
            k, v = (x[ids, h // G].reshape(-1, c["D"])[:n].double() for x in (st["k_cache"], st["v_cache"]))
            z = torch.einsum("td,jd->tj", st["q"][t0:t0 + q, h].double(), k) * st["scale"]
            if st["slopes"] is not None:
                z += st["slopes"][h].double() * (key - pos[:, None])
            out[t0:t0 + q, h] = torch.softmax(z.masked_fill(unseen, -math.inf), -1) @ v
        t0 += q
    return out
