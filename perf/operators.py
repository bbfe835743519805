"""Measured cases of the rotary-position and shared-prefix operators, with their plain forms.

Three operators that a decode or prompt step of a model with rotary positions uses one after another:

``rotary``   y = amplitude * R(pos * f) x on the first R dims of every head of q and k; the inverse direction
             (angles negated) is the gradient of the forward one
``append``   the same rotation of q and k with k and v written to their slots of the paged cache on the way
``shared``   single-token attention over the paged cache for a batch in which the sequences of a group share
             the pages of a long prefix

``own`` False computes them from elementary torch operations in 32 bits (angles in 64), True through
``paper_2505_02351_b200.binding``.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    """The cases.  Head shapes and lengths are those of the named workloads (32/8 and 64/8 heads of a short and a
    large decode batch, 32/4 of the long-sequence batch, 8192 new tokens of the chunked prefill)."""
    rot = dict(op="rotary", D=128, R=128, layout="half", dtype="bf16", scaling="none", inverse=False, far=4096)
    app = dict(op="append", D=128, R=128, layout="half", dtype="bf16", scaling="none", bs=16, fused=False, padded=0, far=4096)
    att = dict(op="shared", Hq=32, Hkv=8, D=128, bs=16, loose=0, alibi=False, lens_seed=0)
    return [
        # four streams that each decode one token: the time of a launch
        dict(rot, name="rotary_4_tokens", T=4, Hq=32, Hkv=8),
        # the prompts of a chunked prefill, positions far past the trained length, frequencies scaled by parts
        dict(rot, name="rotary_prompt_8192", T=8192, Hq=32, Hkv=8, scaling="parts", far=131072),
        # the gradient of an interleaved rotation of half of every head, 32-bit training activations, an odd length
        dict(rot, name="rotary_grad_fp32_4095", T=4095, Hq=64, Hkv=8, R=64, layout="interleaved", dtype="fp32", inverse=True),
        # the new tokens of a decode batch of 32
        dict(app, name="append_32_tokens", T=32, Hq=32, Hkv=8, far=2048),
        # the new tokens of a large batch padded to a captured graph's size; long-context ramp
        dict(app, name="append_256_padded", T=256, Hq=64, Hkv=8, bs=32, layout="interleaved", scaling="ramp", padded=7, far=65536),
        # the chunk of a prefill as it comes out of the fused projection (rows of q, k and v side by side)
        dict(app, name="append_chunk_8192", T=8192, Hq=32, Hkv=8, fused=True, far=6144),
        # a 32-bit cache, a quarter of every head rotated, an odd length
        dict(app, name="append_fp32_1999", T=1999, Hq=16, Hkv=4, D=64, R=16, layout="half", dtype="fp32", scaling="linear", far=32768),
        # four short chats behind one instruction: latency
        dict(att, name="shared_4_short", B=4, groups=1, prefix_lo=512, prefix_hi=512, own_lo=1, own_hi=64),
        # the decode batch of 32 behind one prompt whose length is no multiple of a page
        dict(att, name="shared_32_mid", B=32, groups=1, prefix_lo=1500, prefix_hi=1500, own_lo=64, own_hi=548, lens_seed=1),
        # eight questions about one long document
        dict(att, name="shared_8_document", B=8, Hkv=4, groups=1, prefix_lo=32768, prefix_hi=32768, own_lo=256, own_hi=2048,
             alibi=True, lens_seed=2),
        # a large ragged batch over many prompts, some streams that share nothing
        dict(att, name="shared_256_groups", B=256, Hq=64, bs=32, groups=12, prefix_lo=256, prefix_hi=8192, own_lo=16, own_hi=1024,
             loose=20, lens_seed=3),
        # many samples of one prompt: the products bound it
        dict(att, name="shared_128_samples", B=128, groups=1, prefix_lo=16384, prefix_hi=16384, own_lo=16, own_hi=256, alibi=True,
             lens_seed=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "append", "shared", "shared"])
    if op == "shared":
        while True:
            Hq, Hkv = rng.choice([(32, 8), (32, 4), (64, 8), (16, 8), (8, 8), (16, 4)])
            lo = _log_int(rng, 64, 16384)
            own_lo = _log_int(rng, 1, 256)
            B = _log_int(rng, 2, 256)
            c = dict(op=op, B=B, Hq=Hq, Hkv=Hkv, D=rng.choice([64, 128]), bs=rng.choice([16, 32]),
                     groups=min(B, rng.choice([1, 1, 2, 3, 7, 16])), prefix_lo=lo, prefix_hi=lo + rng.choice([0, rng.randrange(1, lo + 1)]),
                     own_lo=own_lo, own_hi=own_lo + rng.randrange(0, 1024), loose=rng.choice([0, 0, 1, 3]),
                     alibi=rng.random() < 0.5, lens_seed=rng.randrange(1 << 20))
            c["loose"] = min(c["loose"], B - c["groups"])
            w = work(c)
            if w["bytes"] <= 4e8 and w["flops"] <= 1.4e11:
                return c
    dtype = rng.choice(["fp32", "bf16", "bf16"])
    D = rng.choice([64, 128])
    c = dict(op=op, T=_log_int(rng, 1, 8192), D=D, R=rng.choice([D, D, D // 2, D // 4, 3 * D // 4, 2 * rng.randrange(1, D // 2)]),
             layout=rng.choice(["half", "interleaved"]), dtype=dtype, scaling=rng.choice(["none", "linear", "ntk", "parts", "ramp"]),
             far=_log_int(rng, 16, 1 << 20))
    c["Hq"], c["Hkv"] = rng.choice([(32, 8), (32, 4), (16, 4), (8, 8), (4, 2)] if dtype == "fp32" else [(32, 8), (32, 4), (64, 8), (16, 4), (8, 8)])
    if op == "rotary":
        c["inverse"] = rng.random() < 0.5
    else:
        c |= dict(bs=rng.choice([16, 32]), fused=rng.random() < 0.5, padded=rng.choice([0, 0, min(3, c["T"] - 1)]))
    return c


# ------------------------------------------------------------------------------------------------- lengths, sizes
def _lengths(c):
    """(sequences of each group, shared tokens of each group, context length of every sequence): part of the case,
    not of the seed.  The last `loose` sequences belong to no group."""
    rng = np.random.default_rng(c["lens_seed"])
    n_in = c["B"] - c["loose"]
    cuts = np.sort(rng.choice(np.arange(1, n_in), size=c["groups"] - 1, replace=False)) if c["groups"] > 1 else np.zeros(0, dtype=np.int64)
    start = np.concatenate([[0], cuts, [n_in]]).astype(np.int64)
    spread = lambda lo, hi, k: np.rint(np.exp(rng.uniform(np.log(lo), np.log(hi), size=k))).astype(np.int64)  # noqa: E731
    prefix = spread(c["prefix_lo"], c["prefix_hi"], c["groups"])
    mine = spread(c["own_lo"], c["own_hi"], c["B"])
    shared = np.concatenate([np.repeat(prefix, np.diff(start)), np.zeros(c["loose"], dtype=np.int64)])
    return start, shared, shared + mine


def _rope(c):
    """Angles per position in radians (64 bits) and the amplitude of the case's scaling."""
    R, base, factor, trained, low, high = c["R"], 10000.0, 8.0, 8192.0, 1.0, 32.0
    i = np.arange(R // 2, dtype=np.float64)
    kind = c["scaling"] if not (c["scaling"] == "ntk" and R == 2) else "linear"
    if kind == "ntk":
        return (base * factor ** (R / (R - 2))) ** (-2.0 * i / R), 1.0, kind
    f = base ** (-2.0 * i / R)
    if kind == "linear":
        return f / factor, 1.0, kind
    if kind == "parts":
        turns = trained * f / (2 * math.pi)
        w = np.clip((turns - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        return f * (w + (1 - w) / factor), 1.0, kind
    if kind == "ramp":
        at = lambda turns: R * math.log(trained / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(at(high)), 0), min(math.ceil(at(low)), R - 1)
        w = 1.0 - np.clip((i - lo) / max(hi - lo, 0.001), 0.0, 1.0)
        return f * (w + (1 - w) / factor), 0.1 * math.log(factor) + 1.0, kind
    return f, 1.0, kind


def work(case):
    c = case
    if c["op"] == "shared":
        start, shared, n = _lengths(c)
        row = 2 * c["Hkv"] * c["D"] * 2
        once = int(shared[start[:-1]].sum())
        keys = once + int((n - shared).sum())
        return {"bytes": keys * row + 2 * c["B"] * c["Hq"] * c["D"] * 2 + 4 * (keys // c["bs"] + 2 * c["B"]),
                "flops": 4 * int(n.sum()) * c["Hq"] * c["D"]}
    es = 4 if c["dtype"] == "fp32" else 2
    heads = c["Hq"] + c["Hkv"] * (2 if c["op"] == "append" else 1)
    return {"bytes": c["T"] * (2 * heads * c["D"] * es + (12 if c["op"] == "append" else 4)) + 4 * c["R"],
            "flops": c["T"] * (c["Hq"] + c["Hkv"]) * 3 * c["R"]}


# ------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    c = dict(case)
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    rng = np.random.default_rng(int(seed))
    if c["op"] == "shared":
        return _prepare_shared(c, gen, rng, dev)
    dt = DTYPES[c["dtype"]]
    T, Hq, Hkv, D = c["T"], c["Hq"], c["Hkv"], c["D"]
    randn = lambda *s: torch.randn(*s, generator=gen, device=dev).to(dt)  # noqa: E731
    f, amplitude, kind = _rope(c)
    st = {"case": c, "freq": torch.from_numpy(f).to(dev), "amplitude": amplitude}
    # every token has a position of its own, as in a batch whose sequences stand at different places
    st["positions"] = torch.from_numpy(rng.integers(0, c["far"], size=T).astype(np.int32)).to(dev)
    if c["op"] == "append" and c["fused"]:
        rows = randn(T, (Hq + 2 * Hkv) * D)
        q, k, v = rows.split([Hq * D, Hkv * D, Hkv * D], dim=1)
        st["q"], st["k"], st["v"] = q.unflatten(1, (Hq, D)), k.unflatten(1, (Hkv, D)), v.unflatten(1, (Hkv, D))
    else:
        st["q"], st["k"] = randn(T, Hq, D), randn(T, Hkv, D)
    st["q_out"] = torch.empty(T, Hq, D, device=dev, dtype=dt)
    if c["op"] == "rotary":
        st["k_out"] = torch.empty(T, Hkv, D, device=dev, dtype=dt)
    else:
        if not c["fused"]:
            st["v"] = randn(T, Hkv, D)
        bs = c["bs"]
        # a chunk fills its pages; the tokens of a decode batch lie in a page each
        pages = max(2, T // bs + 2) if T > 512 else 2 * T
        st["k_cache"], st["v_cache"] = randn(pages, Hkv, bs, D), randn(pages, Hkv, bs, D)
        slots = rng.permutation(pages * bs)[:T] if T <= 512 else (rng.permutation(pages)[:, None] * bs + np.arange(bs)).reshape(-1)[:T]
        slots = slots.astype(np.int64)
        if c["padded"]:
            slots[-c["padded"]:] = -1
        st["slots"] = torch.from_numpy(slots).to(dev)
    if own:
        from paper_2505_02351_b200 import binding
        scale = {"none": {}, "linear": dict(factor=8.0), "ntk": dict(factor=8.0),
                 "parts": dict(factor=8.0, original_len=8192.0, low_turns=1.0, high_turns=4.0),
                 "ramp": dict(factor=8.0, original_len=8192.0, low_turns=1.0, high_turns=32.0)}[kind]
        st["table"] = binding.rotary_table(binding.rotary_frequencies(c["R"], 10000.0, scaling=kind, **scale), dev)
    return st


def _prepare_shared(c, gen, rng, dev):
    start, shared, n = _lengths(c)
    B, Hq, Hkv, D, bs = c["B"], c["Hq"], c["Hkv"], c["D"], c["bs"]
    pages = -(-n // bs)
    whole = shared // bs                                     # pages a sequence shares with its group
    used = int(whole[start[:-1]].sum() + (pages - whole).sum())
    pool = used + used // 8 + 1
    perm = rng.permutation(pool).astype(np.int32)
    table = np.full((B, int(pages.max())), -1, dtype=np.int32)
    cur = 0
    for g in range(c["groups"]):
        k = int(whole[start[g]])
        table[start[g]:start[g + 1], :k] = perm[cur:cur + k]
        cur += k
    for s in range(B):
        k = int(pages[s] - whole[s])
        table[s, whole[s]:pages[s]] = perm[cur:cur + k]
        cur += k
    randn = lambda *s: torch.randn(*s, generator=gen, device=dev).to(torch.bfloat16)  # noqa: E731
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(dev)  # noqa: E731
    st = {"case": c, "q": randn(B, Hq, D), "k_cache": randn(pool, Hkv, bs, D), "v_cache": randn(pool, Hkv, bs, D),
          "table": i32(table), "lens": i32(n), "group_start": i32(start), "prefix_lens": i32(shared),
          "slopes": torch.exp2(-8.0 * torch.arange(1, Hq + 1, device=dev, dtype=torch.float32) / Hq) if c["alibi"] else None,
          "scale": 1.0 / math.sqrt(D), "out": torch.empty(B, Hq, D, device=dev, dtype=torch.bfloat16),
          # what the program that plans the batch knows on the host
          "most": int(np.diff(start).max()), "prefix_pages": int(whole.max()), "own_pages": int((pages - whole).max()),
          "partitions": max(1, -(-int(n.max()) // 512))}
    if own:
        from paper_2505_02351_b200 import binding
        need = binding.shared_workspace_bytes(B, Hq, Hkv, D, c["groups"], st["partitions"])
        st["workspace"] = torch.empty(need, device=dev, dtype=torch.uint8)
    return st


# ------------------------------------------------------------------------------------------------- one pass
def run(state):
    c = state["case"]
    if own:
        return _run_own(state)
    if c["op"] == "shared":
        return _plain_shared(state)
    angle = state["positions"].double()[:, None] * state["freq"]
    cos, sin = (state["amplitude"] * torch.cos(angle)).float(), (state["amplitude"] * torch.sin(angle)).float()
    if c["op"] == "rotary":
        sin = -sin if c["inverse"] else sin
        return [_rotated(state[x], cos, sin, c) for x in ("q", "k")]
    k = _rotated(state["k"], cos, sin, c)
    slots = state["slots"]
    # a padded token repeats the write of the first one that has a slot
    t = torch.where(slots >= 0, torch.arange(c["T"], device=slots.device), (slots >= 0).long().argmax())
    page, off = slots[t] // c["bs"], slots[t] % c["bs"]
    state["k_cache"][page, :, off] = k[t]
    state["v_cache"][page, :, off] = state["v"][t]
    return [_rotated(state["q"], cos, sin, c), state["k_cache"], state["v_cache"]]


def _rotated(x, cos, sin, c):
    R, dt = c["R"], x.dtype
    cos, sin, y = cos[:, None], sin[:, None], x.float()
    a, b = (y[..., :R // 2], y[..., R // 2:R]) if c["layout"] == "half" else (y[..., 0:R:2], y[..., 1:R:2])
    u, w = a * cos - b * sin, b * cos + a * sin
    first = torch.cat([u, w], -1) if c["layout"] == "half" else torch.stack([u, w], -1).flatten(-2)
    return torch.cat([first, y[..., R:]], -1).to(dt)


def _part(scores, v):
    """(maximum, sum of exponentials, weighted sum of v) of a row over its last axis; -inf scores are keys not seen."""
    m = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - m.clamp_min(-1e30))
    return m, p.sum(-1, keepdim=True), p @ v


def _plain_shared(st):
    c = st["case"]
    B, Hq, Hkv, D, bs, N, M = c["B"], c["Hq"], c["Hkv"], c["D"], c["bs"], c["groups"], st["most"]
    G, dev, table, lens = Hq // Hkv, st["q"].device, st["table"].long(), st["lens"].long()
    q = st["q"].float().view(B, Hkv, G, D)
    slope = torch.zeros(Hq, device=dev) if st["slopes"] is None else st["slopes"]
    slope = slope.view(Hkv, G, 1)
    shared = st["prefix_lens"].long() // bs * bs            # the whole pages of the shared tokens
    # the group pass: keys and values of a group gathered once for all its sequences
    first, size = st["group_start"].long()[:-1], st["group_start"].long().diff()
    rows = (first[:, None] + torch.arange(M, device=dev)).clamp_max(B - 1)
    in_group = torch.arange(M, device=dev) < size[:, None]
    pages = table[first, :st["prefix_pages"]].clamp_min(0)
    L = st["prefix_pages"] * bs
    k = st["k_cache"][pages].float().permute(0, 2, 1, 3, 4).reshape(N, Hkv, L, D)
    v = st["v_cache"][pages].float().permute(0, 2, 1, 3, 4).reshape(N, Hkv, L, D)
    j = torch.arange(L, device=dev)
    s = (q[rows].permute(0, 2, 1, 3, 4).reshape(N, Hkv, M * G, D) @ k.transpose(-1, -2)).view(N, Hkv, M, G, L) * st["scale"]
    s -= slope[:, None] * (lens[rows][:, None, :, None, None] - 1 - j)
    s = torch.where(j < shared[rows][:, None, :, None, None], s, -math.inf).view(N, Hkv, M * G, L)
    part = [x.view(N, Hkv, M, G, -1).transpose(1, 2) for x in _part(s, v)]
    del s, k, v
    # back to the sequences: those of no group have seen nothing yet
    at = torch.where(in_group, rows, B).view(-1)
    m1, l1, a1 = (torch.full((B + 1, Hkv, G, x.shape[-1]), fill, device=dev).index_copy_(0, at, x.reshape(N * M, Hkv, G, -1))[:B]
                  for x, fill in zip(part, (-math.inf, 0.0, 0.0)))
    # the own pass: what is left of every sequence
    S = st["own_pages"] * bs
    at = shared[:, None] // bs + torch.arange(st["own_pages"], device=dev)
    pages = table.gather(1, at.clamp_max(table.shape[1] - 1)).clamp_min(0)
    k = st["k_cache"][pages].float().permute(0, 2, 1, 3, 4).reshape(B, Hkv, S, D)
    v = st["v_cache"][pages].float().permute(0, 2, 1, 3, 4).reshape(B, Hkv, S, D)
    j = (shared[:, None] + torch.arange(S, device=dev))[:, None, None]
    n = lens[:, None, None, None]
    s = torch.where(j < n, (q @ k.transpose(-1, -2)) * st["scale"] - slope * (n - 1 - j), -math.inf)
    m2, l2, a2 = _part(s, v)
    m = torch.maximum(m1, m2)
    w1, w2 = torch.exp(m1 - m), torch.exp(m2 - m)
    return ((w1 * a1 + w2 * a2) / (w1 * l1 + w2 * l2)).view(B, Hq, D).to(torch.bfloat16)


def _run_own(st):
    from paper_2505_02351_b200 import binding
    c = st["case"]
    if c["op"] == "shared":
        binding.paged_attention_decode_shared(st["out"], st["q"], st["k_cache"], st["v_cache"], st["table"], st["lens"],
                                              st["group_start"], st["prefix_lens"], st["slopes"], st["scale"], 512,
                                              st["workspace"], st["partitions"])
        return st["out"]
    layout = binding.ROTARY_HALF if c["layout"] == "half" else binding.ROTARY_INTERLEAVED
    if c["op"] == "rotary":
        binding.rotary(st["q_out"], st["q"], st["positions"], st["table"], layout, k_out=st["k_out"], k=st["k"],
                       amplitude=st["amplitude"], inverse=c["inverse"])
        return [st["q_out"], st["k_out"]]
    binding.rotary_append(st["q_out"], st["q"], st["k"], st["v"], st["k_cache"], st["v_cache"], st["slots"], st["positions"],
                          st["table"], layout, amplitude=st["amplitude"])
    return [st["q_out"], st["k_cache"], st["v_cache"]]


# ------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    c = case
    if c["op"] == "shared":
        start, shared, n = _lengths(c)
        G, bs = c["Hq"] // c["Hkv"], c["bs"]
        out = []
        for s in range(c["B"]):                              # every sequence alone, over its whole context
            length = int(n[s])
            ids = st["table"][s, :-(-length // bs)].long()
            k, v = (x[ids].transpose(1, 2).reshape(-1, c["Hkv"], c["D"])[:length].double() for x in (st["k_cache"], st["v_cache"]))
            q = st["q"][s].double().view(c["Hkv"], G, c["D"])
            z = torch.einsum("hgd,jhd->hgj", q, k) * st["scale"]
            if st["slopes"] is not None:
                back = torch.arange(length - 1, -1, -1, device=z.device, dtype=torch.float64)
                z = z - st["slopes"].double().view(c["Hkv"], G, 1) * back
            out.append(torch.einsum("hgj,jhd->hgd", torch.softmax(z, -1), v).reshape(c["Hq"], c["D"]))
        return torch.stack(out)
    # the rotation as a product of complex numbers
    turn = torch.polar(torch.full((1, 1), float(st["amplitude"]), dtype=torch.float64, device="cuda").expand(c["T"], c["R"] // 2).contiguous(),
                       st["positions"].double()[:, None] * st["freq"])
    if c.get("inverse"):
        turn = turn.conj()

    def rotated(x):
        x = x.double()
        y, R = x.clone(), c["R"]
        z = torch.complex(x[..., :R // 2], x[..., R // 2:R]) if c["layout"] == "half" else torch.view_as_complex(x[..., :R].unflatten(-1, (R // 2, 2)).contiguous())
        z = z * turn[:, None]
        if c["layout"] == "half":
            y[..., :R // 2], y[..., R // 2:R] = z.real, z.imag
        else:
            y[..., 0:R:2], y[..., 1:R:2] = z.real, z.imag
        return y

    if c["op"] == "rotary":
        return [rotated(st["q"]), rotated(st["k"])]
    kc, vc = st["k_cache"].double(), st["v_cache"].double()
    live = st["slots"] >= 0
    slot = st["slots"][live]
    kc[slot // c["bs"], :, slot % c["bs"]] = rotated(st["k"])[live]
    vc[slot // c["bs"], :, slot % c["bs"]] = st["v"].double()[live]
    return [rotated(st["q"]), kc, vc]
