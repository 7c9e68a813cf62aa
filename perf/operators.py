"""Performance cases of the paged 4-bit K/V cache: its pages, its rows, and the
tree-masked verify attention that reads it.

  pages    page_map: pages of the pool handed to growing sequences and taken
           back from shrinking ones, and the slot of every new token
  append   kv4_append and kv4_gather: new K/V rows quantised into the cache at
           their slots, and read back as bf16
  verify   tree_verify_attn_kv4: every node of a draft tree (or, without a
           tree, every query row) against the cache

A cache row is one token of one kv head: 128 E2M1 codes and a power-of-two
scale (an exponent byte with bias 127) for each 32 dimensions, for K and for V.
Keys and values are N(0, 1) with a few wide channels in K; pages of the pool
are in random order and hold older rows where no sequence owns them; page
sizes, lengths and trees are those that a server meets.

With `own` false, `run` computes the operators' plain form: elementary torch
operations in 32 bits, rounded once to bf16 at the end.
"""
import math

import torch

own = False

D = 128       # head dimension
GROUP = 32    # dimensions that share one scale
# The value of each E2M1 code.
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def _verify(name, B, L, Hq, Hkv, W, S, page, ragged=False):
    c = dict(kind="verify", B=B, L=L, Hq=Hq, Hkv=Hkv, W=W, S=S, page=page, ragged=ragged)
    return dict(c, name=name) if name else c


def _append(name, B, N, Hkv, page, accepted):
    c = dict(kind="append", B=B, N=N, Hkv=Hkv, page=page, accepted=accepted)
    return dict(c, name=name) if name else c


def _pages(name, B, L, N, page, ending):
    c = dict(kind="pages", B=B, L=L, N=N, page=page, ending=ending)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One short chat turn with full multi-head attention, one token at a
        # time (W = 0: no tree): launches and memory round trips count.
        _verify("decode_b1_l517_mha32", 1, 517, 32, 32, 0, 0, 16),
        # One user, a few thousand tokens, grouped heads, a tree of 44 nodes.
        _verify("verify_b1_l4096_gqa32x8", 1, 4096, 32, 8, 4, 10, 64),
        # The benchmark's batch: 16 sequences at 8k tokens, trees of 52 nodes.
        _verify("verify_b16_l8192_gqa32x8", 16, 8192, 32, 8, 4, 12, 64),
        # Single-token decoding of a served batch: one pass over the cache.
        _verify("decode_b32_l8192_gqa32x8", 32, 8192, 32, 8, 0, 0, 64),
        # One copied chain of 16 nodes (prompt lookup), pages of 32.
        _verify("verify_b32_l4096_chain16_gqa32x8", 32, 4096, 32, 8, 1, 15, 32),
        # A live server: every sequence at another length and tree size, an
        # odd capacity, 7 query heads per kv head, pages of 16.
        _verify("verify_b24_l6007_ragged_gqa28x4", 24, 6007, 28, 4, 5, 6, 16, True),
        # Long documents, 64 heads over 8, 72 nodes: the largest.
        _verify("verify_b8_l32768_gqa64x8", 8, 32768, 64, 8, 8, 8, 128),
        # The end of an iteration: the accepted nodes (up to 13 of 52) of 16
        # sequences move into the cache.
        _append("append_b16_t52_accepted", 16, 52, 8, 64, 13),
        # Prompts enter: every row of 16 x 2048 tokens.
        _append("append_b16_n2048_prompt", 16, 2048, 8, 64, 0),
        # The same for 4 kv heads, odd lengths and small pages.
        _append("append_b5_n6007_prompt", 5, 6007, 4, 16, 0),
        # A decoding iteration of 64 sequences: up to 13 tokens each, a few
        # sequences end and give their pages back.
        _pages("pages_b64_l2048_decode", 64, 2048, 13, 16, 4),
        # A batch of prompts is admitted while others end.
        _pages("pages_b24_l8192_prompts", 24, 8192, 8192, 64, 8),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    top = work(listed()[6])
    while True:
        kind = rng.choice(["verify"] * 4 + ["append", "append", "pages"])
        page = rng.choice([16, 32, 64, 128, 256])
        if kind == "verify":
            Hq, Hkv = rng.choice([(32, 32), (32, 8), (40, 8), (64, 8), (28, 4), (16, 16), (8, 2)])
            W, S = rng.choice([(0, 0), (0, 0), (1, 15), (rng.randint(1, 8), rng.randint(0, 16))])
            c = _verify(None, _log_int(rng, 1, 64), _log_int(rng, 64, 32768), Hq, Hkv, W, S, page, rng.random() < 0.6)
            w = work(c)
            if w["bytes"] > top["bytes"] or w["flops"] > top["flops"]:
                continue
        elif kind == "append":
            Hkv = rng.choice([2, 4, 8, 16, 32])
            if rng.random() < 0.5:
                T = _log_int(rng, 1, 136)
                c = _append(None, _log_int(rng, 1, 64), T, Hkv, page, rng.randint(1, min(T, 17)))
            else:
                c = _append(None, _log_int(rng, 1, 16), _log_int(rng, 17, 6000), Hkv, page, 0)
        else:
            B, L = _log_int(rng, 1, 256), _log_int(rng, 64, 32768)
            N = rng.choice([rng.randint(1, 17), min(L, _log_int(rng, 64, 8192))])
            c = _pages(None, B, L, N, page, rng.randint(0, B // 2))
            if B * max(N, L) > 1 << 21:
                continue
        return c


# ---------------------------------------------------------------------- sizes

def _lens(c):
    """Context lengths: all L, or from a third of L to L in a fixed order."""
    B, L = c["B"], c["L"]
    if not c["ragged"]:
        return [L] * B
    return [L - (b * 40503 + 977) % 65536 * (2 * L // 3) // 65536 for b in range(B)]


def _tree(c):
    """(rows of the call, node counts): W branches of S + 1 nodes, in a ragged
    batch some branches shorter; without a tree one query row."""
    if c["W"] == 0:
        return 1, [1] * c["B"]
    T = c["W"] * (c["S"] + 1)
    return T, [max(1, T - (b * 5 % 4) * T // 5) if c["ragged"] else T for b in range(c["B"])]


def _adds(c):
    """Rows that each sequence appends: 1 to `accepted` nodes, or the prompt."""
    if c["accepted"]:
        return [1 + (5 * b + 3) % c["accepted"] for b in range(c["B"])]
    return [c["N"] - (b * 37) % (c["N"] // 4 + 1) for b in range(c["B"])]


def _page_lens(c):
    """(lens before, lens after): most sequences grow by up to N, the first
    `ending` end."""
    B, L, N = c["B"], c["L"], c["N"]
    old, new = [], []
    for b in range(B):
        held = (b * 40503 + 977) % 65536 * max(L - N, 0) // 65536
        if b < c["ending"]:
            held = max(held, L // 3)
        old.append(held)
        new.append(0 if b < c["ending"] else min(L, held + 1 + (b * 30011 + 12345) % 65536 * N // 65536))
    return old, new


def work(case):
    c = case
    if c["kind"] == "verify":
        T_max, counts = _tree(c)
        lens = _lens(c)
        row = D // 2 + D // GROUP
        by = fl = 0
        for L, T in zip(lens, counts):
            by += 2 * row * L * c["Hkv"] + 2 * 2 * D * T * c["Hq"] + 4 * T * c["Hq"] + 4 * -(-L // c["page"]) + 8
            fl += 4 * D * L * T * c["Hq"]
            if c["W"]:
                by += 2 * 2 * D * T * c["Hkv"] + 8 * T * -(-T_max // 64)
                fl += 4 * D * c["Hq"] * sum(min(u % (c["S"] + 1) + 1, T) for u in range(T))
        return {"bytes": by, "flops": fl}
    if c["kind"] == "append":
        # bf16 in, codes out, codes in, bf16 out, and a few operations a value
        rows = sum(_adds(c)) * c["Hkv"] * 2
        return {"bytes": rows * 2 * (2 * D + D // 2 + D // GROUP) + 8 * c["B"] * c["N"], "flops": rows * D * 6}
    old, new = _page_lens(c)
    pages = sum(abs(-(-n // c["page"]) - -(-o // c["page"])) for o, n in zip(old, new))
    used = sum(-(-n // c["page"]) - o // c["page"] for o, n in zip(old, new) if n > o)
    return {"bytes": 12 * c["B"] + 8 * pages + 4 * used + 4 * c["B"] * c["N"], "flops": 4 * c["B"] * c["N"]}


# --------------------------------------------------------------------- inputs

def _quantise(x):
    """x float32 [..., D] -> (code 0..15 as int32 [..., D], exponent byte as
    int32 [..., D / GROUP]).  The scale of a group is the power of two X with
    amax < 7 X that is smallest, from the exponent of amax; a value is rounded to the
    nearest multiple that E2M1 holds (ties to the even code), at most 6 X."""
    g = x.view(*x.shape[:-1], D // GROUP, GROUP)
    bits = g.abs().amax(-1).view(torch.int32) >> 16        # of a bf16
    e = (((bits + 0x20) >> 7) - 2).clamp(1, 252)
    y = g.abs() / (e << 23).view(torch.float32).unsqueeze(-1)
    y = torch.where(y < 2, torch.round(y * 2) / 2, torch.where(y < 4, torch.round(y), torch.round(y / 2) * 2)).clamp(max=6)
    code = torch.where(y < 2, y * 2, torch.where(y < 4, y + 2, y / 2 + 4)).to(torch.int32)
    code = code + 8 * torch.signbit(g).to(torch.int32)
    return code.view(x.shape), e


def _values(code, e):
    """The float32 values of codes [..., D] with exponent bytes [..., D / GROUP]."""
    table = torch.tensor(E2M1, dtype=torch.float32, device=code.device)
    v = table[code.long()].view(*e.shape, GROUP)
    return (v * (e.to(torch.int32) << 23).view(torch.float32).unsqueeze(-1)).view(code.shape)


def _unpack(codes):
    """uint8 [..., D / 2] -> codes [..., D]: the even dimension is the low half."""
    return torch.stack((codes & 15, codes >> 4), -1).flatten(-2)


def _pool(n_pages, Hkv, page, gen, wide):
    """Codes and scales of a pool of pages full of rows."""
    codes = torch.empty((n_pages, Hkv, page, D // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((n_pages, Hkv, page, D // GROUP), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 24) // (Hkv * page * D))
    for p in range(0, n_pages, step):
        n = min(step, n_pages - p)
        x = torch.randn((n, Hkv, page, D), generator=gen, device="cuda")
        if wide:
            x[..., ::37] *= 3.0
        code, e = _quantise(x.to(torch.bfloat16).float())
        codes[p:p + n] = (code[..., ::2] | (code[..., 1::2] << 4)).to(torch.uint8)
        scales[p:p + n] = e.to(torch.uint8)
    return codes, scales


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    bf = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    B, page = c["B"], c["page"]
    s = {"case": c}
    if c["kind"] == "verify":
        T_max, counts = _tree(c)
        lens = _lens(c)
        held = [-(-L // page) for L in lens]
        max_pages = -(-c["L"] // page)
        n_pages = sum(held) + 3
        order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
        table = torch.full((B, max_pages), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(held):
            table[b, :n] = order[at:at + n]
            at += n
        s["k_codes"], s["k_scales"] = _pool(n_pages, c["Hkv"], page, gen, True)
        s["v_codes"], s["v_scales"] = _pool(n_pages, c["Hkv"], page, gen, False)
        s.update(page_table=table, lens=i32(lens), node_count=i32(counts), q=bf(B, T_max, c["Hq"], D),
                 k_tree=None, v_tree=None, tree_mask=None,
                 out=torch.zeros((B, T_max, c["Hq"], D), dtype=torch.bfloat16, device="cuda"),
                 lse=torch.zeros((B, c["Hq"], T_max), device="cuda"))
        if c["W"]:
            s["k_tree"], s["v_tree"] = bf(B, T_max, c["Hkv"], D), bf(B, T_max, c["Hkv"], D)
            # chains of S + 1 nodes: a node sees itself and the nodes before it in its chain
            u = torch.arange(T_max, device="cuda")
            sees = (u[:, None] // (c["S"] + 1) == u // (c["S"] + 1)) & (u <= u[:, None])
            nw = -(-T_max // 64)
            bits = torch.zeros((T_max, nw * 64), dtype=torch.int64, device="cuda")
            bits[:, :T_max] = sees
            words = (bits.view(T_max, nw, 64) << torch.arange(64, device="cuda")).sum(-1)
            s["tree_mask"] = words.expand(B, T_max, nw).contiguous()
    elif c["kind"] == "append":
        N, Hkv, adds = c["N"], c["Hkv"], _adds(c)
        R = max(adds)
        n_pages = -(-sum(adds) // page) + 2
        order = torch.randperm(n_pages * page, generator=gen, device="cuda").to(torch.int32)
        if not c["accepted"]:   # a prompt fills whole pages in order
            order = (torch.randperm(n_pages, generator=gen, device="cuda")[:, None] * page
                     + torch.arange(page, device="cuda")).flatten().to(torch.int32)
        slots = torch.full((B, R), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(adds):
            slots[b, :n] = order[at:at + n]
            at += n
        rows = None
        if c["accepted"]:       # the accepted path of each tree, by depth
            rows = torch.rand((B, N), generator=gen, device="cuda").argsort(1)[:, :R].sort(1).values.to(torch.int32)
            rows = rows.contiguous()
        k = torch.randn((B, N, Hkv, D), generator=gen, device="cuda")
        k[..., ::37] *= 3.0
        pool = lambda n: torch.zeros((n_pages, Hkv, page, n), dtype=torch.uint8, device="cuda")  # noqa: E731
        s.update(k_new=k.to(torch.bfloat16), v_new=bf(B, N, Hkv, D), rows=rows, slot_map=slots,
                 k_codes=pool(D // 2), k_scales=pool(D // GROUP), v_codes=pool(D // 2), v_scales=pool(D // GROUP),
                 k_out=torch.zeros((B, R, Hkv, D), dtype=torch.bfloat16, device="cuda"),
                 v_out=torch.zeros((B, R, Hkv, D), dtype=torch.bfloat16, device="cuda"))
    else:
        old, new = _page_lens(c)
        max_pages = -(-c["L"] // page)
        held = [-(-o // page) for o in old]
        want = sum(max(-(-n // page) - h, 0) for n, h in zip(new, held))
        n_pages = sum(held) + want + 5
        order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
        table = torch.full((B, max_pages), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(held):
            table[b, :n] = order[at:at + n]
            at += n
        free = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
        free[:n_pages - at] = order[at:]
        s.update(lens_old=i32(old), lens_new=i32(new), page_table=table, free_pages=free, free_count=i32([n_pages - at]),
                 free_count_out=i32([0]), slot_map=torch.empty((B, c["N"]), dtype=torch.int32, device="cuda"),
                 granted=torch.empty(B, dtype=torch.int32, device="cuda"))
    return s


# ------------------------------------------------------------ the plain forms

def _plain_verify(s):
    c = s["case"]
    B, T_max, Hq, _ = s["q"].shape
    page, Hkv = c["page"], c["Hkv"]
    G = Hq // Hkv
    table = s["page_table"].clamp(min=0).long()
    Lp = table.shape[1] * page

    def context(codes, scales):   # [B, Hkv, Lp, D]
        v = _values(_unpack(codes[table]), scales[table])
        return v.transpose(1, 2).reshape(B, Hkv, Lp, D)

    k, v = context(s["k_codes"], s["k_scales"]), context(s["v_codes"], s["v_scales"])
    seen = torch.arange(Lp, device="cuda") < s["lens"][:, None]
    seen = seen[:, None, :].expand(B, T_max, Lp)
    if s["k_tree"] is not None:
        u = torch.arange(T_max, device="cuda")
        bit = (s["tree_mask"][:, :, u // 64] >> (u % 64)) & 1
        seen = torch.cat((seen, (bit != 0) & (u < s["node_count"][:, None, None])), -1)
        k = torch.cat((k, s["k_tree"].float().transpose(1, 2)), 2)
        v = torch.cat((v, s["v_tree"].float().transpose(1, 2)), 2)
    q = s["q"].float().view(B, T_max, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * T_max, D)
    z = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(D))
    z = z.view(B, Hkv, G, T_max, -1).masked_fill_(~seen[:, None, None], -math.inf)
    m = z.amax(-1, keepdim=True)
    z.sub_(m).exp_()
    total = z.sum(-1, keepdim=True)
    o = torch.matmul(z.view(B, Hkv, G * T_max, -1), v).view(B, Hq, T_max, D) / total.view(B, Hq, T_max, 1)
    lse = (m + torch.log(total)).view(B, Hq, T_max)
    live = torch.arange(T_max, device="cuda") < s["node_count"][:, None]
    out = torch.where(live[:, :, None, None], o.transpose(1, 2).to(torch.bfloat16), s["out"])
    return {"out": out, "lse": torch.where(live[:, None], lse, s["lse"])}


def _plain_append(s):
    slots = s["slot_map"]
    B, R = slots.shape
    rows = s["rows"] if s["rows"] is not None else torch.arange(R, device="cuda").expand(B, R)
    at = rows.long()[:, :, None, None].expand(B, R, s["k_new"].shape[2], D)
    live = (slots >= 0)[:, :, None, None]

    def stored(x, empty):
        v = _values(*_quantise(x.gather(1, at).float()))
        return torch.where(live, v.to(torch.bfloat16), empty)

    return {"k": stored(s["k_new"], s["k_out"]), "v": stored(s["v_new"], s["v_out"])}


def _plain_pages(s):
    c = s["case"]
    page, N = c["page"], c["N"]
    table, free = s["page_table"], s["free_pages"]
    B, max_pages = table.shape
    n_pages = free.shape[0]
    top = max_pages * page
    old, new = s["lens_old"].clamp(0, top).long(), s["lens_new"].clamp(0, top).long()
    held, want = (old + page - 1) // page, (new + page - 1) // page
    back, need = (held - want).clamp(min=0), (want - held).clamp(min=0)
    count = s["free_count"].long()
    i = torch.arange(max_pages, device="cuda")
    # the pages given back go on top of the stack, by sequence and index
    ends = (i >= want[:, None]) & (i < held[:, None])
    to = count + (back.cumsum(0) - back)[:, None] + i - want[:, None]
    stack = torch.cat((free, free.new_zeros(1)))
    stack = stack.scatter(0, torch.where(ends, to, n_pages).flatten(), table.flatten())[:n_pages]
    count = count + back.sum()
    # sequence b is served if the needs up to and including it fit
    upto = need.cumsum(0)
    granted = (upto <= count) | (need == 0)
    take = (i >= held[:, None]) & (i < want[:, None]) & granted[:, None]
    rank = (upto - need)[:, None] + i - held[:, None]
    table = torch.where(take, stack[torch.where(take, count - 1 - rank, 0)], table)
    count = count - torch.where(granted, need, 0).sum()
    p = old[:, None] + torch.arange(N, device="cuda")
    slot = table.gather(1, (p // page).clamp(max=max_pages - 1)) * page + p % page
    slot = torch.where((p < new[:, None]) & granted[:, None], slot, -1)
    return {"page_table": table, "free_pages": stack, "free_count": count.to(torch.int32),
            "slot_map": slot.to(torch.int32), "granted": granted.to(torch.int32)}


def run(state):
    s = state
    kind = s["case"]["kind"]
    if not own:
        return {"verify": _plain_verify, "append": _plain_append, "pages": _plain_pages}[kind](s)
    import paper_2606_05742_amd as adapld
    if "cache" not in s:   # the handle and the workspace are kept, as a decoding loop keeps them
        s["cache"] = adapld.Kv4Cache(**{k: s.get(k) for k in ("k_codes", "k_scales", "v_codes", "v_scales", "page_table",
                                                              "free_pages", "free_count")}, page_size=s["case"]["page"])
    cache = s["cache"]
    if kind == "verify":
        if "ws" not in s:
            B, T_max, Hq, _ = s["q"].shape
            need = adapld.workspace_bytes(adapld.OP_TREE_VERIFY_ATTN_KV4, B, s["case"]["L"], 0, 0, T_max, Hq,
                                          s["case"]["Hkv"], D)
            s["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        out, lse = adapld.tree_verify_attn_kv4(s["q"], cache, s["lens"], s["node_count"], k_tree=s["k_tree"],
                                               v_tree=s["v_tree"], tree_mask=s["tree_mask"], L_max=s["case"]["L"],
                                               out=s["out"], lse=s["lse"], ws=s["ws"])
        return {"out": out, "lse": lse}
    if kind == "append":
        adapld.kv4_append(cache, s["k_new"], s["v_new"], s["slot_map"], rows=s["rows"])
        k, v = adapld.kv4_gather(cache, s["slot_map"], k_out=s["k_out"], v_out=s["v_out"])
        return {"k": k, "v": v}
    slots, granted = adapld.page_map(cache, s["lens_old"], s["lens_new"], slot_map=s["slot_map"], granted=s["granted"],
                                     free_count_out=s["free_count_out"])
    return {"page_table": s["page_table"], "free_pages": s["free_pages"], "free_count": s["free_count_out"],
            "slot_map": slots, "granted": granted}


# ------------------------------------------------- the definition, in 64 bits

def exact(case, seed):
    c = case
    s = prepare(c, seed)
    f64 = torch.float64
    value = torch.tensor(E2M1, dtype=f64, device="cuda")
    if c["kind"] == "verify":
        B, T_max, Hq, _ = s["q"].shape
        Hkv, page = c["Hkv"], c["page"]
        G = Hq // Hkv
        out, lse = s["out"].to(f64), s["lse"].to(f64)
        lens, counts = _lens(c), _tree(c)[1]

        def rows(codes, scales, pages, g, L):
            byte = codes[pages, g].reshape(-1, D // 2)[:L].long()
            v = value[torch.stack((byte % 16, byte // 16), -1).reshape(L, D)]
            e = scales[pages, g].reshape(-1, D // GROUP)[:L].to(f64) - 127
            return v * torch.exp2(e).repeat_interleave(GROUP, 1)

        for b in range(B):
            L, T = lens[b], counts[b]
            pages = s["page_table"][b, :-(-L // page)].long()
            chain = [[v for v in range(u - u % (c["S"] + 1), u + 1)] for u in range(T)] if c["W"] else [[]] * T
            hide = torch.ones((T, T), dtype=torch.bool)
            for u, seen in enumerate(chain):
                hide[u, seen] = False
            hide = hide.cuda()
            for g in range(Hkv):
                k, v = rows(s["k_codes"], s["k_scales"], pages, g, L), rows(s["v_codes"], s["v_scales"], pages, g, L)
                if c["W"]:
                    k = torch.cat((k, s["k_tree"][b, :T, g].to(f64)))
                    v = torch.cat((v, s["v_tree"][b, :T, g].to(f64)))
                for h in range(g * G, g * G + G):
                    z = s["q"][b, :T, h].to(f64) @ k.T / math.sqrt(D)
                    if c["W"]:
                        z[:, L:][hide] = -math.inf
                    m = z.max(1, keepdim=True).values
                    w = torch.exp(z - m)
                    t = w.sum(1, keepdim=True)
                    out[b, :T, h] = w @ v / t
                    lse[b, h, :T] = (m + torch.log(t))[:, 0]
        return {"out": out, "lse": lse}
    if c["kind"] == "append":
        B, R = s["slot_map"].shape
        res = {}
        magnitudes = value[:8]
        for name, x in (("k", s["k_new"]), ("v", s["v_new"])):
            o = s["k_out"].to(f64)
            for b, n in enumerate(_adds(c)):
                at = s["rows"][b, :n].long() if s["rows"] is not None else torch.arange(n, device="cuda")
                g = x[b, at].to(f64).reshape(n, -1, D // GROUP, GROUP)
                # X = 2^(k - 2) for amax in [2^k, 1.75 2^k), 2^(k - 1) from there on
                m, ex = torch.frexp(g.abs().amax(-1, keepdim=True))
                X = torch.exp2((ex - 3 + (m >= 0.875)).clamp(-126, 125).to(f64))
                y = g.abs() / X
                best, off = torch.zeros_like(y), y.clone()
                for j in range(1, 8):   # an even code wins a tie: codes come in ascending order
                    d = (y - magnitudes[j]).abs()
                    win = (d < off) | ((d == off) & (j % 2 == 0))
                    best, off = torch.where(win, magnitudes[j], best), torch.where(win, d, off)
                o[b, :n] = (torch.sign(g) * best * X).reshape(n, -1, D)
            res[name] = o
        return res
    # the stack of free pages, one sequence after another
    old, new = _page_lens(c)
    page, N = c["page"], c["N"]
    table, stack, held = s["page_table"].tolist(), s["free_pages"].tolist(), int(s["free_count"])
    slots, granted = [[-1] * N for _ in old], []
    for b, (o, n) in enumerate(zip(old, new)):
        for i in range(-(-n // page), -(-o // page)):
            stack[held] = table[b][i]
            held += 1
    asked, left = 0, held
    for b, (o, n) in enumerate(zip(old, new)):
        need = max(-(-n // page) - -(-o // page), 0)
        asked += need
        granted.append(int(asked <= held or need == 0))
        if granted[b]:
            for i in range(need):
                left -= 1
                table[b][-(-o // page) + i] = stack[left]
            for i in range(min(N, max(n - o, 0))):
                slots[b][i] = table[b][(o + i) // page] * page + (o + i) % page
    t = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return {"page_table": t(table), "free_pages": t(stack), "free_count": t([left]), "slot_map": t(slots),
            "granted": t(granted)}
