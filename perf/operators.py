"""The operators of the 4-bit paged cache, each in a plain form of elementary torch operations and as a call of the
framework: page tables and slot maps from request lengths, storing prompts and committing accepted paths in 4 bits, and
tree attention over that cache.

The cache's format.  32 neighbouring elements of a token's head share a scale s = (8 + m) 2^(e - 23), a byte 8 e + m with
m < 8 and e < 32; an element is q s with a whole number -8 <= q <= 7 (halves are
rounded away from zero).  A page holds 128 tokens; a layer's pool is
u8 [pages, Hkv, 2 (K and V), 128 (D/2 + D/32)]: the codes q + 8 [128, D/2], then the scales [128, D/32].  In the four bytes
of eight neighbouring elements, the even ones take the lower 16 bits, the odd ones the upper, lowest element lowest."""
import math

import numpy as np
import torch

own = False

PAGE = 128
_SIGMA = 0.6     # of the logarithm of the lengths


# ------------------------------------------------------------------------------------------------- the cases

def listed():
    return [
        # pages and slots of one decode step: every sequence of a running batch takes the room of a full path
        {"name": "pages of a step", "op": "plan", "B": 256, "median": 1500, "most": 8192, "add": 5, "finished": 0},
        # admission of a large batch of prompts beside running sequences, some of which have finished
        {"name": "pages of prompts", "op": "plan", "B": 1021, "median": 700, "most": 4000, "add": 1000, "finished": 100},
        # a handful of tokens into one layer's cache
        {"name": "store few tokens", "op": "store", "T": 37, "Hkv": 2, "D": 64, "skipped": 3},
        # the prompts of a batch into one layer's cache
        {"name": "store prompts", "op": "store", "T": 98304, "Hkv": 8, "D": 128, "skipped": 0},
        # the accepted paths of a round, a long tail of few sequences with large trees
        {"name": "commit few", "op": "commit", "B": 8, "N": 64, "K": 4, "Hkv": 4, "D": 128, "layers": 28, "median": 1000},
        # ... and of a full batch
        {"name": "commit batch", "op": "commit", "B": 256, "N": 16, "K": 4, "Hkv": 2, "D": 128, "layers": 28, "median": 600},
        # a smallest layer, one empty cache and one of a single token among the sequences
        {"name": "attention tiny", "op": "attn", "B": 4, "N": 8, "Hq": 4, "Hkv": 2, "D": 64, "median": 130, "most": 256, "edge": True},
        # plain decoding, one token a sequence
        {"name": "attention one token", "op": "attn", "B": 256, "N": 1, "Hq": 12, "Hkv": 2, "D": 128, "median": 1500, "most": 8192,
         "edge": False},
        # plain decoding at the end of a rollout: few sequences, long ones
        {"name": "attention long tail", "op": "attn", "B": 8, "N": 1, "Hq": 28, "Hkv": 4, "D": 128, "median": 20011, "most": 40000,
         "edge": False},
        # a verification layer with small trees for a full batch
        {"name": "attention small trees", "op": "attn", "B": 256, "N": 8, "Hq": 28, "Hkv": 4, "D": 128, "median": 2000, "most": 8192,
         "edge": False},
        # ... with medium trees
        {"name": "attention trees", "op": "attn", "B": 256, "N": 16, "Hq": 12, "Hkv": 2, "D": 128, "median": 1500, "most": 8192,
         "edge": False},
        # ... with large trees
        {"name": "attention large trees", "op": "attn", "B": 64, "N": 48, "Hq": 40, "Hkv": 8, "D": 128, "median": 4000, "most": 16384,
         "edge": False},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["plan", "store", "commit", "attn", "attn", "attn"])
    if op == "plan":
        B = _log(rng, 1, 1024)
        return {"op": "plan", "B": B, "median": _log(rng, 1, 4000), "most": 8192, "add": _log(rng, 1, 1000),
                "finished": rng.randint(0, B // 4)}
    heads = rng.choice([(4, 2), (12, 2), (28, 4), (40, 8), (8, 8), (16, 1)])
    D = rng.choice([64, 128])
    if op == "store":
        T = _log(rng, 1, 65536)
        return {"op": "store", "T": T, "Hkv": heads[1], "D": D, "skipped": rng.randint(0, min(20, T // 2))}
    if op == "commit":
        N = rng.randint(6, 64)
        return {"op": "commit", "B": _log(rng, 1, 256), "N": N, "K": rng.randint(1, 5), "Hkv": min(heads[1], 4), "D": D,
                "layers": rng.randint(1, 28), "median": _log(rng, 100, 600)}
    case = {"op": "attn", "B": _log(rng, 1, 256), "N": _log(rng, 1, 64), "Hq": heads[0], "Hkv": heads[1], "D": D,
            "median": _log(rng, 1, 16000), "most": 0, "edge": rng.random() < 0.5}
    top = work(listed()[-1])

    def too_much():
        case["most"] = max(1, 4 * case["median"])
        w = work(case)
        return w["bytes"] > 0.8 * top["bytes"] or w["flops"] > 0.8 * top["flops"] or case["B"] * case["median"] * heads[1] > 2 << 20

    while too_much():
        case["B"], case["median"] = max(1, case["B"] * 2 // 3), max(1, case["median"] * 4 // 5)
    return case


def _lengths(n, median, most):
    """Lengths of n sequences, lognormal by their quantiles, so that a case's work goes by the case alone."""
    at = (torch.arange(n, dtype=torch.float64) + 0.5) / n
    return (median * torch.exp(_SIGMA * torch.special.ndtri(at))).round().long().clamp(1, most)


def _attn_lengths(case):
    L = _lengths(case["B"], case["median"], case["most"])
    if case["edge"] and case["B"] >= 3:
        L[:2] = torch.tensor([0, 1])
    return L


def _plan_lengths(case):
    B = case["B"]
    L = _lengths(B, case["median"], case["most"])
    add = _lengths(B, case["add"], 4 * case["add"]) if case["add"] > 8 else torch.full((B,), case["add"])
    if case["add"] > 8:
        L[::2] = 0                       # (prompts: half of the sequences come new)
    if case["finished"]:
        add[torch.linspace(0, B - 1, case["finished"]).long()] = -1
    return L, add


def _ancestors(N):
    """Parents and ancestors (each node its own too) of a tree whose first node has up to four children, the others two."""
    parent = [-1] + [0 if n <= 4 else (n - 5) // 2 + 1 for n in range(1, N)]
    anc = np.eye(N, dtype=bool)
    for n in range(1, N):
        anc[n] |= anc[parent[n]]
    return np.array(parent, np.int32), anc


def _tile(D):
    return PAGE * (D // 2 + D // 32)


def work(case):
    if case["op"] == "plan":
        L, add = _plan_lengths(case)
        had, got = (L + PAGE - 1) // PAGE, (L + add.clamp(min=0) + PAGE - 1) // PAGE
        pages = int(had.sum() + got[add >= 0].sum())
        return {"bytes": 8 * int(add.clamp(min=0).sum()) + 4 * pages + 4 * 5 * case["B"], "flops": 0}
    D, Hkv = case["D"], case["Hkv"]
    row = Hkv * 2 * (D // 2 + D // 32)                      # a token's K and V, in bytes
    if case["op"] == "store":
        T, t = case["T"], max(0, case["T"] - case["skipped"])
        return {"bytes": t * (4 * Hkv * D + 2 * row) + 4 * T * Hkv * D + 8 * T, "flops": 0}
    if case["op"] == "commit":
        rows, t = case["B"] * (case["K"] + 1), case["B"] * (case["K"] / 2 + 1)
        return {"bytes": case["layers"] * (t * (4 * Hkv * D + 2 * row) + 4 * rows * Hkv * D) + 16 * rows, "flops": 0}
    B, N, Hq = case["B"], case["N"], case["Hq"]
    L = int(_attn_lengths(case).sum())
    pairs = N * L + B * int(_ancestors(N)[1].sum())
    return {"bytes": L * row + B * N * (4 * Hq * D + 4 * Hkv * D + 4 * Hq) + L // 32, "flops": 4 * Hq * D * pairs}


# ------------------------------------------------------------------------------------------------- inputs

def _scale_bytes(x):
    """Scale bytes of blocks [..., 32]: the largest magnitude over 7, to four significant bits (halves up)."""
    t = (x.abs().amax(-1).double() / 7).float()
    return (((t.view(torch.int32) + (1 << 19)) >> 20) - 8 * 107).clamp(0, 255)


def _scales(c):
    return (8 + (c & 7)).float() * torch.exp2((c >> 3).float() - 23)


def _quantised(x):
    """Codes and scale bytes of x [..., D]."""
    x = x.float().unflatten(-1, (-1, 32))
    c = _scale_bytes(x)
    t = x.double() / _scales(c).double().unsqueeze(-1)
    q = (torch.sign(t) * torch.floor(t.abs() + 0.5)).clamp(-8, 7)
    return q.flatten(-2).to(torch.int32), c


def _packed(q, c):
    """Pool tiles u8 [..., tile] of codes [..., 128, D] and scale bytes [..., 128, D/32]."""
    n = (q + 8).to(torch.uint8).unflatten(-1, (-1, 4, 2))                # [.., word, pair, even or odd]
    n = n.transpose(-1, -2).unflatten(-1, (2, 2))                        # [.., word, even or odd, byte, nibble]
    codes = n[..., 0] | (n[..., 1] << 4)
    return torch.cat([codes.flatten(-4), c.to(torch.uint8).flatten(-2)], -1)


def _pool(pages, Hkv, D, g):
    out = torch.empty(pages, Hkv, 2, _tile(D), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 25) // (PAGE * Hkv * 2 * D))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        out[p:p + n] = _packed(*_quantised(torch.randn(n, Hkv, 2, PAGE, D, generator=g, device="cuda")))
    return out


def _bf16(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16)


def _table(pages_of, g):
    """Page table and its index of sequences with that many pages, taken in random order from as many."""
    n = int(pages_of.sum())
    indptr = torch.zeros(len(pages_of) + 1, dtype=torch.int32)
    indptr[1:] = pages_of.cumsum(0)
    return torch.randperm(n, generator=g, device="cuda", dtype=torch.int32), indptr.cuda(), n


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    order = lambda n: torch.randperm(n, generator=g, device="cuda").cpu()  # noqa: E731
    s = dict(case)
    if case["op"] == "plan":
        L, add = (v[order(case["B"])] for v in _plan_lengths(case))
        table, indptr, used = _table((L + PAGE - 1) // PAGE, g)
        total = used + int(((add.clamp(min=0) + PAGE - 1) // PAGE + 1).sum()) + 100
        perm = torch.randperm(total, generator=g, device="cuda", dtype=torch.int32)
        s |= {"kv_len": L.int().cuda(), "add": add.int().cuda(), "indptr": indptr, "table": perm[:used][table.long()],
              "free": torch.cat([perm[used:], torch.zeros(used, dtype=torch.int32, device="cuda")]),
              "n_free": torch.tensor([total - used], dtype=torch.int32, device="cuda"),
              "tokens": int(add.clamp(min=0).sum()), "pages": total}
        return s
    Hkv, D = case["Hkv"], case["D"]
    if case["op"] == "store":
        pages = case["T"] // PAGE + 2
        slots = torch.randperm(pages, generator=g, device="cuda")[:, None] * PAGE + torch.arange(PAGE, device="cuda")
        slots = slots.flatten()[torch.arange(case["T"], device="cuda") + 61]
        slots[torch.randperm(case["T"], generator=g, device="cuda")[:case["skipped"]]] = -1
        s |= {"K": _bf16(g, case["T"], Hkv, D), "V": _bf16(g, case["T"], Hkv, D), "slots": slots,
              "pool": torch.zeros(pages, Hkv, 2, _tile(D), dtype=torch.uint8, device="cuda")}
        return s
    B, N = case["B"], case["N"]
    if case["op"] == "commit":
        K = case["K"]
        L = _lengths(B, case["median"], 2 * case["median"])[order(B)]
        table, indptr, pages = _table((L + K + 1 + PAGE - 1) // PAGE, g)
        n_acc = torch.randint(0, K + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        step = torch.arange(K + 1, device="cuda")
        path = (step * max(1, (N - 1) // (K + 1)) + torch.randint(0, max(1, (N - 1) // (K + 1)), (B, K + 1), generator=g, device="cuda"))
        path[:, 0] = 0
        path[step > n_acc[:, None]] = -1
        pos = L.cuda()[:, None] + step
        slots = table[indptr[:-1, None].long() + pos // PAGE].long() * PAGE + pos % PAGE
        slots[step > n_acc[:, None]] = -1
        layer = torch.arange(case["layers"], device="cuda")[:, None] * pages * PAGE
        every = torch.where(slots.flatten() >= 0, slots.flatten() + layer, -1).flatten()      # (slots of the layers' pools as one)
        Kt, Vt = (_bf16(g, case["layers"], B, N, Hkv, D) for _ in range(2))
        pool = torch.zeros(case["layers"], pages, Hkv, 2, _tile(D), dtype=torch.uint8, device="cuda")
        s |= {"Kt": Kt, "Vt": Vt, "pool": pool, "by_layer": (list(Kt), list(Vt), list(pool)), "path": path.int(), "n_acc": n_acc,
              "table": table, "indptr": indptr, "kv_len": L.int().cuda(), "slots": every}
        return s
    L = _attn_lengths(case)[order(B)]
    table, indptr, pages = _table((L + PAGE - 1) // PAGE + 1, g)
    parent, anc = _ancestors(N)
    s |= {"Q": _bf16(g, B, N, case["Hq"], D), "Kt": _bf16(g, B, N, Hkv, D), "Vt": _bf16(g, B, N, Hkv, D),
          "pool": _pool(pages, Hkv, D, g), "table": table, "indptr": indptr, "kv_len": L.int().cuda(),
          "kv_len_host": L.int().numpy(), "longest": int(L.max()), "parent": parent, "anc": torch.from_numpy(anc).cuda()}
    return s


# ------------------------------------------------------------------------------------------------- the plain forms

def _plan(s):
    kv_len, add, indptr, B = s["kv_len"].long(), s["add"].long(), s["indptr"].long(), s["B"]
    live, had = add >= 0, indptr[1:] - indptr[:-1]
    take = torch.where(live, ((kv_len + add + PAGE - 1) // PAGE - had).clamp(min=0), 0)
    owns = torch.where(live, had + take, 0)
    zero = torch.zeros(1, dtype=torch.long, device="cuda")
    new_ptr, tok_ptr, take_ptr = (torch.cat([zero, v.cumsum(0)]) for v in (owns, add.clamp(min=0), take))
    # the tables: a sequence's pages as they were, then pages from the front of the free list
    slot = torch.arange(s["pages"], device="cuda")
    of = torch.searchsorted(new_ptr, slot, right=True) - 1
    seq = of.clamp(max=B - 1)
    i = slot - new_ptr[seq]
    from_old, from_free = indptr[seq] + i, take_ptr[seq] + i - had[seq]
    table = torch.where(i < had[seq], s["table"][from_old.clamp(0, s["table"].numel() - 1)] if s["table"].numel() else 0,
                        s["free"][from_free.clamp(0, s["free"].numel() - 1)])
    table = torch.where(of < B, table, -1)
    # the slots of the new tokens
    t = torch.arange(s["tokens"], device="cuda")
    of_t = torch.searchsorted(tok_ptr, t, right=True) - 1
    pos = kv_len[of_t] + t - tok_ptr[of_t]
    slots = table[new_ptr[of_t] + pos // PAGE].long() * PAGE + pos % PAGE
    # the free list: what was not taken, then the pages of finished sequences
    left = s["n_free"].long() - take_ptr[-1]
    gone = torch.where(live, 0, had)
    gone_ptr = torch.cat([zero, gone.cumsum(0)])
    j = torch.arange(s["free"].numel(), device="cuda")
    of_g = (torch.searchsorted(gone_ptr, j - left, right=True) - 1).clamp(0, B - 1)
    back = indptr[of_g] + j - left - gone_ptr[of_g]
    n_free = left + gone_ptr[-1]
    free = torch.where(j < left, s["free"][(take_ptr[-1] + j).clamp(max=s["free"].numel() - 1)],
                       s["table"][back.clamp(0, s["table"].numel() - 1)] if s["table"].numel() else 0)
    return {"page_table": table, "page_indptr": new_ptr.int(), "tok_indptr": tok_ptr.int(), "slot_map": slots,
            "free_list": torch.where(j < n_free, free, -1), "n_free": n_free.int()}


def _values(x):
    q, c = _quantised(x)
    return (q.float().unflatten(-1, (-1, 32)) * _scales(c).unsqueeze(-1)).flatten(-2)


def _unpacked(tiles, D):
    """Values fp32 [..., 128, D] of pool tiles u8 [..., tile]."""
    codes = tiles[..., :PAGE * D // 2].unflatten(-1, (PAGE, -1, 2, 2))                   # [.., token, word, even or odd, byte]
    n = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).transpose(-1, -2)          # [.., token, word, pair, even or odd]
    q = n.flatten(-3).unflatten(-1, (-1, 32)).float() - 8
    return (q * _scales(tiles[..., PAGE * D // 2:].unflatten(-1, (PAGE, -1)).int()).unsqueeze(-1)).flatten(-2)


def _attention(s):
    B, N, Hq, Hkv, D, T = s["B"], s["N"], s["Hq"], s["Hkv"], s["D"], max(1, s["longest"])
    page = torch.arange((T + PAGE - 1) // PAGE, device="cuda")
    at = (s["indptr"][:-1, None] + page).clamp(max=s["table"].numel() - 1)
    own_page = (page * PAGE) < s["kv_len"][:, None]
    tiles = s["pool"][torch.where(own_page, s["table"][at.long()], 0).long()]            # [B, page, Hkv, 2, tile]
    kv = _unpacked(tiles.permute(3, 0, 2, 1, 4), D).flatten(3, 4)                        # [2, B, Hkv, token, D]
    q = s["Q"].float().unflatten(2, (Hkv, -1)).permute(0, 2, 1, 3, 4).flatten(2, 3)      # [B, Hkv, N G, D]
    past = torch.arange(kv.shape[3], device="cuda") < s["kv_len"][:, None]
    mask = s["anc"].repeat_interleave(Hq // Hkv, 0)                                      # [N G, N]
    kt, vt = (s[k].float().transpose(1, 2) for k in ("Kt", "Vt"))
    a = (q @ kv[0].transpose(-1, -2) * D ** -0.5).masked_fill_(~past[:, None, None], -math.inf)
    b = (q @ kt.transpose(-1, -2) * D ** -0.5).masked_fill_(~mask, -math.inf)
    m = torch.maximum(a.amax(-1), b.amax(-1))
    a, b = a.sub_(m[..., None]).exp_(), b.sub_(m[..., None]).exp_()
    total = a.sum(-1) + b.sum(-1)
    o = (a @ kv[1] + b @ vt) / total[..., None]
    back = lambda v: v.unflatten(2, (N, -1)).transpose(1, 2).flatten(2, 3)  # noqa: E731
    return back(o).bfloat16(), back(m + total.log())


def run(s):
    if own:
        from paper_2608_04962_b200 import binding as S
        if s["op"] == "plan":
            r = S.page_plan(s["kv_len"], s["add"], s["table"], s["indptr"], s["free"], s["n_free"], table_cap=s["pages"],
                            slot_cap=s["tokens"])
            return {k: r[k] for k in ("page_table", "page_indptr", "tok_indptr", "slot_map", "free_list", "n_free")}
        if s["op"] == "store":
            S.kv4_store(s["K"], s["V"], s["slots"], s["pool"])
            return S.kv4_load(s["pool"], s["slots"])
        if s["op"] == "commit":
            lens = torch.empty_like(s["kv_len"])
            Kt, Vt, pool = s["by_layer"]
            S.commit_path_kv4_layers(Kt, Vt, s["path"], s["n_acc"], pool, s["table"], s["indptr"], s["kv_len"], lens)
            return *S.kv4_load(s["pool"].flatten(0, 1), s["slots"]), lens
        return S.tree_attn_kv4(s["Q"], s["pool"], s["table"], s["indptr"], s["kv_len"], s["kv_len_host"], s["Kt"], s["Vt"], s["parent"],
                               want_lse=True)
    if s["op"] == "plan":
        return _plan(s)
    if s["op"] == "store":
        kept = (s["slots"] >= 0)[:, None, None]
        return tuple(torch.where(kept, _values(s[k]), 0).bfloat16() for k in ("K", "V"))
    if s["op"] == "commit":
        seq = torch.arange(s["B"], device="cuda")[:, None]
        kept = (s["path"] >= 0)[None, :, :, None, None]
        rows = (torch.where(kept, _values(s[k][:, seq, s["path"].clamp(min=0).long()]), 0).flatten(0, 2).bfloat16() for k in ("Kt", "Vt"))
        return *rows, s["kv_len"] + s["n_acc"] + 1
    return _attention(s)


# ------------------------------------------------------------------------------------------------- in 64 bits

_STEPS = [(8 + (c % 8)) * 2.0 ** (c // 8 - 23) for c in range(256)]


def _exact_rows(x):
    """Rows of the 4-bit cache from the definition: the scale nearest to the largest magnitude over 7 (halves up), the nearest
    whole multiple of it (halves away from zero)."""
    x = x.double().unflatten(-1, (-1, 32))
    steps = torch.tensor(_STEPS, dtype=torch.float64, device=x.device)
    borders = (steps[1:] + steps[:-1]) / 2
    step = steps[torch.searchsorted(7 * borders, x.abs().amax(-1).contiguous(), right=True)].unsqueeze(-1)
    t = x / step
    return (torch.trunc(t + torch.copysign(torch.full_like(t, 0.5), t)).clamp(-8, 7) * step).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "plan":
        return None
    if case["op"] == "store":
        gone = (s["slots"] < 0)[:, None, None]
        return tuple(_exact_rows(s[k]).masked_fill(gone, 0.0) for k in ("K", "V"))
    if case["op"] == "commit":
        take = s["path"].long().clamp(min=0)[None, :, :, None, None].expand(case["layers"], -1, -1, case["Hkv"], case["D"])
        gone = (s["path"] < 0)[None, :, :, None, None]
        return *(_exact_rows(s[k].gather(2, take)).masked_fill(gone, 0.0).flatten(0, 2) for k in ("Kt", "Vt")), None
    N, Hq, Hkv, D = case["N"], case["Hq"], case["Hkv"], case["D"]
    order = [2 * j + half for half in (0, 1) for j in range(4)]                          # the element of each nibble of a word
    steps = torch.tensor(_STEPS, dtype=torch.float64, device="cuda")
    lens, indptr = s["kv_len_host"].tolist(), s["indptr"].tolist()
    outs, lses = [], []
    for b in range(case["B"]):
        pages = s["table"][indptr[b]:indptr[b + 1]].long()
        halves = []
        for kv in (0, 1):
            tile = s["pool"][pages, :, kv]                                               # [page, Hkv, tile]
            word = tile[..., :PAGE * D // 2].contiguous().view(torch.int32).unflatten(-1, (PAGE, D // 8))
            q = torch.empty(*word.shape, 8, dtype=torch.float64, device="cuda")
            for n, e in enumerate(order):
                q[..., e] = ((word >> (4 * n)) & 15).double() - 8
            step = steps[tile[..., PAGE * D // 2:].long()].unflatten(-1, (PAGE, D // 32)).repeat_interleave(32, -1)
            x = (q.flatten(-2) * step).transpose(1, 2).flatten(0, 1)[:lens[b]]           # [token, Hkv, D]
            halves.append(torch.cat([x, s["Kt" if kv == 0 else "Vt"][b].double()]).repeat_interleave(Hq // Hkv, 1))
        may = torch.cat([torch.ones(N, lens[b], dtype=torch.bool, device="cuda"), s["anc"]], 1)
        score = torch.einsum("nhd,thd->hnt", s["Q"][b].double(), halves[0]) / math.sqrt(D)
        score = torch.where(may, score, torch.full_like(score, -math.inf))
        lse = torch.logsumexp(score, -1)
        outs.append(torch.einsum("hnt,thd->nhd", torch.exp(score - lse[..., None]), halves[1]))
        lses.append(lse.T)
    return torch.stack(outs), torch.stack(lses)
