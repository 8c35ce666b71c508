"""Cases of the 8-bit paged cache: append, attention over it, and the upkeep of its pages.

`run` computes an operator either through the framework (own = True) or in its plain form (elementary torch operations).

The cache: pages of `page` tokens.  A block is one page of one KV head; its 8-bit numbers n (int8, or float8 e4m3) stand for
n * amax / R, with amax the block's largest magnitude and R = 127 (int8) or 448 (e4m3).  Row b of a batch owns the pages
tables[b][0 .. ceil(seq_lens[b] / page)) in order.  Page state: refs[p] = table entries that name page p, free_list[0 .. n_free)
= a stack of the pages that nobody names.
"""
import math
import random

import torch

own = False

R = {"int8": 127.0, "e4m3": 448.0}
F16_MAX = 65504.0


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # one GPT-2 sized attention layer, one sequence of 128 tokens: nothing but latency
        dict(name="attend_gpt2_b1", op="attend", B=1, n_q=12, n_kv=12, d=64, lo=128, hi=128, empty=0, L_q=1, page=16, fmt="int8", fp16=False),
        # a serving batch of ragged rows, four draft tokens to verify per row, some rows not started yet
        dict(name="attend_draft_ragged", op="attend", B=23, n_q=32, n_kv=8, d=128, lo=5, hi=8189, empty=2, L_q=4, page=32, fmt="e4m3", fp16=False),
        # the long-context decode step: 16 rows of 32768 tokens, grouped heads
        dict(name="attend_gqa_32k", op="attend", B=16, n_q=32, n_kv=8, d=128, lo=32768, hi=32768, empty=0, L_q=1, page=64, fmt="int8", fp16=False),
        # a whole prompt attending to itself
        dict(name="attend_prompt_4k", op="attend", B=1, n_q=32, n_kv=8, d=128, lo=4096, hi=4096, empty=0, L_q=4096, page=64, fmt="e4m3", fp16=True),
        # one generated token per row of a GPT-2 sized layer, rows of any length
        dict(name="append_step_b32", op="append", B=32, n_q=12, n_kv=12, d=64, lo=129, hi=1024, empty=0, n=1, ragged=False, page=16, fmt="int8"),
        # prompts of four rows, padded to the longest
        dict(name="append_prompt_4k", op="append", B=4, n_q=32, n_kv=8, d=128, lo=2500, hi=4096, empty=0, n=4096, ragged=True, page=64, fmt="e4m3"),
        # beam search, one token per beam: beams that share their last page get copies of it in every layer's pools
        dict(name="extend_beams", op="extend", B=64, beams=4, lo=130, hi=1020, n=1, page=16, pools=24, page_bytes=16 * 12 * 64, spare=600, max_pages=64),
        # room for the prompts of a large batch: many pages, nothing shared
        dict(name="extend_prompts", op="extend", B=256, beams=1, lo=0, hi=600, n=700, page=16, pools=2, page_bytes=16 * 12 * 64, spare=12000, max_pages=128),
        # beams of 12 sequences reordered after a step
        dict(name="fork_beams", op="fork", B=48, lo=100, hi=1024, page=16, max_pages=64, shared=0.5, dead=0.0, spare=64),
        # a large batch of long rows: some finished (freed), some continued twice
        dict(name="fork_free_large", op="fork", B=256, lo=1000, hi=32768, page=32, max_pages=1024, shared=0.25, dead=0.2, spare=1000),
        # a small cache packed into its front
        dict(name="compact_small", op="compact", B=8, page=16, max_pages=64, n_pages=600, live=0.4, pools=24, page_bytes=16 * 12 * 64),
        # a large cache after most of its rows ended: a quarter of the bytes moves
        dict(name="compact_large", op="compact", B=64, page=64, max_pages=128, n_pages=4096, live=0.5, pools=8, page_bytes=64 * 8 * 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "append", "append", "extend", "fork", "compact"])
    page = rng.choice([16, 32, 64, 128])
    if op in ("attend", "append"):
        n_kv, g, d = rng.choice([(12, 1, 64), (8, 4, 128), (4, 8, 128), (2, 3, 64), (1, 16, 128), (5, 2, 64), (8, 1, 128)])
        case = dict(op=op, n_q=n_kv * g, n_kv=n_kv, d=d, page=page, fmt=rng.choice(["int8", "e4m3"]))
        if op == "attend":
            hi = _log(rng, 1, 32768)
            # a token, drafts, or a prompt's piece; the plain form holds every score at once
            L_q = rng.choice([1, 1, 1, rng.randint(2, 9), _log(rng, 10, 2048)])
            L_q = min(L_q, hi)
            most = min((16 * 8 * 32768) // (n_kv * hi), (1 << 28) // (n_kv * g * hi * L_q), 256)
            if most < 1:
                L_q, most = 1, max(1, (16 * 8 * 32768) // (n_kv * hi))
            B = _log(rng, 1, most) if most > 1 else 1
            return dict(case, B=B, lo=rng.randint(1, hi), hi=hi, empty=rng.choice([0, 0, 1]) if B > 1 else 0, L_q=L_q, fp16=rng.choice([False, True]))
        n = rng.choice([1, 1, rng.randint(2, 40), _log(rng, 41, 4096)])
        B = _log(rng, 1, max(2, min(256, 16384 // n)))
        hi = n + rng.randint(0, 2048)
        return dict(case, B=B, lo=max(1, hi // 2), hi=hi, empty=rng.choice([0, 1]) if B > 1 else 0, n=n, ragged=rng.random() < 0.5)
    if op == "extend":
        beams = rng.choice([1, 2, 4, 5])
        B, n, hi = beams * _log(rng, 1, 200 // beams), rng.choice([1, 1, _log(rng, 2, 600)]), _log(rng, 2, 1500)
        return dict(op=op, B=B, beams=beams, lo=rng.randint(0, hi), hi=hi, n=n, page=page, pools=rng.choice([1, 2, 24]), page_bytes=page * rng.choice([48, 768, 1024]),
                    spare=B * (n // page + 2) + rng.randint(0, 100), max_pages=(hi + n) // page + 1 + rng.randint(0, 9))
    if op == "fork":
        hi = _log(rng, 2, 16384)
        return dict(op=op, B=_log(rng, 1, 256), lo=rng.randint(1, hi), hi=hi, page=page, max_pages=hi // page + 1 + rng.randint(0, 9), shared=rng.uniform(0, 0.9),
                    dead=rng.choice([0.0, 0.3]), spare=rng.randint(0, 500))
    n_pages = _log(rng, 20, 4000)
    return dict(op=op, B=_log(rng, 1, 64), page=page, max_pages=_log(rng, 4, 128), n_pages=n_pages, live=rng.uniform(0.1, 0.9), pools=rng.choice([1, 2, 8, 24]),
                page_bytes=page * rng.choice([48, 256, 512]))


# ------------------------------------------------------------------------------------------------ inputs
def _lens(case):
    """The rows' lengths, a function of the case alone: spread over lo..hi, the first `empty` rows without a token."""
    lo, hi = case["lo"], case["hi"]
    rows = [lo + int((hi - lo) * ((i * 0.6180339887498949 + 0.37) % 1.0) + 0.5) for i in range(case["B"])]
    if lo < hi:
        rows[-1] = hi
    return [0 if i < case.get("empty", 0) else n for i, n in enumerate(rows)]


def _n_new(case, lens):
    """Tokens appended per row: the case's n, or for ragged rows the whole row as far as that goes."""
    return [0 if not n else min(n, case["n"] - (7 * i % case["n"] if case["ragged"] and i % 3 == 2 else 0)) for i, n in enumerate(lens)]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _paged(case, lens, gen, spare):
    """Tables [B][max_pages] of the rows (-1 beyond a row's pages) over randomly placed pages, and the number of pages."""
    need = torch.tensor([-(-n // case["page"]) for n in lens], device="cuda")
    n_pages, width = int(need.sum()) + spare, max(1, int(need.max()))
    perm = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
    at = torch.arange(width, device="cuda")[None]
    flat = ((need.cumsum(0) - need)[:, None] + at).clamp(max=n_pages - 1)
    return torch.where(at < need[:, None], perm[flat], -1).contiguous(), n_pages


def _quantised(shape, fmt, gen):
    """A pool of pages [n_pages][H][page][d] with keys or values of many sizes, and its amax."""
    x = torch.randn(shape, device="cuda", generator=gen)
    x *= torch.exp(0.7 * torch.randn((1, shape[1], 1, shape[3]), device="cuda", generator=gen))
    x *= torch.exp(0.3 * torch.randn((shape[0], shape[1], 1, 1), device="cuda", generator=gen))
    amax = x.abs().amax(dim=(2, 3)).half().float()
    x *= (R[fmt] / amax)[:, :, None, None]
    x.clamp_(-R[fmt], R[fmt])
    return (x.round_().to(torch.int8) if fmt == "int8" else x.to(torch.float8_e4m3fn)), amax


def _cache(case, lens, tables, n_pages, gen):
    H, P, d, fmt = case["n_kv"], case["page"], case["d"], case["fmt"]
    k, ka = _quantised((n_pages, H, P, d), fmt, gen)
    v, va = _quantised((n_pages, H, P, d), fmt, gen)
    # what no sequence holds is left over from earlier use: 0x7f (a NaN in e4m3) behind the rows' ends and in spare pages
    used = torch.zeros(n_pages, dtype=torch.int64, device="cuda")
    at = torch.arange(tables.shape[1], device="cuda")[None] * P
    count = (torch.tensor(lens, device="cuda")[:, None] - at).clamp(0, P)
    used.index_add_(0, tables.clamp(min=0).reshape(-1).long(), count.reshape(-1))
    stale = torch.arange(P, device="cuda")[None] >= used[:, None]
    for t in (k, v):
        t.view(torch.uint8).masked_fill_(stale[:, None, :, None], 0x7F)
    for a in (ka, va):
        a[used == 0] = float("nan")
    return k, ka, v, va


def prepare(case, seed):
    gen = _gen(seed)
    state = dict(case=case)
    if case["op"] in ("attend", "append"):
        lens = _lens(case)
        tables, n_pages = _paged(case, lens, gen, 3)
        state.update(tables=tables, seq_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
        B, H, d = case["B"], case["n_kv"], case["d"]
        if case["op"] == "attend":
            state["cache"] = _cache(case, lens, tables, n_pages, gen)
            q = torch.randn((B, case["n_q"], case["L_q"], d), device="cuda", generator=gen)
            state["q"] = (q * 0.8).half()
        else:
            counts = _n_new(case, lens)
            before = [n - c for n, c in zip(lens, counts)]
            state["cache"] = _cache(case, before, tables, n_pages, gen)
            x = torch.randn((2, B, H, case["n"], d), device="cuda", generator=gen)
            x *= torch.exp(0.7 * torch.randn((2, 1, H, 1, d), device="cuda", generator=gen))
            state["k_new"], state["v_new"] = x[0].half().contiguous(), x[1].half().contiguous()
            state["n_new"] = torch.tensor(counts, dtype=torch.int32, device="cuda")
        return state
    # page state: tables, seq_lens, refs, free_list, n_free; kept twice, so that every pass begins where the first one began
    B, P, W = case["B"], case["page"], case["max_pages"]
    cpu = random.Random(seed)
    if case["op"] == "extend":
        # groups of `beams` rows share all of their pages
        groups = [min(n, W * P - case["n"]) for n in _lens(dict(case, B=-(-B // case["beams"])))]
        lens = [groups[b // case["beams"]] for b in range(B)]
        need = [-(-n // P) for n in groups]
        n_pages = sum(need) + case["spare"]
        perm = list(range(n_pages))
        cpu.shuffle(perm)
        starts = [sum(need[:i]) for i in range(len(need))]
        rows = [perm[starts[b // case["beams"]]:][: need[b // case["beams"]]] for b in range(B)]
        state["n_new"] = torch.full((B,), case["n"], dtype=torch.int32, device="cuda")
    elif case["op"] == "fork":
        # every row shares a leading part of its pages with its left neighbour in a group of four
        lens = _lens(case)
        rows, made = [], 0
        for b, n in enumerate(lens):
            need = -(-n // P)
            keep = 0 if b % 4 == 0 else min(len(rows[-1]), need, int(case["shared"] * need))
            rows.append((rows[-1][:keep] if keep else []) + list(range(made, made + need - keep)))
            made += need - keep
        n_pages = made + case["spare"]
        perm = list(range(n_pages))
        cpu.shuffle(perm)
        rows = [[perm[p] for p in r] for r in rows]
        parents = [-1 if cpu.random() < case["dead"] else min(B - 1, b // 4 * 4 + cpu.randrange(4)) for b in range(B)]
        state["parents"] = torch.tensor(parents, dtype=torch.int32, device="cuda")
    else:
        n_pages = case["n_pages"]
        live = cpu.sample(range(n_pages), max(1, int(case["live"] * n_pages)))
        rows, lens = [], []
        for b in range(B):
            mine = live[b::B][:W]
            rows.append(mine)
            lens.append(max(0, len(mine) * P - cpu.randrange(P)))
    refs = [0] * n_pages
    for r in rows:
        for p in r:
            refs[p] += 1
    free = [p for p in range(n_pages) if not refs[p]]
    cpu.shuffle(free)
    flat = [p for r in rows for p in r + [-1] * (W - len(r))]
    ints = [flat, lens, refs, free + [-1] * (n_pages - len(free)), [len(free)]]
    state["saved"] = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ints]
    state["saved"][0] = state["saved"][0].view(B, W)
    state["parts"] = [x.clone() for x in state["saved"]]
    state["n_pages"] = n_pages
    if "pools" in case:
        state["pools"] = [torch.randint(0, 256, (n_pages, case["page_bytes"]), dtype=torch.uint8, device="cuda", generator=gen) for _ in range(case["pools"])]
    return state


# ------------------------------------------------------------------------------------------------ one pass
_contexts = {}


def _context(n_q, n_kv, d):
    """The framework's context for an attention shape on the current device and stream, made once as a user's program does."""
    device = torch.cuda.current_device()
    key = n_q, n_kv, d, device, torch._C._cuda_getCurrentRawStream(device)
    if key not in _contexts:
        from paper_2601_10155_b200.binding import Lookat
        _contexts[key] = Lookat(n_q, n_kv, d, d, 4, 256, device=device)
    return _contexts[key]


def run(state):
    case = state["case"]
    op = case["op"]
    if op in ("attend", "append"):
        if own:
            if "handle" not in state:                      # a program makes it with its cache and keeps it
                from paper_2601_10155_b200.binding import Q8Cache
                state["handle"] = Q8Cache(*state["cache"])
            lk, cache = _context(case["n_q"], case["n_kv"], case["d"]), state["handle"]
            if op == "attend":
                return lk.lookat_attend_q8(cache, state["q"], state["tables"], state["seq_lens"], out_fp16=case["fp16"])
            lk.lookat_q8_append(cache, state["k_new"], state["v_new"], state["tables"], state["seq_lens"], state["n_new"])
            return list(state["cache"])
        return _plain_attend(state) if op == "attend" else _plain_append(state)
    torch._foreach_copy_(state["parts"], state["saved"])
    tables, seq_lens, refs, free_list, n_free = state["parts"]
    if own:
        if "handle" not in state:
            from paper_2601_10155_b200.binding import PagePools, PageState
            state["handle"] = PageState(tables, seq_lens, refs, free_list, n_free, case["page"]), PagePools(state.get("pools", []))
        lk, (pages, pools) = _context(12, 12, 64), state["handle"]
        if op == "extend":
            lk.lookat_pages_extend(pages, state["n_new"], pools)
        elif op == "fork":
            lk.lookat_pages_fork(pages, state["parents"])
        else:
            lk.lookat_pages_compact(pages, pools)
    else:
        {"extend": _plain_extend, "fork": _plain_fork, "compact": _plain_compact}[op](state, tables, seq_lens, refs, free_list, n_free)
    return [tables, seq_lens, refs, free_list, n_free] + (state["pools"] if "pools" in state else [])


# ---- plain forms
def _plain_attend(state):
    case, q, tables, lens = state["case"], state["q"], state["tables"], state["seq_lens"].long()
    k8, ka, v8, va = state["cache"]
    B, Hq, Lq, d = q.shape
    H, g = case["n_kv"], case["n_q"] // case["n_kv"]
    L = tables.shape[1] * case["page"]
    idx = tables.clamp(min=0).long()
    held = torch.arange(L, device="cuda")[None] < lens[:, None]                                   # [B][L]

    def rows(n8, amax):                                                                           # [B][H][L][d]
        n = (n8.view(torch.uint8)[idx].view(n8.dtype)).float()
        n *= (amax[idx] / R[case["fmt"]])[..., None, None]
        n = n.permute(0, 2, 1, 3, 4).reshape(B, H, L, -1)
        return n.masked_fill_(~held[:, None, :, None], 0.0)

    s = q.float().view(B, H, g * Lq, d) @ rows(k8, ka).transpose(2, 3)
    s = s.view(B, H, g, Lq, L)
    s *= 1.0 / math.sqrt(d)
    last = lens[:, None] - Lq + torch.arange(Lq, device="cuda")[None]                             # [B][Lq]: the query's position
    unseen = torch.arange(L, device="cuda")[None, None] > last[..., None]
    s.masked_fill_(unseen[:, None, None], -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    s -= torch.where(top == -math.inf, 0.0, top)
    s.exp_()
    total = s.sum(dim=-1, keepdim=True)
    o = (s.view(B, H, g * Lq, L) @ rows(v8, va)).view(B, H, g, Lq, -1) / torch.where(total == 0, 1.0, total)
    return o.reshape(B, Hq, Lq, -1).to(torch.float16 if case["fp16"] else torch.float32)


def _round8(x, fmt):
    return x.round().to(torch.int8) if fmt == "int8" else x.to(torch.float8_e4m3fn)


def _plain_append(state):
    case, tables, lens, count = state["case"], state["tables"].long(), state["seq_lens"].long(), state["n_new"].long()
    k8, ka, v8, va = state["cache"]
    B, H, n, P, fmt = case["B"], case["n_kv"], case["n"], case["page"], case["fmt"]
    first = lens - count
    i = torch.arange(n, device="cuda")[None]
    real = i < count[:, None]
    pos = torch.where(real, first[:, None] + i, 0)
    page = tables.gather(1, pos // P)                                                             # [B][n]
    rows, cols = real.nonzero(as_tuple=True)
    page, off = page[rows, cols], (pos % P)[rows, cols]
    begun = ((first % P != 0) & (count > 0)).nonzero()[:, 0]                                      # rows whose first block holds tokens already
    head_page = tables[begun, first[begun] // P]
    older = torch.arange(P, device="cuda")[None] < (first[begun] % P)[:, None]                    # [rows][P]
    for n8, amax, x in ((k8, ka, state["k_new"]), (v8, va, state["v_new"])):
        x = torch.nan_to_num(x.float(), nan=0.0, posinf=F16_MAX, neginf=-F16_MAX).permute(0, 2, 1, 3)[rows, cols]   # [tokens][H][d]
        raw = n8.view(torch.uint8)
        a_old = amax[head_page]                                                                   # [rows][H]
        amax[page] = 0.0
        amax[head_page] = a_old
        amax.index_reduce_(0, page, x.abs().amax(dim=-1), "amax")
        a = amax[head_page]
        had = raw[head_page].view(n8.dtype)
        redone = _round8(torch.where(a > 0, 1.0, 0.0)[..., None, None] * had.float() * a_old[..., None, None] / torch.where(a > 0, a, 1.0)[..., None, None], fmt)
        change = older[:, None, :, None] & (a > a_old)[..., None, None]
        raw[head_page] = torch.where(change, redone.view(torch.uint8), had.view(torch.uint8))
        a = amax[page][..., None]
        raw[page, :, off] = _round8(torch.where(a > 0, R[fmt] * x / torch.where(a > 0, a, 1.0), 0.0), fmt).view(torch.uint8)
    return list(state["cache"])


def _plain_extend(state, tables, seq_lens, refs, free_list, n_free):
    case, n = state["case"], state["n_new"].long()
    P, W, n_pages = case["page"], case["max_pages"], state["n_pages"]
    L = seq_lens.long()
    have, need = -(-L // P), -(-(L + n) // P)
    last = tables.long().gather(1, (have - 1).clamp(min=0)[:, None])[:, 0]
    shares = (n > 0) & (L % P != 0)
    same = shares[:, None] & shares[None] & (last[:, None] == last[None])
    rank = torch.tril(same, diagonal=-1).sum(dim=1)
    copy = shares & (refs.long()[last.clamp(min=0)] - rank > 1)
    take = copy.long() + need - have
    before = take.cumsum(0) - take
    top = n_free.long()
    at = torch.arange(W, device="cuda")[None]
    fresh = (at >= have[:, None]) & (at < need[:, None]) | copy[:, None] & (at == have[:, None] - 1)
    k = before[:, None] + fresh.long().cumsum(1) - 1
    got = free_list.long()[(top - 1 - k).clamp(0, n_pages - 1)]
    rows = copy.nonzero()[:, 0]
    src, dst = last[rows], got[rows, have[rows] - 1]
    refs.index_add_(0, src, -torch.ones_like(src, dtype=torch.int32))
    tables.copy_(torch.where(fresh, got.int(), tables))
    refs[got[fresh]] = 1
    seq_lens += n.int()
    n_free -= take.sum().int()
    for pool in state["pools"]:
        pool[dst] = pool[src]


def _plain_fork(state, tables, seq_lens, refs, free_list, n_free):
    case, parents = state["case"], state["parents"].long()
    P, B, n_pages = case["page"], case["B"], state["n_pages"]
    alive = (parents >= 0) & (parents < B)
    src = parents.clamp(0, B - 1)
    old_lens = seq_lens.long()
    new_lens = torch.where(alive, old_lens[src], 0)
    at = torch.arange(case["max_pages"], device="cuda")[None]
    held, holds = at < -(-old_lens // P)[:, None], at < -(-new_lens // P)[:, None]
    new = torch.where(holds, tables[src], tables)
    old_refs = refs.clone()
    refs.index_add_(0, tables.clamp(min=0).reshape(-1).long(), -held.reshape(-1).int())
    refs.index_add_(0, new.clamp(min=0).reshape(-1).long(), holds.reshape(-1).int())
    freed = ((old_refs > 0) & (refs == 0)).nonzero()[:, 0]
    free_list[n_free.long() + torch.arange(len(freed), device="cuda")] = freed.int()
    n_free += len(freed)
    tables.copy_(new)
    seq_lens.copy_(new_lens)


def _plain_compact(state, tables, seq_lens, refs, free_list, n_free):
    P, n_pages = state["case"]["page"], state["n_pages"]
    live = refs > 0
    used = live.sum()
    ids = torch.arange(n_pages, device="cuda")
    holes, movers = (~live & (ids < used)).nonzero()[:, 0], (live & (ids >= used)).nonzero()[:, 0]
    remap = ids.clone()
    remap[movers] = holes
    held = torch.arange(tables.shape[1], device="cuda")[None] < -(-seq_lens.long() // P)[:, None]
    tables.copy_(torch.where(held, remap[tables.clamp(min=0).long()].int(), tables))
    refs[holes] = refs[movers]
    refs[movers] = 0
    count = n_pages - used
    free_list.copy_(torch.where(ids < count, n_pages - 1 - ids, free_list).int())
    n_free.copy_(count)
    for pool in state["pools"]:
        pool[holes] = pool[movers]


# ------------------------------------------------------------------------------------------------ work
def work(case):
    op = case["op"]
    if op in ("attend", "append"):
        H, d, P = case["n_kv"], case["d"], case["page"]
        lens = _lens(case)
        if op == "attend":
            Lq, Hq = case["L_q"], case["n_q"]
            seen = sum(sum(range(max(0, n - Lq + 1), n + 1)) for n in lens)
            pages = sum(-(-n // P) for n in lens)
            io = case["B"] * Hq * Lq * d * (2 + (2 if case["fp16"] else 4))
            return {"bytes": sum(lens) * H * 2 * d + pages * (8 * H + 4) + io, "flops": 4 * d * Hq * seen}
        new = sum(_n_new(case, lens))
        return {"bytes": new * H * 2 * d * 3 + 8 * H * sum(-(-n // P) for n in _n_new(case, lens)), "flops": 4 * new * H * d}
    B, P, W = case["B"], case["page"], case["max_pages"]
    if op == "extend":
        groups = [min(n, W * P - case["n"]) for n in _lens(dict(case, B=-(-B // case["beams"])))]
        lens = [groups[b // case["beams"]] for b in range(B)]
        copies = sum(groups[g] % P != 0 for b in range(B) for g in [b // case["beams"]] if b % case["beams"])
        fresh = sum(-(-(n + case["n"]) // P) - (-(-n // P)) for n in lens)
        return {"bytes": 2 * copies * case["pools"] * case["page_bytes"] + 16 * (fresh + copies) + 16 * B, "flops": B}
    if op == "fork":
        return {"bytes": 4 * sum(-(-n // P) for n in _lens(case)) * 4 + 12 * B, "flops": B}
    live = max(1, int(case["live"] * case["n_pages"]))
    moved = live * (case["n_pages"] - live) // case["n_pages"]
    return {"bytes": 2 * moved * case["pools"] * case["page_bytes"] + 12 * case["n_pages"] + 8 * live, "flops": case["n_pages"]}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _number8(x, fmt):
    """The 8-bit number nearest to x, ties to the even one, as the value it is."""
    if fmt == "int8":
        return torch.round(x)
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (e - 1).clamp(min=-6) - 3)      # three fraction bits; subnormals below 2^-6
    return (torch.round(x / step) * step).clamp(-448, 448)


def exact(case, seed):
    if case["op"] not in ("attend", "append"):
        return None                                                        # whole numbers only
    state = prepare(case, seed)
    k8, ka, v8, va = state["cache"]
    lens, tables, P, H, fmt = state["seq_lens"].tolist(), state["tables"].tolist(), case["page"], case["n_kv"], case["fmt"]
    if case["op"] == "attend":
        q = state["q"].double()
        g, Lq = case["n_q"] // H, case["L_q"]
        out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            if not n:
                continue
            mine = torch.tensor(tables[b][: -(-n // P)], device="cuda")
            for h in range(H):
                k = (k8.view(torch.uint8)[mine, h].view(k8.dtype).double() * (ka[mine, h].double() / R[fmt])[:, None, None]).reshape(-1, q.shape[-1])[:n]
                v = (v8.view(torch.uint8)[mine, h].view(v8.dtype).double() * (va[mine, h].double() / R[fmt])[:, None, None]).reshape(-1, q.shape[-1])[:n]
                pos = torch.arange(n - Lq, n, device="cuda")
                see = torch.arange(n, device="cuda")[None] <= pos[:, None]
                for r in range(h * g, h * g + g):
                    s = torch.where(see, q[b, r] @ k.T / math.sqrt(q.shape[-1]), -math.inf)
                    out[b, r] = torch.nan_to_num(torch.softmax(s, dim=1), nan=0.0) @ v
        return out
    res = []
    for n8, amax, x in ((k8, ka, state["k_new"]), (v8, va, state["v_new"])):
        num, a = n8.double(), amax.double()
        for b, (n, c) in enumerate(zip(lens, state["n_new"].tolist())):
            for i in range((n - c) // P, -(-n // P)) if c else ():
                lo, hi, p = max(i * P, n - c), min(i * P + P, n), tables[b][i]
                new = x[b, :, lo - (n - c): hi - (n - c)].double()
                was = a[p] if lo > i * P else torch.zeros_like(a[p])
                now = torch.maximum(was, new.abs().amax(dim=(1, 2)))
                if lo > i * P:
                    kept = num[p, :, : lo - i * P]
                    num[p, :, : lo - i * P] = torch.where((now > was)[:, None, None], _number8(kept * was[:, None, None] / now[:, None, None], fmt), kept)
                num[p, :, lo - i * P: hi - i * P] = _number8(R[fmt] * new / now[:, None, None], fmt)
                a[p] = now
        res += [num, a]
    return res
