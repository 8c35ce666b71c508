"""Cases of what a server runs around the 8-bit paged cache: rotary positions, attention of packed prompts, their keys and
values into the cache, and beam search's selection.

`run` computes an operator either through the framework (own = True) or in its plain form (elementary torch operations).

Packed prompts: the tokens of all rows stand one behind the other, row b being tokens starts[b] .. starts[b + 1].  Queries,
keys and values are fp16 and are read where a fused projection leaves them: a token's row of [q heads | k heads | v heads].
The cache is that of operators.py: pages of `page` tokens, a block (one page of one KV head) has 8-bit numbers n that stand for
n * amax / R with amax the block's largest magnitude, R = 127 (int8) or 448 (e4m3).
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
        # one short prompt in one GPT-2 sized layer: nothing but latency
        dict(name="attend_short", op="attend", B=1, n_q=12, n_kv=12, d=64, lo=17, hi=17, empty=0),
        # a serving batch's prompts of any length, grouped heads, one row that is not there
        dict(name="attend_ragged", op="attend", B=23, n_q=32, n_kv=8, d=128, lo=1, hi=1499, empty=1),
        # 32 full contexts of a GPT-2 sized layer
        dict(name="attend_gpt2_b32", op="attend", B=32, n_q=12, n_kv=12, d=64, lo=1024, hi=1024, empty=0),
        # four prompts of 4096 tokens, grouped heads
        dict(name="attend_4k", op="attend", B=4, n_q=32, n_kv=8, d=128, lo=4096, hi=4096, empty=0),
        # one long document
        dict(name="attend_16k", op="attend", B=1, n_q=32, n_kv=8, d=128, lo=16384, hi=16384, empty=0),
        # the generated tokens of 32 rows, far into long contexts
        dict(name="rope_step", op="rope", T=32, n_q=32, n_kv=8, d=128, rotary=128, interleaved=False, scaling="ramp", far=131072),
        # a batch of prompts, the first half of each head rotated in neighbouring pairs
        dict(name="rope_half_head", op="rope", T=5003, n_q=12, n_kv=12, d=64, rotary=32, interleaved=True, scaling="none", far=2048),
        # the prompts of attend_4k
        dict(name="rope_16k", op="rope", T=16384, n_q=32, n_kv=8, d=128, rotary=128, interleaved=False, scaling="bands", far=16384),
        # second pieces of ragged prompts, behind what the rows hold already
        dict(name="append_pieces", op="append", B=23, n_kv=12, d=64, lo=1, hi=500, empty=1, before=700, page=16, fmt="int8"),
        # the prompts of attend_4k
        dict(name="append_4k", op="append", B=4, n_kv=8, d=128, lo=4096, hi=4096, empty=0, before=0, page=64, fmt="e4m3"),
        # a step of the GPT-2 harness's beams
        dict(name="beam_gpt2", op="beam", G=8, W=4, V=50257, max_len=1024, done=0.1, first=False, penalty=0.0),
        # a large batch, wide beams, a large vocabulary
        dict(name="beam_large", op="beam", G=32, W=16, V=131072, max_len=512, done=0.1, first=False, penalty=0.7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_SHAPES = [(12, 1, 64), (8, 4, 128), (4, 8, 128), (2, 3, 64), (1, 16, 128), (5, 2, 64), (8, 1, 128)]


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "rope", "append", "beam"])
    n_kv, g, d = rng.choice(_SHAPES)
    if op == "attend":
        hi = _log(rng, 1, 8192)
        # the plain form holds every score of the padded batch at once
        most = max(1, min(256, (1 << 31) // (n_kv * g * hi * hi), 65536 // hi))
        B = _log(rng, 1, most) if most > 1 else 1
        return dict(op=op, B=B, n_q=n_kv * g, n_kv=n_kv, d=d, lo=rng.randint(1, hi), hi=hi, empty=rng.choice([0, 0, 1]) if B > 1 else 0)
    if op == "rope":
        return dict(op=op, T=_log(rng, 1, 16384), n_q=n_kv * g, n_kv=n_kv, d=d, rotary=rng.choice([d, d, d // 2, d // 4, 20]), interleaved=rng.random() < 0.4,
                    scaling=rng.choice(["none", "linear", "base", "bands", "ramp"]), far=_log(rng, 512, 1 << 20))
    if op == "append":
        hi = _log(rng, 1, 4096)
        B = _log(rng, 1, max(2, min(256, 16384 // hi)))
        return dict(op=op, B=B, n_kv=n_kv, d=d, lo=rng.randint(1, hi), hi=hi, empty=rng.choice([0, 1]) if B > 1 else 0, before=rng.choice([0, rng.randint(1, 1500)]),
                    page=rng.choice([16, 32, 64, 128]), fmt=rng.choice(["int8", "e4m3"]))
    W, V = rng.choice([1, 2, 3, 4, 5, 8, 16, 32]), _log(rng, 40, 131072)
    return dict(op=op, G=_log(rng, 1, max(2, min(128, (1 << 26) // (W * V)))), W=W, V=V, max_len=_log(rng, 16, 1024), done=rng.choice([0.0, 0.1, 0.4]),
                first=rng.random() < 0.25, penalty=rng.choice([0.0, 0.7, 1.0]))


# ------------------------------------------------------------------------------------------------ inputs
def _lens(case):
    """The rows' lengths, a function of the case alone: spread over lo..hi, the first `empty` rows without a token."""
    lo, hi = case["lo"], case["hi"]
    rows = [lo + int((hi - lo) * ((i * 0.6180339887498949 + 0.37) % 1.0) + 0.5) for i in range(case["B"])]
    if lo < hi:
        rows[-1] = hi
    return [0 if i < case["empty"] else n for i, n in enumerate(rows)]


def _starts(lens):
    starts = [0]
    for n in lens:
        starts.append(starts[-1] + n)
    return torch.tensor(starts, dtype=torch.int32, device="cuda")


def _projection(T, n_q, n_kv, d, gen):
    """Queries, keys and values [T][heads][d] as views of one fused projection's output, with heads and dims of many sizes."""
    x = torch.randn((T, n_q + 2 * n_kv, d), device="cuda", generator=gen)
    x *= torch.exp(0.3 * torch.randn((1, n_q + 2 * n_kv, d), device="cuda", generator=gen))
    return x.half().split([n_q, n_kv, n_kv], dim=1)


_ROPE = {"none": dict(), "linear": dict(factor=4.0), "base": dict(factor=8.0), "bands": dict(factor=8.0, original=8192, low=1.0, high=4.0),
         "ramp": dict(factor=16.0, original=8192, low=1.0, high=32.0)}


def _rope_settings(case):
    s = dict(factor=1.0, original=0, low=1.0, high=1.0)
    s.update(_ROPE[case["scaling"]])
    return dict(s, rotary=case["rotary"], base=10000.0 if case["d"] == 64 else 500000.0, scaling=case["scaling"])


def _frequencies(s):
    """Radians per position of each pair, in 64 bits, and the factor on cosine and sine."""
    r, base, scaling, factor = s["rotary"], s["base"], s["scaling"], s["factor"]
    if scaling == "base":
        base *= factor ** (r / (r - 2))
    i = torch.arange(r // 2, dtype=torch.float64, device="cuda")
    f = base ** (-2.0 * i / r)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "bands":                                     # kept, slowed, and what lies between, by turns over the original context
        keep = ((s["original"] * f / (2 * math.pi) - s["low"]) / (s["high"] - s["low"])).clamp(0, 1)
        return f * (keep + (1 - keep) / factor), 1.0
    if scaling == "ramp":                                      # the same along the index, on whole indexes
        at = lambda turns: r * math.log(s["original"] / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(at(s["high"])), 0), min(math.ceil(at(s["low"])), r - 1)
        keep = 1 - ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f * (keep + (1 - keep) / factor), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _number(x, fmt):
    x = x.clamp(-R[fmt], R[fmt])
    return x.round().to(torch.int8) if fmt == "int8" else x.to(torch.float8_e4m3fn)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    state = dict(case=case)
    if op == "attend":
        lens = _lens(case)
        state["starts"], state["longest"] = _starts(lens), max(lens)
        state["q"], state["k"], state["v"] = _projection(sum(lens), case["n_q"], case["n_kv"], case["d"], gen)
    elif op == "rope":
        state["q"], state["k"], _ = _projection(case["T"], case["n_q"], case["n_kv"], case["d"], gen)
        state["positions"] = torch.randint(0, case["far"], (case["T"],), device="cuda", generator=gen, dtype=torch.int32)
        state["settings"] = _rope_settings(case)
        state["frequencies"], state["amplitude"] = _frequencies(state["settings"])
    elif op == "append":
        lens, P, H, d, fmt = _lens(case), case["page"], case["n_kv"], case["d"], case["fmt"]
        held = [case["before"] - 7 * b % (case["before"] + 1) if case["before"] else 0 for b in range(case["B"])]
        whole = [a + n for a, n in zip(held, lens)]
        need = torch.tensor([-(-n // P) for n in whole], device="cuda")
        n_pages, width = int(need.sum()) + 3, max(1, int(need.max()))
        perm = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
        at = torch.arange(width, device="cuda")[None]
        flat = ((need.cumsum(0) - need)[:, None] + at).clamp(max=n_pages - 1)
        state["tables"] = torch.where(at < need[:, None], perm[flat], -1).contiguous()
        state["cache"] = []
        for _ in "kv":                                         # numbers of earlier use everywhere
            x = torch.randn((n_pages, H, P, d), device="cuda", generator=gen) * torch.exp(0.3 * torch.randn((n_pages, H, 1, 1), device="cuda", generator=gen))
            amax = x.abs().amax(dim=(2, 3)).half().float()
            state["cache"] += [_number(x * (R[fmt] / amax)[:, :, None, None], fmt), amax]
        _, state["k"], state["v"] = _projection(sum(lens), H, H, d, gen)
        state["starts"], state["longest"] = _starts(lens), max(lens)
        state["seq_lens"] = torch.tensor(whole, dtype=torch.int32, device="cuda")
    else:
        G, W, V, L = case["G"], case["W"], case["V"], case["max_len"]
        logits = torch.randn((G * W, V), device="cuda", generator=gen)
        logits *= 2.5
        # part of the vocabulary is never generated
        logits[:, V // 3: V // 3 + V // 20] = -math.inf
        state["logits"], state["eos"] = logits, V - 1
        lengths = torch.randint(0, L, (G, 1), device="cuda", generator=gen).expand(G, W).clone()
        scores = -2.0 * torch.rand((G, W), device="cuda", generator=gen) * (1 + lengths).sqrt()
        finished = torch.rand((G, W), device="cuda", generator=gen) < case["done"]
        if case["first"]:                                      # every beam of a group is the same yet: only one counts
            lengths.zero_()
            finished.zero_()
            scores = torch.where(torch.arange(W, device="cuda")[None] == 0, 0.0, -math.inf).expand(G, W)
        tokens = torch.randint(0, V, (G, W, L), device="cuda", generator=gen, dtype=torch.int32)
        # ended beams are up to half as long as the others
        lengths = torch.where(finished, (lengths + 1) // 2 + 1, lengths).clamp(max=L)
        state["saved"] = [scores.float().contiguous(), lengths.int().contiguous(), finished.int().contiguous(), tokens]
        state["parts"] = [x.clone() for x in state["saved"]]
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
    if op == "attend":
        if own:
            return _context(case["n_q"], case["n_kv"], case["d"]).lookat_attend_packed(state["q"], state["k"], state["v"], state["starts"])
        return _plain_attend(state)
    if op == "rope":
        if own:
            if "table" not in state:                           # a program makes it once
                from paper_2601_10155_b200.binding import RopeTable
                s = state["settings"]
                state["table"] = RopeTable(s["rotary"], s["base"], s["scaling"], s["factor"], s["original"], s["low"], s["high"])
            return list(_context(case["n_q"], case["n_kv"], case["d"]).lookat_rope(state["q"], state["k"], state["positions"], state["table"],
                                                                                   interleaved=case["interleaved"]))
        return _plain_rope(state)
    if op == "append":
        if own:
            if "handle" not in state:                          # a program makes it with its cache and keeps it
                from paper_2601_10155_b200.binding import Q8Cache
                state["handle"] = Q8Cache(*state["cache"])
            _context(case["n_kv"], case["n_kv"], case["d"]).lookat_q8_append_packed(state["handle"], state["k"], state["v"], state["starts"], state["tables"],
                                                                                    state["seq_lens"])
            return list(state["cache"])
        return _plain_append(state)
    torch._foreach_copy_(state["parts"], state["saved"])       # every pass begins where the first one began
    if own:
        if "handle" not in state:
            from paper_2601_10155_b200.binding import BeamState
            state["handle"] = BeamState(*state["parts"])
        ids, parents = _context(12, 12, 64).lookat_beam_select(state["handle"], state["logits"], eos=state["eos"], length_penalty=case["penalty"])
    else:
        ids, parents = _plain_beam(state)
    return [*state["parts"], ids, parents]


# ---- plain forms
def _padded(state):
    """Of every place of the padded batch [B][longest]: the token that stands there, and whether there is one."""
    starts = state["starts"].long()
    at = starts[:-1, None] + torch.arange(state["longest"], device="cuda")[None]
    there = at < starts[1:, None]
    return torch.where(there, at, 0), there


def _plain_attend(state):
    case, q, k, v = state["case"], state["q"], state["k"], state["v"]
    at, there = _padded(state)
    B, n = at.shape
    H, g, d = case["n_kv"], case["n_q"] // case["n_kv"], case["d"]
    rows = lambda x: (x[at].float() * there[..., None, None]).permute(0, 2, 1, 3)                # noqa: E731   [B][heads][n][d]
    s = rows(q).reshape(B, H, g * n, d) @ rows(k).transpose(2, 3)
    s = s.view(B, H, g, n, n)
    s *= 1.0 / math.sqrt(d)
    later = torch.ones((n, n), dtype=torch.bool, device="cuda").triu_(1)
    s.masked_fill_(later, -math.inf)
    s -= s.amax(dim=-1, keepdim=True)
    s.exp_()
    total = s.sum(dim=-1, keepdim=True)
    o = (s.view(B, H, g * n, n) @ rows(v)).view(B, H, g, n, d) / total
    return o.permute(0, 3, 1, 2, 4).reshape(B, n, H * g, d)[there].half()


def _plain_rope(state):
    case = state["case"]
    r, c = case["rotary"], case["rotary"] // 2
    angle = state["positions"].double()[:, None] * state["frequencies"]
    cos, sin = ((t * state["amplitude"]).float()[:, None] for t in (angle.cos(), angle.sin()))    # [T][1][pairs]

    def turned(x):
        y = x.float()
        a, b = (y[..., 0:r:2], y[..., 1:r:2]) if case["interleaved"] else (y[..., :c], y[..., c:r])
        pair = a * cos - b * sin, b * cos + a * sin
        front = torch.stack(pair, dim=-1).flatten(-2) if case["interleaved"] else torch.cat(pair, dim=-1)
        return torch.cat([front, y[..., r:]], dim=-1).half()

    return [turned(state["q"]), turned(state["k"])]


def _shrunk(x, fmt):
    return x.round().to(torch.int8) if fmt == "int8" else x.to(torch.float8_e4m3fn)


def _plain_write(state, x, n8, amax, page, off, heads):
    """The new tokens of keys or of values into their blocks; heads: rows whose first block holds tokens already."""
    case, fmt = state["case"], state["case"]["fmt"]
    head_page, older = heads
    x = torch.nan_to_num(x.float(), nan=0.0, posinf=F16_MAX, neginf=-F16_MAX)                     # [tokens][H][d]
    raw = n8.view(torch.uint8)
    a_old = amax[head_page]                                                                       # [rows][H]
    amax[page] = 0.0
    amax[head_page] = a_old
    amax.index_reduce_(0, page, x.abs().amax(dim=-1), "amax")
    a = amax[head_page]
    had = raw[head_page].view(n8.dtype)
    redone = _shrunk(torch.where(a > 0, 1.0, 0.0)[..., None, None] * had.float() * a_old[..., None, None] / torch.where(a > 0, a, 1.0)[..., None, None], fmt)
    change = older[:, None, :, None] & (a > a_old)[..., None, None]
    raw[head_page] = torch.where(change, redone.view(torch.uint8), had.view(torch.uint8))
    a = amax[page][..., None]
    raw[page, :, off] = _shrunk(torch.where(a > 0, R[fmt] * x / torch.where(a > 0, a, 1.0), 0.0), fmt).view(torch.uint8)


def _plain_append(state):
    case, tables = state["case"], state["tables"].long()
    P = case["page"]
    at, there = _padded(state)
    count = there.sum(dim=1)
    first = state["seq_lens"].long() - count
    pos = (first[:, None] + torch.arange(state["longest"], device="cuda")[None])[there]           # of every new token
    row = torch.arange(case["B"], device="cuda")[:, None].expand_as(there)[there]
    page, off = tables[row, pos // P], pos % P
    begun = ((first % P != 0) & (count > 0)).nonzero()[:, 0]
    heads = tables[begun, first[begun] // P], torch.arange(P, device="cuda")[None] < (first[begun] % P)[:, None]
    k8, ka, v8, va = state["cache"]
    _plain_write(state, state["k"], k8, ka, page, off, heads)
    _plain_write(state, state["v"], v8, va, page, off, heads)
    return list(state["cache"])


def _plain_beam(state):
    case, eos = state["case"], state["eos"]
    G, W, V, L = case["G"], case["W"], case["V"], case["max_len"]
    scores, lengths, finished, tokens = state["parts"]
    x = state["logits"].double()
    top = x.amax(dim=-1, keepdim=True)
    x -= top
    lse = torch.log(x.exp().sum(dim=-1, keepdim=True))
    x -= lse
    x += scores.double().view(G * W, 1)
    x = x.view(G, W, V)
    done = finished.bool()
    # an ended beam goes on as it is, under its last token's number
    x.masked_fill_(done[..., None], -math.inf)
    x[..., eos] = torch.where(done, scores.double(), x[..., eos])
    grown = torch.where(done, lengths, lengths + 1)
    x.nan_to_num_(nan=-math.inf, neginf=-math.inf)
    rank = x / grown.clamp(min=1).double().pow(case["penalty"])[..., None]
    # the best, equal ones by their index
    r, i = rank.view(G, W * V).topk(min(W + 8, W * V), dim=-1)
    i, order = i.sort(dim=-1)
    r, order = r.gather(1, order).sort(dim=-1, descending=True, stable=True)
    r, i = r[:, :W], i.gather(1, order)[:, :W]
    if r.shape[1] < W:
        r = torch.nn.functional.pad(r, (0, W - r.shape[1]), value=-math.inf)
        i = torch.nn.functional.pad(i, (0, W - i.shape[1]))
    there = r > -math.inf
    own_place = torch.arange(W, device="cuda")[None].expand(G, W)
    parent = torch.where(there, i // V, own_place)
    ids = torch.where(there, i % V, eos)
    ended = done.gather(1, parent)
    was = lengths.gather(1, parent)
    new = torch.where(there, x.view(G, W * V).gather(1, i), -math.inf).float()
    grows = there & ~ended
    history = tokens.gather(1, parent[..., None].expand(G, W, L))
    slot = torch.arange(L, device="cuda")[None, None] == was[..., None]
    tokens.copy_(torch.where(slot & grows[..., None], ids[..., None].int(), history))
    scores.copy_(new)
    lengths.copy_(was + grows)
    finished.copy_(ended | (grows & (ids == eos)))
    base = W * torch.arange(G, device="cuda")[:, None]
    return ids.int().reshape(-1), (base + parent).int().reshape(-1)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    op = case["op"]
    if op == "attend":
        lens, d = _lens(case), case["d"]
        return {"bytes": sum(lens) * d * 2 * (2 * case["n_q"] + 2 * case["n_kv"]) + 4 * (len(lens) + 1),
                "flops": 4 * d * case["n_q"] * sum(n * (n + 1) // 2 for n in lens)}
    if op == "rope":
        heads = case["n_q"] + case["n_kv"]
        return {"bytes": case["T"] * (heads * case["d"] * 4 + 4), "flops": case["T"] * heads * case["rotary"] * 3}
    if op == "append":
        new, H, d, P = sum(_lens(case)), case["n_kv"], case["d"], case["page"]
        return {"bytes": new * H * 2 * d * 3 + 8 * H * sum(-(-n // P) for n in _lens(case)), "flops": 4 * new * H * d}
    rows = case["G"] * case["W"]
    return {"bytes": rows * (case["V"] * 4 + 2 * 4 * (3 + case["max_len"] // 2) + 8), "flops": 4 * rows * case["V"]}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    op = case["op"]
    state = prepare(case, seed)
    if op == "attend":
        q, k, v, starts = state["q"], state["k"], state["v"], state["starts"].tolist()
        g, out = case["n_q"] // case["n_kv"], torch.zeros(state["q"].shape, dtype=torch.float64, device="cuda")
        for lo, hi in zip(starts[:-1], starts[1:]):
            for h in range(case["n_q"]):
                kk, vv = k[lo:hi, h // g].double(), v[lo:hi, h // g].double()
                for at in range(lo, hi, 2048):
                    end = min(hi, at + 2048)
                    s = q[at:end, h].double() @ kk[: end - lo].T / math.sqrt(case["d"])
                    i, j = torch.arange(at, end, device="cuda"), torch.arange(lo, end, device="cuda")
                    out[at:end, h] = torch.softmax(torch.where(j[None] <= i[:, None], s, -math.inf), dim=1) @ vv[: end - lo]
        return out
    if op == "rope":
        s, p = state["settings"], state["positions"].tolist()
        f, amplitude = _frequencies(s)
        turn = torch.polar(torch.full((len(p), f.numel()), amplitude, dtype=torch.float64, device="cuda"),
                           torch.tensor(p, dtype=torch.float64, device="cuda")[:, None] * f)[:, None]
        res = []
        for x in (state["q"], state["k"]):
            y, r = x.double(), s["rotary"]
            z = torch.view_as_complex(y[..., :r].unflatten(-1, (r // 2, 2) if case["interleaved"] else (2, r // 2)).transpose(-1, -1 if case["interleaved"] else -2).contiguous())
            z = torch.view_as_real(z * turn)
            y[..., :r] = (z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2)
            res.append(y)
        return res
    if op == "beam":
        # the scores of the chosen candidates, by a search over sorted lists of each beam's best
        G, W, V = case["G"], case["W"], case["V"]
        scores, lengths, finished, _ = (x.tolist() if i < 3 else None for i, x in enumerate(state["saved"]))
        best = torch.full((G, W), -math.inf, dtype=torch.float64)
        for gr in range(G):
            found = []
            for w in range(W):
                if scores[gr][w] == -math.inf:
                    continue
                if finished[gr][w]:
                    found.append((scores[gr][w] / max(1, lengths[gr][w]) ** case["penalty"], scores[gr][w]))
                    continue
                p = torch.log_softmax(state["logits"][gr * W + w].double(), dim=0).topk(min(W, V)).values.tolist()
                found += [((scores[gr][w] + y) / (lengths[gr][w] + 1) ** case["penalty"], scores[gr][w] + y) for y in p if y > -math.inf]
            found = sorted(found, key=lambda y: -y[0])[:W]
            best[gr, : len(found)] = torch.tensor([y[1] for y in found], dtype=torch.float64)
        return [best, None, None, None, None, None]
    # the cache: its numbers are whole numbers or have one right value each; only the scales and e4m3's numbers are computed ones
    k8, ka, v8, va = state["cache"]
    lens, tables, P, fmt = state["seq_lens"].tolist(), state["tables"].tolist(), case["page"], case["fmt"]
    starts, res = state["starts"].tolist(), []
    for n8, amax, x in ((k8, ka, state["k"]), (v8, va, state["v"])):
        num, a = n8.double(), amax.double()
        for b, n in enumerate(lens):
            c = starts[b + 1] - starts[b]
            for i in range((n - c) // P, -(-n // P)) if c else ():
                lo, hi, p = max(i * P, n - c), min(i * P + P, n), tables[b][i]
                new = x[starts[b] + lo - (n - c): starts[b] + hi - (n - c)].double().transpose(0, 1)
                was = a[p] if lo > i * P else torch.zeros_like(a[p])
                now = torch.maximum(was, new.abs().amax(dim=(1, 2)))
                if lo > i * P:
                    kept = num[p, :, : lo - i * P]
                    num[p, :, : lo - i * P] = torch.where((now > was)[:, None, None], _number8(kept * was[:, None, None] / now[:, None, None], fmt), kept)
                num[p, :, lo - i * P: hi - i * P] = _number8(R[fmt] * new / now[:, None, None], fmt)
                a[p] = now
        res += [num, a]
    return res


def _number8(x, fmt):
    """The 8-bit number nearest to x, ties to the even one, as the value it is."""
    if fmt == "int8":
        return torch.round(x)
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (e - 1).clamp(min=-6) - 3)      # three fraction bits; subnormals below 2^-6
    return (torch.round(x / step) * step).clamp(-448, 448)
