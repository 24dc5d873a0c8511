"""Decoding with a paged cache of keys and values, as cases that can be timed and whose outputs can be compared: the pages and slots of requests from their lengths,
writing keys and values into the pages (and reading them back), and the attention of one new token of each request over them.

The plain forms below are elementary torch operations in 32 bits, rounded once at the end.  Where `own` is true, run() calls the library.

A request's tokens lie in pages of `page` tokens; table[b, i] is the page of its tokens i page .. i page + page - 1, and slot id page + r is row r of page id.  Free pages are
the stack pool[0:left].  8-bit caches hold codes and a scale for each token and head: scale max|x| / 127 (i8) or / 448 (fp8), 1 where all are zero."""
import math
import random

import torch

own = False

DEV = "cuda"
TORCH_TYPE = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
LARGEST = {"i8": 127.0, "fp8": 448.0}


def listed():
    def tables(name, B, L, page, what):
        return {"name": name, "op": "tables", "B": B, "L": L, "page": page, "what": what}

    def write(name, N, H, D, dtype, source, page=64):
        return {"name": name, "op": "write", "N": N, "H": H, "D": D, "dtype": dtype, "source": source, "page": page}

    def attention(name, B, L, Hq, H, D, dtype, page=64, ragged=False, window=0, source="bf16"):
        return {"name": name, "op": "attention", "B": B, "L": L, "Hq": Hq, "H": H, "D": D, "dtype": dtype, "page": page, "ragged": ragged, "window": window, "source": source}

    return [
        # a decode step: every request of a batch gets one token more, a page now and then
        tables("tables_decode_b64", 64, 2048, 64, "decode"),
        # a step of a busy server: prompts come in, requests go, the others decode
        tables("tables_mixed_b256", 256, 2048, 32, "mixed"),
        # keys and values of one decoded token: nothing but launches
        write("write_n1", 1, 8, 128, "bf16", "bf16"),
        # a prompt of odd length, odd heads, 32-bit activations
        write("write_n777_i8", 777, 5, 80, "i8", "fp32", page=32),
        # a prompt's tokens, quantised on the way
        write("write_n8192_fp8", 8192, 8, 128, "fp8", "bf16"),
        # one short conversation: latency
        attention("attend_b1_l500", 1, 500, 32, 8, 128, "bf16"),
        # one long document
        attention("attend_b1_l131072", 1, 131072, 28, 4, 128, "bf16", page=128),
        # a served batch, requests of all lengths
        attention("attend_b64_ragged", 64, 16384, 32, 8, 128, "bf16", ragged=True),
        # the same from a cache of half the bytes
        attention("attend_b64_ragged_fp8", 64, 16384, 32, 8, 128, "fp8", ragged=True),
        # few requests, odd sizes, 32-bit queries
        attention("attend_b7_i8_odd", 7, 3001, 15, 5, 80, "i8", page=32, ragged=True, source="fp32"),
        # heads of their own keys, of which only the last are seen
        attention("attend_b16_window", 16, 8192, 16, 16, 64, "fp16", page=32, window=1500),
        # a large batch
        attention("attend_b256_l4096", 256, 4096, 28, 4, 128, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(28, 4), (32, 8), (8, 8), (12, 2), (16, 1), (15, 5), (40, 2), (1, 1)]
MAX_WRITE = 8192 * 8 * 128
MAX_CACHED = 256 * 4096 * 4 * 128                       # values of keys


def draw(rng):
    """One operator over the whole ranges: 1 .. 256 requests, contexts 1 .. 131072 tokens, heads of 16 .. 256 values, query heads 1 .. 20 to a head of keys, pages of 32 .. 256."""
    op = rng.choice(["tables", "write", "attention", "attention", "attention"])
    page = rng.choice([32, 64, 128, 256])
    if op == "tables":
        return {"op": op, "B": _log_int(rng, 1, 256), "L": _log_int(rng, 16, 2048), "page": page, "what": rng.choice(["decode", "mixed", "mixed", "full"])}
    Hq, H = rng.choice(HEADS)
    D = rng.choice([64, 80, 96, 128, 128, 192, 256, rng.randint(16, 256)])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp8", "i8"])
    source = rng.choice(["bf16", "bf16", "fp32"])
    while True:
        if op == "write":
            c = {"op": op, "N": _log_int(rng, 1, 8192), "H": H, "D": D, "dtype": dtype, "source": source, "page": page}
            if c["N"] * H * D <= MAX_WRITE:
                return c
        else:
            L = _log_int(rng, 1, 131072)
            c = {"op": op, "B": _log_int(rng, 1, 256), "L": L, "Hq": Hq, "H": H, "D": D, "dtype": dtype, "page": page, "ragged": rng.random() < 0.5,
                 "window": _log_int(rng, 1, L) if rng.random() < 0.25 else 0, "source": source}
            if c["B"] * (L + page) * H * D <= MAX_CACHED:
                return c


# ---- lengths, which are the case's own -------------------------------------------------------------------------------------------

def _lengths(case):
    """Tokens of each request: L each, or spread over their logarithm up to L with an empty one now and then."""
    B, L = case["B"], case["L"]
    if not case["ragged"]:
        return [L] * B
    rng = random.Random(B * 1000003 + L)
    return [L] + [0 if rng.random() < 0.02 else _log_int(rng, max(1, L // 64), L) for _ in range(B - 1)]


def _requests(case):
    """(lengths, wanted lengths, free pages) of a step."""
    B, L, page = case["B"], case["L"], case["page"]
    rng = random.Random(B * 1000003 + L)
    if case["what"] == "decode":
        lens = [rng.randint(1, L - 1) for _ in range(B)]
        want = [n + 1 for n in lens]
    else:
        kind = [rng.random() for _ in range(B)]
        lens = [0 if k < 0.25 else rng.randint(1, L - 1) for k in kind]
        want = [rng.randint(1, L) if k < 0.25 else 0 if k < 0.4 else max(n - 3, 0) if k < 0.45 else n + 1 for k, n in zip(kind, lens)]
    more = sum(max(0, -(-w // page) - -(-n // page)) for w, n in zip(want, lens))
    return lens, want, max(1, more // 2) if case["what"] == "full" else more + 8       # full: half of what it takes, so that some are left out


def _new_tokens(case):
    lens, want, _ = _requests(case)
    return max(1, sum(max(0, w - n) for w, n in zip(want, lens)) + 7)     # a batch is padded


# ---- the plain forms ---------------------------------------------------------------------------------------------------------

def plain_tables(s):
    page, N, W, P = s["page"], s["N"], s["table"].shape[1], s["pool"].shape[0]
    lens, want, left = s["lens"].long(), s["want"].long(), s["left"].long()
    have, need = (lens + page - 1) // page, (want + page - 1) // page
    ends = torch.cumsum((want - lens).clamp(min=0), 0)
    starts = ends - (want - lens).clamp(min=0)
    possible = (need <= W) & (ends <= N)
    more = torch.where(possible, (need - have).clamp(min=0), 0)
    columns = torch.arange(W, device=lens.device)
    freed = ((columns >= need[:, None]) & (columns < have[:, None])).reshape(-1)
    place = torch.where(freed, left + torch.cumsum(freed.long(), 0) - 1, P)
    pool = torch.cat([s["pool"], s["pool"][:1]])
    pool.scatter_(0, place, s["table"].reshape(-1))
    s["pool"].copy_(pool[:P])
    pages = left + freed.sum()
    upto = torch.cumsum(more, 0)
    served = (want <= lens) | (possible & ((more == 0) | (upto <= pages)))
    taken = torch.where(served & (more > 0), upto, 0).amax()
    i = torch.arange(N, device=lens.device)
    b = (i[:, None] >= ends).sum(1)
    there = b < lens.shape[0]
    b = b.clamp(max=lens.shape[0] - 1)
    position = lens[b] + i - starts[b]
    column = position // page
    there = there & served[b]
    new = there & (column >= have[b])
    from_pool = pool[torch.where(new, pages - 1 - (upto[b] - more[b] + column - have[b]), 0)]
    cell = b * W + torch.where(there, column, 0)
    ids = torch.where(new, from_pool, s["table"].reshape(-1)[cell])
    slots = torch.where(there, ids.long() * page + position % page, -1)
    table = torch.cat([s["table"].reshape(-1), s["pool"][:1]])
    table.scatter_(0, torch.where(new, cell, table.shape[0] - 1), ids)
    s["table"].copy_(table[:-1].view(-1, W))
    offsets = torch.cat([torch.zeros_like(ends[:1]), ends]).clamp(max=N)
    return {"lens": torch.where(served, want, lens).int(), "left": (pages - taken).int(), "slots": slots.int(), "offsets": offsets.int(), "table": s["table"], "pool": s["pool"]}


def _e4m3(x):
    """The nearest of the 8-bit values, ties to even, as a number in the type of x; |x| <= 448."""
    exponent = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(exponent - 3)
    return torch.round(x / step) * step


def plain_codes(x, dtype):
    """x[..., D] -> what the cache holds of it: values of 16 bits and no scales, or codes (as numbers of 16 bits, which hold them exactly) and scales[...]."""
    if dtype not in LARGEST:
        return x.to(TORCH_TYPE[dtype]), None
    x = x.float()
    largest = x.abs().amax(-1)
    some = largest > 0
    inverse = torch.where(some, LARGEST[dtype] / largest, 1.0)
    y = (x * inverse[..., None]).clamp(-LARGEST[dtype], LARGEST[dtype])
    y = torch.round(y) if dtype == "i8" else _e4m3(y)
    return y.to(torch.bfloat16), torch.where(some, largest / LARGEST[dtype], 1.0)


def plain_values(codes, scales):
    return codes.float() if scales is None else codes.float() * scales[..., None]


def plain_write(s):
    """Into the cache at the tokens' slots, and out of it again."""
    slots, out = s["slots"].long(), []
    for name in ("K", "V"):
        codes, scales = plain_codes(s[name], s["dtype"])
        s["codes_" + name][slots] = codes
        held = s["codes_" + name][slots]
        if scales is not None:
            s["scales_" + name][slots] = scales
            scales = s["scales_" + name][slots]
        out.append(plain_values(held, scales).to(s[name].dtype))
    return {"K": out[0], "V": out[1]}


def plain_attention(s):
    B, Hq, D = s["q"].shape
    H, page = s["H"], s["page"]
    token = (s["table"].long()[:, :, None] * page + torch.arange(page, device=s["q"].device)).view(B, -1)
    k, v = (plain_values(s["codes_" + n][token], None if s["scales_" + n] is None else s["scales_" + n][token]).transpose(1, 2) for n in ("K", "V"))      # [B, H, tokens, D]
    q = s["q"].float().view(B, H, Hq // H, D)
    scores = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(D)
    t = torch.arange(token.shape[1], device=q.device)
    lens = s["lens"].long()[:, None]
    seen = (t < lens) & (t >= (lens - s["window"] if s["window"] else 0))
    scores = torch.where(seen[:, None, None, :], scores, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    return out.view(B, Hq, D).to(torch.bfloat16)


# ---- inputs --------------------------------------------------------------------------------------------------------------------

def _keys(g, N, H, D, dtype):
    """Keys or values of N tokens as rows of a projection's result: N(0, 1) with a few channels 8 times as large, as keys have them."""
    x = torch.randn((N, H * D), generator=g, device=DEV)
    x[:, torch.randint(0, H * D, (max(1, H * D // 64),), generator=g, device=DEV)] *= 8
    return x.to(dtype).view(N, H, D)


def _pages_of(g, counts, W, spare=3):
    """A table of W columns whose rows name counts[b] pages of a cache in any order, and the number of pages; the free ones are those behind."""
    used = sum(counts)
    order = torch.randperm(used + spare, generator=g, device=DEV).int()
    B = len(counts)
    count = torch.tensor(counts, device=DEV)
    column = torch.arange(W, device=DEV)
    place = torch.where(column < count[:, None], torch.cumsum(count, 0)[:, None] - count[:, None] + column, used + spare)
    table = torch.cat([order, torch.zeros(1, dtype=torch.int32, device=DEV)])[place]
    return table.view(B, W).contiguous(), order, used


def _cache(s, case, P):
    """An empty cache: the library's pages, or rows of codes by slot."""
    if own:
        from paper_2603_05232_amd import binding
        s["pages"] = torch.zeros((P, binding.kv_page_bytes(case["H"], case["page"], case["D"], case["dtype"])), dtype=torch.uint8, device=DEV)
        return
    held = TORCH_TYPE.get(case["dtype"], torch.bfloat16)
    for n in ("K", "V"):
        s["codes_" + n] = torch.zeros((P * case["page"], case["H"], case["D"]), dtype=held, device=DEV)
        s["scales_" + n] = torch.ones((P * case["page"], case["H"]), device=DEV) if case["dtype"] in LARGEST else None


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    op, page = case["op"], case["page"]
    s = {"op": op, "page": page}
    if op == "tables":
        lens, want, free = _requests(case)
        turn = torch.randperm(case["B"], generator=g, device=DEV).tolist()
        lens, want = [lens[i] for i in turn], [want[i] for i in turn]
        W = -(-(case["L"] + 1) // page)
        s["table"], order, used = _pages_of(g, [-(-n // page) for n in lens], W, spare=free)
        s["pool"] = torch.cat([order[used:], order[:used]])                # used ones lie above the free ones, where they do not count
        s["left"] = torch.tensor([free], dtype=torch.int32, device=DEV)
        s["lens"], s["want"] = (torch.tensor(n, dtype=torch.int32, device=DEV) for n in (lens, want))
        s["N"] = _new_tokens(case)
        if own:
            from paper_2603_05232_amd import binding
            n = binding.kv_tables_workspace_bytes(case["B"], s["N"])
            s["workspace"] = torch.empty((n,), dtype=torch.uint8, device=DEV) if n else None
        return s
    s.update(dtype=case["dtype"], H=case["H"], D=case["D"])
    source = TORCH_TYPE[case["source"]]
    if op == "write":                                   # one prompt, or the piece of one that begins where a page is half full
        N, at = case["N"], page // 2 + 1 if case["N"] % 2 else 0
        table, _, used = _pages_of(g, [-(-(N + at) // page)], -(-(N + at) // page))
        position = torch.arange(N, device=DEV) + at
        s["slots"] = (table[0].long()[position // page] * page + position % page).int()
        s["K"], s["V"] = (_keys(g, N, case["H"], case["D"], source) for _ in "KV")
        _cache(s, case, used + 3)
        return s
    lens, H, D = _lengths(case), case["H"], case["D"]
    W = max(1, -(-max(lens) // page))
    counts = [-(-n // page) for n in lens]
    s["table"], _, used = _pages_of(g, counts, W)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["q"] = _keys(g, case["B"], case["Hq"], D, source)
    s["window"] = case["window"]
    P = used + 3
    _cache(s, case, P)
    step = max(page, 1 << 18)
    for first in range(0, P * page, step):              # every slot holds something, also those that nobody sees
        n = min(step, P * page - first)
        k, v = (_keys(g, n, H, D, torch.bfloat16) for _ in "KV")
        if own:
            from paper_2603_05232_amd import binding
            binding.kv_write(k, v, torch.arange(first, first + n, dtype=torch.int32, device=DEV), s["pages"], page, case["dtype"])
        else:
            for name, x in (("K", k), ("V", v)):
                codes, scales = plain_codes(x, case["dtype"])
                s["codes_" + name][first:first + n] = codes
                if scales is not None:
                    s["scales_" + name][first:first + n] = scales
    if own:
        n = binding.kv_attention_workspace_bytes(case["B"], case["Hq"], H, D)
        s["workspace"] = torch.empty((n,), dtype=torch.uint8, device=DEV) if n else None
    return s


def run(s):
    op = s["op"]
    if own:
        from paper_2603_05232_amd import binding
        if op == "tables":
            lens, left, slots, offsets = binding.kv_tables(s["lens"], s["want"], s["table"], s["pool"], s["left"], s["page"], s["N"], workspace=s["workspace"])
            return {"lens": lens, "left": left, "slots": slots, "offsets": offsets, "table": s["table"], "pool": s["pool"]}
        if op == "write":
            binding.kv_write(s["K"], s["V"], s["slots"], s["pages"], s["page"], s["dtype"])
            return dict(zip("KV", binding.kv_read(s["pages"], s["slots"], s["H"], s["D"], s["page"], s["dtype"], s["K"].dtype)))
        return binding.kv_attention(s["q"], s["pages"], s["table"], s["lens"], s["H"], s["page"], s["dtype"], window=s["window"], workspace=s["workspace"])
    return {"tables": plain_tables, "write": plain_write, "attention": plain_attention}[op](s)


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------------

def _exact_held(x, dtype):
    """What an 8-bit or 16-bit cache holds of x."""
    if dtype not in LARGEST:
        return x.to(TORCH_TYPE[dtype]).double()
    x = x.double()
    a = x.abs().amax(-1, keepdim=True)
    unit = torch.where(a > 0, a / LARGEST[dtype], 1.0)
    y = x / unit
    if dtype == "fp8":
        step = torch.exp2(torch.frexp(y)[1].double().clamp(min=-5) - 4)
        return torch.round(y / step) * step * unit
    return torch.round(y) * unit


def exact(case, seed):
    global own
    if case["op"] == "tables":                          # whole numbers
        return None
    was, own = own, False                               # rows of codes, not the library's pages
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "write":
        return {n: _exact_held(s[n], case["dtype"]) for n in ("K", "V")}
    lens, page, H, D = _lengths(case), case["page"], case["H"], case["D"]
    out = torch.zeros((case["B"], case["Hq"], D), dtype=torch.float64, device=DEV)
    for b, n in enumerate(lens):
        first = max(0, n - case["window"]) if case["window"] else 0
        if n == first:
            continue
        t = torch.arange(first, n, device=DEV)
        rows = s["table"][b].long()[t // page] * page + t % page
        k, v = (s["codes_" + x][rows].double() * (1.0 if s["scales_" + x] is None else s["scales_" + x][rows].double()[..., None]) for x in "KV")
        q = s["q"][b].double().view(H, -1, D)
        p = torch.softmax(torch.bmm(q, k.permute(1, 2, 0).contiguous()) * D ** -0.5, dim=-1)
        out[b] = torch.bmm(p, v.transpose(0, 1).contiguous()).reshape(-1, D)
    return out


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------------

HELD_BYTES = {"bf16": 2, "fp16": 2, "fp8": 1, "i8": 1}


def work(case):
    if case["op"] == "tables":                          # lengths in and out, slots, table entries that are read or written, offsets
        lens, want, _ = _requests(case)
        pages = sum(abs(-(-w // case["page"]) - -(-n // case["page"])) for w, n in zip(want, lens))
        return {"bytes": 16 * case["B"] + 4 * _new_tokens(case) + 8 * pages + 8, "flops": 0}
    held = HELD_BYTES[case["dtype"]]
    per = case["H"] * (2 * case["D"] * held + (8 if held == 1 else 0))       # bytes of a token's keys and values
    es = 4 if case["source"] == "fp32" else 2
    if case["op"] == "write":                           # values in, codes out; codes in, values out
        values = 2 * case["N"] * case["H"] * case["D"]
        return {"bytes": 2 * values * es + 2 * case["N"] * per + 8 * case["N"], "flops": 4 * values}
    tokens = sum(min(n, case["window"]) if case["window"] else n for n in _lengths(case))
    rows = case["B"] * case["Hq"] * case["D"]
    return {"bytes": tokens * per + rows * (es + 2) + 4 * case["B"] + 4 * tokens // case["page"], "flops": 4 * case["Hq"] * case["D"] * tokens}
