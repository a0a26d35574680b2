"""The paged key/value cache as a server uses it, as cases that can be timed and compared.

Three operators of ``paper_2601_21896_b200.binding``: the block tables and slot map of a step from
the requests' lengths (``pafu_paged_tables``), the new tokens' rows written into the pages
(``pafu_paged_append``) and the attention of one new token a request over its pages
(``pafu_paged_attn``).  ``run`` computes them in elementary torch operations, or calls the library
where ``own`` is true.  Lengths are drawn from the seed between the case's bounds.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
E4M3_MAX = 448.0


def listed():
    return [
        # the smallest call: one request of 97 tokens, heads of the Tiny configuration (2 x 64); latency only
        dict(name="attn_one_short", op="attn", requests=1, lo=97, hi=97, heads=2, kv_heads=2, d=64, page=16, layout="tokens",
             type="bf16", cache="bf16", sink=0, recent=-1),
        # a batch of short prompts answered by a small model with one shared key head; a few requests have not begun (length 0)
        dict(name="attn_many_short", op="attn", requests=512, lo=0, hi=300, heads=16, kv_heads=1, d=64, page=16, layout="tokens",
             type="f16", cache="f16", sink=0, recent=-1),
        # an ordinary serving batch: grouped heads, 16-token pages, ragged lengths
        dict(name="attn_batch", op="attn", requests=64, lo=100, hi=8192, heads=32, kv_heads=8, d=128, page=16, layout="tokens",
             type="bf16", cache="bf16", sink=0, recent=-1),
        # the repository's layer (12 heads x 128, a head of keys for each) over four videos, a page for each frame of 1560 tokens
        dict(name="attn_frames", op="attn", requests=4, lo=9360, hi=46800, heads=12, kv_heads=12, d=128, page=1560, layout="tokens",
             type="bf16", cache="bf16", sink=0, recent=-1),
        # the same batch size with 40 heads in 8 groups and a cache in 8 bits, pages laid out head by head
        dict(name="attn_e4m3", op="attn", requests=32, lo=1000, hi=16384, heads=40, kv_heads=8, d=128, page=64, layout="heads",
             type="bf16", cache="e4m3", sink=0, recent=-1),
        # one long document: the split over the cache's length
        dict(name="attn_long", op="attn", requests=1, lo=200003, hi=200003, heads=32, kv_heads=4, d=128, page=32, layout="tokens",
             type="bf16", cache="bf16", sink=0, recent=-1),
        # long streams that attend to their first tokens and a recent window, as the retention rule keeps them
        dict(name="attn_sink_recent", op="attn", requests=128, lo=500, hi=20000, heads=32, kv_heads=8, d=128, page=16, layout="heads",
             type="f16", cache="f16", sink=4, recent=1021),
        # one new token of each of 64 requests, rows of 12 heads x 128; latency only
        dict(name="append_decode", op="append", tokens=64, kv_heads=12, d=128, page=16, layout="tokens", type="bf16", cache="bf16",
             fused=True, spare=512),
        # the repository's chunk of 4680 tokens, 40 heads, copied into pages that are laid out head by head
        dict(name="append_chunk", op="append", tokens=4680, kv_heads=40, d=128, page=64, layout="heads", type="f16", cache="f16",
             fused=False, spare=1000),
        # a cache of 28080 tokens filled in 8 bits from fused query/key/value rows
        dict(name="append_prefill_e4m3", op="append", tokens=28080, kv_heads=12, d=128, page=60, layout="tokens", type="bf16",
             cache="e4m3", fused=True, spare=1000),
        # a step of 256 requests that each get one token
        dict(name="tables_decode", op="tables", requests=256, width=512, page=16, lo=1, hi=8000, grow=1, begin=0.0, end=0.0, pad=0),
        # a busy step: many requests, a few begin with long prompts, a few end and give their pages back
        dict(name="tables_admission", op="tables", requests=2000, width=1024, page=16, lo=1, hi=12000, grow=1, begin=0.03, end=0.05,
             pad=100),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "append", "append", "tables"])
    page = rng.choice([1, 8, 16, 16, 24, 32, 60, 64, 128, 1560])
    layout = rng.choice(["tokens", "heads"])
    d = rng.choice([64, 128])
    t = rng.choice(["bf16", "f16"])
    cache = rng.choice([t, t, "e4m3"])
    if op == "attn":
        kv, group = rng.choice([(1, 1), (1, 8), (1, 16), (2, 1), (2, 7), (4, 8), (8, 4), (8, 5), (8, 1), (12, 1), (40, 1), (2, 20)])
        requests = _logint(rng, 1, 300)
        page = 64 if page > 128 and requests > 8 else page       # a pool of mostly empty pages is no use to anyone
        # at most about 0.8 GB of cache in 16 bits
        most = int(8e8 / (requests * kv * d * 4))
        hi = _logint(rng, 1, max(2, min(200000, most)))
        lo = rng.choice([0, 1, hi // 2, hi])
        sink, recent = rng.choice([(0, -1), (0, -1), (4, 256), (0, 1000), (64, 0)])
        return dict(op="attn", requests=requests, lo=min(lo, hi), hi=hi, heads=kv * group, kv_heads=kv, d=d, page=page,
                    layout=layout, type=t, cache=cache, sink=sink, recent=recent)
    if op == "append":
        kv = rng.choice([1, 2, 8, 12, 40])
        tokens = _logint(rng, 1, min(28080, int(1.5e8 / (kv * d * 4))))
        return dict(op="append", tokens=tokens, kv_heads=kv, d=d, page=page, layout=layout, type=t, cache=cache,
                    fused=rng.choice([True, False]), spare=_logint(rng, 1, 1000))
    requests = _logint(rng, 1, 2000)
    page = rng.choice([8, 16, 24, 32, 60])
    hi = _logint(rng, 10, 12000)
    return dict(op="tables", requests=requests, width=-(-(hi + 4) // page) + rng.randint(0, 100), page=page, lo=rng.choice([0, 1, hi // 2]),
                hi=hi, grow=rng.choice([1, 1, 4]), begin=rng.choice([0.0, 0.02, 0.1]), end=rng.choice([0.0, 0.05, 0.2]),
                pad=rng.choice([0, 1, 100]))


def _pool(pages, page, kv, d, layout, dtype, gen):
    """[pages, page, kv, d], stored token by token or head by head in a page."""
    shape = (pages, page, kv, d) if layout == "tokens" else (pages, kv, page, d)
    x = torch.randn(shape, device="cuda", dtype=torch.float16 if dtype == torch.float8_e4m3fn else dtype, generator=gen)
    if dtype == torch.float8_e4m3fn:
        x = (x * 80).clamp_(-E4M3_MAX, E4M3_MAX).to(dtype)      # what a scale of about 1 / 80 makes of values of size 1
    return x if layout == "tokens" else x.transpose(1, 2)


def _lengths(n, lo, hi, cpu):
    return torch.randint(lo, hi + 1, (n,), generator=cpu)


def prepare(case, seed):
    cpu = torch.Generator().manual_seed(seed)
    gen = torch.Generator("cuda").manual_seed(seed)
    return {"attn": _prepare_attn, "append": _prepare_append, "tables": _prepare_tables}[case["op"]](case, cpu, gen)


def _scales(n, gen):
    return (0.01 + 0.005 * torch.rand(n, device="cuda", generator=gen)).float()


def _prepare_attn(c, cpu, gen):
    R, kv, d, page = c["requests"], c["kv_heads"], c["d"], c["page"]
    lens = _lengths(R, c["lo"], c["hi"], cpu)
    if R > 1:
        lens[-1] = c["hi"]
    count = (lens + page - 1) // page
    width, total = max(1, int(count.max())), int(count.sum())
    n_pages = max(1, total + total // 16)
    # the pages of a request lie anywhere in the pool; table entries behind a request's last page are never read
    order = torch.randperm(n_pages, generator=cpu)[:total]
    table = torch.full((R, width), -1, dtype=torch.int64)
    table[torch.arange(width)[None, :] < count[:, None]] = order
    s = dict(c=c, lens=lens.int().cuda(), table=table.int().cuda())
    s["K"] = _pool(n_pages, page, kv, d, c["layout"], DTYPES[c["cache"]], gen)
    s["V"] = _pool(n_pages, page, kv, d, c["layout"], DTYPES[c["cache"]], gen)
    s["ks"] = s["vs"] = None
    if c["cache"] == "e4m3":
        s["ks"], s["vs"] = _scales(kv, gen), _scales(kv, gen)
    t = DTYPES[c["type"]]
    # the new token's queries come out of a fused projection: rows of query, key and value heads
    qkv = torch.randn((R, c["heads"] + 2 * kv, d), device="cuda", generator=gen, dtype=t) * 2
    s["Q"] = qkv[:, : c["heads"]]
    if own:
        from paper_2601_21896_b200 import binding as B
        s["O"] = torch.empty((R, c["heads"], d), device="cuda", dtype=t)
        s["LSE"] = torch.empty((c["heads"], R), device="cuda")
        s["cache"] = B.PagedCache(s["K"], s["V"], s["table"], c["heads"], dtype=t, k_scale=s["ks"], v_scale=s["vs"])
        s["ws"] = torch.zeros(B.pafu_paged_workspace_bytes(s["cache"]), dtype=torch.uint8, device="cuda")
    return s


def _prepare_append(c, cpu, gen):
    n, kv, d, page = c["tokens"], c["kv_heads"], c["d"], c["page"]
    n_pages = -(-(n + c["spare"]) // page)
    slots = torch.randperm(n_pages, generator=cpu)[:, None] * page + torch.arange(page)[None, :]
    slots = slots.reshape(-1)[:n].clone()
    if n > 8:
        slots[n - n // 8:] = -1                 # a padded batch: the last rows belong to no request
    s = dict(c=c, slots=slots.cuda())
    s["K"] = _pool(n_pages, page, kv, d, c["layout"], DTYPES[c["cache"]], gen)
    s["V"] = _pool(n_pages, page, kv, d, c["layout"], DTYPES[c["cache"]], gen)
    s["ks"] = s["vs"] = None
    if c["cache"] == "e4m3":
        s["ks"], s["vs"] = _scales(kv, gen), _scales(kv, gen)
    t = DTYPES[c["type"]]
    if c["fused"]:
        qkv = torch.randn((n, 3 * kv, d), device="cuda", generator=gen, dtype=t)
        s["Kn"], s["Vn"] = qkv[:, kv: 2 * kv], qkv[:, 2 * kv:]
    else:
        s["Kn"] = torch.randn((n, kv, d), device="cuda", generator=gen, dtype=t)
        s["Vn"] = torch.randn((n, kv, d), device="cuda", generator=gen, dtype=t)
    if own:
        from paper_2601_21896_b200 import binding as B
        table = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
        s["cache"] = B.PagedCache(s["K"], s["V"], table, kv, dtype=t, k_scale=s["ks"], v_scale=s["vs"])
        s["ws"] = torch.zeros(B.pafu_paged_workspace_bytes(s["cache"]), dtype=torch.uint8, device="cuda")
    return s


def _begin_end(c):
    return int(c["requests"] * c["begin"]), int(c["requests"] * c["end"])


def _new_tokens(c):
    begin, end = _begin_end(c)
    return (c["requests"] - begin - end) * c["grow"] + begin // 2 * (c["lo"] + c["hi"]) + begin % 2 * c["hi"]


def _prepare_tables(c, cpu, gen):
    R, page, width = c["requests"], c["page"], c["width"]
    old = _lengths(R, c["lo"], c["hi"], cpu)
    new = old + c["grow"]
    # who begins and who ends is drawn; how many do, and the tokens of the step, are the case's, as under a scheduler's
    # token budget: prompts come in pairs of lo + hi tokens
    begin, end = _begin_end(c)
    who = torch.randperm(R, generator=cpu)
    first, last = who[:begin], who[R - end:]
    new[first[1::2]] = c["lo"] + c["hi"] - old[first[: begin // 2 * 2: 2]]
    new[first[::2]] = old[first[::2]]
    if begin % 2:
        new[first[-1]] = c["hi"]
    old[first] = 0
    new[last] = 0
    have = (old + page - 1) // page
    need = ((new + page - 1) // page - have).clamp(min=0)
    held = int(have.sum())
    n_pages = R * -(-(c["hi"] + c["grow"]) // page)
    order = torch.randperm(n_pages, generator=cpu)
    table = torch.full((R, width), -1, dtype=torch.int64)
    table[torch.arange(width)[None, :] < have[:, None]] = order[:held]
    count = int(need.sum()) + min(16, n_pages - held - int(need.sum()))
    free = torch.full((n_pages,), -1, dtype=torch.int64)
    free[:count] = order[held: held + count]
    n_slots = _new_tokens(c) + c["pad"]
    s = dict(c=c, old=old.int().cuda(), new=new.int().cuda(), table=table.int().cuda(), free=free.int().cuda(),
             n_free=torch.tensor([count], dtype=torch.int32, device="cuda"), n_slots=n_slots)
    if own:
        from paper_2601_21896_b200 import binding as B
        s["n_free_out"] = torch.empty(1, dtype=torch.int32, device="cuda")
        s["lens"] = torch.empty(R, dtype=torch.int32, device="cuda")
        s["slots"] = torch.empty(n_slots, dtype=torch.int64, device="cuda")
        s["cu"] = torch.empty(R + 1, dtype=torch.int32, device="cuda")
        pool = torch.empty((n_pages, page, 1, 64), dtype=torch.float8_e4m3fn, device="cuda")
        s["cache"] = B.PagedCache(pool, pool, s["table"], 1, dtype=torch.bfloat16)
        s["ws"] = torch.zeros(B.pafu_paged_workspace_bytes(s["cache"]), dtype=torch.uint8, device="cuda")
    return s


def run(s):
    c = s["c"]
    if own:
        from paper_2601_21896_b200 import binding as B
        if c["op"] == "attn":
            B.pafu_paged_attn(s["cache"], s["Q"], s["lens"], s["O"], s["LSE"], n_sink=c["sink"], n_recent=c["recent"], ws=s["ws"])
            return s["O"], s["LSE"]
        if c["op"] == "append":
            B.pafu_paged_append(s["cache"], s["Kn"], s["Vn"], s["slots"], ws=s["ws"])
            return s["K"], s["V"]
        B.pafu_paged_tables(s["cache"], s["old"], s["new"], s["free"], s["n_free"], s["n_free_out"], s["lens"], s["slots"],
                            s["cu"], ws=s["ws"])
        return s["table"], s["free"], s["n_free_out"], s["lens"], s["slots"], s["cu"]
    return {"attn": _plain_attn, "append": _plain_append, "tables": _plain_tables}[c["op"]](s)


# ------------------------------------------------------------------------------ plain forms
def _plain_attn(s):
    c, T = s["c"], s["lens"]
    R, kv, d, page = c["requests"], c["kv_heads"], c["d"], c["page"]
    group = c["heads"] // kv
    # the kept positions side by side: the first tokens, then the recent ones moved up to them
    longest = s["table"].shape[1] * page
    kept = T.long()
    if c["recent"] >= 0:
        longest = min(longest, c["sink"] + c["recent"])
        kept = kept.clamp(max=c["sink"] + c["recent"])
    j = torch.arange(longest, device="cuda")
    keep = j < kept[:, None]
    pos = torch.where(keep, j + (j >= c["sink"]) * (T - kept)[:, None], torch.zeros_like(j))
    pages = s["table"].long().clamp(min=0).gather(1, pos // page)
    K = s["K"][pages, pos % page].float()                                    # [R, L, kv, d]
    if s["ks"] is not None:
        K = K * s["ks"][:, None]
    q = s["Q"].float().reshape(R, kv, group, d) * (1.0 / math.sqrt(d))
    logits = torch.matmul(q, K.permute(0, 2, 3, 1))                          # [R, kv, group, L]
    del K
    logits = torch.where(keep[:, None, None, :], logits, torch.full_like(logits, -math.inf))
    top = logits.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    V = s["V"][pages, pos % page].float()
    if s["vs"] is not None:
        V = V * s["vs"][:, None]
    V = torch.where(keep[:, :, None, None], V, torch.zeros_like(V))
    o = torch.matmul(p, V.permute(0, 2, 1, 3)) / torch.where(total == 0, torch.ones_like(total), total)
    lse = (top + torch.log(total)).reshape(R, c["heads"]).transpose(0, 1).contiguous()
    return o.reshape(R, c["heads"], d).to(s["Q"].dtype), lse


def _plain_append(s):
    page = s["c"]["page"]
    mine = s["slots"] >= 0
    slots = s["slots"][mine]
    for pool, rows, scale in ((s["K"], s["Kn"], s["ks"]), (s["V"], s["Vn"], s["vs"])):
        rows = rows[mine]
        if pool.dtype == torch.float8_e4m3fn:
            x = (rows.float() / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX)
            pool.view(torch.uint8)[slots // page, slots % page] = x.to(pool.dtype).view(torch.uint8)
        else:
            pool[slots // page, slots % page] = rows
    return s["K"], s["V"]


def _plain_tables(s):
    page, width = s["c"]["page"], s["c"]["width"]
    old, new, table, free = s["old"].long(), s["new"].long(), s["table"].long(), s["free"].long()
    F = s["n_free"].long()
    have, want = (old + page - 1) // page, (new + page - 1) // page
    need, back = (want - have).clamp(min=0), (have - want).clamp(min=0)
    need_end, back_end = need.cumsum(0), back.cumsum(0)
    col = torch.arange(width, device="cuda")
    leaves = (col >= want[:, None]) & (col < have[:, None])
    stack = torch.cat([free, free.new_zeros(1)])
    at = F + (back_end - back)[:, None] + col - want[:, None]
    # released pages on top of the stack; entries that leave nothing go to a place behind it
    stack.index_put_((torch.where(leaves, at, torch.full_like(at, free.numel())),), torch.where(leaves, table, torch.zeros_like(table)))
    stack = stack[:-1]
    height = F + back_end[-1]
    takes = (col >= have[:, None]) & (col < want[:, None])
    i = (need_end - need)[:, None] + col - have[:, None]
    table = torch.where(takes, stack[(height - 1 - i).clamp(0, free.numel() - 1)], table)
    left = height - need_end[-1]
    place = torch.arange(free.numel(), device="cuda")
    free = torch.where((place >= F) & (place < left), stack, free)
    cu = torch.cat([old.new_zeros(1), (new - old).clamp(min=0).cumsum(0)])
    j = torch.arange(s["n_slots"], device="cuda")
    r = torch.searchsorted(cu[1:].contiguous(), j, right=True).clamp(max=old.numel() - 1)
    t = old[r] + j - cu[r]
    slots = torch.where(j < cu[-1], table[r, (t // page).clamp(0, width - 1)] * page + t % page, torch.full_like(j, -1))
    return table.int(), free.int(), left.int(), s["new"], slots, cu.int()


# ------------------------------------------------------------------------------ work and exact values
def _kept(c, T):
    if c["recent"] < 0:
        return T
    return T if T <= c["sink"] + c["recent"] else c["sink"] + c["recent"]


def work(case):
    c = case
    size = {"bf16": 2, "f16": 2, "e4m3": 1}
    if c["op"] == "attn":
        mean = 0.5 * (_kept(c, c["lo"]) + _kept(c, c["hi"]))
        if c["recent"] >= 0 and c["lo"] != c["hi"]:         # lengths are even between lo and hi; the kept part stops growing
            stop = c["sink"] + c["recent"]
            mean = sum(_kept(c, c["lo"] + (c["hi"] - c["lo"]) * (i + 0.5) / 1000) for i in range(1000)) / 1000 if stop else 0
        keys = c["requests"] * mean
        return {"bytes": keys * c["kv_heads"] * c["d"] * 2 * size[c["cache"]] + keys / c["page"] * 4 + c["requests"] * 4
                + 2 * c["requests"] * c["heads"] * c["d"] * size[c["type"]] + c["requests"] * c["heads"] * 4,
                "flops": 4 * keys * c["heads"] * c["d"]}
    if c["op"] == "append":
        n = c["tokens"] - (c["tokens"] // 8 if c["tokens"] > 8 else 0)
        values = 2 * n * c["kv_heads"] * c["d"]
        return {"bytes": values * (size[c["type"]] + size[c["cache"]]) + 8 * c["tokens"], "flops": values if c["cache"] == "e4m3" else 0}
    R, mean = c["requests"], 0.5 * (c["lo"] + c["hi"])
    begin, end = _begin_end(c)
    pages = (_new_tokens(c) + end * mean) / c["page"]
    return {"bytes": R * (8 + 4 + 4 + 4) + 8 * (_new_tokens(c) + c["pad"]) + 8 * pages, "flops": 0}


def exact(case, seed):
    c = case
    if c["op"] == "tables":
        return None                     # whole numbers
    s = prepare(case, seed)
    page, kv, d = c["page"], c["kv_heads"], c["d"]
    if c["op"] == "append":
        got = []
        slots = s["slots"].cpu()
        rows = (slots >= 0).nonzero()[:, 0]
        where = slots[rows]
        for pool, new, scale in ((s["K"], s["Kn"], s["ks"]), (s["V"], s["Vn"], s["vs"])):
            full = pool.double()
            x = new.double()[rows.cuda()]
            if scale is not None:
                x = torch.clamp(x / scale.double().reshape(1, kv, 1), -E4M3_MAX, E4M3_MAX)
            full[(where // page).cuda(), (where % page).cuda()] = x
            got.append(full)
        return tuple(got)
    R, N = c["requests"], c["heads"]
    O = torch.zeros((R, N, d), dtype=torch.float64, device="cuda")
    LSE = torch.full((N, R), -math.inf, dtype=torch.float64, device="cuda")
    for r, T in enumerate(s["lens"].tolist()):
        first = 0 if c["recent"] < 0 else max(0, T - c["recent"])
        kept = list(range(min(c["sink"], first))) + list(range(first, T))
        if not kept:
            continue
        t = torch.tensor(kept, device="cuda")
        own_pages = s["table"][r].long()[t // page]
        for h in range(kv):
            k = s["K"][own_pages, t % page, h].double() * (1.0 if s["ks"] is None else s["ks"][h].double())
            v = s["V"][own_pages, t % page, h].double() * (1.0 if s["vs"] is None else s["vs"][h].double())
            heads = slice(h * (N // kv), (h + 1) * (N // kv))
            z = s["Q"][r, heads].double() @ k.t() / d ** 0.5
            LSE[heads, r] = torch.logsumexp(z, -1)
            O[r, heads] = torch.softmax(z, -1) @ v
    return O, LSE
