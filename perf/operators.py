"""Serving from a paged KV cache, as timed cases: what follows a sparse prefill in a program that answers requests.

A case is a dict of plain values.  `op` names the operator that a pass goes through:

  plan    block tables and slot maps of one step from the requests' lengths (paged_plan)
  append  keys and values of a step's new tokens into their pages (paged_append)
  attn    attention of the new tokens of every request over its paged keys and values (paged_attn)

`batch` requests hold between `ctx_lo` and `ctx_hi` cached tokens and bring between `new_lo` and `new_hi` new ones; `long` of them
bring `new_hi` (a step that mixes chunks of prompts with single tokens).  Pages hold `page` tokens and lie in a random order.
`sink` and `window` (tokens) are the A-shape of decoding: the first `sink` keys and the last `window` ones (0: every causal key);
`softcap` bounds the logits by a tanh, `slopes` adds a bias that falls with the distance.  32 query / 8 KV heads of 128 are the
8B-class GQA models that the sparse prefill serves, its pages the blocks of 64 and 128 tokens that it selects by.
"""
import math

import torch

own = False
DEVICE = "cuda" if torch.cuda.is_available() else "cpu"


def _case(name=None, *, op, batch, ctx_lo, ctx_hi, new_lo=1, new_hi=1, long=0, page=64, q_heads=32, kv_heads=8, head_dim=128, sink=0,
          window=0, softcap=0.0, slopes=False, lse=False):
    c = dict(op=op, batch=batch, ctx_lo=ctx_lo, ctx_hi=ctx_hi, new_lo=new_lo, new_hi=new_hi, long=long, page=page, q_heads=q_heads,
             kv_heads=kv_heads, head_dim=head_dim, sink=sink, window=window, softcap=softcap, slopes=slopes, lse=lse)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # the bookkeeping of a decode step: one token for each of 64 requests
        _case("plan_decode_64", op="plan", batch=64, ctx_lo=0, ctx_hi=8191),
        # the bookkeeping of a step that takes in many prompts at once
        _case("plan_prompts_512", op="plan", batch=512, ctx_lo=0, ctx_hi=2000, new_lo=1, new_hi=401, page=16),
        # single tokens of 256 requests go to their pages
        _case("append_decode_256", op="append", batch=256, ctx_lo=0, ctx_hi=500),
        # prompts of odd lengths, some behind a cached prefix that ends inside a page
        _case("append_prompts_16k", op="append", batch=8, ctx_lo=0, ctx_hi=300, new_lo=1500, new_hi=2600, page=128),
        # the smallest call: one request, a short context; launches and latency are all there is
        _case("decode_1", op="attn", batch=1, ctx_lo=500, ctx_hi=500),
        # ordinary decoding: 64 requests of different lengths
        _case("decode_64", op="attn", batch=64, ctx_lo=200, ctx_hi=8191),
        # few requests behind the long prompts that sparse prefill is made for; the log-sum-exp is kept to merge partial attention
        _case("decode_4_128k", op="attn", batch=4, ctx_lo=90000, ctx_hi=131071, page=128, lse=True),
        # A-shape decoding with capped logits, the smaller head size, small pages
        _case("decode_32_sink_window", op="attn", batch=32, ctx_lo=3000, ctx_hi=32767, page=16, q_heads=40, head_dim=64, sink=64, window=4096, softcap=30.0),
        # four drafted tokens of each of 32 requests are verified at once
        _case("verify_32", op="attn", batch=32, ctx_lo=100, ctx_hi=4000, new_lo=4, new_hi=4, page=32, lse=True),
        # a chunk of a long prompt over the cache that holds the rest
        _case("chunk_2k_at_96k", op="attn", batch=1, ctx_lo=98304, ctx_hi=98304, new_lo=2048, new_hi=2048),
        # fresh prompts of odd lengths, bias by distance, head_dim 64
        _case("prompts_4x4k_slopes", op="attn", batch=4, ctx_lo=0, ctx_hi=0, new_lo=2500, new_hi=4001, page=128, q_heads=16, kv_heads=16, head_dim=64, slopes=True),
        # a mixed step: three chunks among single tokens, capped logits
        _case("mixed_12", op="attn", batch=12, ctx_lo=0, ctx_hi=16000, new_lo=1, new_hi=515, long=3, page=16, softcap=50.0),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    op = rng.choice(("plan", "append", "attn", "attn", "attn", "attn"))
    q_heads, kv_heads = rng.choice(((32, 8), (32, 8), (40, 8), (16, 2), (16, 16), (8, 1)))
    c = dict(op=op, page=rng.choice((16, 32, 64, 64, 128)), q_heads=q_heads, kv_heads=kv_heads, head_dim=rng.choice((64, 128, 128)))
    if op == "plan":
        new = rng.choice((1, 1, _log_uniform(rng, 2, 700)))
        c.update(batch=_log_uniform(rng, 1, 512), ctx_lo=0, ctx_hi=_log_uniform(rng, 10, 20000), new_lo=1, new_hi=new)
    elif op == "append":
        new = rng.choice((1, _log_uniform(rng, 2, 3000)))
        c.update(batch=_log_uniform(rng, 1, 256 if new == 1 else 8), ctx_lo=0, ctx_hi=_log_uniform(rng, 10, 600), new_lo=(new + 1) // 2, new_hi=new)
    else:
        kind = rng.choice(("decode", "decode", "verify", "chunk", "mixed"))
        ctx = _log_uniform(rng, 30, 100000)
        if kind == "decode":
            c.update(batch=_log_uniform(rng, 1, 128), ctx_lo=ctx // 8, ctx_hi=ctx)
        elif kind == "verify":
            n = rng.randint(2, 9)
            c.update(batch=_log_uniform(rng, 1, 64), ctx_lo=ctx // 8, ctx_hi=ctx, new_lo=n, new_hi=n)
        elif kind == "chunk":
            n = _log_uniform(rng, 20, 4000)
            c.update(batch=rng.randint(1, 3), ctx_lo=ctx // 2, ctx_hi=ctx, new_lo=(n + 1) // 2, new_hi=n)
        else:
            c.update(batch=rng.randint(3, 16), ctx_lo=0, ctx_hi=ctx, new_lo=1, new_hi=_log_uniform(rng, 20, 700), long=rng.randint(1, 2))
        if rng.random() < 0.3:
            c.update(sink=rng.randint(0, 130), window=_log_uniform(rng, 1, 8000))
        c.update(softcap=rng.choice((0.0, 0.0, 20.0, 50.0)), slopes=rng.random() < 0.25, lse=rng.random() < 0.3)
    return _case(**c)


def _padded(c):
    """Keys and scores of the batch padded to its longest request: what the plain form holds."""
    keys = c["batch"] * (c["ctx_hi"] + c["new_hi"])
    return keys * c["kv_heads"] * c["head_dim"], keys * c["new_hi"] * c["q_heads"]


def draw(rng):
    chunk = next(c for c in listed() if c["name"] == "chunk_2k_at_96k")
    while True:
        c = _draw_once(rng)
        if c["op"] != "attn" or (_padded(c)[0] <= 2 ** 30 and _padded(c)[1] <= _padded(chunk)[1] and work(c)["flops"] <= work(chunk)["flops"]):
            return c


def _lengths(c):
    """Cached and new tokens of every request, the same for every seed: a case is of one size."""
    n = c["batch"]
    ctx = [c["ctx_lo"] + (c["ctx_hi"] - c["ctx_lo"]) * ((7919 * (b + 1)) % 1013) // 1012 for b in range(n)]
    new = [c["new_lo"] + (c["new_hi"] - c["new_lo"]) * ((4057 * (b + 1)) % 509) // 508 for b in range(n)]
    if c["long"]:
        new = [c["new_hi"] if b * c["long"] // n != (b + 1) * c["long"] // n else c["new_lo"] for b in range(n)]
    return ctx, new


def prepare(case, seed):
    """The requests' lengths, the cache with its tables and a step's inputs, from `seed` alone."""
    c = case
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    ctx, new = _lengths(c)
    page, Hq, Hkv, D, B, T = c["page"], c["q_heads"], c["kv_heads"], c["head_dim"], c["batch"], sum(new)
    columns = max(-(-(x + n) // page) for x, n in zip(ctx, new))
    have, want = [-(-x // page) for x in ctx], [-(-(x + n) // page) for x, n in zip(ctx, new)]
    n_pages = sum(want) + 7
    ids = torch.randperm(n_pages, generator=g, device=DEVICE).to(torch.int32)
    t = dict(dtype=torch.int32, device=DEVICE)
    s = dict(case=c, n_pages=n_pages, max_new=max(new), n_tokens=T, ctx_lens=torch.tensor(ctx, **t), new_lens=torch.tensor(new, **t))
    filled = have if c["op"] == "plan" else want
    at = torch.tensor([sum(filled[:b]) for b in range(B)], device=DEVICE)[:, None] + torch.arange(columns, device=DEVICE)
    there = torch.arange(columns, device=DEVICE) < torch.tensor(filled, device=DEVICE)[:, None]
    s["block_table"] = torch.where(there, ids[at.clamp(max=n_pages - 1)], -1).to(torch.int32)
    if c["op"] == "plan":
        s["free_pages"], s["free_range"] = ids[sum(have):].contiguous(), torch.tensor([0, n_pages - sum(have)], **t)
        return s

    def values(*shape):
        return torch.randn(shape, generator=g, device=DEVICE).to(torch.bfloat16)

    s["k_pages"], s["vt_pages"] = values(n_pages, Hkv, page, D), values(n_pages, Hkv, D, page)
    starts = torch.tensor([sum(new[:b]) for b in range(B + 1)], **t)
    if c["op"] == "append":
        of = torch.repeat_interleave(torch.arange(B, device=DEVICE), s["new_lens"].long())
        pos = s["ctx_lens"].long()[of] + torch.arange(T, device=DEVICE) - starts.long()[of]
        s["slots"] = (s["block_table"].long()[of, pos // page] * page + pos % page).to(torch.int32)
        s["k"], s["v"] = values(T, Hkv, D), values(T, Hkv, D)
        return s
    s["q"] = values(T, Hq, D) * 2
    s["q_starts"], s["kv_lens"] = starts, s["ctx_lens"] + s["new_lens"]
    s["slopes"] = torch.exp2(-8.0 * torch.arange(1, Hq + 1, device=DEVICE) / Hq) if c["slopes"] else None
    return s


def run(state):
    return _own(state) if own else {"plan": _plan, "append": _append, "attn": _attn}[state["case"]["op"]](state)


def _own(s):
    import paper_2602_21233_amd as spa
    c = s["case"]
    if c["op"] == "plan":
        starts, kv_lens, slots, positions, taken = spa.paged_plan(s["block_table"], s["ctx_lens"], s["new_lens"], s["free_pages"], s["free_range"],
                                                                  s["n_tokens"], c["page"], s["n_pages"])
        return dict(block_table=s["block_table"], q_starts=starts, kv_lens=kv_lens, slots=slots, positions=positions, taken=taken)
    if c["op"] == "append":
        spa.paged_append(s["k"], s["v"], s["slots"], s["k_pages"], s["vt_pages"])
        return dict(k_pages=s["k_pages"], vt_pages=s["vt_pages"])
    got = spa.paged_attn(s["q"], s["k_pages"], s["vt_pages"], s["block_table"], s["q_starts"], s["kv_lens"], max_new_tokens=s["max_new"],
                         n_sink_tokens=c["sink"], window_tokens=c["window"], softcap=c["softcap"], slopes=s["slopes"], return_lse=c["lse"])
    return dict(out=got[0], lse=got[1]) if c["lse"] else dict(out=got)


def _plan(s):
    """Requests in order take the pages that they need from the free list; one for which it has too few is left out."""
    page, table, n = s["case"]["page"], s["block_table"], s["n_tokens"]
    ctx, new, first = s["ctx_lens"].long(), s["new_lens"].long(), s["free_range"][0].long()
    room = s["free_range"][1] - first
    have = (ctx + page - 1) // page
    need = (ctx + new + page - 1) // page - have
    before = need.cumsum(0) - need
    goes = (need == 0) | (before + need <= room)
    taken = torch.where(goes, need, 0).sum()
    columns = torch.arange(table.shape[1], device=table.device)
    fresh = goes[:, None] & (columns >= have[:, None]) & (columns < (have + need)[:, None])
    last = s["free_pages"].numel() - 1
    table.copy_(torch.where(fresh, s["free_pages"][(first + before[:, None] + columns - have[:, None]).clamp(0, last)], table))
    starts = torch.cat([torch.zeros_like(new[:1]), new.cumsum(0)])
    token = torch.arange(n, device=table.device)
    of = torch.searchsorted(starts[1:], token, right=True).clamp(max=ctx.numel() - 1)
    there = token < starts[-1]
    pos = ctx[of] + token - starts[of]
    slots = table[of, (pos // page).clamp(max=table.shape[1] - 1)].long() * page + pos % page
    return dict(block_table=table, q_starts=starts.int(), kv_lens=torch.where(goes, ctx + new, 0).int(),
                slots=torch.where(there & goes[of], slots, -1).int(), positions=torch.where(there, pos, 0).int(),
                taken=torch.stack([taken, (~goes).sum()]).int())


def _append(s):
    page, slots = s["case"]["page"], s["slots"].long()
    s["k_pages"][slots // page, :, slots % page] = s["k"]
    s["vt_pages"][slots // page, :, :, slots % page] = s["v"]
    return dict(k_pages=s["k_pages"], vt_pages=s["vt_pages"])


def _attn(s):
    """The batch padded to its longest request, in 32 bits."""
    c, q, n = s["case"], s["q"], s["max_new"]
    B, Hq, Hkv, D, G = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["q_heads"] // c["kv_heads"]
    pages = s["block_table"].long().clamp(min=0)
    keys = pages.shape[1] * c["page"]
    k = s["k_pages"][pages].float().permute(0, 2, 4, 1, 3).reshape(B, Hkv, D, keys)
    v = s["vt_pages"][pages].float().permute(0, 2, 1, 4, 3).reshape(B, Hkv, keys, D)
    starts, kv = s["q_starts"].long(), s["kv_lens"].long()
    row = (starts[:-1, None] + torch.arange(n, device=q.device)).clamp(max=q.shape[0] - 1)
    x = q[row].float().view(B, n, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * n, D)
    x = torch.matmul(x, k).mul_(1.0 / math.sqrt(D)).view(B, Hkv, G, n, keys)
    if c["softcap"]:
        x = x.div_(c["softcap"]).tanh_().mul_(c["softcap"])
    at = (kv - (starts[1:] - starts[:-1]))[:, None] + torch.arange(n, device=q.device)
    back = at[:, :, None] - torch.arange(keys, device=q.device)
    if c["slopes"]:
        x -= s["slopes"].view(Hkv, G, 1, 1) * back[:, None, None].float()
    seen = back >= 0
    if c["window"]:
        seen &= (back < c["window"]) | (torch.arange(keys, device=q.device) < c["sink"])
    x.masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True).clamp(min=-1e30)
    x = x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x.view(B, Hkv, G * n, keys), v).view(B, Hkv, G, n, D) / total
    token = torch.arange(q.shape[0], device=q.device)
    of = torch.searchsorted(starts[1:], token, right=True)
    got = dict(out=out.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, D)[of, token - starts[of]].to(torch.bfloat16))
    if c["lse"]:
        got["lse"] = (m + total.log()).permute(0, 3, 1, 2, 4).reshape(B, n, Hq)[of, token - starts[of]]
    return got


def work(case):
    c = case
    ctx, new = _lengths(c)
    row = c["kv_heads"] * c["head_dim"] * 2
    if c["op"] == "plan":
        pages = sum(-(-(x + n) // c["page"]) - -(-x // c["page"]) for x, n in zip(ctx, new))
        return {"bytes": 4.0 * (2 * pages + 2 * sum(new) + 4 * c["batch"]), "flops": 0.0}
    if c["op"] == "append":
        return {"bytes": sum(new) * (4.0 * row + 4.0), "flops": 0.0}
    keys = pairs = 0
    for x, n in zip(ctx, new):
        w = c["window"] or x + n
        keys += min(x + n, min(n + w, x + n) + min(c["sink"], max(0, x - w)))
        pairs += sum(min(p + 1, w + min(c["sink"], max(0, p + 1 - w))) for p in range(x, x + n))
    return {"bytes": keys * 2.0 * row + sum(new) * c["q_heads"] * (4.0 * c["head_dim"] + 4.0 * c["lse"]), "flops": 4.0 * c["head_dim"] * c["q_heads"] * pairs}


def exact(case, seed):
    """Request by request and head by head, in 64 bits."""
    c = case
    if c["op"] == "plan":       # whole numbers
        return None
    s = prepare(case, seed)
    ctx, new = _lengths(c)
    page, Hkv, G, D = c["page"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["head_dim"]
    if c["op"] == "append":
        k, vt = s["k_pages"].double(), s["vt_pages"].double()
        order = s["slots"].long()
        rows = k.permute(0, 2, 1, 3).contiguous().view(-1, Hkv, D).index_copy_(0, order, s["k"].double())
        cols = vt.permute(0, 3, 1, 2).contiguous().view(-1, Hkv, D).index_copy_(0, order, s["v"].double())
        return dict(k_pages=rows.view(-1, page, Hkv, D).permute(0, 2, 1, 3), vt_pages=cols.view(-1, page, Hkv, D).permute(0, 2, 3, 1))
    out = torch.zeros(sum(new), c["q_heads"], D, dtype=torch.float64, device=DEVICE)
    lse = torch.zeros(sum(new), c["q_heads"], dtype=torch.float64, device=DEVICE)
    first = 0
    for b, (x, n) in enumerate(zip(ctx, new)):
        ids = s["block_table"][b, :-(-(x + n) // page)].long()
        i, j = torch.arange(x, x + n, device=DEVICE)[:, None], torch.arange(x + n, device=DEVICE)[None, :]
        hidden = j > i
        if c["window"]:
            hidden = hidden | ((i - j >= c["window"]) & (j >= c["sink"]))
        for h in range(Hkv):
            k = s["k_pages"][ids, h].double().reshape(-1, D)[:x + n]
            v = s["vt_pages"][ids, h].double().transpose(1, 2).reshape(-1, D)[:x + n]
            for e in range(h * G, h * G + G):
                z = s["q"][first:first + n, e].double() @ k.T / math.sqrt(D)
                if c["softcap"]:
                    z = c["softcap"] * torch.tanh(z / c["softcap"])
                if c["slopes"]:
                    z = z + s["slopes"][e].double() * (j - i)
                z[hidden] = -math.inf
                lse[first:first + n, e] = torch.logsumexp(z, 1)
                out[first:first + n, e] = torch.exp(z - lse[first:first + n, e, None]) @ v
        first += n
    return dict(out=out, lse=lse) if c["lse"] else dict(out=out)
