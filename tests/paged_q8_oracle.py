"""Plain 64-bit forms of the quantised paged cache and of shared prompts, on the CPU, and the inputs that their tests share."""
import math

import torch

import paged_oracle

E4M3 = torch.float8_e4m3fn


def e4m3_values():
    """What each of the 256 codes stands for."""
    out = []
    for code in range(256):
        exponent, mantissa = code >> 3 & 15, code & 7
        x = math.ldexp(8 + mantissa, exponent - 10) if exponent else math.ldexp(mantissa, -9)
        out.append(math.nan if code & 127 == 127 else -x if code >> 7 else x)
    return torch.tensor(out, dtype=torch.float64)


VALUES = e4m3_values()


def quantise(x):
    """(codes, exponents) of rows of bf16 values, each value to the nearest of the 127 magnitudes, of two as near to the one with an even code."""
    x = x.double()
    amax = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    e = torch.full(amax.shape, -126)
    for at in range(-126, 128):
        e = torch.where((amax > 448.0 * 2.0 ** at) & (e == at), at + 1, e)
    y = torch.ldexp(x, -e[..., None])
    size, grid = y.abs(), VALUES[:127]
    above = torch.searchsorted(grid, size.contiguous()).clamp(max=126)         # first not below
    below = (above - 1).clamp(min=0)
    up, down = grid[above] - size, size - grid[below]
    code = torch.where((up < down) | ((up == down) & (above % 2 == 0)), above, below)
    code = torch.where(torch.isfinite(x), code, 127) + torch.where(torch.signbit(y), 128, 0)
    return code.to(torch.uint8), (e + 127).to(torch.uint8)


def values_of(codes, exps):
    """What rows of codes with an exponent each stand for, in 64 bits."""
    return torch.ldexp(VALUES[codes.long()], exps.int()[..., None] - 127)


def append_q8(k, v, slots, k_codes, vt_codes, k_exp, v_exp):
    page = k_codes.shape[2]
    k_codes, vt_codes, k_exp, v_exp = (x.clone() for x in (k_codes, vt_codes, k_exp, v_exp))
    (kc, ke), (vc, ve) = quantise(k), quantise(v)
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < k_codes.shape[0] * page:
            b, o = s // page, s % page
            k_codes[b, :, o], k_exp[b, :, o] = kc[t], ke[t]
            vt_codes[b, :, :, o], v_exp[b, :, o] = vc[t], ve[t]
    return k_codes, vt_codes, k_exp, v_exp


def shares(table, starts, kv_lens, page, min_tokens):
    """The rules of sparse_prefill_paged_shares, one request after the other."""
    B = len(kv_lens)
    whole = [max(0, kv_lens[b] - (starts[b + 1] - starts[b])) // page for b in range(B)]
    common = [0] * (B + 1)
    for b in range(1, B):
        n = 0
        while n < min(whole[b], whole[b - 1]) and table[b, n] == table[b - 1, n]:
            n += 1
        common[b] = n * page
    groups = []
    for b in range(B):
        beside = max(common[b - 1], common[b + 1]) if b else 0
        if b and common[b] >= max(min_tokens, 1) and 2 * common[b] >= beside:
            groups[-1].append(b)
        else:
            groups.append([b])
    out = torch.zeros(3, B, dtype=torch.int32)
    for g in groups:
        for b in g:
            out[0, b], out[1, b], out[2, b] = g[0], len(g), min([common[x] for x in g[1:]], default=0)
    return out


class Step:
    """A serving step on the CPU: groups of requests (prefix, [(cached tokens of its own, new ones), ..]).  Whatever no query may see is NaN, with
    any exponent, table entries that no query needs are wild.  q8: quantised pages, whose values (exact in bf16) are the keys and values."""

    def __init__(self, seed, groups, page=64, q_heads=4, kv_heads=2, head_dim=128, q8=False, padding=0, peak=1.0, spare=3):
        g = torch.Generator().manual_seed(seed)
        randn = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16)  # noqa: E731
        self.page, self.q8, H, D = page, q8, kv_heads, head_dim
        own = [r for _, requests in groups for r in requests]
        self.new = [n for _, n in own]
        self.kv_lens = [p // page * page + c + n for p, requests in groups for c, n in requests]
        B = len(own)
        self.starts = [sum(self.new[:b]) for b in range(B + 1)]
        self.T = self.starts[-1] + padding
        self.q = (randn(max(self.T, 1), q_heads, D) * peak).to(torch.bfloat16)
        self.leaders = [0]
        for _, requests in groups:
            self.leaders.append(self.leaders[-1] + len(requests))
        common = [p // page for p, _ in groups for _ in range(len(_))]
        group = [x for x, (_, requests) in enumerate(groups) for _ in requests]
        pages = [-(-n // page) for n in self.kv_lens]
        n_pages = sum(p // page for p, _ in groups) + sum(n - c for n, c in zip(pages, common)) + spare
        ids = torch.randperm(n_pages, generator=g).tolist()
        C = max(pages + [1])
        self.table = torch.tensor([-1, 2 ** 31 - 1, -2 ** 31, n_pages] * (C * B), dtype=torch.int32)[:C * B].view(B, C).clone()
        code = torch.uint8 if q8 else torch.bfloat16
        self.k_pages = torch.full((n_pages, H, page, D), 127 if q8 else math.nan, dtype=code)
        self.vt_pages = torch.full((n_pages, H, D, page), 255 if q8 else math.nan, dtype=code)
        any_exp = lambda: torch.randint(0, 256, (n_pages, H, page), generator=g).to(torch.uint8)  # noqa: E731
        self.k_exp, self.v_exp = (any_exp(), any_exp()) if q8 else (None, None)

        def cached(n):
            """n tokens' values and what the pages hold of them"""
            x = randn(H, n, D) * torch.exp2(torch.randint(-2, 3, (H, n, 1), generator=g).float())
            if not q8:
                return x.to(torch.bfloat16), x.to(torch.bfloat16), None
            codes, e = quantise(x.to(torch.bfloat16))
            return values_of(codes, e).to(torch.bfloat16), codes, e

        def put(number, at, k, v, j0):
            n = min(page, k[1].shape[1] - j0)
            self.k_pages[number, :, :n], self.vt_pages[number, :, :, :n] = k[1][:, j0:j0 + n], v[1][:, j0:j0 + n].transpose(1, 2)
            if q8:
                self.k_exp[number, :, :n], self.v_exp[number, :, :n] = k[2][:, j0:j0 + n], v[2][:, j0:j0 + n]

        self.keys, self.values = [], []
        fronts = []
        for p, _ in groups:
            k, v, numbers = cached(p // page * page), cached(p // page * page), [ids.pop() for _ in range(p // page)]
            for j, number in enumerate(numbers):
                put(number, j, k, v, j * page)
            fronts.append((k, v, numbers))
        for b in range(B):
            front = fronts[group[b]]
            self.table[b, :common[b]] = torch.tensor(front[2], dtype=torch.int32)
            k, v = cached(self.kv_lens[b] - common[b] * page), cached(self.kv_lens[b] - common[b] * page)
            for j in range(common[b], pages[b]):
                self.table[b, j] = ids.pop()
                put(int(self.table[b, j]), j, k, v, (j - common[b]) * page)
            self.keys.append(torch.cat([front[0][0], k[0]], 1))
            self.values.append(torch.cat([front[1][0], v[0]], 1))
        self.shares = torch.tensor([[self.leaders[x] for x in group], [self.leaders[x + 1] - self.leaders[x] for x in group],
                                    [c * page if len(groups[x][1]) > 1 else 0 for x, c in zip(group, common)]], dtype=torch.int32)

    def hide(self, sink, window):
        """Pages whose keys no query of the step sees any more: NaN there, and forgotten in the tables."""
        needed = set()
        for b, n in enumerate(self.kv_lens):
            first = n - self.new[b] - window + 1
            for j in range(-(-n // self.page)):
                if j * self.page < sink or (j + 1) * self.page > first:
                    needed.add(int(self.table[b, j]))
        for b, n in enumerate(self.kv_lens):
            for j in range(-(-n // self.page)):
                number = int(self.table[b, j])
                if number >= 0 and number not in needed:
                    self.k_pages[number] = self.vt_pages[number] = 127 if self.q8 else math.nan
                    self.table[b, j] = -7

    def cache(self):
        """(k_pages, vt_pages, k_exp, v_exp) on the GPU"""
        if not self.q8:
            return self.k_pages.cuda(), self.vt_pages.cuda(), None, None
        return self.k_pages.cuda().view(E4M3), self.vt_pages.cuda().view(E4M3), self.k_exp.cuda(), self.v_exp.cuda()

    def want(self, **how):
        return paged_oracle.attn(self.q, self.keys, self.values, self.starts, self.kv_lens, **how)


def alone(ctx, new):
    """Requests that share nothing."""
    return [(0, [(c, n)]) for c, n in zip(ctx, new)]
