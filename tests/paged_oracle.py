"""Plain 64-bit forms of the paged-KV-cache calls, request by request on the CPU, and the inputs that their tests share."""
import math

import torch


def plan(block_table, ctx, new, free_pages, free_range, n_tokens, page, n_pages):
    """The rules of sparse_prefill_paged_plan, one token after the other.  Returns (table, starts, kv_lens, slots, positions, taken)."""
    table, B, C = block_table.clone(), len(ctx), block_table.shape[1]
    first = min(max(free_range[0], 0), len(free_pages))
    end = min(max(free_range[1], first), len(free_pages))
    starts, kv, slots, positions = [0], [], [-1] * n_tokens, [0] * n_tokens
    tokens = pages = taken = left_out = 0
    for b in range(B):
        more = max(new[b], 0)
        at = tokens
        tokens += more
        sound = ctx[b] >= 0 and new[b] >= 0 and ctx[b] + more <= C * page and tokens <= n_tokens
        have = -(-ctx[b] // page)
        need = -(-(ctx[b] + more) // page) - have if sound else 0
        goes = sound and (need == 0 or pages + need <= end - first)
        for j in range(need if goes else 0):
            table[b, have + j] = free_pages[first + pages + j]
        taken += need if goes else 0
        pages += need
        left_out += not goes
        kv.append(ctx[b] + more if goes else 0)
        starts.append(min(tokens, n_tokens))
        for t in range(at, min(tokens, n_tokens)):
            pos = ctx[b] + t - at
            positions[t] = (pos + 2 ** 31) % 2 ** 32 - 2 ** 31       # of an absurd length, as 32 bits hold it
            if goes:
                number = int(table[b, pos // page])
                slots[t] = number * page + pos % page if 0 <= number < n_pages else -1
    i32 = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    return table, i32(starts), i32(kv), i32(slots), i32(positions), i32([taken, left_out])


def append(k, v, slots, k_pages, vt_pages):
    page = k_pages.shape[2]
    k_pages, vt_pages = k_pages.clone(), vt_pages.clone()
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < k_pages.shape[0] * page:
            k_pages[s // page, :, s % page] = k[t]
            vt_pages[s // page, :, :, s % page] = v[t]
    return k_pages, vt_pages


def attn(q, keys, values, starts, kv_lens, scale=None, sink=0, window=0, softcap=0.0, slopes=None):
    """q [T, Hq, D]; keys[b], values[b] [Hkv, n, D] with n >= kv_lens[b].  Returns out, lse in 64 bits, and for both the most that a
    kernel may be off which works in fp32, rounds the weights to bf16 once and the output once: per output value
      2^-8 (sum_j p_j |v_j| + |out|)    half a step of bf16 for each weight, and for the result
      + 4 e sum_j p_j |v_j|             e: error of a logit, which scales its weight and the denominator
    with e = 2^-24 ((D + 8) scale sum_d |q_d k_d| + 8 |x|) for the sum of products and the steps to x (cap and bias: of the size of
    the cap and of the bias) + 2^-21 for the exponential, the largest among the keys that weigh anything (2^-30), and per log-sum-exp e + (n + 8) 2^-24 for the sum of n positive terms + 2^-22 (1 + |lse|)."""
    T, Hq, D = q.shape
    out = torch.zeros(T, Hq, D, dtype=torch.float64)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64)
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    for b, n_keys in enumerate(kv_lens):
        first, n = starts[b], starts[b + 1] - starts[b]
        if n_keys == 0 or n == 0:
            continue
        i = torch.arange(n_keys - n, n_keys)[:, None]
        j = torch.arange(n_keys)[None, :]
        seen = j <= i
        if window:
            seen &= (i - j < window) | (j < sink)
        for h in range(Hq):
            kv_head = h // (Hq // keys[b].shape[0])
            k, v = keys[b][kv_head, :n_keys].double(), values[b][kv_head, :n_keys].double()
            x = q[first:first + n, h].double()
            size = (D + 8) * scale * (x.abs() @ k.abs().T) * 2 ** -24
            z = x @ k.T * scale
            if softcap:
                z = softcap * torch.tanh(z / softcap)
                size = size + 8 * softcap * 2 ** -24
            if slopes is not None:
                z = z - float(slopes[h]) * (i - j)
                size = size + 8 * abs(float(slopes[h])) * (i - j).abs() * 2 ** -24
            size = torch.where(seen, size + 8 * z.abs() * 2 ** -24, 0.0)
            z = torch.where(seen, z, -math.inf)
            some = seen.any(1)
            total = torch.logsumexp(z, 1)
            p = torch.where(seen, torch.exp(z - total[:, None]), 0.0)
            p[~some] = 0.0
            o, mass = p @ v, p @ v.abs()
            e = torch.where(p > 2 ** -30, size, 0.0).amax(1) + 2 ** -21
            rows = slice(first, first + n)
            out[rows, h], lse[rows, h] = o, torch.where(some, total, -math.inf)
            out_tol[rows, h] = 1.01 * 2 ** -8 * (mass + o.abs()) + 4 * e[:, None] * mass + 1e-30
            lse_tol[rows, h] = torch.where(some, e + (n_keys + 8) * 2 ** -24 + 2 ** -22 * (1 + total.abs()), 0.0)
    return out, lse, out_tol, lse_tol


class Step:
    """A serving step on the CPU: `ctx` cached and `new` new tokens of every request, their keys and values, and the cache that
    holds them.  Whatever no query may see is NaN, table entries that no query needs are wild."""

    def __init__(self, seed, ctx, new, page=64, q_heads=4, kv_heads=2, head_dim=128, spare=3, padding=0, peak=1.0):
        g = torch.Generator().manual_seed(seed)
        randn = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16)  # noqa: E731
        self.page, B = page, len(ctx)
        self.kv_lens = [c + n for c, n in zip(ctx, new)]
        self.starts = [sum(new[:b]) for b in range(B + 1)]
        self.T = self.starts[-1] + padding
        self.q = (randn(max(self.T, 1), q_heads, head_dim) * peak).to(torch.bfloat16)
        self.keys = [randn(kv_heads, n, head_dim) for n in self.kv_lens]
        self.values = [randn(kv_heads, n, head_dim) for n in self.kv_lens]
        pages = [-(-n // page) for n in self.kv_lens]
        n_pages = sum(pages) + spare
        ids = torch.randperm(n_pages, generator=g).tolist()
        self.table = torch.tensor([-1, 2 ** 31 - 1, -2 ** 31, n_pages] * (max(pages + [1]) * B), dtype=torch.int32)[:max(pages + [1]) * B].view(B, -1).clone()
        self.k_pages = torch.full((n_pages, kv_heads, page, head_dim), math.nan, dtype=torch.bfloat16)
        self.vt_pages = torch.full((n_pages, kv_heads, head_dim, page), math.nan, dtype=torch.bfloat16)
        for b in range(B):
            for j in range(pages[b]):
                number = ids.pop()
                self.table[b, j] = number
                at = slice(j * page, min((j + 1) * page, self.kv_lens[b]))
                self.k_pages[number, :, :at.stop - at.start] = self.keys[b][:, at]
                self.vt_pages[number, :, :, :at.stop - at.start] = self.values[b][:, at].transpose(1, 2)

    def hide(self, sink, window, new):
        """Pages whose keys no query of the step sees any more: forgotten in the table, NaN in the lists' places."""
        for b, n in enumerate(self.kv_lens):
            first = n - new[b] - window + 1
            for j in range(-(-n // self.page)):
                if j * self.page >= sink and (j + 1) * self.page <= first:
                    number = int(self.table[b, j])
                    self.k_pages[number] = self.vt_pages[number] = math.nan
                    self.table[b, j] = -7

    def want(self, **how):
        return attn(self.q, self.keys, self.values, self.starts, self.kv_lens, **how)
