"""Set-up and 64-bit references of the tests of card_kv_attend, card_kv_copy_pages, card_kv_move_slots and card_logprobs.
Written from the definitions, for any device; the library is not used here."""
from __future__ import annotations

import math

import torch

PAGE = 16


def k_places(tokens, h):
    """Where the elements of these places of a page lie in a K page of one head, [tokens][h]."""
    j, t = torch.arange(h), tokens.view(-1, 1)
    return (j // 8 * PAGE + t) * 8 + j % 8


def v_places(tokens, h):
    j, t = torch.arange(h), tokens.view(-1, 1)
    return (j // 32 * 64 + t // 4 * 16 + j % 16) * 8 + j // 16 % 2 * 4 + t % 4


class Batch:
    """A ragged batch on pools of `layers` layers: lens = [(tokens in the cache, new tokens)].  fill: what pages
    hold where nothing was stored."""

    def __init__(self, heads, lens, dtype, layers=2, layer=1, seed=0, fill=math.nan, extra_rows=0, order="rows", spare=2, slack=0):
        self.q_heads, self.kv_heads, self.h = heads
        self.lens, self.layer, self.dtype = lens, layer, dtype
        g = torch.Generator().manual_seed(seed)
        need = [(c + n + PAGE - 1) // PAGE for c, n in lens]
        self.n_pages = sum(need) + spare
        perm = torch.randperm(self.n_pages, generator=g).tolist()
        self.width = max(need + [1]) + slack
        self.tables = torch.full((len(lens), self.width), 2 ** 30, dtype=torch.int32)
        for s, n in enumerate(need):
            self.tables[s, :n] = torch.tensor([perm.pop() for _ in range(n)], dtype=torch.int32)
        self.starts = torch.tensor([0] + [n for _, n in lens]).cumsum(0).to(torch.int32)
        self.ctx = torch.tensor([c for c, _ in lens], dtype=torch.int32)
        self.n_rows = int(self.starts[-1]) + extra_rows
        shape = (layers, self.n_pages, self.kv_heads, PAGE * self.h)
        self.k_pool = torch.full(shape, fill, dtype=torch.bfloat16)
        self.v_pool = torch.full(shape, fill, dtype=torch.bfloat16)
        # what the sequences hold, in plain order: [tokens][kv heads][h]
        self.keys = [torch.randn((c, self.kv_heads, self.h), generator=g).bfloat16() for c, _ in lens]
        self.values = [torch.randn((c, self.kv_heads, self.h), generator=g).bfloat16() for c, _ in lens]
        for s, (c, _) in enumerate(lens):
            if c:
                self.put(self.k_pool, self.v_pool, s, torch.arange(c), self.keys[s], self.values[s])

        def rows(heads_):
            if order == "heads":  # [heads][rows][h]
                return torch.randn((heads_, self.n_rows, self.h), generator=g).to(dtype).transpose(0, 1)
            return torch.randn((self.n_rows, heads_, self.h), generator=g).to(dtype)

        if order == "fused":  # side by side in a row
            x = torch.randn((self.n_rows, (self.q_heads + 2 * self.kv_heads) * self.h), generator=g).to(dtype)
            x = x.view(self.n_rows, -1, self.h)
            self.q, self.k, self.v = x.split([self.q_heads, self.kv_heads, self.kv_heads], 1)
        else:
            self.q, self.k, self.v = rows(self.q_heads), rows(self.kv_heads), rows(self.kv_heads)
        self.mask = self.mask_base = None

    def put(self, k_pool, v_pool, s, positions, k, v):
        page = self.tables[s, positions // PAGE].long()
        for head in range(self.kv_heads):
            k_pool[self.layer, page[:, None], head, k_places(positions % PAGE, self.h)] = k[:, head]
            v_pool[self.layer, page[:, None], head, v_places(positions % PAGE, self.h)] = v[:, head]

    def tree_mask(self, seed=1, density=0.4, words=None, bases=None, empty=False):
        """Random masks from a multiple of 16 on; every other row of an empty one sees nothing."""
        g = torch.Generator().manual_seed(seed)
        if bases is None:
            bases = [0 if empty else c // PAGE * PAGE for c, _ in self.lens]
        self.mask_base = torch.tensor(bases, dtype=torch.int32)
        most = max(c + n - b for (c, n), b in zip(self.lens, bases))
        words = words or max(1, (most + 31) // 32)
        bits = torch.rand((self.n_rows, words, 32), generator=g) < density
        if empty:
            bits[::2] = False
        value = (bits.long() << torch.arange(32)).sum(-1)
        self.bits = bits.view(self.n_rows, -1)
        self.mask = torch.where(value >= 1 << 31, value - (1 << 32), value).to(torch.int32)
        return self

    def reference(self):
        """(out in 64 bits, sum p |v| / sum p, largest error of a score per unit of rounding, pools); rows behind the last sequence are nan."""
        out = torch.full((self.n_rows, self.q_heads, self.h), math.nan, dtype=torch.float64)
        mean_abs, score_abs = torch.zeros_like(out), 0.0
        k_pool, v_pool = self.k_pool.clone(), self.v_pool.clone()
        group = self.q_heads // self.kv_heads
        for s, (c, n) in enumerate(self.lens):
            if n == 0:
                continue
            r0 = int(self.starts[s])
            k_new, v_new = self.k[r0:r0 + n].bfloat16(), self.v[r0:r0 + n].bfloat16()
            self.put(k_pool, v_pool, s, torch.arange(c, c + n), k_new, v_new)
            k = torch.cat([self.keys[s], k_new]).double()
            v = torch.cat([self.values[s], v_new]).double()
            j = torch.arange(c + n)
            if self.mask is None:
                seen = j[None, :] <= c + torch.arange(n)[:, None]
            else:
                bit = j - int(self.mask_base[s])
                bits = self.bits[r0:r0 + n]
                seen = (bit < 0)[None, :] | (bits[:, bit.clamp(0, bits.shape[1] - 1)] & ((bit >= 0) & (bit < bits.shape[1]))[None, :])
            for head in range(self.q_heads):
                q = self.q[r0:r0 + n, head].double()
                kk, vv = k[:, head // group], v[:, head // group]
                score = (q @ kk.T / math.sqrt(self.h)).masked_fill(~seen, -math.inf)
                score_abs = max(score_abs, float((q.abs() @ kk.abs().T / math.sqrt(self.h)).max()))
                top = score.max(-1, keepdim=True).values
                weight = (score - torch.where(top == -math.inf, 0.0, top)).exp()
                total = weight.sum(-1, keepdim=True)
                p = torch.where(total > 0, weight / total, 0.0)
                out[r0:r0 + n, head] = p @ vv
                mean_abs[r0:r0 + n, head] = p @ vv.abs()
        return out, mean_abs, score_abs, k_pool, v_pool

    def tolerance(self, out, mean_abs, score_abs):
        """Per element.  Keys and values are exact bf16 on both sides.  A score is a sum of 3 h products in fp32 (h for bf16 queries)
        and two roundings of the scale; the weight of a key follows its score's error, both in the sum of weights and in the output;
        exp2 is off by 2 ulp; sums over n keys are off by n + 32 roundings at most.  bf16: weights are
        rounded to it once, and so is the output."""
        ulp = 2.0 ** -24
        n = max(c + n for c, n in self.lens)
        tol = mean_abs * (2 * (3 * self.h + 4) * ulp * score_abs + 2 * (n + 32) * ulp)
        if self.dtype == torch.bfloat16:
            tol = tol + (mean_abs + out.abs()) * 2.0 ** -8 * (1 + 2.0 ** -8)
        else:
            tol = tol + out.abs() * 4 * ulp
        return tol


def logprob_reference(logits, tokens, temperature, top):
    """64 bits, row by row, with the rules for rows without a finite logit and for void ones."""
    rows, vocab = logits.shape
    logprob, entropy = torch.zeros(rows, dtype=torch.float64), torch.zeros(rows, dtype=torch.float64)
    top_tokens = torch.full((rows, top), -1, dtype=torch.int64)
    top_logprobs = torch.full((rows, top), -math.inf, dtype=torch.float64)
    for r in range(rows):
        x = logits[r].double()
        tok = -1 if tokens is None else int(tokens[r])
        if bool(torch.isnan(x).any()) or bool((x == math.inf).any()):
            p = torch.full_like(x, math.nan)
            entropy[r], top_logprobs[r] = math.nan, math.nan
        elif bool((x == -math.inf).all()):
            p = torch.full_like(x, -math.inf)
        else:
            d = (x - x.max()) / temperature
            p = d - d.exp().sum().log()
            entropy[r] = -torch.where(p == -math.inf, 0.0, p.exp() * p).sum()
            order = x.sort(descending=True, stable=True).indices[:top]
            order = order[x[order] > -math.inf]
            top_tokens[r, :len(order)] = order
            top_logprobs[r, :len(order)] = p[order]
        logprob[r] = 0.0 if tok < 0 else (math.nan if tok >= vocab else p[tok])
    return logprob, entropy, top_tokens, top_logprobs
