"""Set-up and 64-bit references of the tests of the cache of 4 bits, and of rotation with storing.  Written from the definitions, for any
device; the library is not used here."""
from __future__ import annotations

import math

import torch

from serving_common import PAGE, Batch


def quantised(x):
    """fp32 [..., h] -> codes int64 [..., h], words int32 [..., h / 64], as the definition says it, each operation rounded to fp32."""
    x = x.float().unflatten(-1, (-1, 64))
    low, high = x.min(-1).values, x.max(-1).values
    most = torch.maximum(-low, high)
    scale = ((high - low) * (17 / 256) + most * (1 / 1024)).bfloat16()
    want = (low - most * (1 / 128)) - scale.float() * 16
    lower, bits = scale.view(torch.int16).int(), want.view(torch.int32)
    word = ((bits - lower + 0x8000) & -0x10000) | lower
    inverse = torch.where(scale > 0, 1 / scale.float(), 0.0)
    code = ((x - word.view(torch.float32)[..., None]) * inverse[..., None]).round() - 16
    return code.nan_to_num(0).clamp(0, 15).long().flatten(-2), word


def values(codes, words):
    """What codes [..., h] and words [..., h / 64] stand for, in 64 bits."""
    scale, offset = (words << 16).view(torch.float32).double(), words.view(torch.float32).double()
    return (scale[..., None] * (16 + codes.unflatten(-1, (-1, 64))) + offset[..., None]).flatten(-2)


def magnitudes(codes, words):
    """What the two terms of a value come to: roundings are relative to this."""
    scale, offset = (words << 16).view(torch.float32).double(), words.view(torch.float32).double()
    return (scale[..., None] * (16 + codes.unflatten(-1, (-1, 64))) + offset.abs()[..., None]).flatten(-2)


def k_nibbles(t, h):
    """Where, in nibbles, the codes of tokens t lie in a K page of one head: [tokens][h]."""
    c, t = torch.arange(h), t.view(-1, 1)
    return ((c // 8 % 4 * PAGE + t) * (h // 32) + c // 32) * 8 + c % 2 * 4 + c % 8 // 2


def v_nibbles(t, h):
    c, t = torch.arange(h), t.view(-1, 1)
    return ((((t // 4 * 16 + c % 16) * 2 + t // 2 % 2) * (h // 64) + c // 64) * 2 + t % 2) * 4 + c // 16 % 4


def put_codes(page, where, codes):
    """page: uint8 [9 h]; where, codes: [tokens][h]."""
    nibbles = torch.stack((page & 15, page >> 4), -1).flatten()
    nibbles[where.flatten()] = codes.flatten().to(torch.uint8)
    page[:] = nibbles[0::2] | nibbles[1::2] << 4


def put_tokens(pool, page, t, codes, words, nibbles):
    """pool: uint8 [pages][heads][9 h]; tokens t (places, [n]) of one page; codes [n][heads][h], words [n][heads][h / 64]."""
    heads, h = pool.shape[1], pool.shape[2] // 9
    for a in range(heads):
        put_codes(pool[page, a], nibbles(t, h), codes[:, a])
        w = pool[page, a].view(torch.int32)
        for g in range(h // 64):
            w[2 * h + g * PAGE + t] = words[:, a, g]


class Batch4(Batch):
    """A ragged batch on pools of 4 bits."""

    def __init__(self, heads, lens, dtype, fill=0xFF, **more):
        super().__init__(heads, [(0, n) for _, n in lens], dtype, **dict(more, spare=more.pop("spare", 2) + sum((c + n + 15) // 16 for c, n in lens)))
        g = torch.Generator().manual_seed(more.get("seed", 0) + 1000)
        self.lens = lens
        self.ctx = torch.tensor([c for c, _ in lens], dtype=torch.int32)
        need = [(c + n + PAGE - 1) // PAGE for c, n in lens]
        self.width = max(need + [1]) + more.get("slack", 0)
        perm = torch.randperm(self.n_pages, generator=g).tolist()
        self.tables = torch.full((len(lens), self.width), 2 ** 30, dtype=torch.int32)
        for s, n in enumerate(need):
            self.tables[s, :n] = torch.tensor([perm.pop() for _ in range(n)], dtype=torch.int32)
        layers = self.k_pool.shape[0]
        # 0xFF: words of NaN in all that nothing was stored to
        self.k_pool, self.v_pool = (torch.full((layers, self.n_pages, self.kv_heads, 9 * self.h), fill, dtype=torch.uint8) for _ in range(2))
        gain = torch.where(torch.rand(self.kv_heads, self.h, generator=g) < 0.03, 5.0, 1.0)
        self.keys = [quantised(torch.randn((c, self.kv_heads, self.h), generator=g) * gain) for c, _ in lens]
        self.values = [quantised(torch.randn((c, self.kv_heads, self.h), generator=g)) for c, _ in lens]
        for s, (c, _) in enumerate(lens):
            self.put4(self.k_pool, self.v_pool, s, 0, self.keys[s], self.values[s])

    def put4(self, k_pool, v_pool, s, first, k, v):
        """Tokens first .. of sequence s."""
        n = len(k[0])
        for p in range(first // PAGE, (first + n + PAGE - 1) // PAGE):
            at = torch.arange(max(first, p * PAGE), min(first + n, p * PAGE + PAGE))
            page = int(self.tables[s, p])
            put_tokens(k_pool[self.layer], page, at % PAGE, k[0][at - first], k[1][at - first], k_nibbles)
            put_tokens(v_pool[self.layer], page, at % PAGE, v[0][at - first], v[1][at - first], v_nibbles)

    def new_tokens(self, s, k=None, v=None):
        r0, r1 = int(self.starts[s]), int(self.starts[s + 1])
        return quantised((self.k if k is None else k)[r0:r1]), quantised((self.v if v is None else v)[r0:r1])

    def reference(self):
        out = torch.full((self.n_rows, self.q_heads, self.h), math.nan, dtype=torch.float64)
        tol = torch.zeros_like(out)
        k_pool, v_pool = self.k_pool.clone(), self.v_pool.clone()
        group, ulp = self.q_heads // self.kv_heads, 2.0 ** -24
        parts, weight_error, rounding = (3, 2.0 ** -24, ulp) if self.dtype == torch.float32 else (1, 2.0 ** -16, 2.0 ** -8)
        for s, (c, n) in enumerate(self.lens):
            if n == 0:
                continue
            r0 = int(self.starts[s])
            new = self.new_tokens(s)
            self.put4(k_pool, v_pool, s, c, *new)
            (kc, kw), (vc, vw) = ([torch.cat(x) for x in zip(old, fresh)] for old, fresh in zip((self.keys[s], self.values[s]), new))
            k, v, k_abs, v_abs = values(kc, kw), values(vc, vw), magnitudes(kc, kw), magnitudes(vc, vw)
            seen = self.seen(s)
            for head in range(self.q_heads):
                q = self.q[r0:r0 + n, head].double()
                a = head // group
                score = (q @ k[:, a].T / math.sqrt(self.h)).masked_fill(~seen, -math.inf)
                top = score.max(-1, keepdim=True).values
                weight = (score - torch.where(top == -math.inf, 0.0, top)).exp()
                total = weight.sum(-1, keepdim=True)
                p = torch.where(total > 0, weight / total, 0.0)
                out[r0:r0 + n, head] = p @ v[:, a]
                # Codes are exact.  A score is a sum of `parts` h products in fp32, of two terms a group, and twice rounded when it is scaled and the largest
                # is taken off: each rounding is relative to what the terms come to.  A weight follows its score's error, in the sum of weights and in
                # the output; exp2 is off by 2 ulp; weights enter the products, multiplied by a scale, with two parts or three; sums over n keys, of two
                # terms each, are off by 2 n + 32 roundings at most.
                score_abs = float((q.abs() @ k_abs[:, a].T / math.sqrt(self.h)).masked_fill(~seen, 0.0).max())
                mean_abs = p @ v_abs[:, a]
                tol[r0:r0 + n, head] = mean_abs * (2 * (parts * self.h + 8) * ulp * score_abs + 2 * (2 * (c + n) + 32) * ulp + 2 * weight_error) \
                    + out[r0:r0 + n, head].abs() * rounding * (1 + rounding)
        return out, tol, k_pool, v_pool

    def seen(self, s):
        c, n = self.lens[s]
        j, r0 = torch.arange(c + n), int(self.starts[s])
        if self.mask is None:
            return j[None, :] <= c + torch.arange(n)[:, None]
        bit, bits = j - int(self.mask_base[s]), self.bits[r0:r0 + n]
        return (bit < 0)[None, :] | (bits[:, bit.clamp(0, bits.shape[1] - 1)] & ((bit >= 0) & (bit < bits.shape[1]))[None, :])


def rotated(x, positions, freqs):
    """[rows][heads][h] at positions [rows], in 64 bits, and the sum of the magnitudes of both products."""
    h = x.shape[-1]
    angle = (positions.double()[:, None] * torch.tensor(freqs, dtype=torch.float64))[:, None, :]
    a, b = x.double()[..., :h // 2], x.double()[..., h // 2:]
    c, s = angle.cos(), angle.sin()
    return torch.cat((a * c - b * s, b * c + a * s), -1), torch.cat(((a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()), -1)


def model_freqs(theta, h):
    return [theta ** (-2 * j / h) for j in range(h // 2)]
