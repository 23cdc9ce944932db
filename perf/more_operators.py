"""The operators of a program with its own layers that serves texts, or searches with beams, on a paged cache: rotation of queries and
keys with the storing of keys and values, attention over a cache of 4 bits a value, and the selection of beams.

Pages, layers and head layouts are those of the library's caches.  Their plain forms below are elementary torch operations in 32 bits, angles and the
scores of beams in 64.
"""
import math

import torch

own = False

# query heads, key/value heads, head size and vocabulary of the shapes in card_inputs/configs.py, and one of odd sizes
HEADS = {
    "tiny": (4, 2, 64, 1024),
    "odd": (10, 2, 128, 3001),
    "llama1b": (32, 8, 64, 128256),
    "llama8b": (32, 8, 128, 128256),
    "llama70b": (64, 8, 128, 128256),
    "qwen7b": (28, 4, 128, 152064),
}
PAGE = 16
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
THETA = 1e4


def _append(model, bits, seqs, new, ctx, type="bf16", tree=False, scaled=False):
    """seqs sequences of up to `ctx` tokens in a cache of `bits` bits and up to `new` new ones each (one of them has as many); tree: positions of their
    own; scaled: frequencies of the caller's."""
    return {"op": "append", "model": model, "bits": bits, "seqs": seqs, "new": new, "ctx": ctx, "type": type, "tree": tree, "scaled": scaled}


def _attend(model, seqs, new, ctx, mask="causal", type="bf16"):
    return {"op": "attend", "model": model, "bits": 4, "seqs": seqs, "new": new, "ctx": ctx, "mask": mask, "type": type}


def _beam(model, groups, beams, out_beams, length, type="f32", temperature=1.0):
    """groups searches of `beams` beams that go on with out_beams; texts of `length` tokens so far; some beams have ended."""
    return {"op": "beam", "model": model, "groups": groups, "beams": beams, "out_beams": out_beams, "length": length, "type": type,
            "temperature": temperature}


def listed():
    cases = {
        # a token each of a batch of texts of different lengths
        "append decode": _append("llama8b", 16, 48, 1, 4000),
        # a level of the draft's tree, activations in 32 bits as the library keeps them
        "append tree f32": _append("llama1b", 16, 1, 100, 1024, "f32", tree=True),
        # the last chunk of a long prompt
        "append prompt": _append("llama70b", 16, 1, 2000, 14000),
        # chunks of three prompts of a model with stretched frequencies, to a cache of 4 bits, and what that then holds
        "append chunks 4 bits": _append("qwen7b", 4, 3, 1000, 3500, scaled=True),
        # one token each for three short texts of the smallest shape: latency
        "attend tiny": _attend("tiny", 3, 1, 100),
        # plain decoding of a batch of texts of different lengths
        "attend decode": _attend("llama8b", 64, 1, 8000),
        # a chain of five candidates of one very long text
        "attend long": _attend("llama70b", 1, 5, 120000),
        # the last chunk of a long prompt
        "attend prompt": _attend("llama8b", 1, 2000, 14000),
        # a level of the draft's tree
        "attend tree f32": _attend("llama1b", 1, 100, 1024, "tree", "f32"),
        # three searches of a small vocabulary: latency
        "beam tiny": _beam("tiny", 3, 3, 3, 20),
        # one search
        "beam step": _beam("llama8b", 1, 4, 4, 300),
        # a batch of searches
        "beam batch": _beam("qwen7b", 40, 6, 6, 900, "bf16", 0.8),
    }
    return [dict(case, name=name) for name, case in cases.items()]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    model = rng.choice(list(HEADS))
    q_heads, kv_heads, h, _ = HEADS[model]
    op = rng.choice(["append", "append", "attend", "attend", "attend", "beam"])
    type = rng.choice(["bf16", "bf16", "f32"])
    if op == "append":
        bits, tree, scaled = rng.choice([4, 16]), rng.random() < 0.3, rng.random() < 0.3
        if rng.random() < 0.5:
            return _append(model, bits, _log_uniform(rng, 1, 64), rng.choice([1, rng.randint(2, 8)]), _log_uniform(rng, 1, 4000), type, tree, scaled)
        return _append(model, bits, rng.randint(1, 4), _log_uniform(rng, 9, 500), _log_uniform(rng, 1, 3500), type, tree, scaled)
    if op == "attend":
        if rng.random() < 0.25:
            return _attend(model, rng.randint(1, 4), rng.randint(2, 128), _log_uniform(rng, 1, 2000), "tree", type)
        if rng.random() < 0.5:
            seqs = _log_uniform(rng, 1, 64)
            return _attend(model, seqs, rng.choice([1, 1, rng.randint(2, 8)]), _log_uniform(rng, 1, min(60000, 200000 // seqs)), "causal", type)
        # (the plain form holds all scores: sequences x new x query heads x length in 32 bits)
        seqs, new = rng.randint(1, 4), _log_uniform(rng, 9, 2000)
        most = 2000 * 16000 * 32 // (seqs * new * q_heads) - new
        return _attend(model, seqs, new, _log_uniform(rng, 1, max(2, min(14000, most))), "causal", type)
    beams = rng.randint(1, 12)
    out_beams = beams if rng.random() < 0.6 else rng.randint(1, 20)
    return _beam(model, _log_uniform(rng, 1, max(1, 100 // beams)), beams, out_beams, _log_uniform(rng, 1, 1000), type, rng.choice([1.0, 0.8, 1.3]))


# ---- inputs ---------------------------------------------------------------------------------------


def _generator(seed, stream, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed((seed * 1000003 + stream * 7919 + 17) & 0x7FFFFFFFFFFFFFFF)
    return g


class _State:
    pass


def _lengths(case):
    """Tokens in the cache and new tokens of each sequence, the same for every seed: the first has the most of both."""
    n, g = case["seqs"], _generator(0, 3, "cpu")
    ctx = (torch.rand(n, generator=g) * 0.9 + 0.1).mul(case["ctx"]).long()
    new = (torch.rand(n, generator=g) * case["new"]).long().add(1).clamp(max=case["new"])
    ctx[0], new[0] = case["ctx"], case["new"]
    return ctx, new


def _normal(shape, seed, stream):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=_generator(seed, stream))


def _pools(s, case, pages, seed):
    _, kv_heads, h, _ = HEADS[case["model"]]
    s.layers, s.pages = 2, pages
    if case["bits"] == 16:
        shape = (s.layers, pages, kv_heads, PAGE * h)
        s.k_pool, s.v_pool = (_normal(shape, seed, i).to(torch.bfloat16) for i in (1, 2))
        return
    s.k_pool, s.v_pool = (torch.zeros((s.layers, pages, kv_heads, 9 * h), dtype=torch.uint8, device="cuda") for _ in range(2))
    # some channels of keys are far larger than the others
    gain = torch.where(torch.rand(kv_heads, 1, h, generator=_generator(seed, 20), device="cuda") < 0.03, 6.0, 1.0)
    _k4_codes(s.k_pool[1], h)[:], _words(s.k_pool[1], h)[:] = _k4_page(*_quantised(_normal((pages, kv_heads, PAGE, h), seed, 1) * gain))
    _v4_codes(s.v_pool[1], h)[:], _words(s.v_pool[1], h)[:] = _v4_page(*_quantised(_normal((pages, kv_heads, PAGE, h), seed, 2)))


def _prepare_batch(s, case, seed):
    q_heads, kv_heads, h, _ = HEADS[case["model"]]
    ctx, new = _lengths(case)
    need = (ctx + new + PAGE - 1) // PAGE
    total, most = int(need.sum()), int(need.max())
    _pools(s, case, total + 3, seed)
    order = torch.randperm(total + 3, generator=_generator(seed, 4, "cpu"))[:total]
    tables = torch.zeros((case["seqs"], most), dtype=torch.int32)
    tables[torch.arange(most)[None, :] < need[:, None]] = order.to(torch.int32)
    starts = torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)])
    s.n_rows, s.max_new, s.max_len = int(starts[-1]), int(new.max()), int((ctx + new).max())
    s.tables, s.ctx, s.starts = tables.cuda(), ctx.to(torch.int32).cuda(), starts.to(torch.int32).cuda()
    # queries, keys and values as a fused projection leaves them: side by side in a row
    qkv = _normal((s.n_rows, (q_heads + 2 * kv_heads) * h), seed, 5).to(TYPES[case["type"]])
    s.q = qkv[:, : q_heads * h].view(s.n_rows, q_heads, h)
    s.k = qkv[:, q_heads * h: (q_heads + kv_heads) * h].view(s.n_rows, kv_heads, h)
    s.v = qkv[:, (q_heads + kv_heads) * h:].view(s.n_rows, kv_heads, h)
    s.out = torch.zeros((s.n_rows, q_heads, h), dtype=qkv.dtype, device="cuda")
    s.k_out, s.v_out = (torch.zeros((s.n_rows, kv_heads, h), dtype=qkv.dtype, device="cuda") for _ in range(2))
    row_of = torch.arange(s.n_rows) - torch.repeat_interleave(starts[:-1], new)
    s.positions = s.freqs = s.mask = s.mask_base = None
    if case.get("tree"):
        depth = torch.randint(0, 12, (s.n_rows,), generator=_generator(seed, 21, "cpu"))
        s.positions = (torch.repeat_interleave(ctx, new) + depth).to(torch.int32).cuda()
    if case.get("scaled"):  # the low frequencies four times lower
        s.freqs = [THETA ** (-2 * j / h) / (1.0 if j < h // 4 else 4.0) for j in range(h // 2)]
    if case.get("mask") == "tree":
        # every node sees the context and itself, and a third of the other nodes' slots (ancestors)
        words = (s.max_new + PAGE + 31) // 32
        base = ctx // PAGE * PAGE
        past = torch.repeat_interleave(ctx - base, new)  # context slots behind the mask's begin
        bit = torch.arange(32 * words)[None, :]
        seen = torch.rand((s.n_rows, 32 * words), generator=_generator(seed, 6, "cpu")) < 0.33
        seen = (seen & (bit < (past + row_of)[:, None])) | (bit < past[:, None]) | (bit == (past + row_of)[:, None])
        value = (seen.view(s.n_rows, words, 32).long() << torch.arange(32)).sum(-1)
        s.mask = torch.where(value >= 1 << 31, value - (1 << 32), value).to(torch.int32).cuda()
        s.mask_base = base.to(torch.int32).cuda()
    if own:
        s.plan = _batch_plan(s, case)


def _prepare_beams(s, case, seed):
    _, _, _, vocab = HEADS[case["model"]]
    n, b, k = case["groups"], case["beams"], case["out_beams"]
    # logits as a vocabulary head gives them: a bell with a few tokens that stand out
    x = torch.empty((n * b, vocab), dtype=torch.float32, device="cuda").normal_(0.0, 2.0, generator=_generator(seed, 8))
    likely = torch.randint(0, vocab, (n * b, 6), device="cuda", generator=_generator(seed, 9))
    x.scatter_add_(1, likely, torch.rand((n * b, 6), device="cuda", generator=_generator(seed, 10)) * 14.0)
    s.logits = x.to(TYPES[case["type"]])
    s.scores = torch.rand((n, b), device="cuda", generator=_generator(seed, 11)) * -3.0 - 0.9 * case["length"]
    s.done = (torch.rand((n, b), device="cuda", generator=_generator(seed, 12)) < 0.15).to(torch.int32)
    s.done[:, 0] = 0
    s.eos = 7
    s.history = torch.randint(0, vocab, (n, b, case["length"] + 16), device="cuda", generator=_generator(seed, 13)).to(torch.int32)
    s.lengths = torch.full((n,), case["length"], dtype=torch.int32, device="cuda")
    s.lengths[1::2] -= 1  # some are a token behind
    i32 = dict(dtype=torch.int32, device="cuda")
    s.out = {"scores": torch.empty((n, k), dtype=torch.float32, device="cuda"), "tokens": torch.empty((n, k), **i32), "parents": torch.empty((n, k), **i32),
             "done": torch.empty((n, k), **i32), "history": torch.zeros((n, k, s.history.shape[2]), **i32)}
    if own:
        s.plan = _beam_plan(s, case)


def prepare(case, seed):
    s = _State()
    s.case = case
    if case["op"] == "beam":
        _prepare_beams(s, case, seed)
    else:
        _prepare_batch(s, case, seed)
    return s


# ---- the framework's calls ------------------------------------------------------------------------


def _batch_plan(s, case):
    import paper_2508_04462_amd as card

    q_heads, kv_heads, h, vocab = HEADS[case["model"]]
    # (of a model, these operators take the layers, heads, head size and the base of the frequencies)
    s.cfg = card.CardModelCfg(s.layers, 512, q_heads, kv_heads, h, 512, vocab, THETA, 1e-5, PAGE, 1 << 20, 32, 0)
    s.batch = card.CardKVBatch(s.k_pool.data_ptr(), s.v_pool.data_ptr(), s.pages, case["seqs"], s.tables.data_ptr(), s.tables.shape[1],
                               s.n_rows, s.ctx.data_ptr(), s.starts.data_ptr(), s.max_new, s.max_len)
    if case["op"] == "append":
        return card.card_rotation(s.freqs, s.positions)
    mask = None
    if s.mask is not None:
        mask = card.CardRowMask(s.mask.data_ptr(), s.mask_base.data_ptr(), s.mask.shape[1])
    return mask, torch.empty(card.card_kv4_attend_workspace_bytes(s.cfg, s.batch), dtype=torch.uint8, device="cuda")


def _beam_plan(s, case):
    import paper_2508_04462_amd as card

    n, b, k = case["groups"], case["beams"], case["out_beams"]
    o = s.out
    beams = card.CardBeams(n, b, k, s.eos, s.scores.data_ptr(), s.done.data_ptr(), s.history.data_ptr(), s.lengths.data_ptr(), s.history.shape[2],
                           o["scores"].data_ptr(), o["tokens"].data_ptr(), o["parents"].data_ptr(), o["done"].data_ptr(), o["history"].data_ptr())
    return beams, torch.empty(card.card_beam_select_workspace_bytes(n, b, k, s.logits.shape[1]), dtype=torch.uint8, device="cuda")


def _run_own(s):
    import paper_2508_04462_amd as card

    case, stream = s.case, torch.cuda.current_stream().cuda_stream
    if case["op"] == "beam":
        status, got = card.card_beam_select(s.logits, s.plan[0], case["temperature"], s.plan[1], stream), s.out
    elif case["op"] == "attend":
        mask, workspace = s.plan
        status = card.card_kv4_attend(s.cfg, s.batch, 1, card.card_rows(s.q), None, None, card.card_rows(s.out), mask, workspace, stream)
        got = {"out": s.out}
    else:
        call = card.card_kv_append if case["bits"] == 16 else card.card_kv4_append
        status = call(s.cfg, s.batch, 1, s.plan, card.card_rows(s.q), card.card_rows(s.out), card.card_rows(s.k), card.card_rows(s.v), stream)
        got = {"q": s.out, "k_cache": s.k_pool[1], "v_cache": s.v_pool[1]}
        if case["bits"] == 4 and status == card.CARD_OK:
            status = card.card_kv4_read(s.cfg, s.batch, 1, card.card_rows(s.k_out), card.card_rows(s.v_out), stream)
            got = {"q": s.out, "k": s.k_out, "v": s.v_out}
    if status != card.CARD_OK:
        raise card.CardError(status, case["op"])
    return got


# ---- caches ---------------------------------------------------------------------------------------
# Order of the elements of a page of one head in 16 bits: K [h / 8][16 tokens][8]; V [h / 32][4][16][2][4], which are
# channel / 32, token / 4, channel % 16, channel / 16 % 2, token % 4.


def _k_view(pool, h):
    return pool.unflatten(-1, (h // 8, PAGE, 8))


def _v_view(pool, h):
    return pool.unflatten(-1, (h // 32, 4, 16, 2, 4))


# In 4 bits: 8 h bytes of codes, then a word for every 64 channels of a token, [h / 64][16 tokens]: its lower half is a scale in bf16, the whole of it
# in fp32 an offset; code c stands for scale * (16 + c) + offset.  Codes, a nibble each, from the lowest bits on: K [4][16 tokens][h / 32][2][4], which are channel / 8 % 4,
# token, channel / 32, channel % 2, channel % 8 / 2; V [4][16][2][h / 64][2][4], which are token / 4, channel % 16, token / 2 % 2, channel / 64,
# token % 2, channel / 16 % 4.


def _k4_codes(pool, h):
    return pool[..., : 8 * h].unflatten(-1, (4, PAGE, h // 32, 4))


def _v4_codes(pool, h):
    return pool[..., : 8 * h].unflatten(-1, (4, 16, 2, h // 64, 2, 2))


def _words(pool, h):
    return pool.view(torch.int32)[..., 2 * h:].unflatten(-1, (h // 64, PAGE))


def _quantised(x):
    """[..., h] in 32 bits -> codes [..., h] and words [..., h / 64]."""
    x = x.unflatten(-1, (-1, 64))
    low, high = x.amin(-1), x.amax(-1)
    most = torch.maximum(-low, high)
    scale = (high - low) * (17 / 256) + most * (1 / 1024)
    scale = scale.to(torch.bfloat16).float()
    bits = scale.view(torch.int32) >> 16
    offset = (low - most * (1 / 128)) - scale * 16
    word = ((offset.view(torch.int32) - bits + 0x8000) & -0x10000) | bits
    code = ((x - word.view(torch.float32)[..., None]) * (1 / scale)[..., None]).round() - 16
    code = torch.where(scale[..., None] > 0, code, 0).clamp(0, 15)
    return code.flatten(-2).to(torch.uint8), word


def _bytes(nibbles):
    return nibbles[..., 0::2] | nibbles[..., 1::2] << 4


def _k4_tokens(codes):
    """Codes [..., h] of tokens -> bytes [..., 4, h / 32, 4]."""
    x = codes.unflatten(-1, (-1, 4, 4, 2))  # channel / 32, / 8 % 4, % 8 / 2, % 2
    return _bytes(x.movedim(-4, -3).transpose(-1, -2).flatten(-2))


def _v4_tokens(codes):
    """-> bytes [..., 16, h / 64, 2]."""
    x = codes.unflatten(-1, (-1, 4, 16))  # channel / 64, / 16 % 4, % 16
    return _bytes(x.movedim(-1, -3))


def _k4_page(codes, words):
    """Codes [..., 16 tokens, h] and words [..., 16, h / 64] in the order of a page."""
    return _k4_tokens(codes).movedim(-4, -3), words.transpose(-1, -2)


def _v4_page(codes, words):
    x = _v4_tokens(codes).unflatten(-4, (4, 2, 2))  # token / 4, / 2 % 2, % 2; channel % 16, / 64, byte
    return x.movedim((-6, -3, -5, -2, -4, -1), (-6, -5, -4, -3, -2, -1)), words.transpose(-1, -2)


def _nibbles(b):
    return torch.stack((b & 15, b >> 4), -1).flatten(-2)


def _values(codes, words, dtype=torch.float32):
    """Codes [..., h] and words [..., h / 64] -> the values that they stand for."""
    scale, offset = (words << 16).view(torch.float32).to(dtype), words.view(torch.float32).to(dtype)
    return (scale[..., None] * (codes.unflatten(-1, (-1, 64)).to(dtype) + 16) + offset[..., None]).flatten(-2)


def _k4_rows(pages, h):
    """[..., pages, heads, 9 h] -> [..., heads, pages * 16, h] in 32 bits."""
    x = _nibbles(_k4_codes(pages, h)).unflatten(-1, (2, 4)).transpose(-1, -2).flatten(-2)  # [4][16][h / 32][8]
    x = x.movedim(-4, -2).flatten(-3)
    return _values(x, _words(pages, h).transpose(-1, -2)).movedim(-4, -3).flatten(-3, -2)


def _v4_rows(pages, h):
    x = _nibbles(_v4_codes(pages, h))  # [4][16][2][h / 64][2][4]: token / 4, channel % 16, token / 2 % 2, channel / 64, token % 2, channel / 16 % 4
    x = x.movedim((-6, -5, -4, -3, -2, -1), (-6, -1, -5, -3, -4, -2)).flatten(-3).flatten(-4, -2)
    return _values(x, _words(pages, h).transpose(-1, -2)).movedim(-4, -3).flatten(-3, -2)


# ---- the plain forms ------------------------------------------------------------------------------


def _places(s):
    """Sequence, slot, page and place of each row."""
    ctx, starts = s.ctx.long(), s.starts.long()
    row = torch.arange(s.n_rows, device="cuda")
    seq = torch.searchsorted(starts[1:], row, right=True)
    slot = ctx[seq] + row - starts[seq]
    return seq, slot, s.tables[seq, slot // PAGE].long(), slot % PAGE


def _plain_append(s):
    _, _, h, _ = HEADS[s.case["model"]]
    _, slot, page, place = _places(s)
    position = slot if s.positions is None else s.positions
    if s.freqs is None:
        freqs = THETA ** (torch.arange(h // 2, dtype=torch.float64, device="cuda") * (-2 / h))
    else:
        freqs = torch.tensor(s.freqs, dtype=torch.float64, device="cuda")
    angle = (position.double()[:, None] * freqs)[:, None, :]
    cos, sin = angle.cos().float().double(), angle.sin().float().double()

    def rotated(x):
        a, b = x.double().split(h // 2, -1)
        return torch.cat((a * cos - b * sin, b * cos + a * sin), -1).float()

    kp, vp = s.k_pool[1], s.v_pool[1]
    k, v = rotated(s.k), s.v.float()
    s.out.copy_(rotated(s.q))
    if s.case["bits"] == 16:
        _k_view(kp, h)[page, :, :, place] = k.to(kp.dtype).unflatten(-1, (h // 8, 8))
        _v_view(vp, h)[page, :, :, place // 4, :, :, place % 4] = v.to(vp.dtype).unflatten(-1, (h // 32, 2, 16)).transpose(-1, -2)
        return {"q": s.out, "k_cache": kp, "v_cache": vp}
    codes, words = _quantised(k)
    _k4_codes(kp, h)[page, :, :, place], _words(kp, h)[page, :, :, place] = _k4_tokens(codes), words
    s.k_out.copy_(_values(codes, words))
    codes, words = _quantised(v)
    _v4_codes(vp, h)[page, :, place // 4, :, place // 2 % 2, :, place % 2], _words(vp, h)[page, :, :, place] = _v4_tokens(codes), words
    s.v_out.copy_(_values(codes, words))
    return {"q": s.out, "k": s.k_out, "v": s.v_out}


def _plain_attend(s):
    q_heads, kv_heads, h, _ = HEADS[s.case["model"]]
    group, seqs = q_heads // kv_heads, s.case["seqs"]
    ctx, starts = s.ctx.long(), s.starts.long()
    used = (s.max_len + PAGE - 1) // PAGE
    tables = s.tables[:, :used].long()
    k, v = _k4_rows(s.k_pool[1][tables], h), _v4_rows(s.v_pool[1][tables], h)  # [seqs, kv heads, keys, h]
    # the rows of each sequence, filled up to the longest chunk
    i = torch.arange(s.max_new, device="cuda")
    at = (starts[:-1, None] + i).clamp(max=s.n_rows - 1)
    there = i < (starts[1:] - starts[:-1])[:, None]
    q = s.q[at].float().view(seqs, s.max_new, kv_heads, group, h).permute(0, 2, 1, 3, 4).flatten(2, 3)
    score = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(1.0 / math.sqrt(h)).view(seqs, kv_heads, s.max_new, group, -1)
    key = torch.arange(used * PAGE, device="cuda")
    if s.mask is None:
        seen = key <= (ctx[:, None] + i)[:, :, None]
    else:
        base = s.mask_base.long()
        bit = key - base[:, None]
        word = s.mask[at].long().gather(2, (bit.clamp(0, 32 * s.mask.shape[1] - 1) // 32)[:, None, :].expand(-1, s.max_new, -1))
        seen = ((word >> (bit % 32)[:, None, :]) & 1).bool() & (bit < 32 * s.mask.shape[1])[:, None, :]
        seen = (seen | (bit < 0)[:, None, :]) & (key < (ctx + starts[1:] - starts[:-1])[:, None])[:, None, :]
    score.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = weight.sum(-1, keepdim=True)
    out = torch.matmul(weight.flatten(2, 3), v).view(seqs, kv_heads, s.max_new, group, h) / total
    out = torch.where(total > 0, out, 0.0).permute(0, 2, 1, 3, 4).flatten(2, 3)
    s.out[at[there]] = out[there].to(s.out.dtype)
    return {"out": s.out}


def _plain_beam(s):
    case = s.case
    n, b, k = case["groups"], case["beams"], case["out_beams"]
    vocab = s.logits.shape[1]
    x = s.logits.double() / case["temperature"]
    x = x - x.amax(-1, keepdim=True)
    total = (x - x.exp().sum(-1, keepdim=True).log()).view(n, b, vocab) + s.scores.double()[:, :, None]
    # a beam that has ended goes on as it is
    ended = s.done.bool()
    token = torch.arange(vocab, device="cuda")
    total = torch.where(ended[:, :, None], torch.where(token == s.eos, s.scores.double()[:, :, None], -math.inf), total).flatten(1)
    # equal scores: the first beam, of its tokens the lowest, first
    best, at = (t[:, :k] for t in total.sort(dim=-1, descending=True, stable=True))
    parent, token = at // vocab, at % vocab
    o = s.out
    o["scores"].copy_(best)
    o["tokens"].copy_(token)
    o["parents"].copy_(parent)
    o["done"].copy_(ended.gather(1, parent) | (token == s.eos))
    place = torch.arange(s.history.shape[2], device="cuda")
    moved = s.history.gather(1, parent[:, :, None].expand(-1, -1, s.history.shape[2]))
    length = s.lengths[:, None, None]
    moved = torch.where(place == length, token[:, :, None].to(torch.int32), moved)
    o["history"].copy_(torch.where(place <= length, moved, o["history"]))
    return o


def run(state):
    if own:
        return _run_own(state)
    return {"append": _plain_append, "attend": _plain_attend, "beam": _plain_beam}[state.case["op"]](state)


# ---- what a pass cannot do without, and its values in 64 bits ----------------------------------------


def work(case):
    q_heads, kv_heads, h, vocab = HEADS[case["model"]]
    size = 2 if case["type"] == "bf16" else 4
    if case["op"] == "beam":
        rows, n = case["groups"] * case["beams"], case["groups"] * case["out_beams"]
        return {"bytes": rows * (vocab * size + 8) + n * 16 + 2 * n * case["length"] * 4, "flops": 5 * rows * vocab}
    ctx, new = _lengths(case)
    cached, rows = int(ctx.sum()), int(new.sum())
    token = 2 * kv_heads * (2 * h if case["bits"] == 16 else 9 * h // 16)  # bytes of a token in the cache
    if case["op"] == "append":
        moved = rows * (2 * (q_heads + kv_heads) * h * size + token)
        if case["bits"] == 4:  # and read again
            moved += rows * (token + 2 * kv_heads * h * size)
        return {"bytes": moved, "flops": 3 * rows * (q_heads + kv_heads) * h}
    keys = int((new * ctx).sum()) + int((new * (new + 1)).sum()) // 2
    return {"bytes": (cached + rows) * token + rows * 2 * q_heads * h * size, "flops": 4 * keys * q_heads * h}


def _exact_token(pool, page, place, h, values):
    """Channels of tokens from a pool of 4 bits, one by one: [n, heads, h] in 64 bits."""
    c = torch.arange(h, device="cuda")
    place = place[:, None]
    if values == "k":
        nibble = ((c // 8 % 4 * PAGE + place) * (h // 32) + c // 32) * 8 + c % 2 * 4 + c % 8 // 2
    else:
        nibble = ((((place // 4 * 16 + c % 16) * 2 + place // 2 % 2) * (h // 64) + c // 64) * 2 + place % 2) * 4 + c // 16 % 4
    rows = pool[page]  # [n, heads, 9 h]
    byte = rows.gather(2, (nibble // 2)[:, None, :].expand(-1, rows.shape[1], -1)).int()
    code = torch.where(nibble[:, None, :] % 2 == 1, byte >> 4, byte & 15)
    word = pool.view(torch.int32)[page].gather(2, (2 * h + c // 64 * PAGE + place)[:, None, :].expand(-1, rows.shape[1], -1))
    return (word << 16).view(torch.float32).double() * (16.0 + code) + word.view(torch.float32).double()


def _exact_quantised(x):
    """What a cache of 4 bits holds of [n, heads, h]."""
    out = torch.empty_like(x, dtype=torch.float64)
    for g in range(0, x.shape[-1], 64):
        y = x[..., g: g + 64].double()
        low, high = y.min(-1, keepdim=True).values, y.max(-1, keepdim=True).values
        most = y.abs().max(-1, keepdim=True).values
        scale = ((68 * (high - low) + most) / 1024).float().to(torch.bfloat16)
        want = (low - most / 128 - 16 * scale.double()).float()
        # of the words whose lower half is the scale's, the nearest
        lower, bits = scale.view(torch.int16).long(), want.view(torch.int32).long()
        at = torch.stack([(bits >> 16) + step << 16 | lower for step in (-1, 0, 1)])
        word = at.gather(0, (at - bits).abs().argmin(0, keepdim=True))[0]
        offset = word.to(torch.int32).view(torch.float32).double()
        out[..., g: g + 64] = offset + scale.double() * ((y - offset) / scale.double()).round().clamp(16, 31)
    return out


def _exact_append(s):
    _, _, h, _ = HEADS[s.case["model"]]
    got = {"q": torch.empty(s.q.shape, dtype=torch.float64, device="cuda")}
    k = torch.empty(s.k.shape, dtype=torch.float64, device="cuda")
    _, slot, page, place = _places(s)
    position = (slot if s.positions is None else s.positions).double()
    for j in range(h // 2):
        f = THETA ** (-2 * j / h) if s.freqs is None else s.freqs[j]
        turn = torch.polar(torch.ones_like(position), position * f)[:, None]
        for x, y in ((s.q, got["q"]), (s.k, k)):
            z = torch.complex(x[..., j].double(), x[..., j + h // 2].double()) * turn
            y[..., j], y[..., j + h // 2] = z.real, z.imag
    if s.case["bits"] == 4:
        return dict(got, k=_exact_quantised(k.float()), v=_exact_quantised(s.v))
    kp, vp = s.k_pool[1].clone(), s.v_pool[1].clone()
    j, t, heads = torch.arange(h, device="cuda"), place[:, None], kp.shape[1]
    k_at, v_at = (j // 8 * PAGE + t) * 8 + j % 8, (j // 32 * 64 + t // 4 * 16 + j % 16) * 8 + j // 16 % 2 * 4 + t % 4
    for head in range(heads):
        kp[page[:, None], head, k_at] = k[:, head].float().to(kp.dtype)
        vp[page[:, None], head, v_at] = s.v[:, head].to(vp.dtype)
    return dict(got, k_cache=kp, v_cache=vp)


def _exact_attend(s):
    """Sequence by sequence and head by head, keys and values put in order token by token."""
    q_heads, kv_heads, h, _ = HEADS[s.case["model"]]
    out = torch.zeros(s.out.shape, dtype=torch.float64, device="cuda")
    ctx, starts, tables = s.ctx.tolist(), s.starts.tolist(), s.tables.long()
    for n in range(s.case["seqs"]):
        r0, r1 = starts[n], starts[n + 1]
        t = torch.arange(ctx[n] + r1 - r0, device="cuda")
        page, place = tables[n, t // PAGE], t % PAGE
        k, v = (_exact_token(pool[1], page, place, h, name) for pool, name in ((s.k_pool, "k"), (s.v_pool, "v")))
        if s.mask is None:
            seen = t[None, :] <= ctx[n] + torch.arange(r1 - r0, device="cuda")[:, None]
        else:
            bit = t - int(s.mask_base[n])
            words = s.mask[r0:r1].long() & 0xFFFFFFFF
            seen = (words[:, bit.clamp(min=0) // 32] >> (bit.clamp(min=0) % 32)) & 1
            seen = (seen == 1) | (bit < 0)[None, :]
        for a in range(q_heads):
            score = s.q[r0:r1, a].double() @ k[:, a // (q_heads // kv_heads)].T.contiguous() / math.sqrt(h)
            out[r0:r1, a] = torch.softmax(score.masked_fill(~seen, -math.inf), -1) @ v[:, a // (q_heads // kv_heads)].contiguous()
    return {"out": out}


def _exact_beam(s):
    """Beam by beam, the best of its tokens; whole numbers are the plain form's to say."""
    case = s.case
    scores = []
    for g in range(case["groups"]):
        found = []
        for b in range(case["beams"]):
            if int(s.done[g, b]):
                found.append(s.scores[g, b: b + 1].double())
                continue
            p = torch.log_softmax(s.logits[g * case["beams"] + b].double() / case["temperature"], -1)
            found.append(p.topk(min(case["out_beams"], p.numel())).values + s.scores[g, b].double())
        scores.append(torch.cat(found).sort(descending=True).values[: case["out_beams"]])
    return {"scores": torch.stack(scores), "tokens": None, "parents": None, "done": None, "history": None}


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "beam": _exact_beam}[case["op"]](s)
