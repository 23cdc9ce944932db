"""The operators of a program that serves several texts from one paged cache, at the sizes that it calls them: attention of each
text's new tokens, page copies (a fork copies the page it goes on writing), moves of tokens between slots (accepted nodes of
the draft's tree join the text; a text gives up tokens) and log probabilities of tokens.

Pages, layers and head layouts are those of the library's cache.  Their plain forms below are elementary torch operations in 32 bits.
"""
import ctypes
import math

import torch

own = False

# query heads, key/value heads, head size, layers and vocabulary of the shapes in card_inputs/configs.py, and one of odd sizes
HEADS = {
    "tiny": (4, 2, 64, 2, 1024),
    "odd": (10, 2, 128, 3, 3001),
    "llama1b": (32, 8, 64, 16, 128256),
    "llama8b": (32, 8, 128, 32, 128256),
    "llama70b": (64, 8, 128, 80, 128256),
    "qwen7b": (28, 4, 128, 28, 152064),
}
PAGE = 16
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _attend(model, seqs, new, ctx, mask="causal", type="bf16"):
    """seqs sequences of up to `ctx` tokens in the cache and up to `new` new ones each (one of them has as many)."""
    return {"op": "attend", "model": model, "seqs": seqs, "new": new, "ctx": ctx, "mask": mask, "type": type}


def _copy(model, layers, pages):
    return {"op": "copy", "model": model, "layers": layers, "pages": pages}


def _move(model, layers, texts, tokens, reach):
    """`tokens` tokens of each text move to the front of the reach * tokens last slots of it."""
    return {"op": "move", "model": model, "layers": layers, "texts": texts, "tokens": tokens, "reach": reach}


def _logprobs(model, rows, top, type="f32", temperature=1.0):
    return {"op": "logprobs", "model": model, "rows": rows, "top": top, "type": type, "temperature": temperature}


def listed():
    cases = {
        # one token each for three short texts of the smallest shape: latency
        "attend tiny": _attend("tiny", 3, 1, 100),
        # plain decoding of a batch of texts of different lengths
        "attend decode": _attend("llama8b", 48, 1, 4000),
        # a chain of five candidates of one long text
        "attend long": _attend("llama70b", 1, 5, 32700),
        # chunks of three prompts behind what their texts hold already
        "attend chunks": _attend("qwen7b", 3, 1000, 3500),
        # the last chunk of a long prompt
        "attend prompt": _attend("llama8b", 1, 2000, 14000),
        # a level of the draft's tree, activations in 32 bits as the library keeps them
        "attend tree f32": _attend("llama1b", 1, 100, 1024, "tree", "f32"),
        # the fork of one short text
        "copy tail": _copy("tiny", 2, 1),
        # a batch of forks, or a text of 2500 tokens copied whole
        "copy text": _copy("llama8b", 32, 157),
        # the accepted nodes of eight draft trees
        "move paths": _move("llama1b", 16, 8, 4, 6),
        # a text that gives up every third token or so
        "move text": _move("llama8b", 32, 1, 1500, 1.4),
        # the rows of one verification step, with alternatives
        "logprobs step": _logprobs("llama8b", 8, 5),
        # the tokens of a prompt
        "logprobs prompt": _logprobs("qwen7b", 1000, 1, "bf16", 0.7),
    }
    return [dict(case, name=name) for name, case in cases.items()]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    model = rng.choice(list(HEADS))
    q_heads, kv_heads, h, layers, vocab = HEADS[model]
    op = rng.choice(["attend", "attend", "attend", "copy", "move", "logprobs", "logprobs"])
    if op == "attend":
        type = rng.choice(["bf16", "bf16", "f32"])
        if rng.random() < 0.25:
            return _attend(model, rng.randint(1, 4), rng.randint(2, 128), _log_uniform(rng, 1, 2000), "tree", type)
        if rng.random() < 0.5:
            seqs = _log_uniform(rng, 1, 64)
            return _attend(model, seqs, rng.choice([1, 1, rng.randint(2, 8)]), _log_uniform(rng, 1, min(32000, 200000 // seqs)), "causal", type)
        # (the plain form holds all scores: sequences x new x query heads x length in 32 bits)
        seqs, new = rng.randint(1, 4), _log_uniform(rng, 9, 2000)
        most = 2000 * 16000 * 32 // (seqs * new * q_heads) - new
        return _attend(model, seqs, new, _log_uniform(rng, 1, max(2, min(14000, most))), "causal", type)
    if op == "copy":
        layers = rng.randint(1, min(layers, 32))
        return _copy(model, layers, _log_uniform(rng, 1, max(1, 157 * 32 * 8 * 128 // (layers * kv_heads * h))))
    if op == "move":
        layers = rng.randint(1, min(layers, 32))
        tokens = _log_uniform(rng, 1, 1500)
        return _move(model, layers, rng.randint(1, max(1, min(8, 1500 // tokens))), tokens, rng.choice([1.2, 1.4, 3, 6]))
    type = rng.choice(["f32", "bf16"])
    return _logprobs(model, _log_uniform(rng, 1, 1000 if type == "bf16" else 500), rng.choice([0, 1, 5, 20]), type, rng.choice([1.0, 0.7, 1.3]))


# ---- inputs ---------------------------------------------------------------------------------------


def _generator(seed, stream, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed((seed * 1000003 + stream * 7919 + 17) & 0x7FFFFFFFFFFFFFFF)
    return g


class _State:
    pass


def _pools(s, case, layers, pages, seed):
    _, kv_heads, h, _, _ = HEADS[case["model"]]
    s.layers, s.pages = layers, pages
    shape = (layers, pages, kv_heads, PAGE * h)
    s.k_pool = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=_generator(seed, 1))
    s.v_pool = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=_generator(seed, 2))


def _lengths(case):
    """Tokens in the cache and new tokens of each sequence, the same for every seed: the first has the most of both."""
    n, g = case["seqs"], _generator(0, 3, "cpu")
    ctx = (torch.rand(n, generator=g) * 0.9 + 0.1).mul(case["ctx"]).long()
    new = (torch.rand(n, generator=g) * case["new"]).long().add(1).clamp(max=case["new"])
    ctx[0], new[0] = case["ctx"], case["new"]
    return ctx, new


def _prepare_attend(s, case, seed):
    q_heads, kv_heads, h, _, _ = HEADS[case["model"]]
    ctx, new = _lengths(case)
    need = (ctx + new + PAGE - 1) // PAGE
    total, most = int(need.sum()), int(need.max())
    _pools(s, case, 2, total + 3, seed)
    order = torch.randperm(total + 3, generator=_generator(seed, 4, "cpu"))[:total]
    tables = torch.zeros((case["seqs"], most), dtype=torch.int32)
    tables[torch.arange(most)[None, :] < need[:, None]] = order.to(torch.int32)
    starts = torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)])
    s.n_rows, s.max_new, s.max_len = int(starts[-1]), int(new.max()), int((ctx + new).max())
    s.tables, s.ctx, s.starts = tables.cuda(), ctx.to(torch.int32).cuda(), starts.to(torch.int32).cuda()
    # queries, keys and values as a fused projection leaves them: side by side in a row
    width = (q_heads + 2 * kv_heads) * h
    qkv = torch.empty((s.n_rows, width), dtype=torch.float32, device="cuda").normal_(generator=_generator(seed, 5))
    qkv = qkv.to(TYPES[case["type"]])
    s.q = qkv[:, : q_heads * h].view(s.n_rows, q_heads, h)
    s.k = qkv[:, q_heads * h: (q_heads + kv_heads) * h].view(s.n_rows, kv_heads, h)
    s.v = qkv[:, (q_heads + kv_heads) * h:].view(s.n_rows, kv_heads, h)
    s.out = torch.zeros((s.n_rows, q_heads, h), dtype=qkv.dtype, device="cuda")
    s.mask = s.mask_base = None
    if case["mask"] == "tree":
        # every node sees the context and itself, and a third of the other nodes' slots (ancestors)
        words = (s.max_new + PAGE + 31) // 32
        base = ctx // PAGE * PAGE
        row_of = torch.arange(s.n_rows) - torch.repeat_interleave(starts[:-1], new)
        past = torch.repeat_interleave(ctx - base, new)  # context slots behind the mask's begin
        bit = torch.arange(32 * words)[None, :]
        seen = torch.rand((s.n_rows, 32 * words), generator=_generator(seed, 6, "cpu")) < 0.33
        seen = (seen & (bit < (past + row_of)[:, None])) | (bit < past[:, None]) | (bit == (past + row_of)[:, None])
        value = (seen.view(s.n_rows, words, 32).long() << torch.arange(32)).sum(-1)
        s.mask = torch.where(value >= 1 << 31, value - (1 << 32), value).to(torch.int32).cuda()
        s.mask_base = base.to(torch.int32).cuda()
    if own:
        s.plan = _attend_plan(s, case)


def _moves(case, seed):
    """Slots (page * 16 + place) that tokens come from and go to, text by text, and the number of pages."""
    g, tokens = _generator(seed, 7, "cpu"), case["tokens"]
    span = max(tokens + 1, int(tokens * case["reach"]))
    pages = (span + 2 * PAGE - 1) // PAGE
    order = torch.randperm(case["texts"] * pages, generator=g).view(case["texts"], pages)
    src, dst = [], []
    for text in range(case["texts"]):
        first = int(torch.randint(0, PAGE, (1,), generator=g))
        kept = torch.randperm(span - 1, generator=g)[:tokens].sort().values + first + 1
        to = torch.arange(tokens) + first
        src.append(order[text][kept // PAGE] * PAGE + kept % PAGE)
        dst.append(order[text][to // PAGE] * PAGE + to % PAGE)
    return torch.cat(src), torch.cat(dst), case["texts"] * pages


def prepare(case, seed):
    s = _State()
    s.case = case
    if case["op"] == "attend":
        _prepare_attend(s, case, seed)
        return s
    if case["op"] == "logprobs":
        _, _, _, _, vocab = HEADS[case["model"]]
        rows = case["rows"]
        # logits as a vocabulary head gives them: a bell with a few tokens that stand out
        x = torch.empty((rows, vocab), dtype=torch.float32, device="cuda").normal_(0.0, 2.0, generator=_generator(seed, 8))
        likely = torch.randint(0, vocab, (rows, 4), device="cuda", generator=_generator(seed, 9))
        x.scatter_add_(1, likely, torch.rand((rows, 4), device="cuda", generator=_generator(seed, 10)) * 12.0)
        s.logits = x.to(TYPES[case["type"]])
        s.tokens = torch.randint(0, vocab, (rows,), device="cuda", generator=_generator(seed, 11)).to(torch.int32)
        s.tokens[::2] = likely[::2, 0].to(torch.int32)
        s.logprob = torch.empty(rows, dtype=torch.float32, device="cuda")
        s.entropy = torch.empty(rows, dtype=torch.float32, device="cuda")
        s.top_tokens = torch.empty((rows, case["top"]), dtype=torch.int32, device="cuda")
        s.top_logprobs = torch.empty((rows, case["top"]), dtype=torch.float32, device="cuda")
        if own:
            s.plan = _logprobs_plan(s, case)
        return s
    if case["op"] == "copy":
        n = case["pages"]
        _pools(s, case, case["layers"], 2 * n + 1, seed)
        order = torch.randperm(2 * n + 1, generator=_generator(seed, 12, "cpu"))
        src, dst = order[:n], order[n: 2 * n]
    else:
        src, dst, pages = _moves(case, seed)
        _pools(s, case, case["layers"], pages, seed)
    s.src, s.dst = src.cuda(), dst.cuda()
    # the lists as the host's bookkeeping holds them
    s.src_host, s.dst_host = ((ctypes.c_int32 * len(x))(*x.tolist()) for x in (src, dst))
    if own:
        s.plan = _pool_plan(s, case)
    return s


# ---- the framework's calls ------------------------------------------------------------------------


def _cfg(case, layers):
    import paper_2508_04462_amd as card

    q_heads, kv_heads, h, _, vocab = HEADS[case["model"]]
    # (of a model, these operators take the layers, heads and head size)
    return card.CardModelCfg(layers, 512, q_heads, kv_heads, h, 512, vocab, 1e4, 1e-5, PAGE, 1 << 20, 32, 0)


def _pool_plan(s, case):
    import paper_2508_04462_amd as card

    return _cfg(case, s.layers), card.CardKV(s.k_pool.data_ptr(), s.v_pool.data_ptr(), None, s.pages, -1)


def _attend_plan(s, case):
    import paper_2508_04462_amd as card

    cfg = _cfg(case, s.layers)
    batch = card.CardKVBatch(s.k_pool.data_ptr(), s.v_pool.data_ptr(), s.pages, case["seqs"], s.tables.data_ptr(), s.tables.shape[1],
                             s.n_rows, s.ctx.data_ptr(), s.starts.data_ptr(), s.max_new, s.max_len)
    mask = None
    if s.mask is not None:
        mask = card.CardRowMask(s.mask.data_ptr(), s.mask_base.data_ptr(), s.mask.shape[1])
    workspace = torch.empty(card.card_kv_attend_workspace_bytes(cfg, batch), dtype=torch.uint8, device="cuda")
    return cfg, batch, mask, workspace


def _logprobs_plan(s, case):
    import paper_2508_04462_amd as card

    rows, vocab = s.logits.shape
    return torch.empty(card.card_logprobs_workspace_bytes(rows, vocab, case["top"]), dtype=torch.uint8, device="cuda")


def _run_own(s):
    import paper_2508_04462_amd as card

    case, stream = s.case, torch.cuda.current_stream().cuda_stream
    if case["op"] == "attend":
        cfg, batch, mask, workspace = s.plan
        status = card.card_kv_attend(cfg, batch, 1, card.card_rows(s.q), card.card_rows(s.k), card.card_rows(s.v), card.card_rows(s.out),
                                     mask, workspace, stream)
        got = {"out": s.out, "k_cache": s.k_pool[1], "v_cache": s.v_pool[1]}
    elif case["op"] == "logprobs":
        status = card.card_logprobs(s.logits, s.tokens, case["temperature"], case["top"], s.logprob, s.entropy, s.top_tokens,
                                    s.top_logprobs, s.plan, stream)
        got = _logprobs_outputs(case, s.logprob, s.entropy, s.top_tokens, s.top_logprobs)
    else:
        call = card.card_kv_copy_pages if case["op"] == "copy" else card.card_kv_move_slots
        status = call(*s.plan, s.src_host, s.dst_host, stream)
        got = {"k_cache": s.k_pool, "v_cache": s.v_pool}
    if status != card.CARD_OK:
        raise card.CardError(status, case["op"])
    return got


# ---- the plain forms ------------------------------------------------------------------------------
# Order of the elements of a page of one head: K [h / 8][16 tokens][8]; V [h / 32][4][16][2][4], which are
# channel / 32, token / 4, channel % 16, channel / 16 % 2, token % 4.


def _k_view(pool, h):
    return pool.unflatten(-1, (h // 8, PAGE, 8))


def _v_view(pool, h):
    return pool.unflatten(-1, (h // 32, 4, 16, 2, 4))


def _k_rows(pages, h):
    """[..., pages, heads, 16 h] -> [..., heads, pages * 16, h] in 32 bits."""
    x = _k_view(pages, h).movedim(-2, -3).flatten(-2)
    return x.movedim(-4, -3).flatten(-3, -2).float()


def _v_rows(pages, h):
    x = _v_view(pages, h).movedim((-4, -1, -5, -2, -3), (-5, -4, -3, -2, -1)).flatten(-3).flatten(-3, -2)
    return x.movedim(-4, -3).flatten(-3, -2).float()


def _logprobs_outputs(case, logprob, entropy, top_tokens, top_logprobs):
    got = {"logprob": logprob, "entropy": entropy}
    if case["top"]:
        got.update(top_tokens=top_tokens, top_logprobs=top_logprobs)
    return got


def _plain_attend(s):
    q_heads, kv_heads, h, _, _ = HEADS[s.case["model"]]
    group, seqs = q_heads // kv_heads, s.case["seqs"]
    ctx, starts = s.ctx.long(), s.starts.long()
    row = torch.arange(s.n_rows, device="cuda")
    seq = torch.searchsorted(starts[1:], row, right=True)
    slot = ctx[seq] + row - starts[seq]
    page, place = s.tables[seq, slot // PAGE].long(), slot % PAGE
    kp, vp = s.k_pool[1], s.v_pool[1]
    _k_view(kp, h)[page, :, :, place] = s.k.to(kp.dtype).unflatten(-1, (h // 8, 8))
    v = s.v.to(vp.dtype).unflatten(-1, (h // 32, 2, 16)).transpose(-1, -2)
    _v_view(vp, h)[page, :, :, place // 4, :, :, place % 4] = v
    used = (s.max_len + PAGE - 1) // PAGE
    tables = s.tables[:, :used].long()
    k, v = _k_rows(kp[tables], h), _v_rows(vp[tables], h)  # [seqs, kv heads, keys, h]
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
    return {"out": s.out, "k_cache": kp, "v_cache": vp}


def _plain_move(s):
    _, _, h, _, _ = HEADS[s.case["model"]]
    k, v = _k_view(s.k_pool, h), _v_view(s.v_pool, h)
    p, t, to, u = s.src // PAGE, s.src % PAGE, s.dst // PAGE, s.dst % PAGE
    k[:, to, :, :, u] = k[:, p, :, :, t]
    v[:, to, :, :, u // 4, :, :, u % 4] = v[:, p, :, :, t // 4, :, :, t % 4]
    return {"k_cache": s.k_pool, "v_cache": s.v_pool}


def _plain_logprobs(s):
    case = s.case
    x = s.logits.float() / case["temperature"]
    d = x - x.amax(-1, keepdim=True)
    e = d.exp()
    total = e.sum(-1, keepdim=True)
    log_total = total.log()
    logprob = d.gather(1, s.tokens.long()[:, None]) - log_total
    entropy = log_total - (e * d).sum(-1, keepdim=True) / total
    # equal logits: the lowest token first
    order = s.logits.float().sort(dim=-1, descending=True, stable=True).indices[:, : case["top"]]
    top = d.gather(1, order) - log_total
    return _logprobs_outputs(case, logprob[:, 0], entropy[:, 0], order.to(torch.int32), top)


def run(state):
    if own:
        return _run_own(state)
    op = state.case["op"]
    if op == "attend":
        return _plain_attend(state)
    if op == "logprobs":
        return _plain_logprobs(state)
    if op == "copy":
        state.k_pool[:, state.dst] = state.k_pool[:, state.src]
        state.v_pool[:, state.dst] = state.v_pool[:, state.src]
        return {"k_cache": state.k_pool, "v_cache": state.v_pool}
    return _plain_move(state)


# ---- what a pass cannot do without, and its values in 64 bits ----------------------------------------


def work(case):
    q_heads, kv_heads, h, _, vocab = HEADS[case["model"]]
    if case["op"] == "logprobs":
        size = 4 if case["type"] == "f32" else 2
        return {"bytes": case["rows"] * (vocab * size + 12 + 8 * case["top"]), "flops": 5 * case["rows"] * vocab}
    if case["op"] == "copy":
        return {"bytes": 2 * case["pages"] * case["layers"] * kv_heads * PAGE * h * 4, "flops": 0}
    if case["op"] == "move":
        return {"bytes": 2 * case["texts"] * case["tokens"] * case["layers"] * kv_heads * h * 4, "flops": 0}
    ctx, new = _lengths(case)
    size = 4 if case["type"] == "f32" else 2
    cached, rows = int(ctx.sum()), int(new.sum())
    keys = int((new * ctx).sum()) + int((new * (new + 1)).sum()) // 2
    moved = cached * kv_heads * h * 4 + rows * (2 * q_heads + 2 * kv_heads) * h * size + rows * kv_heads * h * 4
    return {"bytes": moved, "flops": 4 * keys * q_heads * h}


def _exact_attend(s):
    """Sequence by sequence and head by head, keys and values put in order token by token."""
    q_heads, kv_heads, h, _, _ = HEADS[s.case["model"]]
    out = torch.zeros(s.out.shape, dtype=torch.float64, device="cuda")
    kp, vp = s.k_pool[1].clone(), s.v_pool[1].clone()
    j = torch.arange(h, device="cuda")
    ctx, starts, tables = s.ctx.tolist(), s.starts.tolist(), s.tables.long()
    for n in range(s.case["seqs"]):
        r0, r1 = starts[n], starts[n + 1]
        length = ctx[n] + r1 - r0
        t = torch.arange(length, device="cuda")
        page, place = tables[n, t // PAGE], (t % PAGE)[:, None]
        k_at = (j // 8 * PAGE + place) * 8 + j % 8
        v_at = ((j // 32 * 64 + place // 4 * 16 + j % 16) * 8) + j // 16 % 2 * 4 + place % 4
        for head in range(kv_heads):
            index = (page[ctx[n]:, None], head)
            kp[index[0], head, k_at[ctx[n]:]] = s.k[r0:r1, head].to(kp.dtype)
            vp[index[0], head, v_at[ctx[n]:]] = s.v[r0:r1, head].to(vp.dtype)
            k, v = kp[page[:, None], head, k_at].double(), vp[page[:, None], head, v_at].double()
            if s.mask is None:
                seen = t[None, :] <= ctx[n] + torch.arange(r1 - r0, device="cuda")[:, None]
            else:
                bit = t - int(s.mask_base[n])
                words = s.mask[r0:r1].long() & 0xFFFFFFFF
                seen = (words[:, bit.clamp(min=0) // 32] >> (bit.clamp(min=0) % 32)) & 1
                seen = (seen == 1) | (bit < 0)[None, :]
            for g in range(head * (q_heads // kv_heads), (head + 1) * (q_heads // kv_heads)):
                score = s.q[r0:r1, g].double() @ k.T.contiguous() / math.sqrt(h)
                weight = torch.softmax(score.masked_fill(~seen, -math.inf), -1)
                out[r0:r1, g] = weight @ v
    return {"out": out, "k_cache": kp, "v_cache": vp}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attend":
        return _exact_attend(s)
    if case["op"] == "logprobs":
        x = s.logits.double() / case["temperature"]
        p = torch.log_softmax(x, -1)
        entropy = -torch.special.xlogy(p.exp(), p.exp()).sum(-1)
        token = s.tokens.long()
        logprob = p[torch.arange(len(token), device="cuda"), token]
        top = p.topk(case["top"], -1).values if case["top"] else None
        # (which tokens they are: where two logits are equal, only the rule on ties says)
        return _logprobs_outputs(case, logprob, entropy, None, top)
    _, _, h, _, _ = HEADS[case["model"]]
    pools = {}
    for name, pool in (("k_cache", s.k_pool), ("v_cache", s.v_pool)):
        flat = pool.clone()
        if case["op"] == "copy":
            flat.index_copy_(1, s.dst, pool.index_select(1, s.src))
        else:
            j = torch.arange(h, device="cuda")

            def places(t):
                t = (t % PAGE)[:, None]
                if name == "k_cache":
                    return (j // 8 * PAGE + t) * 8 + j % 8
                return ((j // 32 * 64 + t // 4 * 16 + j % 16) * 8) + j // 16 % 2 * 4 + t % 4

            for layer in range(s.layers):
                for head in range(pool.shape[2]):
                    flat[layer, s.dst[:, None] // PAGE, head, places(s.dst)] = pool[layer, s.src[:, None] // PAGE, head, places(s.src)]
        pools[name] = flat
    return pools
