"""Several sequences on one pair of page pools: bookkeeping on the host, pages on the device."""
from __future__ import annotations

from typing import Dict, List, Optional, Sequence

import torch

from . import binding as B
from .runtime import _check, make_cfg


class _Sequence:
    def __init__(self, table: torch.Tensor):
        self.pages: List[int] = []
        self.length = 0
        self.table = table  # on the device: what steps, prompts and card_kv_gather read


class AttendPlan:
    """What the attention calls of one batch share, layer after layer: lengths, row starts and block tables on the device, and a
    workspace.  Made by SequencePool.plan; it holds as long as its sequences keep its tokens on its pages, and for calls that store, its rows' pages
    to themselves.  Calls of one plan run one after the other."""

    def __init__(self, pool: "SequencePool", seqs: Sequence[int], new: Sequence[int]):
        dev = pool.device
        held = [pool._seqs[s] for s in seqs]
        self._pool, self._changes = pool, None
        self._rows = [(s, list(h.pages), h.length - n, h.length) for s, h, n in zip(seqs, held, new)]
        width = max(1, max(len(h.pages) for h in held))
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        self.n_rows, self.n_seqs = starts[-1], len(held)
        self.stream = torch.cuda.current_stream(dev)
        self.ctx_lens = torch.tensor([h.length - n for h, n in zip(held, new)], dtype=torch.int32, device=dev)
        self.row_starts = torch.tensor(starts, dtype=torch.int32, device=dev)
        self.tables = torch.tensor([h.pages + [0] * (width - len(h.pages)) for h in held], dtype=torch.int32, device=dev)
        self.batch = B.CardKVBatch(pool.k_pages.data_ptr(), pool.v_pages.data_ptr(), pool.n_pages, self.n_seqs, self.tables.data_ptr(), width,
                                   self.n_rows, self.ctx_lens.data_ptr(), self.row_starts.data_ptr(), max(new), max(h.length for h in held))
        need = B.card_kv_attend_workspace_bytes if pool.bits == 16 else B.card_kv4_attend_workspace_bytes
        self.workspace = torch.empty(need(pool.cfg, self.batch), dtype=torch.uint8, device=dev)

    def _look_again(self) -> None:
        """What the pool's changes since the last look leave of the plan."""
        pool = self._pool
        if self._changes == pool._changes:
            return
        self._changes = pool._changes
        self._reads = all(s in pool._seqs and pool._seqs[s].length >= end and pool._seqs[s].pages[:len(pages)] == pages for s, pages, _, end in self._rows)
        self._stores = self._reads and all(pool.writable(s, first, end) for s, _, first, end in self._rows)


class SequencePool:
    """Pages of one model's cache, shared by sequences that come and go.  A sequence has a length and the pages for it; a fork shares
    the pages that are full and copies the last one.  Pages that several sequences hold are never written: what would write to one
    gets a copy first.  A new page's values are zero, whoever held it before: steps and prompts multiply the places behind a text's end with weights of
    zero.  One thread at a time; device work goes to the current stream, in the order of the calls.

    Steps and prompts of a Target run on a sequence after Target.attach; a program with its own layers rotates and stores through append(), or
    stores what it has rotated through attend(), and attends through attend().

    bits=4: codes of 4 bits with a scale and an offset for each 64 channels of a token, 3.5 times as many tokens in the same memory (card_kv4_append).
    Such a pool is for append() and attend(); a Target does not run on it."""

    bits = 16

    def __init__(self, shape, n_pages: int, max_ctx: int, device: str = "cuda:0", bits: int = 16):
        if not torch.cuda.is_available():
            raise RuntimeError("libcard needs a GPU: there is no CPU path")
        self._setup(make_cfg(shape, max_ctx), n_pages, torch.device(device), bits)

    def _setup(self, cfg, n_pages: int, device, bits: int = 16) -> None:
        if bits not in (16, 4):
            raise ValueError("bits: 16 or 4")
        self.cfg, self.n_pages, self.bits = cfg, int(n_pages), bits
        nbytes = (B.card_kv_pool_bytes if bits == 16 else B.card_kv4_pool_bytes)(self.cfg, self.n_pages)
        if nbytes == 0:
            raise B.CardError(B.CARD_EINVAL, "card_kv_pool_bytes")
        self.k_pages = torch.zeros(nbytes, dtype=torch.uint8, device=device)
        self.v_pages = torch.zeros(nbytes, dtype=torch.uint8, device=device)
        self.device = self.k_pages.device  # ("cuda" has become the device that was current)
        self._free = list(range(self.n_pages - 1, -1, -1))
        self._users = [0] * self.n_pages
        self._written = [False] * self.n_pages  # pages that some sequence has held
        self._seqs: Dict[int, _Sequence] = {}
        self._next = 0
        self._changes = 0  # of what sequences hold and share

    # -- bookkeeping
    @property
    def free_pages(self) -> int:
        return len(self._free)

    def length(self, seq: int) -> int:
        return self._seqs[seq].length

    def new(self) -> int:
        """An empty sequence; returns its number."""
        seq, self._next = self._next, self._next + 1
        self._seqs[seq] = _Sequence(torch.zeros(self.cfg.max_ctx // 16, dtype=torch.int32, device=self.device))
        return seq

    def free(self, seq: int) -> None:
        self._changes += 1
        for p in self._seqs.pop(seq).pages:
            self._release(p)

    def truncate(self, seq: int, length: int) -> None:
        """Forget the tokens from `length` on."""
        s = self._seqs[seq]
        if not 0 <= length <= s.length:
            raise B.CardError(B.CARD_ERANGE, "truncate")
        self._changes += 1
        keep = (length + 15) // 16
        for p in s.pages[keep:]:
            self._release(p)
        del s.pages[keep:]
        s.length = length

    def extend(self, seq: int, n: int) -> None:
        """Room for n more tokens, which the caller stores.  CARD_ECAPACITY, and nothing changes, where there are no pages for them."""
        s = self._seqs[seq]
        if n < 0:
            raise B.CardError(B.CARD_ERANGE, "extend")
        self._changes += 1
        if s.length + n > self.cfg.max_ctx:
            raise B.CardError(B.CARD_ECAPACITY, "extend")
        need = (s.length + n + 15) // 16 - len(s.pages)
        shared = self._shared(s, s.length, s.length + n)
        if need + len(shared) > len(self._free):
            raise B.CardError(B.CARD_ECAPACITY, "extend")
        self._own(s, shared)
        if need > 0:
            again = any(self._written[p] for p in self._free[-need:])
            s.pages += [self._take() for _ in range(need)]
            self._upload(s)
            if again and self.bits == 16:  # (of 4 bits, places behind an end are never multiplied)
                values = self.v_pages.view(torch.int64).view(self.cfg.n_layers, self.n_pages, -1)
                values.index_fill_(1, s.table[len(s.pages) - need:len(s.pages)].long(), 0)
        s.length += n

    def fork(self, seq: int) -> int:
        """A sequence of the same tokens: full pages are shared, the last one, which both may go on writing, is copied as the calls before have
        left it."""
        s = self._seqs[seq]
        tail = s.length % 16 != 0
        if tail and not self._free:
            raise B.CardError(B.CARD_ECAPACITY, "fork")
        self._changes += 1
        other = self.new()
        t = self._seqs[other]
        t.length, t.pages = s.length, list(s.pages)
        for p in t.pages:
            self._users[p] += 1
        if tail:
            self._own(t, [len(t.pages) - 1])
        self._upload(t)
        return other

    def compact(self, seq: int, first: int, positions: Sequence[int]) -> None:
        """The tokens at `positions` (ascending, from `first` on at the earliest) move to first, first + 1, ..., in all layers; the
        sequence ends behind them.  The accepted nodes of a draft's tree become text; tokens that a text gives up leave no gaps."""
        s = self._seqs[seq]
        pos = [int(p) for p in positions]
        if not 0 <= first <= s.length or any(b <= a for a, b in zip(pos, pos[1:])) or (pos and (pos[0] < first or pos[-1] >= s.length)):
            raise B.CardError(B.CARD_ERANGE, "compact")
        moves = [(p, first + i) for i, p in enumerate(pos) if p != first + i]
        if moves:
            shared = self._shared(s, moves[0][1], first + len(pos))
            if len(shared) > len(self._free):
                raise B.CardError(B.CARD_ECAPACITY, "compact")
            self._own(s, shared)
            slot = lambda p: s.pages[p // 16] * 16 + p % 16  # noqa: E731
            with torch.cuda.device_of(self.k_pages):
                move = B.card_kv_move_slots if self.bits == 16 else B.card_kv4_move_slots
                _check(move(self.cfg, self._pools(), [slot(p) for p, _ in moves], [slot(q) for _, q in moves], self._stream()), "card_kv_move_slots")
        self.truncate(seq, first + len(pos))

    def reorder(self, seqs: Sequence[int], parents: Sequence[int]) -> List[int]:
        """Beams that go on: sequence number i of the result continues seqs[parents[i]], and what no parent names is freed.  The first that continues a
        sequence keeps it, the others are forks of it: full pages are shared, last pages copied in one call.  CARD_ECAPACITY, and nothing changes,
        where there are no pages for that."""
        parents = [int(p) for p in parents]
        if len(set(seqs)) != len(seqs) or any(not 0 <= p < len(seqs) for p in parents):
            raise ValueError("each sequence once, and parents among them")
        held = [self._seqs[s] for s in seqs]
        tails = [p for i, p in enumerate(parents) if p in parents[:i] and held[p].length % 16 != 0]
        gone = [s for i, s in enumerate(seqs) if i not in parents]
        users: Dict[int, int] = {}
        for s in gone:
            for page in self._seqs[s].pages:
                users[page] = users.get(page, 0) + 1
        if len(tails) > len(self._free) + sum(self._users[page] == n for page, n in users.items()):
            raise B.CardError(B.CARD_ECAPACITY, "reorder")
        for s in gone:
            self.free(s)
        self._changes += 1
        result, src, dst, forks = [], [], [], []
        for i, p in enumerate(parents):
            if p not in parents[:i]:
                result.append(seqs[p])
                continue
            result.append(self.new())
            t = self._seqs[result[-1]]
            t.length, t.pages = held[p].length, list(held[p].pages)
            whole = t.length // 16
            for page in t.pages[:whole]:
                self._users[page] += 1
            if t.length % 16 != 0:
                src.append(t.pages[-1])
                t.pages[-1] = self._take()
                dst.append(t.pages[-1])
            forks.append(t)
        if src:
            self._copy_pages(src, dst)
        if forks:  # (their tables in one upload)
            width = max(len(t.pages) for t in forks)
            rows = torch.tensor([t.pages + [0] * (width - len(t.pages)) for t in forks], dtype=torch.int32, device=self.device)
            for t, row in zip(forks, rows):
                t.table[:len(t.pages)] = row[:len(t.pages)]
        return result

    def writable(self, seq: int, first: int, end: int) -> bool:
        """Whether positions [first, end) are the sequence's, on pages of its own."""
        s = self._seqs[seq]
        return 0 <= first <= end <= s.length and not self._shared(s, first, end)

    # -- device side
    def kv(self, seq: int, pending: int = -1) -> B.CardKV:
        """The sequence as steps, prompts and card_kv_gather take it, of a pool of 16 bits: they would read far behind the end of one of 4."""
        if self.bits != 16:
            raise ValueError("a pool of 4 bits: steps, prompts and card_kv_gather take 16")
        return B.CardKV(self.k_pages.data_ptr(), self.v_pages.data_ptr(), self._seqs[seq].table.data_ptr(), self.n_pages, int(pending))

    def plan(self, seqs: Sequence[int], new: Sequence[int]) -> AttendPlan:
        """A batch: the last new[i] tokens of sequence seqs[i] (extended by them before) are the rows of the calls.  Uploads lengths and tables, and so waits
        for the current stream, as extend, fork and compact do where a sequence's pages change."""
        if not seqs or len(seqs) != len(new) or len(set(seqs)) != len(seqs):
            raise ValueError("as many numbers of new tokens as sequences, at least one, each sequence once")
        for s, n in zip(seqs, new):
            if n < 0 or not self.writable(s, self.length(s) - n, self.length(s)):
                raise B.CardError(B.CARD_EINVAL, "plan")
        return AttendPlan(self, seqs, new)

    def append(self, plan: AttendPlan, layer: int, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, positions: Optional[torch.Tensor] = None,
               freqs: Optional[Sequence[float]] = None, out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """card_kv_append (or card_kv4_append) of the plan's rows: k and v [rows][kv heads][h] go to their pages, k rotated, and q
        [rows][query heads][h] comes back rotated (in `out`, which may be q), for attend() without k and v.  positions: int32 [rows] on the pool's
        device, where they are not the places in the sequences; freqs: h / 2 frequencies, where they are not the model's.  CARD_ESTALE as attend()."""
        cfg = self.cfg
        if q is not None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
        elif out is not None:
            raise ValueError("out without q")
        self._look_at_rows(plan, (q, cfg.n_q_heads), (out, cfg.n_q_heads), (k, cfg.n_kv_heads), (v, cfg.n_kv_heads))
        if positions is not None and (tuple(positions.shape) != (plan.n_rows,) or positions.dtype != torch.int32 or not positions.is_contiguous() or
                                      positions.device != self.k_pages.device):
            raise ValueError("positions: int32 [rows], on the pool's device")
        if plan.n_rows == 0:
            return out
        self._still_holds(plan, True, "append")
        rows = [None if t is None else B.card_rows(t) for t in (q, out, k, v)]
        call = B.card_kv_append if self.bits == 16 else B.card_kv4_append
        with torch.cuda.device_of(self.k_pages):
            _check(call(cfg, plan.batch, layer, B.card_rotation(freqs, positions), *rows, self._stream()), "card_kv_append")
        return out

    def read(self, seq: int, layer: int, first: int = 0, end: Optional[int] = None, dtype: torch.dtype = torch.float32):
        """card_kv4_read: keys and values [end - first][kv heads][h] of tokens first .. end - 1 of a sequence (to its end), as a pool of 4 bits holds them."""
        if self.bits != 4:
            raise ValueError("of pools of 4 bits (else card_kv_gather)")
        s, cfg = self._seqs[seq], self.cfg
        end = s.length if end is None else end
        if not 0 <= first <= end <= s.length:
            raise B.CardError(B.CARD_ERANGE, "read")
        n = end - first
        k, v = (torch.empty((n, cfg.n_kv_heads, cfg.head_dim), dtype=dtype, device=self.device) for _ in range(2))
        if n > 0:
            at = torch.tensor([first, 0, n], dtype=torch.int32, device=self.device)
            batch = B.CardKVBatch(self.k_pages.data_ptr(), self.v_pages.data_ptr(), self.n_pages, 1, s.table.data_ptr(), s.table.numel(), n, at.data_ptr(),
                                  at.data_ptr() + 4, n, end)
            with torch.cuda.device_of(self.k_pages):
                _check(B.card_kv4_read(cfg, batch, layer, B.card_rows(k), B.card_rows(v), self._stream()), "card_kv4_read")
        return k, v

    def _look_at_rows(self, plan: AttendPlan, *rows) -> None:
        for t, heads in rows:
            if t is not None and (tuple(t.shape) != (plan.n_rows, heads, self.cfg.head_dim) or t.device != self.k_pages.device):
                raise ValueError(f"expected [{plan.n_rows}][{heads}][{self.cfg.head_dim}] on {self.k_pages.device}, got {tuple(t.shape)} on {t.device}")

    def _still_holds(self, plan: AttendPlan, stores: bool, where: str) -> None:
        if plan._pool is not self:
            raise ValueError("a plan of another pool")
        plan._look_again()
        if not (plan._stores if stores else plan._reads):
            raise B.CardError(B.CARD_ESTALE, where)
        stream = torch.cuda.current_stream(self.device)
        if stream != plan.stream:  # the plan may be dropped before that stream has got to the call
            for t in (plan.ctx_lens, plan.row_starts, plan.tables, plan.workspace):
                t.record_stream(stream)

    def attend(self, plan: AttendPlan, layer: int, q: torch.Tensor, k: Optional[torch.Tensor], v: Optional[torch.Tensor],
               out: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None, mask_base: Optional[torch.Tensor] = None) -> torch.Tensor:
        """card_kv_attend (or card_kv4_attend) of the plan's rows: q and out [rows][query heads][h], k and v [rows][kv heads][h] (None: stored before), bf16 or
        fp32; mask int32 [rows][words] with mask_base int32 [sequences].  CARD_ESTALE, and nothing happens, where the plan does not hold any more: its
        sequences have given up its tokens or pages, or it is to store to pages that a fork holds since."""
        cfg = self.cfg
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
        self._look_at_rows(plan, (q, cfg.n_q_heads), (k, cfg.n_kv_heads), (v, cfg.n_kv_heads), (out, cfg.n_q_heads))
        row_mask = None
        if mask is not None:
            if mask_base is None or mask.dim() != 2 or mask.shape[0] != plan.n_rows or not mask.is_contiguous() or not mask_base.is_contiguous() or \
                    mask_base.numel() != plan.n_seqs or mask.dtype != torch.int32 or mask_base.dtype != torch.int32 or \
                    mask.device != self.k_pages.device or mask_base.device != self.k_pages.device:
                raise ValueError("masks: int32 [rows][words], with mask_base int32 [sequences], on the pool's device")
            row_mask = B.CardRowMask(mask.data_ptr(), mask_base.data_ptr(), mask.shape[1])
        if plan.n_rows == 0:
            return out
        self._still_holds(plan, k is not None, "attend")
        rows = [None if t is None else B.card_rows(t) for t in (q, k, v, out)]
        call = B.card_kv_attend if self.bits == 16 else B.card_kv4_attend
        with torch.cuda.device_of(self.k_pages):
            _check(call(cfg, plan.batch, layer, *rows, row_mask, plan.workspace, self._stream()), "card_kv_attend")
        return out

    def _stream(self) -> int:
        return torch.cuda.current_stream(self.device).cuda_stream

    def _take(self) -> int:
        p = self._free.pop()
        self._users[p], self._written[p] = 1, True
        return p

    def _release(self, p: int) -> None:
        self._users[p] -= 1
        if self._users[p] == 0:
            self._free.append(p)

    def _shared(self, s: _Sequence, first: int, end: int) -> List[int]:
        """Which of the sequence's pages that hold positions [first, end) others hold, too."""
        if first >= end:
            return []
        return [i for i in range(first // 16, min((end + 15) // 16, len(s.pages))) if self._users[s.pages[i]] > 1]

    def _own(self, s: _Sequence, places: Sequence[int]) -> None:
        """Copies of these shared pages take their places."""
        if not places:
            return
        self._changes += 1
        dst = [self._take() for _ in places]
        self._copy_pages([s.pages[i] for i in places], dst)
        for i, d in zip(places, dst):
            self._release(s.pages[i])
            s.pages[i] = d
        self._upload(s)

    def _pools(self) -> B.CardKV:
        return B.CardKV(self.k_pages.data_ptr(), self.v_pages.data_ptr(), None, self.n_pages, -1)

    def _copy_pages(self, src: Sequence[int], dst: Sequence[int]) -> None:
        with torch.cuda.device_of(self.k_pages):
            copy = B.card_kv_copy_pages if self.bits == 16 else B.card_kv4_copy_pages
            _check(copy(self.cfg, self._pools(), src, dst, self._stream()), "card_kv_copy_pages")

    def _upload(self, s: _Sequence) -> None:
        s.table[:len(s.pages)] = torch.tensor(s.pages, dtype=torch.int32, device=self.device)


def token_logprobs(logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, top: int = 0, temperature: float = 1.0) -> Dict:
    """card_logprobs of logits [rows][vocab] (bf16 or fp32): "entropy" [rows], "logprob" [rows] of tokens (int32 [rows], negative: none),
    "top_tokens" and "top_logprobs" [rows][top].  No synchronisation."""
    rows, vocab = logits.shape
    dev = logits.device
    if tokens is not None and (tokens.shape != (rows,) or tokens.dtype != torch.int32 or not tokens.is_contiguous() or tokens.device != dev):
        raise ValueError("tokens: int32 [rows], beside the logits")
    res = {"entropy": torch.empty(rows, dtype=torch.float32, device=dev)}
    if tokens is not None:
        res["logprob"] = torch.empty(rows, dtype=torch.float32, device=dev)
    if top > 0:
        res["top_tokens"] = torch.empty((rows, top), dtype=torch.int32, device=dev)
        res["top_logprobs"] = torch.empty((rows, top), dtype=torch.float32, device=dev)
    ws = torch.empty(B.card_logprobs_workspace_bytes(rows, vocab, top), dtype=torch.uint8, device=dev)
    with torch.cuda.device(dev):
        _check(B.card_logprobs(logits, tokens, temperature, top, res.get("logprob"), res["entropy"], res.get("top_tokens"), res.get("top_logprobs"),
                               ws, torch.cuda.current_stream(dev).cuda_stream), "card_logprobs")
    return res


def beam_select(logits: torch.Tensor, scores: torch.Tensor, out_beams: Optional[int] = None, done: Optional[torch.Tensor] = None, eos: int = -1,
                temperature: float = 1.0, history: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None) -> Dict:
    """card_beam_select of logits [groups * beams][vocab] (bf16 or fp32) and scores fp32 [groups][beams]: "scores", "tokens", "parents" and "done"
    [groups][out_beams] (as many as beams, unless it is given).  done: int32 [groups][beams]; history: int32 [groups][beams][most] with lengths int32
    [groups], then "history" [groups][out_beams][most] has the new texts, zeros behind them.  SequencePool.reorder lets the sequences follow the
    parents.  No synchronisation."""
    groups, beams = scores.shape
    rows, vocab = logits.shape
    dev, n = logits.device, beams if out_beams is None else int(out_beams)
    if (history is None) != (lengths is None):
        raise ValueError("history and lengths: both or neither")
    most = 0 if history is None else history.shape[-1]
    for t, shape, dtype in ((scores, (groups, beams), torch.float32), (done, (groups, beams), torch.int32), (history, (groups, beams, most), torch.int32),
                            (lengths, (groups,), torch.int32)):
        if t is not None and (tuple(t.shape) != shape or t.dtype != dtype or not t.is_contiguous() or t.device != dev):
            raise ValueError(f"expected {dtype} {shape}, contiguous, beside the logits")
    if rows != groups * beams:
        raise ValueError("a row of logits for each beam")
    whole = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=dev)  # noqa: E731
    res = {"scores": torch.empty((groups, n), dtype=torch.float32, device=dev), "tokens": whole(groups, n), "parents": whole(groups, n), "done": whole(groups, n)}
    if history is not None:
        res["history"] = whole(groups, n, most)
    at = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    args = B.CardBeams(groups, beams, n, int(eos), at(scores), at(done), at(history), at(lengths), most, at(res["scores"]), at(res["tokens"]),
                       at(res["parents"]), at(res["done"]), at(res.get("history")))
    ws = torch.empty(B.card_beam_select_workspace_bytes(groups, beams, n, vocab), dtype=torch.uint8, device=dev)
    with torch.cuda.device(dev):
        _check(B.card_beam_select(logits, args, temperature, ws, torch.cuda.current_stream(dev).cuda_stream), "card_beam_select")
    return res
