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
        self.workspace = torch.empty(B.card_kv_attend_workspace_bytes(pool.cfg, self.batch), dtype=torch.uint8, device=dev)

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

    Steps and prompts of a Target run on a sequence after Target.attach; a program with its own layers stores and attends
    through attend()."""

    def __init__(self, shape, n_pages: int, max_ctx: int, device: str = "cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("libcard needs a GPU: there is no CPU path")
        self._setup(make_cfg(shape, max_ctx), n_pages, torch.device(device))

    def _setup(self, cfg, n_pages: int, device) -> None:
        self.cfg, self.n_pages = cfg, int(n_pages)
        nbytes = B.card_kv_pool_bytes(self.cfg, self.n_pages)
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
            if again:
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
                _check(B.card_kv_move_slots(self.cfg, self.kv(seq), [slot(p) for p, _ in moves], [slot(q) for _, q in moves], self._stream()),
                       "card_kv_move_slots")
        self.truncate(seq, first + len(pos))

    def writable(self, seq: int, first: int, end: int) -> bool:
        """Whether positions [first, end) are the sequence's, on pages of its own."""
        s = self._seqs[seq]
        return 0 <= first <= end <= s.length and not self._shared(s, first, end)

    # -- device side
    def kv(self, seq: int, pending: int = -1) -> B.CardKV:
        """The sequence as steps, prompts and card_kv_gather take it."""
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

    def attend(self, plan: AttendPlan, layer: int, q: torch.Tensor, k: Optional[torch.Tensor], v: Optional[torch.Tensor],
               out: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None, mask_base: Optional[torch.Tensor] = None) -> torch.Tensor:
        """card_kv_attend of the plan's rows: q and out [rows][query heads][h], k and v [rows][kv heads][h] (None: stored before), bf16 or
        fp32; mask int32 [rows][words] with mask_base int32 [sequences].  CARD_ESTALE, and nothing happens, where the plan does not hold any more: its
        sequences have given up its tokens or pages, or it is to store to pages that a fork holds since."""
        cfg = self.cfg
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
        for t, heads in ((q, cfg.n_q_heads), (k, cfg.n_kv_heads), (v, cfg.n_kv_heads), (out, cfg.n_q_heads)):
            if t is not None and (tuple(t.shape) != (plan.n_rows, heads, cfg.head_dim) or t.device != self.k_pages.device):
                raise ValueError(f"expected [{plan.n_rows}][{heads}][{cfg.head_dim}] on {self.k_pages.device}, got {tuple(t.shape)} on {t.device}")
        row_mask = None
        if mask is not None:
            if mask_base is None or mask.dim() != 2 or mask.shape[0] != plan.n_rows or not mask.is_contiguous() or not mask_base.is_contiguous() or \
                    mask_base.numel() != plan.n_seqs or mask.dtype != torch.int32 or mask_base.dtype != torch.int32 or \
                    mask.device != self.k_pages.device or mask_base.device != self.k_pages.device:
                raise ValueError("masks: int32 [rows][words], with mask_base int32 [sequences], on the pool's device")
            row_mask = B.CardRowMask(mask.data_ptr(), mask_base.data_ptr(), mask.shape[1])
        if plan.n_rows == 0:
            return out
        if plan._pool is not self:
            raise ValueError("a plan of another pool")
        plan._look_again()
        if not (plan._reads if k is None else plan._stores):
            raise B.CardError(B.CARD_ESTALE, "attend")
        rows = [None if t is None else B.card_rows(t) for t in (q, k, v, out)]
        stream = torch.cuda.current_stream(self.device)
        if stream != plan.stream:  # the plan may be dropped before that stream has got to the call
            for t in (plan.ctx_lens, plan.row_starts, plan.tables, plan.workspace):
                t.record_stream(stream)
        with torch.cuda.device_of(self.k_pages):
            _check(B.card_kv_attend(cfg, plan.batch, layer, *rows, row_mask, plan.workspace, self._stream()), "card_kv_attend")
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
        src = [s.pages[i] for i in places]
        dst = [self._take() for _ in places]
        kv = B.CardKV(self.k_pages.data_ptr(), self.v_pages.data_ptr(), None, self.n_pages, -1)
        with torch.cuda.device_of(self.k_pages):
            _check(B.card_kv_copy_pages(self.cfg, kv, src, dst, self._stream()), "card_kv_copy_pages")
        for i, d in zip(places, dst):
            self._release(s.pages[i])
            s.pages[i] = d
        self._upload(s)

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
