"""KV blocks of one instance, kept in a page pool: what a decision places, moves and gives up.

``BlockPool`` holds the 8-bit blocks of a batch of sequences (one slot each) and runs the
calls of ``netkv.h`` on them: new tokens in (``append``), blocks back as rows (``read``), one
decode step's attention (``attend``), a chunk of new tokens a slot, turned by their positions,
stored and attended (``extend``, ``attend_chunk``), and the eviction of the blocks that have drawn
the least attention (``evict``).  ``move`` carries a sequence from one pool to another, as the transfer that
``netkv_schedule_streams`` prices does between instances.

Pages are handed out on the host; device work is enqueued on torch's current stream.  Calls that
change a pool come one after another; ``read`` and ``attend_chunk`` do not, and may overlap.  Only
``evict`` waits for the device: it reads which pages became free.
"""
from __future__ import annotations

import ctypes
import math
from typing import List, Optional, Sequence

import torch

from . import netkv

BLOCK = netkv.NETKV_BLOCK_TOKENS
LOG2_E = 1.0 / math.log(2.0)
FORMATS = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def bytes_per_token(layers: int, kv_heads: int, dim: int) -> int:
    """Bytes that a token of an 8-bit cache takes on the wire (Eq. 1 with a byte an element, and
    4 bytes a block and head for each scale), rounded up: for ``netkv_weights``."""
    per_block = 2 * layers * kv_heads * (dim * BLOCK + 4)
    return -(-per_block // BLOCK)


def blocks_of(tokens: int) -> int:
    return -(-tokens // BLOCK)


class BlockPool:
    def __init__(self, n_pages: int, kv_heads: int, dim: int, slots: int, width: int,
                 fmt: str = "int8", device="cuda"):
        """slots sequences of up to width blocks over n_pages pages."""
        shape = (n_pages, kv_heads, BLOCK, dim)
        self.pages = netkv.KvPages(torch.zeros(shape, dtype=FORMATS[fmt], device=device),
                                   torch.zeros(shape, dtype=FORMATS[fmt], device=device),
                                   torch.zeros(shape[:2], device=device),
                                   torch.zeros(shape[:2], device=device))
        self.table = torch.full((slots, width), -1, dtype=torch.int32, device=device)
        self.mass = torch.zeros((slots, width), device=device)
        self.length = torch.zeros(slots, dtype=torch.int32, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.tokens: List[int] = [0] * slots          # length, on the host
        self.seen: List[int] = [0] * slots            # tokens ever, evicted ones too: the next position
        self.page_of: List[List[int]] = [[] for _ in range(slots)]
        self.free = list(range(n_pages - 1, -1, -1))
        self._spare = (torch.empty_like(self.table), torch.empty_like(self.length),
                       torch.empty_like(self.mass), torch.empty_like(self.table),
                       torch.empty_like(self.length))

    @property
    def slots(self) -> int:
        return len(self.tokens)

    def _dev(self, x, dtype=torch.int32):
        """A list on the device, sent from pinned memory: a copy from elsewhere waits for the stream."""
        cuda = self.table.device.type == "cuda"
        t = torch.tensor(list(x), dtype=dtype, pin_memory=cuda)
        return t.to(self.table.device, non_blocking=True)

    def _offsets(self, counts: Sequence[int]):
        off = [0]
        for c in counts:
            off.append(off[-1] + c)
        return self._dev(off, torch.int64)

    def _counts(self, counts: Sequence[int], *rows: torch.Tensor) -> List[int]:
        """counts as integers: one a slot, none below 0, not more in all than any of the rows."""
        out = [int(c) for c in counts]
        if len(out) != self.slots or any(c < 0 or c != d for c, d in zip(out, counts)):
            raise ValueError(f"{self.slots} counts of 0 or more expected, got {list(counts)}")
        if any(sum(out) > len(x) for x in rows):
            raise ValueError(f"{sum(out)} rows expected, got {[len(x) for x in rows]}")
        return out

    def reserve(self, counts: Sequence[int]) -> None:
        """Pages for counts[i] more tokens of each slot; nothing changes where they do not fit."""
        self._take(self._counts(counts))

    def _take(self, counts: List[int]) -> List[int]:
        """reserve(); how many pages each slot was given."""
        need = [max(0, blocks_of(t + c) - len(p))
                for t, c, p in zip(self.tokens, counts, self.page_of)]
        if sum(need) > len(self.free):
            raise MemoryError(f"{sum(need)} pages needed, {len(self.free)} free")
        if any(blocks_of(t + c) > self.table.shape[1] for t, c in zip(self.tokens, counts)):
            raise ValueError(f"a slot holds at most {self.table.shape[1]} blocks")
        at, pages = [], []
        for s, n in enumerate(need):
            for _ in range(n):
                page = self.free.pop()
                at.append(s * self.table.shape[1] + len(self.page_of[s]))
                pages.append(page)
                self.page_of[s].append(page)
        self._enter(at, pages)
        return need

    def _enter(self, at: List[int], pages: List[int]) -> None:
        """Pages into the table's entries, which have drawn nothing yet."""
        if at:
            at = self._dev(at, torch.int64)
            self.table.view(-1)[at] = self._dev(pages)
            self.mass.view(-1).index_fill_(0, at, 0.0)

    def _give_back(self, taken: List[int]) -> None:
        for pages, n in zip(reversed(self.page_of), reversed(taken)):
            for _ in range(n):
                self.free.append(pages.pop())

    def append(self, k: torch.Tensor, v: torch.Tensor, counts: Sequence[int]) -> None:
        """Rows k, v [sum(counts), kv_heads, dim]: counts[i] new tokens of slot i each.  Nothing
        changes where a call is refused."""
        counts = self._counts(counts, k, v)
        taken = self._take(counts)
        try:
            netkv.netkv_kv_store(self.pages, k, v, self._offsets(counts), self.length, self.table,
                                 status=self.status)
        except Exception:
            self._give_back(taken)
            raise
        self._grow(counts)

    def _grow(self, counts: List[int]) -> None:
        more = self._dev(counts)
        self.tokens = [t + c for t, c in zip(self.tokens, counts)]
        self.seen = [t + c for t, c in zip(self.seen, counts)]
        self.length += more

    def read(self, k: torch.Tensor, v: torch.Tensor, counts: Sequence[int]) -> None:
        """The first counts[i] tokens of each slot into the rows k, v."""
        counts = self._counts(counts, k, v)
        if any(c > t for c, t in zip(counts, self.tokens)):
            raise ValueError("more tokens asked for than a slot holds")
        netkv.netkv_kv_load(self.pages, k, v, self._offsets(counts), None, self.table,
                            status=self.status)

    def attend(self, q: torch.Tensor, scale=None):
        """One query row a slot, [slots, heads, dim]: (out, lse); the blocks' weights add up in
        ``mass``."""
        need = netkv.netkv_attn_decode_workspace_size(self.pages, self.slots, q.shape[1],
                                                      self.table.shape[1], True)
        # of the call's own: the last one's may still be in use on another stream
        workspace = torch.empty(need, dtype=torch.uint8, device=self.table.device)
        out = torch.empty_like(q)
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        netkv.netkv_attn_decode(self.pages, q, self.length, self.table, out, lse=lse,
                                mass_in=self.mass, mass_out=self.mass, scale=scale,
                                workspace=workspace, status=self.status)
        return out, lse

    def _chunk_bytes(self, q: torch.Tensor, scale) -> int:
        """Workspace of the queries' attention; a ValueError where that would be refused."""
        # as the call gets it: what is above 0 as a Python number may be 0 in 32 bits
        if scale is not None and not 0.0 < ctypes.c_float(scale).value * LOG2_E <= 3.4028235e38:
            raise ValueError(f"a scale above 0, and finite times log2(e), expected, got {scale}")
        need = netkv.netkv_attn_chunk_workspace_size(self.pages, q.shape[0], self.slots, q.shape[1])
        if need == 0:
            raise ValueError(f"query heads in groups of {self.pages.heads_dim[0]} expected, got {q.shape[1]}")
        return need

    def _chunk_outputs(self, q: torch.Tensor, rows: int, scale):
        """Output, lse and workspace of the attention of q's first rows, all that it may want of the
        allocator: a workspace of the call's own, as calls on other streams may overlap with it."""
        workspace = torch.empty(self._chunk_bytes(q, scale), dtype=torch.uint8, device=self.table.device)
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        if rows < len(q):  # the call leaves a padded batch's other rows as they are
            out[rows:].zero_()
            lse[rows:].fill_(-math.inf)
        return out, lse, workspace

    def _attend_chunk(self, q: torch.Tensor, off: torch.Tensor, scale, out, lse, workspace):
        netkv.netkv_attn_chunk(self.pages, q, off, self.length, self.table, out, lse=lse, scale=scale,
                               workspace=workspace, status=self.status)
        return out, lse

    def attend_chunk(self, q: torch.Tensor, counts: Sequence[int], scale=None):
        """Rows q [sum(counts), heads, dim] are the queries of the last counts[i] tokens of each slot i:
        (out, lse), each row over its own token and those before it.  Rows of q behind these, as of a padded
        batch, give 0 and -inf.  The blocks' ``mass`` stays."""
        counts = self._counts(counts, q)
        return self._attend_chunk(q, self._offsets(counts), scale,
                                  *self._chunk_outputs(q, sum(counts), scale))

    def extend(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, counts: Sequence[int],
               rotary: "netkv.Rotary", positions: Optional[torch.Tensor] = None, scale=None):
        """counts[i] new tokens of each slot i, as a layer has them: queries and keys turned by their
        positions, keys and values into blocks, and attention over the blocks: (out, lse), with 0 and -inf
        in rows behind these.

        positions [axes, rows] int32; by default a token's number in its slot, counting tokens that
        have been evicted.  The blocks' ``mass`` stays: where only extend() runs, evict() takes the oldest
        blocks between the first and the last ones.  Nothing changes where the call is refused."""
        counts = self._counts(counts, q, k, v)
        outputs = self._chunk_outputs(q, sum(counts), scale)
        if positions is None and rotary.axes > 1:
            raise ValueError("positions of every axis expected")
        if positions is None and any(c and s != t for c, s, t in zip(counts, self.seen, self.tokens)):
            at = [s + i for s, c in zip(self.seen, counts) for i in range(c)]
            positions = self._dev(at + [0] * (k.shape[0] - len(at)))
        off, turned, taken, grown = self._offsets(counts), torch.empty_like(q), self._take(counts), False
        try:
            netkv.netkv_kv_append(self.pages, k, v, off, self.length, self.table, rotary, pos=positions, q=q,
                                  q_out=turned, status=self.status)
            self._grow(counts)
            grown = True
            return self._attend_chunk(turned, off, scale, *outputs)
        except Exception:
            if grown:
                self._grow([-c for c in counts])
            self._give_back(taken)
            raise

    def evict(self, budget: Sequence[int], sink: int = 4, recent: int = 4) -> List[List[int]]:
        """Cuts slot i to max(budget[i], sink + recent) blocks; the pages that became free."""
        table, length, mass, freed, n_freed = self._spare
        netkv.netkv_kv_evict(self.table, self.length, self.mass, self._dev(budget), sink, recent,
                             table, length, mass, freed, n_freed, status=self.status)
        self._spare = (self.table, self.length, self.mass, freed, n_freed)
        self.table, self.length, self.mass = table, length, mass
        gone = [row[:n] for row, n in zip(freed.tolist(), n_freed.tolist())]
        at, ahead = [], []  # pages for tokens to come, which the call does not know of
        for s, pages in enumerate(gone):
            out = set(pages)
            self.page_of[s] = [p for p in self.page_of[s] if p not in out]
            self.tokens[s] -= BLOCK * len(pages)
            self.free.extend(pages)
            used = blocks_of(self.tokens[s])
            at.extend(s * self.table.shape[1] + i for i in range(used, len(self.page_of[s])))
            ahead.extend(self.page_of[s][used:])
        self._enter(at, ahead)
        return gone

    def release(self, slot: int) -> None:
        """Gives all of a slot's pages back."""
        self.free.extend(self.page_of[slot])
        self.page_of[slot] = []
        self.tokens[slot] = self.seen[slot] = 0
        self.table[slot].fill_(-1)
        self.length[slot].fill_(0)


def move(src: BlockPool, slot: int, dst: BlockPool, to: int) -> int:
    """Slot `slot` of src into the empty slot `to` of dst, block by block, with the weight that each
    block has drawn; the bytes of blocks moved.  The slot of src stays as it is until release()."""
    if dst.tokens[to]:
        raise ValueError(f"slot {to} is in use")
    # codes are copied as they are, page by page
    kind = lambda pool: (tuple(pool.pages.tensors[0].shape[1:]), pool.pages.tensors[0].dtype)  # noqa: E731
    if kind(src) != kind(dst):
        raise ValueError(f"pools of one shape and format expected, got {kind(src)} and {kind(dst)}")
    n = src.tokens[slot]
    counts = [0] * dst.slots
    counts[to] = n
    taken = dst._take(counts)
    # either slot may hold pages beyond its tokens
    blocks = blocks_of(n)
    here, there = src.page_of[slot][:blocks], dst.page_of[to][:blocks]
    one = src.pages.tensors[0][0].numel()
    try:
        netkv.netkv_copy_group_async([(dst.pages.tensors[i][b], src.pages.tensors[i][a], one)
                                      for a, b in zip(here, there) for i in (0, 1)])
    except Exception:
        dst._give_back(taken)
        raise
    # scales are kv_heads floats a page, less than a copy's 16 bytes for some shapes
    a, b = src._dev(here, torch.int64), dst._dev(there, torch.int64)
    for i in (2, 3):
        dst.pages.tensors[i][b] = src.pages.tensors[i][a]
    dst.mass[to, :blocks] = src.mass[slot, :blocks]
    dst.tokens[to] = n
    dst.seen[to] = src.seen[slot]
    dst.length[to].fill_(n)
    return 2 * blocks * (one + src.pages.tensors[2][0].numel() * 4)
