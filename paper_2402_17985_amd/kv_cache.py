"""Buffer bookkeeping for the paged 8-bit key / value cache of one attention layer: owns the pages, their scales and the page table, hands out
pages, and forwards to the fq_* calls.  No arithmetic."""
from . import binding as B


class FqKvCache:
    """`pages` pages of `page_size` tokens, shared by up to `batch` sequences of at most `max_len` tokens each.

    Calls go to the current stream.  attend() may run on several streams at once; reserve(), release(), append(), fork() and compact() change the table and the
    pages, and the caller orders them with what else uses the cache.  append() and attend() copy their counts from the host, which waits for the stream (so do
    fork() and compact() with page numbers): inside a captured graph use the fq_* calls with counts on the device.  A sequence's last tokens (rejected drafts) are dropped by setting lengths[b] to what stays: the next
    ones take their places; its pages stay with it.

    Sequences that fork() made from one another share pages.  An append copies what it would change of them first, so that each sequence keeps its own
    past; appending takes pages for that.  (The fq_* calls know nothing of shared pages: give a sequence its own, by an append here, before they write.)"""

    def __init__(self, pages: int, batch: int, max_len: int, heads_kv: int, head_dim: int, page_size: int = 64, rope_cos=None, rope_sin=None,
                 interleaved: bool = False, device="cuda:0"):
        """rope_cos, rope_sin: fp32 device tensors [positions, rope_dim / 2] with at least max_len rows, or None: no rotation."""
        import torch
        self.torch = torch
        self.device, self.page_size, self.max_len, self.batch = device, page_size, max_len, batch
        self.rope_cos, self.rope_sin, self.interleaved = rope_cos, rope_sin, interleaved
        if rope_cos is not None and rope_cos.shape[0] < max_len:
            raise ValueError(f"{rope_cos.shape[0]} positions of rope_cos for sequences of up to {max_len} tokens")
        new = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=device)  # noqa: E731
        self.k_cache, self.v_cache = new((pages, heads_kv, page_size, head_dim), torch.int8), new((pages, heads_kv, head_dim, page_size), torch.int8)
        self.k_scale, self.v_scale = new((pages, heads_kv), torch.float32), new((pages, heads_kv), torch.float32)
        self.page_table = torch.full((batch, -(-max_len // page_size)), -1, dtype=torch.int32, device=device)
        self.held = [[] for _ in range(batch)]      # page numbers of each sequence
        self.lengths = [0] * batch
        self._free = list(range(pages - 1, -1, -1))
        self._users = [0] * pages                   # sequences that hold a page
        self._shared = 0                            # pages that several hold

    def _i32(self, values):
        return self.torch.tensor(values, dtype=self.torch.int32, device=self.device)

    @staticmethod
    def _offsets(counts):
        at = [0]
        for n in counts:
            at.append(at[-1] + n)
        return at

    def _check_counts(self, name, counts, rows_of, rows):
        if min(counts, default=0) < 0:
            raise ValueError(f"{name} has a negative count")
        if len(counts) != self.batch or sum(counts) != rows:
            raise ValueError(f"{name} must say for each sequence how many of {rows_of}'s rows are its own")

    def reserve(self, b: int, tokens: int) -> None:
        """Pages for the first `tokens` tokens of sequence b; raises if it may not grow so long, or no page is free (nothing changes then)."""
        if tokens > self.max_len:
            raise ValueError(f"sequence {b} would hold {tokens} tokens, more than {self.max_len}")
        have, need = len(self.held[b]), -(-tokens // self.page_size)
        if need - have > len(self._free):
            raise RuntimeError(f"{need - have} pages wanted, {len(self._free)} free")
        if need > have:
            self.held[b] += [self._take() for _ in range(need - have)]
            self.page_table[b, have:need] = self._i32(self.held[b][have:])

    def _take(self) -> int:
        page = self._free.pop()
        self._users[page] = 1
        return page

    def _drop(self, page: int) -> None:
        self._users[page] -= 1
        if self._users[page] == 0:
            self._free.append(page)
        elif self._users[page] == 1:
            self._shared -= 1

    def release(self, b: int) -> None:
        """Sequence b ends: pages that no other sequence shares are free again."""
        for page in reversed(self.held[b]):
            self._drop(page)
        self.held[b], self.lengths[b] = [], 0
        self.page_table[b].fill_(-1)

    def fork(self, b: int, into) -> None:
        """The sequences `into` (which must hold nothing) continue sequence b's tokens: they share its pages, and nothing is copied until one of them grows."""
        into = list(into)
        if len(set(into)) < len(into) or any(not 0 <= c < self.batch for c in [b] + into):
            raise ValueError(f"fork of sequence {b} into {into} of {self.batch}")
        if any(self.held[c] for c in into):
            raise ValueError(f"sequences {[c for c in into if self.held[c]]} hold pages: release them first")
        used = -(-self.lengths[b] // self.page_size)          # pages reserved ahead stay b's own
        pages = self.held[b][:used]
        for c in into:
            for page in pages:
                self._users[page] += 1
                self._shared += self._users[page] == 2
            self.held[c], self.lengths[c] = list(pages), self.lengths[b]
        if pages and into:
            self.page_table[self._i64(into), :used] = self._i32(pages)

    def _i64(self, values):
        return self.torch.tensor(values, dtype=self.torch.int64, device=self.device)

    def _copy(self, src, dst) -> None:
        if src:
            B.fq_kv_copy_pages(self.k_cache, self.v_cache, self.k_scale, self.v_scale, self._i32(src), self._i32(dst))

    def _writes(self, b: int, grown: int):
        """Places in held[b] of the shared pages that appending up to `grown` tokens writes to: whose past must stay with the others."""
        first, end = self.lengths[b] // self.page_size, -(-grown // self.page_size)
        return [i for i in range(first, min(end, len(self.held[b]))) if self._users[self.held[b][i]] > 1]

    def _replaced(self, grown):
        """(sequence, place in held[b]) of the shared pages for which an append up to `grown` tokens needs pages of the sequence's own: one for each
        writer, but for the last of a page that all its holders write, which keeps it."""
        left, places = {}, []               # left: holders of a page that would still share it
        for b, n in enumerate(grown):
            for i in self._writes(b, n) if n > self.lengths[b] else ():
                page = self.held[b][i]
                left[page] = left.get(page, self._users[page]) - 1
                if left[page]:
                    places.append((b, i))
        return places

    def compact(self) -> int:
        """Moves pages so that those in use are the first ones of the pool, and returns their number.  Sequences keep what they hold."""
        live = sum(1 for n in self._users if n)
        moved = [page for page in range(live, len(self._users)) if self._users[page]]
        room = [page for page in range(live) if not self._users[page]]
        to = dict(zip(moved, room))
        self._copy(moved, room)
        for old, new in to.items():
            self._users[new], self._users[old] = self._users[old], 0
        for b, held in enumerate(self.held):
            if any(page in to for page in held):
                self.held[b] = [to.get(page, page) for page in held]
                self.page_table[b, :len(held)] = self._i32(self.held[b])
        self._free = list(range(len(self._users) - 1, live - 1, -1))
        return live

    def append(self, Q, K, V, new, Q_out=None, K_out=None) -> None:
        """Append new[b] tokens to every sequence b (0: none): the rows of K, V (and Q) in order.  See fq_kv_append."""
        self._check_counts("new", new, "K", K.shape[0])
        grown = [n + m for n, m in zip(self.lengths, new)]
        replaced = self._replaced(grown) if self._shared else []
        places = replaced + [(b, i) for b, (n, h) in enumerate(zip(grown, self.held)) for i in range(len(h), -(-n // self.page_size))]
        wanted, free = len(places), len(self._free)
        if wanted > free or max(grown) > self.max_len:
            raise RuntimeError(f"{wanted} pages wanted, {free} free; longest sequence {max(grown)} of {self.max_len}")
        fresh = self._free[free - wanted:][::-1]
        # Copies go before any change of what the sequences hold: where one is refused, no past is lost.  (A page that a sequence starts anew has nothing to copy.)
        copies = [(self.held[b][i], page) for (b, i), page in zip(replaced, fresh) if self.lengths[b] > i * self.page_size]
        self._copy([old for old, _ in copies], [page for _, page in copies])
        del self._free[free - wanted:]
        for (b, i), page in zip(places, fresh):
            self._users[page] = 1
            if i < len(self.held[b]):
                self._drop(self.held[b][i])
            self.held[b][i:i + 1] = [page]
        if places:                              # one write to the device for all sequences
            at, pages = self._i32([[b * self.page_table.shape[1] + i for b, i in places], fresh])
            self.page_table.view(-1)[at] = pages
        B.fq_kv_append(Q, K, V, self._i32(self._offsets(new)), self._i32(self.lengths), max(1, max(new)), self.k_cache, self.v_cache, self.k_scale,
                       self.v_scale, self.page_table, rope_cos=self.rope_cos, rope_sin=self.rope_sin, interleaved=self.interleaved,
                       Q_out=Q_out, K_out=K_out)
        self.lengths = grown

    def attend(self, Q, queries, scale: float, Y=None):
        """Attention of the last queries[b] tokens of every sequence over all that the cache holds of it.  See fq_attn_cache."""
        self._check_counts("queries", queries, "Q", Q.shape[0])
        if Y is None:
            Y = self.torch.empty(Q.shape, dtype=Q.dtype, device=Q.device)
        max_q, max_len = max(1, max(queries)), max(1, max(self.lengths))
        size = B.fq_attn_cache_workspace_bytes(self.batch, Q.shape[0], max_q, max_len, Q.shape[1], self.k_cache.shape[1], Q.shape[2])
        # of this call: torch's allocator gives it to no other stream before the kernels are through
        workspace = self.torch.empty(size, dtype=self.torch.uint8, device=self.device)
        B.fq_attn_cache(Q, self._i32(self._offsets(queries)), self._i32(self.lengths), max_q, max_len, self.k_cache, self.v_cache, self.k_scale,
                        self.v_scale, self.page_table, scale, Y, workspace)
        return Y
