"""Buffer bookkeeping for the paged 8-bit key / value cache of one attention layer: owns the pages, their scales and the page table, hands out
pages, and forwards to the fq_* calls.  No arithmetic."""
from . import binding as B


class FqKvCache:
    """`pages` pages of `page_size` tokens, shared by up to `batch` sequences of at most `max_len` tokens each.

    Calls go to the current stream.  attend() may run on several streams at once; reserve(), release() and append() change the table and the pages, and the
    caller orders them with what else uses the cache.  append() and attend() copy their counts from the host, which waits for the stream: inside a captured
    graph use the fq_* calls with counts on the device.  A sequence's last tokens (rejected drafts) are dropped by setting lengths[b] to what stays: the next
    ones take their places; its pages stay with it."""

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
            self.held[b] += [self._free.pop() for _ in range(need - have)]
            self.page_table[b, have:need] = self._i32(self.held[b][have:])

    def release(self, b: int) -> None:
        """Sequence b ends: its pages are free again."""
        self._free += reversed(self.held[b])
        self.held[b], self.lengths[b] = [], 0
        self.page_table[b].fill_(-1)

    def append(self, Q, K, V, new, Q_out=None, K_out=None) -> None:
        """Append new[b] tokens to every sequence b (0: none): the rows of K, V (and Q) in order.  See fq_kv_append."""
        self._check_counts("new", new, "K", K.shape[0])
        grown = [n + m for n, m in zip(self.lengths, new)]
        wanted = sum(max(0, -(-n // self.page_size) - len(h)) for n, h in zip(grown, self.held))
        if wanted > len(self._free) or max(grown) > self.max_len:
            raise RuntimeError(f"{wanted} pages wanted, {len(self._free)} free; longest sequence {max(grown)} of {self.max_len}")
        for b, n in enumerate(grown):
            self.reserve(b, n)
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
