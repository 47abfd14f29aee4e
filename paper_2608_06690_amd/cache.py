"""PagedCache: the attention state of a batch of requests, in pages that belong to a policy decision (App. B.2:
caches are tagged with the policy decision, the model revision and the checkpoint fingerprint, and reuse across
tags is refused). It keeps the books of the pages on the host and passes pointers; all computation happens in
libpmpe (pmpe_kv_write, pmpe_kv_read, pmpe_attn_decode)."""
from __future__ import annotations

from typing import Any, List, Optional, Sequence

import torch

from . import _native as N
from .policy import policy_word, request_offsets

_FREE = -1  # the tag of a page that belongs to no decision: refused to every request
_NONE = -1  # the page of a column that a request does not have: out of the pool, so refused


def _as_int32(word: int) -> int:
    return word - (1 << 32) if word >= 1 << 31 else word


class PagedCache:
    """Keys and values of up to `requests` requests of one layer, in `n_pages` pages of `page_size` rows, of which a
    request has max_pages at most.

    `open` gives a request its decision, which its pages carry from then on; `write` adds rows to the requests of a
    batch (the new token of each in a decoding step, a prompt before it), `attend` is the attention of each request's
    newest token, `share` lets a request begin with another's first pages where their cache tags are equal. The
    kernels refuse a page of the other decision whatever the block table says: the bits of `dev_status`, which the
    caller reads when it likes, tell. The books are the host's, their device copies follow on the stream of each call (the
    current one without `stream`): an object's calls go to one stream, or the caller orders its streams."""

    def __init__(self, requests: int, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, max_pages: int,
                 model_revision: bytes, checkpoint_fingerprint: bytes, bf16: bool = True, fp8: bool = False, device="cuda"):
        self.desc = N.make_cache_desc(n_pages, page_size, n_kv_heads, head_dim, max_pages, bf16, fp8)
        self.revision, self.fingerprint = model_revision, checkpoint_fingerprint
        N.make_cache_tag(0, model_revision, checkpoint_fingerprint)  # (their lengths)
        dt = torch.uint8 if fp8 else torch.bfloat16 if bf16 else torch.float32
        i32 = dict(dtype=torch.int32, device=device)
        shape, sshape = (n_pages, n_kv_heads, page_size, head_dim), (n_pages, n_kv_heads, head_dim // 32, page_size)
        self.k, self.v = (torch.zeros(shape, dtype=dt, device=device) for _ in range(2))
        self.k_scale, self.v_scale = ((torch.zeros(sshape, dtype=torch.uint8, device=device) if fp8 else None) for _ in range(2))
        self.block_table = torch.full((requests, max_pages), _NONE, **i32)
        self.page_tag = torch.full((n_pages,), _FREE, **i32)
        self.words, self.seq_len = torch.zeros(requests, **i32), torch.zeros(requests, **i32)
        self.dev_status = torch.zeros(1, **i32)
        self.lengths: List[int] = [0] * requests       # rows of each request
        self.decision: List[Optional[int]] = [None] * requests  # 1 allow, 0 deny, None: not open
        self._pages: List[List[int]] = [[] for _ in range(requests)]
        self._users = [0] * n_pages
        self._free = list(range(n_pages - 1, -1, -1))
        self._ws = {}

    @property
    def requests(self) -> int:
        return len(self.lengths)

    def tag(self, r: int) -> N.CacheTag:
        """The cache tag of an open request."""
        if self.decision[r] is None:
            raise ValueError(f"request {r} is not open")
        return N.make_cache_tag(self.decision[r], self.revision, self.fingerprint)

    def open(self, r: int, meta: Any, stream=None) -> None:
        """Request r begins anew, with the decision that its trusted metadata resolve to (missing or malformed: deny)."""
        self.close(r, stream)
        word = policy_word(meta)
        with torch.cuda.stream(stream):
            self.decision[r] = int(word == N.PMPE_POLICY_ALLOW)
            self.words[r] = _as_int32(word)

    def close(self, r: int, stream=None) -> None:
        """Request r gives its pages back; those that no other request has belong to no decision then."""
        with torch.cuda.stream(stream):
            self._give_back(r, 0)
            self.lengths[r], self.decision[r] = 0, None
            self.words[r] = 0
            self.seq_len[r] = 0

    def _give_back(self, r: int, keep: int) -> None:
        """The pages of request r but the first `keep`. Their columns of the table name none from then on: a length that
        runs ahead of the pages (a captured step replayed too often) must not meet another request's rows."""
        free, had = [], len(self._pages[r])
        if had > keep:
            self.block_table[r, keep:had] = _NONE
        for p in self._pages[r][keep:]:
            self._users[p] -= 1
            if self._users[p] == 0:
                free.append(p)
        if free:
            self._free.extend(reversed(free))
            self.page_tag[torch.tensor(free, device=self.page_tag.device)] = _FREE
        del self._pages[r][keep:]

    def share(self, r: int, source: int, rows: int, tag: Optional[N.CacheTag] = None, stream=None) -> int:
        """Request r, open and empty, begins with the rows of the whole pages among the first `rows` of `source`. tag:
        the cache tag that these rows were made under (default: the source's). Returns the number of rows it has then;
        raises PmpeError where the tags differ."""
        if rows < 0:
            raise ValueError(f"{rows} rows cannot be shared")
        if self.lengths[r] or self._pages[r] or r == source:
            raise ValueError(f"request {r} must be empty, without pages, and another than its source")
        if not N.pmpe_cache_tag_check(self.tag(source) if tag is None else tag, self.tag(r)):
            raise N.PmpeError(N.PMPE_ERR_TAG_MISMATCH, "pmpe_cache_tag_check")
        if self.decision[source] != self.decision[r]:  # (whatever tag was given: the pages are the source's)
            raise N.PmpeError(N.PMPE_ERR_TAG_MISMATCH, "pmpe_cache_tag_check")
        n = min(rows, self.lengths[source]) // self.desc.page_size
        pages = self._pages[source][:n]
        for p in pages:
            self._users[p] += 1
        self._pages[r], self.lengths[r] = list(pages), n * self.desc.page_size
        with torch.cuda.stream(stream):
            if n:
                self.block_table[r, :n] = self.block_table[source, :n]
            self.seq_len[r] = self.lengths[r]
        return self.lengths[r]

    def _counts(self, counts: Sequence[int]) -> List[int]:
        counts = [int(n) for n in counts]
        if len(counts) != self.requests:
            raise ValueError(f"{self.requests} counts are needed, not {len(counts)}")
        return counts

    def reserve(self, counts: Sequence[int], stream=None) -> None:
        """Pages for counts[r] rows of each request behind those that it has, or none at all (ValueError): a captured
        write takes none itself, so its replays go as far as pages are reserved and are refused behind that."""
        counts = self._counts(counts)
        with torch.cuda.stream(stream):
            self._reserve(counts)

    def advance(self, stream=None) -> List[int]:
        """Brings the host's lengths to the device's, which alone has counted the rows of replayed writes: after replays,
        and before the next call that goes by the requests' lengths (write, read, share, reserve). Rows that were refused
        because no page was there are in neither then. Waits for the stream; returns the rows that each request gained."""
        with torch.cuda.stream(stream):
            torch.minimum(self.seq_len, torch.tensor(self._most(), dtype=torch.int32).to(self.seq_len.device), out=self.seq_len)
            have = self.seq_len.tolist()
        gained = [a - b for a, b in zip(have, self.lengths)]
        self.lengths = have
        return gained

    def _most(self) -> List[int]:
        """Rows that the pages of each request hold."""
        return [len(p) * self.desc.page_size for p in self._pages]

    def _reserve(self, counts: Sequence[int]) -> List[int]:
        """Pages for counts[r] more rows of each request, or none at all. Returns the request of each page taken."""
        size, need = self.desc.page_size, []
        for r, n in enumerate(counts):
            if n < 0 or (n > 0 and self.decision[r] is None):
                raise ValueError(f"request {r} is not open")
            total = -(-(self.lengths[r] + n) // size)
            if total > self.desc.max_pages:
                raise ValueError(f"request {r} would have {total} pages, more than {self.desc.max_pages}")
            need += [r] * (total - len(self._pages[r]))
        if len(need) > len(self._free):
            raise ValueError(f"{len(need)} pages are needed, {len(self._free)} are free")
        if not need:
            return need
        if self.k.is_cuda and torch.cuda.is_current_stream_capturing():
            raise ValueError("a captured write cannot take pages: they have to be reserved before")
        rows, cols, pages, tags, n = [], [], [], [], [len(p) for p in self._pages]
        for r, p in zip(need, reversed(self._free)):
            rows.append(r)
            cols.append(n[r])
            pages.append(p)
            tags.append(_as_int32(N.PMPE_POLICY_ALLOW if self.decision[r] else N.PMPE_POLICY_DENY))
            n[r] += 1
        n, i = len(need), torch.tensor(rows + cols + pages + tags + self._most(), dtype=torch.int64).to(self.page_tag.device)
        # (a length that replays have taken past the pages of now counts rows that were refused: the new pages, and what
        # they held before, must not stand in for them)
        torch.minimum(self.seq_len, i[4 * n:].int(), out=self.seq_len)
        self.block_table[i[:n], i[n:2 * n]] = i[2 * n:3 * n].int()
        self.page_tag[i[2 * n:3 * n]] = i[3 * n:4 * n].int()
        for r, p in zip(rows, pages):  # (the books last: where the device's part fails, they are as they were)
            self._pages[r].append(self._free.pop())
            self._users[p] = 1
        return need

    def write(self, k: torch.Tensor, v: torch.Tensor, counts: Sequence[int], req_offset: Optional[torch.Tensor] = None,
              stream=None) -> None:
        """The rows k and v [sum(counts), n_kv_heads, head_dim] (slices of a projection will do) behind those that the
        requests have: counts[r] of request r, in order. req_offset: request_offsets(counts) on the device, if the
        caller has it (a captured write needs it). With a stream, the books' small copies are made on it, too. Nothing is
        written while a graph captures the call, so the host's lengths stay: `reserve` before, `advance` after replays."""
        counts = self._counts(counts)
        if sum(counts) != k.shape[0]:
            raise ValueError(f"the counts must have a sum of {k.shape[0]}")
        act = torch.bfloat16 if self.desc.act_dtype == N.PMPE_BF16 else torch.float32
        for t in (k, v):  # (before the books change)
            if t.shape != (k.shape[0], self.desc.n_kv_heads, self.desc.head_dim) or t.dtype != act or t.device != self.k.device:
                raise ValueError(f"k and v must be {[k.shape[0], self.desc.n_kv_heads, self.desc.head_dim]} of {act} on {self.k.device}")
        with torch.cuda.stream(stream):
            if req_offset is None:
                req_offset = request_offsets(counts, self.seq_len.device)
            elif req_offset.shape != (self.requests + 1,) or req_offset.dtype != torch.int32 or req_offset.device != self.k.device:
                raise ValueError(f"req_offset must be [{self.requests + 1}] of torch.int32 on {self.k.device}")
            taken = self._reserve(counts)
            more = counts[0] if all(n == counts[0] for n in counts) else req_offset[1:] - req_offset[:-1]
            self.seq_len.add_(more)
            try:
                N.pmpe_kv_write(self.desc, k, v, req_offset, self.seq_len, self.block_table, self.page_tag, self.words, self.k,
                                self.v, self.k_scale, self.v_scale, self.dev_status)
            except Exception:  # nothing was written: a length ahead of the rows would show what the pages held before
                self.seq_len.sub_(more)
                for r in set(taken):  # (no others: pages reserved ahead may hold rows of replays)
                    self._give_back(r, len(self._pages[r]) - taken.count(r))
                raise
            if not (self.k.is_cuda and torch.cuda.is_current_stream_capturing()):
                self.lengths = [a + b for a, b in zip(self.lengths, counts)]
            if stream is not None:
                req_offset.record_stream(stream)

    def attend(self, q: torch.Tensor, scale: float, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
               first: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Attention of each request's newest row: q [requests, n_heads, head_dim]; first [requests] int32: positions
        before it are out of the window. A request without rows has zeros. The workspace is the object's: its calls,
        and graphs that hold one, follow one another."""
        heads = q.shape[1]
        with torch.cuda.stream(stream):  # (new memory belongs to the stream that writes it)
            if out is None:
                out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            if heads not in self._ws:  # (kept: a captured step may hold it)
                self._ws[heads] = torch.empty(max(16, N.pmpe_attn_decode_workspace_bytes(self.desc, self.requests, heads)),
                                              dtype=torch.uint8, device=q.device)
        N.pmpe_attn_decode(self.desc, q, first, self.seq_len, self.block_table, self.page_tag, self.words, self.k, self.v,
                           self.k_scale, self.v_scale, scale, out, lse, self.dev_status, self._ws[heads], stream)
        return out

    def read(self, counts: Sequence[int], first: Optional[Sequence[int]] = None, stream=None):
        """Rows first[r] .. first[r] + counts[r] - 1 of each request back in the activation type: (k, v)."""
        first = [0] * self.requests if first is None else [int(f) for f in first]
        for r, n in enumerate(counts):
            if n < 0 or (n > 0 and not 0 <= first[r] <= self.lengths[r] - n):
                raise ValueError(f"request {r} has {self.lengths[r]} rows")
        dev = self.k.device
        dt = torch.bfloat16 if self.desc.act_dtype == N.PMPE_BF16 else torch.float32
        with torch.cuda.stream(stream):
            k, v = (torch.empty(sum(counts), self.desc.n_kv_heads, self.desc.head_dim, dtype=dt, device=dev) for _ in range(2))
            N.pmpe_kv_read(self.desc, k, v, request_offsets(counts, dev), torch.tensor(first, dtype=torch.int32).to(dev),
                           self.block_table, self.page_tag, self.words, self.k, self.v, self.k_scale, self.v_scale, self.dev_status)
        return k, v


class Sampler:
    """Draws a token per row of logits with parameters of each row (pmpe_sample); its buffers hold the last draw, so
    its calls, and graphs that hold one, follow one another.
    Parameters [rows]: temperature, top_p and min_p (more than 1 counts as 1) fp32, top_k int32, each may be None."""

    def __init__(self, rows: int, vocab: int, temperature=None, top_k=None, top_p=None, min_p=None, device="cuda"):
        self.temperature, self.top_k, self.top_p, self.min_p = temperature, top_k, top_p, min_p
        self.token, self.kept = (torch.empty(rows, dtype=torch.int32, device=device) for _ in range(2))
        self.prob = torch.empty(rows, dtype=torch.float32, device=device)
        self.ws = torch.empty(max(16, N.pmpe_sample_workspace_bytes(rows, vocab)), dtype=torch.uint8, device=device)

    def __call__(self, logits: torch.Tensor, u: torch.Tensor, stream=None) -> torch.Tensor:
        """Tokens [rows] int32 of logits [rows, vocab], by the uniform numbers u [rows]."""
        N.pmpe_sample(logits, self.temperature, self.top_k, self.top_p, self.min_p, u, self.token, self.prob, self.kept, self.ws,
                      stream)
        return self.token
