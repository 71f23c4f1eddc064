"""Buffers and call order of the hot path for one layer (marshalling only; all compute is in the library).

prefill():  ec_prefill_score -> ec_select_anchors -> ec_merge_compact      (Sec. 3.3 Instruction Encoding)
decode():   ec_evict_index (host) -> ec_decode_step                        (Sec. 3.3 Output Generation)
extend():   ec_chunk_score -> ec_select_anchors -> ec_remerge_compact      (a later turn: chat history is
                                                                            compressed again with the new chunk)

PagedBatch holds the compressed caches of sequences that come and go in pages of one pool per layer:
admit() / store() -> begin() -> decode() or decode_scored() in every layer -> end(), shrink() when memory runs short, release()

PagedTokens does so for steps of any number of new tokens a sequence, with pages given out on the device and positions by rotation:
admit() -> begin() -> attend() in every layer, release()
"""
from __future__ import annotations

import math

import torch

from . import binding as ec


class LayerState:
    """Device buffers of one layer's compressed cache plus the bookkeeping integers of Alg. 1."""

    def __init__(self, B, H, D, T, n_anchor, cap, dtype: torch.dtype, gamma, G=1, recent=25,
                 protect_first=1, protect_last=1, device="cuda", keep_assign=False):
        self.B, self.H, self.D, self.T, self.G = B, H, D, T, G
        self.n_anchor, self.cap, self.gamma, self.recent = n_anchor, cap, gamma, recent
        self.protect_first, self.protect_last = protect_first, protect_last
        self.k_cache = torch.zeros((B, H, cap, D), dtype=dtype, device=device)
        self.v_cache = torch.zeros((B, H, cap, D), dtype=dtype, device=device)
        self.pos = torch.zeros((B, G, cap), dtype=torch.int32, device=device)
        self.score = torch.empty((B, G, T), dtype=torch.float32, device=device)
        self.anchor_idx = torch.empty((B, G, n_anchor), dtype=torch.int32, device=device)
        self.counts = torch.empty((B, G, n_anchor), dtype=torch.int32, device=device)
        self.assign = torch.empty((B, G, T), dtype=torch.int32, device=device) if keep_assign else None
        self.cache_len = 0
        self.n_seen = 0

    def prefill(self, q, k, v, scale, ws_prefill, out=None, lse=None):
        ec.ec_prefill_score(q, k, v, out, lse, self.score, scale, ws_prefill)
        ec.ec_select_anchors(self.score, self.n_anchor, self.protect_first, self.protect_last, self.anchor_idx)
        ec.ec_merge_compact(k, v, self.anchor_idx, self.k_cache, self.v_cache, self.counts, self.assign, self.pos)
        self.cache_len = self.n_anchor
        self.n_seen = self.T

    def decode(self, q, k_new, v_new, scale, out, ws_decode):
        self.n_seen += 1
        idx = ec.ec_evict_index(self.n_seen, self.cache_len + 1, self.gamma[0], self.gamma[1],
                                recent=self.recent, protect_first=self.protect_first)
        ec.ec_decode_step(q, k_new, v_new, self.k_cache, self.v_cache, self.pos, self.cache_len, idx,
                          self.n_seen - 1, scale, out, ws_decode)
        if idx < 0:
            self.cache_len += 1
        return idx

    def extend(self, q, k, v, scale, ws_chunk, out=None, lse=None):
        """A later multi-token pass: the chunk's K/V rows go behind the cache rows, the chunk's queries score
        every row of [cache | chunk], and the rows are merged again (Alg. 1's plain mean) into
        ceil(gamma * tokens seen) rows."""
        T_new = q.shape[2]
        P, L = self.cache_len, self.cache_len + T_new
        if L > self.cap:
            raise ValueError(f"cache capacity {self.cap} cannot hold {P} rows + a chunk of {T_new}")
        self.k_cache[:, :, P:L].copy_(k)
        self.v_cache[:, :, P:L].copy_(v)
        self.pos[:, :, P:L] = torch.arange(self.n_seen, self.n_seen + T_new, dtype=torch.int32, device=self.pos.device)
        self.n_seen += T_new
        n_new = -(-self.gamma[0] * self.n_seen // self.gamma[1])
        n_new = max(min(n_new, L), self.protect_first + self.protect_last)
        dev = self.k_cache.device
        self.score = torch.empty((self.B, self.G, L), dtype=torch.float32, device=dev)
        ec.ec_chunk_score(q, self.k_cache, self.v_cache, P, out, lse, self.score, scale, ws_chunk)
        self.anchor_idx = torch.empty((self.B, self.G, n_new), dtype=torch.int32, device=dev)
        ec.ec_select_anchors(self.score, n_new, self.protect_first, self.protect_last, self.anchor_idx)
        src_pos = self.pos[:, :, :L].clone()  # the merge writes self.pos while it reads the old map
        k_next, v_next = torch.zeros_like(self.k_cache), torch.zeros_like(self.v_cache)
        self.counts = torch.empty((self.B, self.G, n_new), dtype=torch.int32, device=dev)
        ec.ec_remerge_compact(self.k_cache, self.v_cache, L, self.anchor_idx, k_next, v_next, src_pos=src_pos,
                              counts=self.counts, pos=self.pos)
        self.k_cache, self.v_cache = k_next, v_next
        self.n_anchor = self.cache_len = n_new
        return n_new


class PagedBatch:
    """The caches of up to `places` sequences in pages, for all layers of a model: one pool of n_pages pages of `page` rows per layer and one page
    table that the layers share.  The host keeps the free pages and the length of every sequence; nothing is read back from the device.

        batch.admit([0, 1], [n_anchor, n_anchor], [T, T])        # two sequences get pages ...
        for i, state in enumerate(layers):
            batch.store(i, [0, 1], state.k_cache, state.v_cache, state.pos, mass)   # ... and their compressed prompts' rows
        for q, k, v in generated_tokens:
            batch.begin()                                        # room for a row
            for i in range(n_layers):
                batch.decode_scored(i, q[i], k[i], v[i], scale, out[i], keep)       # attention, masses, and the lightest row goes
            batch.end(keep)
        batch.shrink(keep // 2)                                  # all but the heaviest rows go, their pages are free
    """

    def __init__(self, layers, places, H, Hkv, D, page, n_pages, max_pages, dtype: torch.dtype, G=1, recent=25, protect_first=1, device="cuda"):
        self.H, self.Hkv, self.D, self.G, self.page, self.max_pages = H, Hkv, D, G, page, max_pages
        self.recent, self.protect_first = recent, protect_first
        self.k_pages, self.v_pages = (torch.zeros((layers, n_pages, Hkv, page, D), dtype=dtype, device=device) for _ in range(2))
        self.pos_pages = torch.zeros((layers, n_pages, G, page), dtype=torch.int32, device=device)
        self.mass_pages = torch.zeros((layers, n_pages, G, page), dtype=torch.float32, device=device)
        self.rows, self.seen = [-1] * places, [0] * places  # rows of every sequence, -1: no sequence; tokens seen
        self.held = [[] for _ in range(places)]
        self.free = list(range(n_pages - 1, -1, -1))
        self.table = torch.full((places, max_pages), -1, dtype=torch.int32, device=device)
        # rows before the step, behind it, tokens seen before it and behind it
        self.numbers = torch.zeros((4, places), dtype=torch.int32, device=device)
        self.len_b, self.len_after, self.pos_b, self.seen_b = self.numbers
        dt = ec.dtype_code(self.k_pages)
        self.ws = ec.new_workspace(ec.EC_FN_PAGED_DECODE_SCORE_STEP, places, H, max_pages * page, D, dt, device)
        self.ws_one = ec.new_workspace(ec.EC_FN_PAGED_EVICT_MIN, places, G, 1, D, dt, device)
        self.budgets = {}  # by budget, for the batch's lifetime: a graph may hold them
        self.changes = {}  # entries of the table that are not on the device yet, by their place in it
        self._upload()

    def _eager(self, what):
        """A replay would send the lengths and pages of the capture again, out of memory that holds something else by then."""
        if self.table.is_cuda and torch.cuda.is_current_stream_capturing():
            raise RuntimeError(f"PagedBatch.{what}() cannot be captured: it sends what the host knows now (a token's graph holds its decode calls)")

    def _send(self, x):
        """A host tensor on the device, without waiting (torch keeps pinned memory until the copy out of it has ended)."""
        return x.pin_memory().to(self.table.device, non_blocking=True) if self.table.is_cuda else x

    def _ints(self, x):
        return self._send(torch.tensor(x, dtype=torch.int32))

    def _upload(self):
        x = torch.tensor([self.rows, [n + 1 for n in self.rows], self.seen, [n + 1 for n in self.seen]], dtype=torch.int32)
        self.numbers.copy_(x.pin_memory() if self.table.is_cuda else x, non_blocking=True)

    def _budget(self, keep):
        """`keep` for every place: the layers of a token share the tensor, and so do graphs captured after a token with that budget. A graph captured
        before one has a tensor of its own in every layer, filled by its replays."""
        if keep not in self.budgets:
            made = torch.full_like(self.len_b, keep)
            if self.table.is_cuda and torch.cuda.is_current_stream_capturing():
                return made
            self.budgets[keep] = made
        return self.budgets[keep]

    def _room(self, rows):
        """Refuses, before anything is changed, what the free pages and a sequence's table do not hold: rows by place."""
        for b, n in rows.items():
            if -(-n // self.page) > self.max_pages:
                raise ValueError(f"sequence {b}: {-(-n // self.page)} pages for {n} rows, but a sequence has {self.max_pages} at most")
        more = {b: -(-n // self.page) - len(self.held[b]) for b, n in rows.items()}
        if sum(max(n, 0) for n in more.values()) > len(self.free):
            raise ValueError(f"{[n for n in more.values() if n > 0]} more pages for sequences {[b for b, n in more.items() if n > 0]}, but {len(self.free)} are free")

    def _hold(self, place, rows):
        """Exactly the pages that `rows` rows need, taken from the free ones or given back to them; _upload_table() sends what has changed."""
        held, need, first = self.held[place], -(-rows // self.page), place * self.max_pages
        while len(held) < need:
            held.append(self.free.pop())
            self.changes[first + len(held) - 1] = held[-1]
        while len(held) > need:
            self.free.append(held.pop())
            self.changes[first + len(held)] = -1

    def _upload_table(self):
        if not self.changes:
            return
        n = len(self.changes)  # their places (64 bits), then their contents, in one copy
        x = torch.empty(3 * n, dtype=torch.int32)
        x[:2 * n].view(torch.int64).copy_(torch.tensor(list(self.changes)))
        x[2 * n:] = torch.tensor(list(self.changes.values()), dtype=torch.int32)
        x = self._send(x)
        self.table.view(-1).index_copy_(0, x[:2 * n].view(torch.int64), x[2 * n:])
        self.changes = {}

    def _places(self, places):
        """Places of the batch, each named once."""
        places = list(places)
        if len(set(places)) != len(places) or any(not 0 <= b < len(self.rows) for b in places):
            raise ValueError(f"{places} are not different places of 0 .. {len(self.rows) - 1}")
        return places

    def admit(self, places, rows, seen):
        """Pages for sequences that start with `rows` rows of a prompt of `seen` tokens; store() brings the rows of every layer."""
        self._eager("admit")
        places = self._places(places)
        if not len(places) == len(rows) == len(seen) or any(n < 0 for n in rows):
            raise ValueError(f"places {places}, rows {list(rows)} and seen {list(seen)} do not belong together")
        for b in places:
            if self.rows[b] >= 0:
                raise ValueError(f"place {b} holds a sequence")
        self._room(dict(zip(places, rows)))
        for b, n, t in zip(places, rows, seen):
            self._hold(b, n)
            self.rows[b], self.seen[b] = n, t
        self._upload_table()
        self._upload()

    def release(self, place):
        self._eager("release")
        self._places([place])
        self._hold(place, 0)
        self.rows[place], self.seen[place] = -1, 0
        self._upload_table()
        self._upload()

    def store(self, layer, places, k, v, pos, mass):
        """Rows 0.. of k, v [len(places),Hkv,n,D], pos and mass [len(places),G,n] as the sequences' rows (their first rows[place] ones)."""
        self._eager("store")
        places = self._places(places)
        if any(self.rows[b] > k.shape[2] for b in places):
            raise ValueError(f"{k.shape[2]} rows for sequences of {[self.rows[b] for b in places]}")
        table = self.table.index_select(0, self._send(torch.tensor(places, dtype=torch.int64)))
        ec.ec_paged_store(k, v, pos, mass, table, self.k_pages[layer], self.v_pages[layer], self.pos_pages[layer], self.mass_pages[layer], None,
                          self._ints([self.rows[b] for b in places]))

    def begin(self):
        """Room for one more row of every sequence."""
        self._eager("begin")
        rows = {b: n + 1 for b, n in enumerate(self.rows) if n >= 0}
        self._room(rows)
        for b, n in rows.items():
            self._hold(b, n)
        self._upload_table()

    def decode(self, layer, q, k_new, v_new, scale, out):
        """One layer of a token: append and attend (places without a sequence get zeros).  Masses are left alone, so that new rows have none of
        their own: before shrink() they are stored, or the tokens take decode_scored()."""
        ec.ec_paged_decode_step(q, k_new, v_new, self.k_pages[layer], self.v_pages[layer], self.pos_pages[layer], self.table, self.len_b, self.pos_b,
                                scale, out, self.ws)

    def decode_scored(self, layer, q, k_new, v_new, scale, out, keep: int):
        """One layer of a token under the frequency policy: append, attend, add to the masses, and a sequence of more than `keep` rows loses its
        lightest."""
        ec.ec_paged_decode_score_step(q, k_new, v_new, self.k_pages[layer], self.v_pages[layer], self.pos_pages[layer], self.mass_pages[layer],
                                      self.table, self.len_b, self.pos_b, scale, out, self.ws)
        ec.ec_paged_evict_min(self.k_pages[layer], self.v_pages[layer], self.pos_pages[layer], self.mass_pages[layer], self.table, self.len_after,
                              self._budget(keep), self.seen_b, 1, self.protect_first, self.recent, self.ws_one)

    def end(self, keep: int | None = None):
        """Behind the last layer of a token; keep as in decode_scored, None after decode."""
        self._eager("end")
        if any(n >= len(held) * self.page for n, held in zip(self.rows, self.held)):
            raise ValueError("a token ends, but begin() has not made room for its row")
        for b, n in enumerate(self.rows):
            if n >= 0:
                self.rows[b] = n if keep is not None and n + 1 > keep else n + 1
                self.seen[b] += 1
        self._upload()

    def shrink(self, keep: int):
        """Sequences of more than `keep` rows keep the heaviest, in every layer; the pages behind are free."""
        self._eager("shrink")
        if keep < 0:
            raise ValueError(f"keep is {keep}")
        most = max(max(self.rows) - keep, 0)
        if not most:
            return
        ws = ec.new_workspace(ec.EC_FN_PAGED_EVICT_MIN, len(self.rows), self.G, most, self.D, ec.dtype_code(self.k_pages), self.table.device)
        for layer in range(self.k_pages.shape[0]):
            ec.ec_paged_evict_min(self.k_pages[layer], self.v_pages[layer], self.pos_pages[layer], self.mass_pages[layer], self.table, self.len_b,
                                  self._budget(keep), self.pos_b, most, self.protect_first, self.recent, ws)
        for b, n in enumerate(self.rows):
            if n > keep:
                self.rows[b] = keep
                self._hold(b, keep)
        self._upload_table()
        self._upload()


def rotary_frequencies(rot: int, base: float = 10000.0, factor: float = 1.0, kind: str = "linear", trained: int = 4096, low: float = 1.0, high: float = 32.0,
                       device="cuda"):
    """(freq f32 [rot/2], mscale) for ec_paged_rotary_store: base^(-2i/rot) radians a position, stretched for contexts `factor` times as long as the `trained` one:
      linear  every frequency divided by the factor
      base    the base raised, so that the slowest pair is divided by the factor and the fastest stays: base * factor^(rot/(rot-2))
      parts   pairs that turn more than `high` times over the trained context stay, those that turn less than `low` times are divided by the factor, those
              between in proportion; mscale = 0.1 ln(factor) + 1"""
    if rot < 2 or rot % 2 or not 1.0 <= factor < math.inf or not 0.0 < base < math.inf or kind not in ("linear", "base", "parts"):
        raise ValueError(f"rot {rot} must be even, the factor {factor} at least 1, the base {base} above 0, the kind {kind!r} one of linear, base, parts")
    if kind == "parts" and not (low < high and trained > 0):
        raise ValueError(f"the pairs between low {low} and high {high} need low < high and a trained context, not {trained}")
    if kind == "base" and factor > 1.0:
        if rot == 2:
            raise ValueError("a raised base needs more than one pair")
        base = base * factor ** (rot / (rot - 2))
    freq = torch.tensor(base, dtype=torch.float64) ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    mscale = 1.0
    if kind == "linear":
        freq = freq / factor
    elif kind == "parts":
        kept = ((freq * trained / (2 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        freq = freq * kept + freq / factor * (1.0 - kept)
        mscale = 0.1 * math.log(factor) + 1.0
    return freq.float().to(device), mscale


class PagedTokens:
    """The caches of up to `places` sequences in pages for steps of any number of new tokens a sequence, up to `tokens` in all: chunks of prompts, drafted tokens and
    single ones side by side. Lengths, the page table and the free pages live on the device, and begin() and attend() send nothing from the host and read nothing
    back, so that a step can be captured and replayed with other numbers of tokens.

        batch.admit([0, 1])                                  # two new sequences
        batch.new_b.copy_(new)                               # int32 [places]: tokens of each sequence in this step
        batch.begin()                                        # pages, rows and positions for them
        for i in range(n_layers):
            batch.attend(i, q[i], k[i], v[i], scale, out[i]) # [tokens,H or Hkv,D] packed, sequence after sequence (batch.token_start)

    A sequence that the free pages do not hold, or whose tokens end behind the last of `tokens`, keeps what it has: its tokens get zeros, len_b and seen_b do not
    grow, start_b is -1. Rows of out behind the last sequence's tokens are left as they are.
    Compressed prompts come in as rows: admit(places, rows, seen), which takes their pages or is refused, then store() in every layer before the first step that has
    tokens for them (until then the pages hold what others left there).
    New rows' masses are 0 (what adds to masses is ec_paged_decode_score_step)."""

    def __init__(self, layers, places, tokens, H, Hkv, D, page, n_pages, max_pages, dtype: torch.dtype, freq, mscale=1.0, interleaved=False, G=1, device="cuda"):
        self.page, self.mscale, self.interleaved = page, mscale, interleaved
        self.k_pages, self.v_pages = (torch.zeros((layers, n_pages, Hkv, page, D), dtype=dtype, device=device) for _ in range(2))
        self.pos_pages = torch.zeros((layers, n_pages, G, page), dtype=torch.int32, device=device)
        self.mass_pages = torch.zeros((layers, n_pages, G, page), dtype=torch.float32, device=device)
        ints = lambda *s, fill=0: torch.full(s, fill, dtype=torch.int32, device=device)  # noqa: E731
        self.table, self.held = ints(places, max_pages, fill=-1), ints(places)
        self.free_pages = torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device)
        self.n_free = ints(1, fill=n_pages)
        self.len_b, self.seen_b, self.new_b = ints(places, fill=-1), ints(places), ints(places)  # rows (-1: no sequence), tokens seen, tokens of the next step
        self.start_b, self.token_start = ints(places, fill=-1), ints(places + 1)
        self.rows, self.pos = torch.full((tokens,), -1, dtype=torch.int64, device=device), ints(tokens)
        self.prompts = set()  # places that were admitted with rows
        self.freq = freq
        self.turned = torch.zeros((tokens, H, D), dtype=dtype, device=device)
        self.ws = ec.new_workspace(ec.EC_FN_PAGED_CHUNK_STEP, places, H, tokens, D, ec.dtype_code(self.k_pages), device)

    def _set(self, places, rows, seen):
        if self.table.is_cuda and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("PagedTokens: sequences come and go outside a capture (a step's graph holds begin() and attend())")
        places = list(places)
        if len(set(places)) != len(places) or any(not 0 <= b < self.table.shape[0] for b in places):
            raise ValueError(f"{places} are not different places of 0 .. {self.table.shape[0] - 1}")
        self.prompts.difference_update(places)
        at = torch.tensor(places, dtype=torch.int64).to(self.table.device)
        for x, values in ((self.len_b, rows), (self.seen_b, seen)):
            x.index_copy_(0, at, torch.tensor(values, dtype=torch.int32).to(x.device))

    def admit(self, places, rows=None, seen=None):
        """Sequences that start with `rows` rows of prompts of `seen` tokens, none by default; a place's earlier sequence is gone. Rows get their pages here, and where
        the free ones (those of places released before among them) or a table do not hold them all, the places are left free. Pages of tokens come with begin()."""
        places = list(places)
        rows, seen = (list(x) if x is not None else [0] * len(places) for x in (rows, seen))
        if not len(places) == len(rows) == len(seen) or any(n < 0 for n in rows):
            raise ValueError(f"places {places}, rows {rows} and seen {seen} do not belong together")
        self._set(places, rows, seen)
        if not any(rows):
            return
        start, nothing, first = torch.empty_like(self.len_b), torch.zeros_like(self.new_b), torch.empty_like(self.token_start)
        ec.ec_paged_plan(self.len_b, nothing, self.table, self.held, self.free_pages, self.n_free, self.page, start, self.len_b, first, T=1)
        start = start.tolist()
        refused = [b for b in places if start[b] < 0]
        if refused:
            self._set(places, [-1] * len(places), [0] * len(places))
            raise ValueError(f"{[n for b, n in zip(places, rows) if b in refused]} rows for places {refused}: too few free pages, or more rows than a table holds")
        self.prompts.update(b for b, n in zip(places, rows) if n)

    def release(self, places):
        """Sequences that are over; their pages are free with the next begin() or the next rows that admit() takes in."""
        places = list(places)
        self._set(places, [-1] * len(places), [0] * len(places))

    def begin(self):
        """Pages, rows and positions for new_b more tokens of every sequence."""
        ec.ec_paged_plan(self.len_b, self.new_b, self.table, self.held, self.free_pages, self.n_free, self.page, self.start_b, self.len_b, self.token_start,
                         self.rows, self.pos, seen_b=self.seen_b, seen_after_b=self.seen_b)

    def store(self, layer, places, k, v, pos, mass, n_rows_b=None):
        """Rows 0.. of k, v [len(places),Hkv,n,D], pos and mass [len(places),G,n] as the first rows of the sequences (n_rows_b int32 of each, all by default)."""
        places = list(places)
        if not self.prompts.issuperset(places):
            raise ValueError(f"places {[b for b in places if b not in self.prompts]} were not admitted with rows")
        table = self.table.index_select(0, torch.tensor(places, dtype=torch.int64).to(self.table.device))
        ec.ec_paged_store(k, v, pos, mass, table, self.k_pages[layer], self.v_pages[layer], self.pos_pages[layer], self.mass_pages[layer], None, n_rows_b)

    def attend(self, layer, q, k, v, scale, out, lse=None):
        """One layer of the step that begin() has planned: q, out [tokens,H,D], k, v [tokens,Hkv,D] (q, k and v may be parts of one projection's output)."""
        ec.ec_paged_rotary_store(q, k, v, self.pos, self.rows, self.freq, self.turned, self.k_pages[layer], self.v_pages[layer], self.pos_pages[layer],
                                 self.mass_pages[layer], interleaved=self.interleaved, mscale=self.mscale)
        ec.ec_paged_chunk_step(self.turned, self.k_pages[layer], self.v_pages[layer], self.table, self.start_b, self.token_start, scale, out, self.ws, lse=lse)
