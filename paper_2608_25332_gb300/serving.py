"""Questions about one pruned image or video, from the pruning step to the answers.

After the pruning layers a sample's sequence is [system rows | kept visual rows | text]. Where
several questions are asked about the same image or video, the system and visual rows are
the same for all of them: their keys and values are computed, pruned and stored once, and
every question's prompt and every decoded token attends over them and over its own rows.

``QuestionCache`` keeps that state for the LLM layers behind the pruning: one paged pool of
key/value rows per layer, one set of block tables for all layers. The LLM itself is the
caller's: it hands each layer's queries, keys and values in and gets the attention's output
back. All calls enqueue on the current stream; nothing synchronises with the host.

    cache = QuestionCache(layers, B, H_q, H_kv, page_size, n_pages, max_len, dtype, bits=4, rotary=P.Rotary(...))
    cache.set_prefix(K, V)                # per layer: rows of a compaction, system + visual
    cache.begin(new_len)                  # prompts: the questions' lengths, 0 for an idle slot
    for each layer: out = cache.prompt(layer, Q, K, V, pos=pos)      # packed rows of all questions
    while ...:
        cache.begin(ones)                 # 1: one more token, -1: the question is answered
        for each layer: out = cache.decode(layer, Q, K, V, pos=pos)  # one row per request

With a rotary, queries and keys come as the projections leave them: prompt and decode norm them
where the model has norms and rotate them by the rows' position ids, on the way into the cache.
Without one they come rotated, and pos is left out. The prefix's keys are a compaction's, which
are rotated already.
"""
from __future__ import annotations

import torch

from . import provip as P


class QuestionCache:
    """Paged keys and values of B concurrent questions over one shared prefix.

    layers: LLM layers behind the pruning; n_pages pages of page_size rows per layer, for the
    prefix and the questions; max_len: own tokens of a question at most (prompt and answer),
    rounded up to whole pages; max_new: new tokens of one step over all questions at most (default
    B * max_len). bits: 16 for pages of dtype, 4 for pages of 4 bits (72 bytes for a head's 128 values
    instead of 256 in bf16): what is decoded from, and what prompts see of the prefix; a prompt's own
    rows see each other unrounded. rotary, norms, eps: the rotation of queries and keys (P.Rotary),
    their norms as a pair of weights [128] a layer, and what is added to the mean square.
    """

    def __init__(self, layers, B, H_q, H_kv, page_size, n_pages, max_len, dtype=torch.bfloat16, device="cuda",
                 max_new=None, algo=P.ALGO_AUTO, bits=16, rotary=None, norms=None, eps=1e-6):
        dev = torch.device(device)
        P._dtype_of(dtype)  # (refused here, not by the first append)
        if bits not in (4, 16):
            raise P.ProvipError(P.ERR_INVALID_ARG, f"QuestionCache: pages of {bits} bits")
        if norms is not None and (rotary is None or len(norms) != layers):
            raise P.ProvipError(P.ERR_INVALID_ARG, "QuestionCache: norms are a pair a layer, beside a rotary")
        self.bits, self.rotary, self.norms, self.eps = bits, rotary, norms, float(eps)
        self.B, self.H_q, self.H_kv, self.page_size = int(B), int(H_q), int(H_kv), int(page_size)
        self.max_len = -(-int(max_len) // self.page_size) * self.page_size  # what the tables may hand out
        self.dtype, self.device, self.algo = dtype, dev, algo
        self.pools = [tuple(P.pages4(n_pages, page_size, H_kv, dev) if bits == 4 else
                            torch.zeros(n_pages, page_size, H_kv, 128, dtype=dtype, device=dev) for _ in range(2))
                      for _ in range(layers)]
        self.free = torch.arange(n_pages, dtype=torch.int32, device=dev)
        self.n_free = torch.full((1,), n_pages, dtype=torch.int32, device=dev)
        self.tables = torch.zeros(B, self.max_len // self.page_size, dtype=torch.int32, device=dev)
        self.kv_len = torch.zeros(B, dtype=torch.int32, device=dev)
        self.planner = P.PageTables(B, page_size, B * self.max_len if max_new is None else max_new, dev)
        self._slot_map = torch.full((self.planner.T_max + 1,), -1, dtype=torch.int32, device=dev)  # the last stays -1
        self.planner.slot_map, self._first_row = self._slot_map[:-1], self.planner.row_start[:-1]
        self.prefix, self.prefix_len, self.prefix_table = [], 0, None
        self._prefix_held = torch.zeros(2, dtype=torch.int32, device=dev)  # rows that the prefix has in pages; 0
        # the step's new tokens, and the tokens held before it (at one place for good, as all that the
        # planner writes, so that a layer's calls can be captured in a graph)
        self.new_len, self.held = torch.zeros_like(self.kv_len), torch.zeros_like(self.kv_len)
        self._derived = {}
        self.plan = None
        self._prompt = self._decode = None  # the steps' buffers: of the last size only
        # rotated queries (and keys) of prompts, of the last size only, and of decoding, at one place for good as
        # a captured step writes there; in 4 bits, the prefix read back for prompts, and its slots
        self._turned, self._turned_one, self._read = (), (), ()

    def set_prefix(self, K, V):
        """K, V: a [n, H_kv, 128] tensor per layer (for instance rows [:vis_start + keep] of a
        compaction's K_out[b] and V_out[b]), copied here: they may change afterwards. Their pages
        come off the free stack, and those of the prefix before go back onto it (its questions
        should have ended); more rows than the pool holds are refused. Where the questions leave
        too few pages, the prefix gets none: every decode() then reports it in the device status,
        and its result is meaningless."""
        n, layers = K[0].shape[0] if len(K) else 0, len(self.pools)
        if len(K) != layers or len(V) != layers or any(
                x.shape != (n, self.H_kv, 128) or x.dtype is not self.dtype or x.device != self.kv_len.device for x in (*K, *V)):
            raise P.ProvipError(P.ERR_INVALID_ARG, f"set_prefix: K and V must be {layers} tensors [n, {self.H_kv}, 128] each, "
                                                   f"of as many rows, {self.dtype} on {self.kv_len.device}")
        need, pages = -(-n // self.page_size), self.free.numel()
        if need > pages:
            raise P.ProvipError(P.ERR_INVALID_ARG, f"set_prefix: {n} rows take {need} pages, the pool has {pages}")
        # prompts read rows of their own, not the caller's, which the next pruning may overwrite (4 bits: from pages). All
        # that may be refused or lack memory comes before any page changes hands
        prefix = [tuple(x if self.bits == 4 and self._packed(x) else x.clone(memory_format=torch.contiguous_format) for x in kv)
                  for kv in zip(K, V)]
        read = tuple(torch.zeros(n, self.H_kv, 128, dtype=self.dtype, device=self.device) for _ in range(2)) if self.bits == 4 else ()
        # two requests of the tables: the prefix before, which ends, and this one. (-1: no page.
        # Where the questions hold too many, the prefix gets none and decoding reports it)
        before = 0 if self.prefix_table is None else self.prefix_table.numel()
        table = torch.full((2, max(need, before)), -1, dtype=torch.int32, device=self.device)
        if before:
            table[0, :before] = self.prefix_table
        new = torch.full((2,), n, dtype=torch.int32, device=self.device)
        new[0].fill_(-1)
        plan = P.PageTables(2, self.page_size, n, self.device)(self._prefix_held, new, self.free, self.n_free, table)
        self.n_free.copy_(plan["free_count"])
        self._prefix_held[0].copy_(plan["kv_len"][1])
        for (kp, vp), (k, v) in zip(self.pools, prefix):
            (P.provip_kv_append4 if self.bits == 4 else P.provip_kv_append)(k, v, plan["slot_map"], kp, vp)
        self._drop(self.prefix_table, self._prompt, self._decode, *(x for kv in self.prefix for x in kv), *self._read)
        if self.bits == 4:
            # prompts read the rows back from the pages, one layer's at a time (a row without a slot is reported there)
            read = (*read, torch.where(plan["slot_map"] < 0, 2 ** 31 - 1, plan["slot_map"]))
            prefix = []
        self.prefix, self.prefix_len, self.prefix_table, self._read = prefix, n, table[1, :need], read
        self._prompt = self._decode = None

    def begin(self, new_len):
        """The next step's new tokens per question (int32 [B] on the device): pages and slots for
        them; -1 returns an answered question's pages (its slot can take another question).
        A question that the free pages do not suffice for keeps its length: read kv_len where
        that can happen."""
        if new_len.dtype is not torch.int32 or new_len.device != self.kv_len.device or not new_len.is_contiguous() or \
                new_len.numel() < self.B:
            raise P.ProvipError(P.ERR_INVALID_ARG, f"begin: new_len must be a contiguous int32 tensor of {self.B} entries on "
                                                   f"{self.kv_len.device}")
        self._drop(*self._derived.values())
        self._derived.clear()
        if new_len.numel() > self.B:
            new_len = new_len.view(-1)[:self.B]
        self.new_len.copy_(new_len)  # (the caller may write the next step's into it)
        self.held.copy_(self.kv_len)
        self.plan = self.planner(self.kv_len, self.new_len, self.free, self.n_free, self.tables, inplace=True)
        return self.plan

    def prompt(self, layer, Q, K, V, max_rows=None, pos=None):
        """Prompts of the step begun: the questions' rows packed in request order, Q [T, H_q, 128],
        K and V [T, H_kv, 128] (T >= the step's new tokens). Every row sees the prefix and the
        step's rows of its question up to itself, so a question with new rows must hold no token
        yet (one that was not begun, or ended by -1): what it holds lies in pages, which the
        prompts' attention does not read. A question that does is reported in the device status,
        its rows go into the cache, and their output is left untouched. max_rows: the longest
        question (default max_len). pos: the rows' position ids [axes, T] (int32), with a rotary. The
        result is overwritten by the next call (another layer's)."""
        T, longest = Q.shape[0], min(self.max_len, Q.shape[0]) if max_rows is None else int(max_rows)
        self._check_rows("prompt", T, K, V)
        self._check_pos("prompt", T, pos)
        if self._prompt is None or self._prompt.shape[0] != T or self._prompt.shape[4] != longest:
            self._drop(self._prompt)
            self._prompt = P.PromptAttention(T, self.B, self.H_q, self.H_kv, longest, longest, self.prefix_len, True, None,
                                             self.dtype, self.device, self.algo, want_lse=False)
        start, n = self.plan["row_start"], self._once("rows", self._prompt_rows)
        kp, vp = self.pools[layer]
        rows = min(T, self.planner.T_max)  # (rows behind the last question have no slot)
        Q, K = self._append(layer, Q, K, V, self.plan["slot_map"][:rows], pos, rows, True)
        pre = (None, None)
        if self.prefix_len:
            pre = self.prefix[layer] if self.bits == 16 else P.provip_kv_read4(self._read[2], kp, vp, out=self._read[:2])
        return self._prompt(Q, K, V, start, n, start, n, *pre)["out"]

    def decode(self, layer, Q, K, V, pos=None):
        """One token per question: Q [B, H_q, 128], K and V [B, H_kv, 128] in request order, all of
        the step's new lengths 1 (or -1, whose rows are skipped: their output is that of an empty
        question; a longer one is reported in the device status and taken for an empty question).
        pos: the rows' position ids [axes, B] (int32), with a rotary. The result is overwritten by the
        next call."""
        if Q.shape[0] != self.B:
            raise P.ProvipError(P.ERR_INVALID_ARG, f"decode: Q must have {self.B} rows")
        self._check_rows("decode", self.B, K, V)
        self._check_pos("decode", self.B, pos)
        if self._decode is None:
            shape = (self.B, self.H_q, self.H_kv, self.max_len, self.prefix_len, None, self.dtype, self.device)
            self._decode = P.DecodeAttention4(*shape, want_lse=False) if self.bits == 4 else \
                P.DecodeAttention(*shape, self.algo, want_lse=False)
        kp, vp = self.pools[layer]
        Q, _ = self._append(layer, Q, K, V, self._once("slots", self._token_slots), pos, self.B, False)
        n = self._once("lengths", lambda: torch.where(self.new_len > 1, -1, self.kv_len))  # -1: reported
        return self._decode(Q, kp, vp, self.tables, n, self.prefix_table if self.prefix_len else None)["out"]

    @staticmethod
    def _packed(x):
        """whether rows [n, H, 128] lie as the 4-bit append takes them: a row's heads side by side, at 16 bytes"""
        n, H, _ = x.shape
        s0, s1, s2 = x.stride()
        return s2 == 1 and (H == 1 or s1 == 128) and x.data_ptr() % 16 == 0 and \
            (n <= 1 or (s0 >= H * 128 and s0 * x.element_size() % 16 == 0))

    @staticmethod
    def _check_rows(what, n, *tensors):
        if any(x.shape[0] != n for x in tensors):
            raise P.ProvipError(P.ERR_INVALID_ARG, f"{what}: K and V must have as many rows as Q, {n}")

    def _check_pos(self, what, n, pos):
        if (pos is None) != (self.rotary is None) or (pos is not None and (pos.dim() != 2 or pos.shape[1] != n)):
            raise P.ProvipError(P.ERR_INVALID_ARG, f"{what}: position ids [axes, {n}] go with a rotary, and with one only")

    def _append(self, layer, Q, K, V, slots, pos, rows, want_k):
        """The first `rows` keys and values into the layer's pages, rotated on the way where there is a rotary.
        Returns the queries and (want_k) keys to attend with; rows past the step's last stay unrotated."""
        kp, vp = self.pools[layer]
        if self.rotary is None:
            (P.provip_kv_append4 if self.bits == 4 else P.provip_kv_append)(K[:rows], V[:rows], slots, kp, vp)
            return Q, K
        zeros = lambda n, h: torch.zeros(n, h, 128, dtype=self.dtype, device=self.device)
        if not want_k:
            self._turned_one = self._turned_one or (zeros(self.B, self.H_q), None)
        elif not self._turned or self._turned[0].shape[0] != Q.shape[0]:
            self._drop(*self._turned)
            self._turned = zeros(Q.shape[0], self.H_q), zeros(Q.shape[0], self.H_kv)
        q, k = self._turned if want_k else self._turned_one
        count = self.plan["row_start"][self.B:] if want_k else None  # (a decode step's rows are by question, not packed)
        w_q, w_k = (None, None) if self.norms is None else self.norms[layer]
        P.provip_rotate_append(Q[:rows], K[:rows], V[:rows], pos[:, :rows], self.rotary, slots, kp, vp, w_q, w_k, self.eps,
                               out=(q[:rows], k[:rows] if want_k else None), n_rows=count)
        return q, k

    @staticmethod
    def _drop(*held):
        """Tensors, or steps with theirs, that the cache lets go of: their memory is handed out again
        behind what the current stream has under way, whichever stream it was allocated on."""
        held = [t for x in held if x is not None for t in ((x,) if isinstance(x, torch.Tensor) else (x.out, x.ws)) if t.is_cuda]
        stream = torch.cuda.current_stream(held[0].device) if held else None
        for t in held:
            t.record_stream(stream)

    def _once(self, name, make):
        """What a step's layers share, worked out at its first use; in a graph at every use, as
        its replays follow steps that are begun later."""
        if self.device.type == "cuda" and torch.cuda.is_current_stream_capturing():
            return make()
        if name not in self._derived:
            self._derived[name] = make()
        return self._derived[name]

    def _prompt_rows(self):
        """The questions' rows for prompt(): -1, which is reported, where tokens are held already."""
        return torch.where(torch.minimum(self.new_len, self.held) > 0, -1, self.new_len.clamp(min=0))

    def _token_slots(self):
        """Slots of the questions' new tokens in request order, -1 for a question without one.
        Packed rows skip such questions: the token of question b is row row_start[b], which for
        those behind the step's last row may lie past the map's end (it has max_new slots): they
        take the entry behind it, -1."""
        n = self.planner.T_max
        rows = torch.where(self.new_len > 0, self._first_row, n).clamp_(max=n)
        return self._slot_map.index_select(0, rows)
