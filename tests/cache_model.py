"""The binding's cache and attention calls restated in plain Python and 64 bits on the CPU,
from their contract in include/provip.h, so that what calls them can be tested without a
GPU. A condition that a kernel would report in the device status is listed in ``reports``."""
import math
import weakref

import torch

from paper_2608_25332_gb300 import provip as P

DH = 128


def _ceil(a, b):
    return -(-a // b)


class Model:
    """monkeypatch.setattr-s itself in the place of the binding's calls."""

    def __init__(self, monkeypatch):
        self.reports, self.made = [], []
        for name in ("PageTables", "PromptAttention", "DecodeAttention"):
            monkeypatch.setattr(P, name, self._bound(getattr(self, name)))
        monkeypatch.setattr(P, "provip_kv_append", self.append)

    def _bound(self, cls):
        def make(*a, **kw):
            step = cls(self, *a, **kw)
            self.made.append((cls.__name__, weakref.ref(step)))
            return step
        return make

    def kept(self, name):
        return sum(n == name and step() is not None for n, step in self.made)

    @staticmethod
    def _rows(n, t, what):
        if t.dtype is not torch.int32 or not t.is_contiguous() or t.numel() < n:
            raise P.ProvipError(P.ERR_INVALID_ARG, what)

    def append(self, K, V, slot_map, k_pages, v_pages):
        self._rows(K.shape[0], slot_map, "slot_map")
        for x, pages in ((K, k_pages), (V, v_pages)):
            flat = pages.view(-1, *pages.shape[2:])
            for t in range(x.shape[0]):
                s = int(slot_map[t])
                if s >= flat.shape[0]:
                    self.reports.append("slot")
                elif s >= 0:
                    flat[s] = x[t]

    class PageTables:
        def __init__(self, model, B, page_size, T_max, device="cpu"):
            self.model, self.B, self.page, self.T_max = model, B, page_size, T_max
            self.kv_len = torch.zeros(B, dtype=torch.int32)
            self.free_count = torch.zeros(1, dtype=torch.int32)
            self.slot_map, self.row_start = torch.zeros(T_max, dtype=torch.int32), torch.zeros(B + 1, dtype=torch.int32)

        def __call__(self, kv_len, new_len, free_pages, free_count, block_table, inplace=False):
            kv, new, n = kv_len.tolist(), new_len.tolist(), int(free_count)
            assert block_table.shape[0] == self.B and len(kv) >= self.B and len(new) >= self.B
            stack = free_pages[:n].tolist()
            for b in range(self.B):
                if new[b] < 0:
                    stack += block_table[b, :_ceil(kv[b], self.page)].tolist()
                    kv[b] = 0
            start, slots, short = [0], [], False
            for b in range(self.B):
                add = max(new[b], 0)
                held, want = _ceil(kv[b], self.page), _ceil(kv[b] + add, self.page)
                fits = want <= block_table.shape[1] and start[-1] + add <= self.T_max
                if not fits:
                    self.model.reports.append("tables")
                short = short or want - held > len(stack)
                ok = fits and (want == held or not short)
                for i in range(held, want if ok else held):
                    block_table[b, i] = stack.pop()
                for t in range(kv[b], kv[b] + add):
                    slots.append(int(block_table[b, t // self.page]) * self.page + t % self.page if ok else -1)
                start.append(start[-1] + add)
                kv[b] += add if ok else 0
            free_pages[:len(stack)] = torch.tensor(stack, dtype=torch.int32)
            self.slot_map[:] = torch.tensor((slots + [-1] * self.T_max)[:self.T_max], dtype=torch.int32)
            kv_out, fc_out = (kv_len, free_count) if inplace else (self.kv_len, self.free_count)
            kv_out[:] = torch.tensor(kv, dtype=torch.int32)
            fc_out[:] = len(stack)
            self.row_start[:] = torch.tensor(start, dtype=torch.int32)
            return dict(kv_len=kv_out, row_start=self.row_start, slot_map=self.slot_map, free_count=fc_out)

    @staticmethod
    def attend(q, k, v, scale):
        """q [H_q, 128] over k, v [n, H_kv, 128] in 64 bits"""
        if k.shape[0] == 0:
            return torch.zeros(q.shape, dtype=torch.float64)
        R = q.shape[0] // k.shape[1]
        kk, vv = (x.double().repeat_interleave(R, 1) for x in (k, v))
        p = torch.softmax(torch.einsum("hd,jhd->hj", q.double(), kk) * scale, 1)
        return torch.einsum("hj,jhd->hd", p, vv)

    class PromptAttention:
        def __init__(self, model, T_q, B, H_q, H_kv, q_len_max, k_len_max, prefix_len=0, causal=True, scale=None, dtype=None,
                     device="cpu", algo=0, want_lse=True):
            self.model, self.shape, self.causal = model, (T_q, B, H_q, H_kv, q_len_max, k_len_max, prefix_len), causal
            self.scale = DH ** -0.5 if scale is None else scale
            self.out = torch.full((T_q, H_q, DH), math.nan, dtype=torch.float64)
            self.ws = self.out[:0]

        def __call__(self, Q, K, V, q_start, q_len, k_start, k_len, K_prefix=None, V_prefix=None):
            T_q, B, _, _, qm, km, n = self.shape
            if Q.shape[0] != T_q or qm > T_q or km > K.shape[0] or (n and (K_prefix is None or K_prefix.shape[0] < n)):
                raise P.ProvipError(P.ERR_INVALID_ARG, "prompt_attention")
            for t in (q_start, q_len, k_start, k_len):
                Model._rows(B, t, "starts or lengths")
            for b in range(B):
                q0, lq, k0, lk = (int(t[b]) for t in (q_start, q_len, k_start, k_len))
                if not (0 <= lq <= qm and 0 <= q0 <= T_q - lq and 0 <= lk <= km and 0 <= k0 <= K.shape[0] - lk):
                    self.model.reports.append("sequence")
                    continue
                for i in range(lq):
                    see = max(lk - lq + i + 1, 0) if self.causal else lk
                    k, v = K[k0:k0 + see], V[k0:k0 + see]
                    if n:
                        k, v = torch.cat([K_prefix[:n], k]), torch.cat([V_prefix[:n], v])
                    self.out[q0 + i] = Model.attend(Q[q0 + i], k, v, self.scale)
            return dict(out=self.out, lse=None)

    class DecodeAttention:
        def __init__(self, model, B, H_q, H_kv, kv_len_max, prefix_len=0, scale=None, dtype=None, device="cpu", algo=0,
                     want_lse=True):
            self.model, self.shape = model, (B, kv_len_max, prefix_len)
            self.scale = DH ** -0.5 if scale is None else scale
            self.out = torch.full((B, H_q, DH), math.nan, dtype=torch.float64)
            self.ws = self.out[:0]

        def __call__(self, Q, k_pages, v_pages, block_table, kv_len, prefix_table=None):
            B, km, n = self.shape
            ps, pages = k_pages.shape[1], k_pages.shape[0]
            if km > block_table.shape[1] * ps or Q.shape[0] != B:
                raise P.ProvipError(P.ERR_INVALID_ARG, "decode_attention")
            Model._rows(B, kv_len, "kv_len")

            def rows(table, m):
                if any(not 0 <= int(p) < pages for p in table[:_ceil(m, ps)]):
                    self.model.reports.append("page")
                j = torch.arange(m)
                return [x[table.long().clamp(0, pages - 1)[j // ps], j % ps] for x in (k_pages, v_pages)]

            if n:
                Model._rows(_ceil(n, ps), prefix_table, "prefix_table")
                pre = rows(prefix_table, n)
            for b in range(B):
                m = int(kv_len[b])
                if not 0 <= m <= km:
                    self.model.reports.append("kv_len")
                    m = 0
                k, v = rows(block_table[b], m)
                if n:
                    k, v = torch.cat([pre[0], k]), torch.cat([pre[1], v])
                self.out[b] = Model.attend(Q[b], k, v, self.scale)
            return dict(out=self.out, lse=None)
