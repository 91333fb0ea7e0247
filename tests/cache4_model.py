"""cache_model's Model with the rotating and 4-bit calls of the binding, restated in plain Python."""
import numpy as np
import torch

import cache4_ref as ref
from cache_model import Model
from paper_2608_25332_gb300 import provip as P


class Model4(Model):
    def __init__(self, monkeypatch):
        super().__init__(monkeypatch)
        monkeypatch.setattr(P, "DecodeAttention4", self._bound(self.DecodeAttention4))
        for name in ("provip_rotate_append", "provip_kv_append4", "provip_kv_read4"):
            monkeypatch.setattr(P, name, getattr(self, name[7:]))

    def kv_append4(self, K, V, slot_map, k_pages, v_pages):
        self._rows(K.shape[0], slot_map, "slot_map")
        page = k_pages.shape[2] // P.ROW4
        for x, pages in ((K, k_pages), (V, v_pages)):
            codes, bits = ref.pack(x.float().numpy().reshape(-1, 128))
            for t in range(x.shape[0]):
                s = int(slot_map[t])
                if s >= pages.shape[0] * page:
                    self.reports.append("slot")
                elif s >= 0:
                    for h in range(x.shape[1]):
                        ref.put(pages, page, s, h, codes[t * x.shape[1] + h], bits[t * x.shape[1] + h])

    def kv_read4(self, slot_map, k_pages, v_pages, dtype=torch.bfloat16, out=None):
        page = k_pages.shape[2] // P.ROW4
        for pages, to in ((k_pages, out[0]), (v_pages, out[1])):
            for t, s in enumerate(slot_map.tolist()):
                if s >= pages.shape[0] * page:
                    self.reports.append("slot")
                elif s >= 0:
                    to[t] = ref.values(pages, page, torch.tensor([s]))[0].to(to.dtype)
        return out

    def rotate_append(self, Q, K, V, pos, rotary, slot_map, k_pages, v_pages, q_norm=None, k_norm=None, eps=1e-6, out=None,
                      want_k=False, n_rows=None):
        n = Q.shape[0] if n_rows is None else int(n_rows)
        if not 0 <= n <= Q.shape[0]:
            self.reports.append("rows")
            n = min(max(n, 0), Q.shape[0])
        assert pos.dtype is torch.int32 and pos.shape[0] >= rotary.n_axes and pos.shape[1] == Q.shape[0]
        q, k = (ref.turn(x[:n], pos[:, :n], list(rotary.inv_freq), list(rotary.axis), w, eps, rotary.factor)[0].to(x.dtype)
                for x, w in ((Q, q_norm), (K, k_norm)))
        out[0][:n] = q
        if out[1] is not None:
            out[1][:n] = k
        put = self.kv_append4 if k_pages.dtype is torch.uint8 else self.append
        put(k, V[:n], slot_map[:n].contiguous(), k_pages, v_pages)
        return out

    class DecodeAttention4:
        def __init__(self, model, B, H_q, H_kv, kv_len_max, prefix_len=0, scale=None, dtype=None, device="cpu", want_lse=True):
            self.inner = Model.DecodeAttention(model, B, H_q, H_kv, kv_len_max, prefix_len, scale)
            self.out, self.ws = self.inner.out, self.inner.ws

        def __call__(self, Q, k_pages, v_pages, block_table, kv_len, prefix_table=None):
            page = k_pages.shape[2] // P.ROW4
            slots = torch.arange(k_pages.shape[0] * page)
            pools = [ref.values(x, page, slots).view(x.shape[0], page, x.shape[1], 128) for x in (k_pages, v_pages)]
            return self.inner(Q, *pools, block_table, kv_len, prefix_table)


def held(x):
    """what rows [n, H, 128] stand for in 4 bits, in 64 bits"""
    codes, bits = ref.pack(x.detach().float().cpu().numpy().reshape(-1, 128))
    d = ref.bf16_value(bits).astype(np.float64)
    v = (codes.reshape(-1, 4, 32) - 8) * d[..., None]
    return torch.from_numpy(v.reshape(x.shape)).to(x.device)
