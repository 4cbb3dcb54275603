"""A paged cache with tracking records for the tests of attention that records weights and of eviction: contents made on the host,
pages scattered over the pool, everything around the tokens poisoned."""
from __future__ import annotations

import numpy as np
import torch

from paper_2511_11729_amd import binding as hb

DEV = "cuda:0"
P = 16


class CacheCase:
    def __init__(self, lengths, n_q, n_kv, d, *, dtype="bf16", layers=1, seed=0, poison=True, extra_pages=3, block=None, room=0, table_pad=1):
        """room: tokens a sequence may still append."""
        self.n = np.asarray(lengths, np.int32)
        self.B, self.n_q, self.n_kv, self.d, self.L, self.dtype = len(self.n), n_q, n_kv, d, layers, dtype
        eb = 4 if dtype == "f32" else 2
        row = n_kv * d * eb
        page_bytes = P * row
        block = block or max(1 << 16, 1 << (4 * page_bytes - 1).bit_length())
        r = np.random.default_rng(seed)
        pages = np.maximum(1, -(-(self.n.astype(np.int64) + room) // P))
        self.max_pages = int(pages.max()) + table_pad
        ppb = block // page_bytes
        chunks = -(-(int(pages.sum()) + extra_pages) // ppb)
        self.n_pages = chunks * ppb
        self.slab_bytes = chunks * layers * 2 * block
        tdt = torch.float32 if dtype == "f32" else torch.bfloat16
        ids = r.permutation(self.n_pages)[: int(pages.sum())]
        self.table = np.full((self.B, self.max_pages), -1, np.int32)
        at = 0
        for b in range(self.B):
            self.table[b, : pages[b]] = ids[at: at + pages[b]]
            at += pages[b]
        self.slab = torch.zeros(self.slab_bytes, dtype=torch.uint8, device=DEV)
        self.view = torch.as_strided(self.slab.view(tdt), (chunks, layers, 2, ppb, n_kv, P, d),
                                     (layers * 2 * block // eb, 2 * block // eb, block // eb, P * n_kv * d, P * d, d, 1))
        self.cache = torch.full((chunks, layers, 2, ppb, n_kv, P, d), float("nan") if poison else 0.0, dtype=tdt)
        self.records = np.zeros((layers, self.n_pages, n_kv, P), [("w", np.float32), ("p", np.int32)])
        self.records["w"] = np.nan if poison else 0.0
        self.records["p"] = -77
        self.K = []                    # [layer][sequence] -> (K, V) fp64 [n, n_kv, d], as stored
        for l in range(layers):
            seqs = []
            for b in range(self.B):
                kv = torch.from_numpy(r.standard_normal((2, int(self.n[b]), n_kv, d)).astype(np.float32)).to(tdt)
                t = np.arange(int(self.n[b]))
                page = self.table[b, t // P]
                for which in (0, 1):
                    self.cache[page // ppb, l, which, page % ppb, :, t % P] = kv[which]
                self.records["w"][l, page, :, t % P] = r.lognormal(-3.0, 2.0, (len(t), n_kv)).astype(np.float32)
                self.records["p"][l, page, :, t % P] = t[:, None]
                seqs.append(tuple(kv.double().numpy()))
            self.K.append(seqs)
        self.ppb = ppb
        self.pool = hb.Pool(self.slab, self.slab_bytes, block_bytes=block, n_layers=layers, kv_row_bytes=row)
        w = torch.zeros(max(n_q * d, 16) * 16, dtype=tdt, device=DEV)
        g = torch.ones(16, device=DEV)
        self.layer = dict.fromkeys(("wq", "wk", "wv", "wo", "wg", "wu", "wd"), w) | {"g1": g, "g2": g}
        self.longest = max(1, int(self.n.max()) + room)
        self.ctx = hb.Context(self.pool, n_layers=layers, hidden=16, n_q_heads=n_q, n_kv_heads=n_kv, head_dim=d, ffn=16,
                              dtype=hb.HARLI_F32 if dtype == "f32" else hb.HARLI_BF16, max_batch=self.B, max_seq_len=self.longest,
                              layers=[self.layer] * layers)
        self.workspace = torch.empty(self.ctx.kv_attend_workspace_bytes(self.B, self.longest), dtype=torch.uint8, device=DEV)
        self.reset()

    def reset(self):
        self.view.copy_(self.cache.to(DEV))
        self.track = torch.from_numpy(self.records.view(np.int32).reshape(self.records.shape + (2,)).copy()).to(DEV)
        self.table_dev = torch.from_numpy(self.table).to(DEV)
        self.n_dev = torch.from_numpy(self.n).to(DEV)

    def attend(self, q, out, *, layer=0, track=True, stream=None, **kw):
        args = dict(layer=layer, batch=self.B, q=q, out=out, n_tokens=self.n_dev, page_table=self.table_dev, max_pages=self.max_pages,
                    max_kv_len=self.longest, track=self.track if track else None, workspace=self.workspace, stream=stream)
        self.ctx.kv_attend(**dict(args, **kw))

    def evict(self, keep, **kw):
        self.keep_dev = torch.from_numpy(np.asarray(keep, np.int32)).to(DEV)
        args = dict(batch=self.B, n_tokens=self.n_dev, keep=self.keep_dev, page_table=self.table_dev, max_pages=self.max_pages,
                    max_kv_len=self.longest, track=self.track)
        self.ctx.kv_evict(**dict(args, **kw))

    def got_records(self):
        return self.track.cpu().numpy().view([("w", np.float32), ("p", np.int32)])[..., 0]

    def slots(self, b, n):
        """Page and slot of the first n tokens of sequence b."""
        t = np.arange(n)
        return self.table[b, t // P], t % P
