"""Scenes of the growing cache for the GPU tests: a batch of requests whose pages lie in
random order in a supply with spare pages, everything filled with values of its own."""
import numpy as np
import torch

import paper_2607_17715_amd as c2kv

ACT = {"f32": torch.float32, "bf16": torch.bfloat16, "i8": torch.bfloat16}


def f64(t):
    return t.detach().double().cpu().numpy()


class Scene:
    def __init__(self, store, n, ctx, hq=8, hkv=2, d=128, page=64, base=5e5, seed=0, pad_rows=0,
                 spare_pages=2, fused=False, far=0):
        g = torch.Generator().manual_seed(1000 + seed)
        normal = lambda *s: torch.randn(s, generator=g)
        self.store, self.hq, self.hkv, self.d, self.page, self.base = store, hq, hkv, d, page, base
        self.n, self.B = list(n), len(n)
        self.act = ACT[store]
        act_name = "f32" if store == "f32" else "bf16"
        self.cfg = c2kv.attn_cfg(hq, hkv, d, act_name, base)
        kv = [a + b for a, b in zip(n, ctx)]
        need = [-(-x // page) for x in kv]
        self.n_pages = sum(need) + spare_pages
        ids = torch.randperm(self.n_pages, generator=g).tolist()
        self.max_pages = max(max(need), 1) + 1
        table = np.full((self.B, self.max_pages), -1, np.int32)
        for b in range(self.B):
            for i in range(need[b]):
                table[b, i] = ids.pop()
        self.table, self.kv_len = table, np.array(kv, np.int32)
        self.tok_off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        self.n_tokens = int(self.tok_off[-1]) + pad_rows
        N = self.n_tokens
        if fused:
            qkv = normal(N, hq + 2 * hkv, d).to(self.act).cuda()
            self.q, self.k, self.v = (qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:])
        else:
            self.q, self.k, self.v = (normal(N, h, d).to(self.act).cuda() for h in (hq, hkv, hkv))
        self.pos = (torch.arange(N, dtype=torch.int32) * 3 + 17 + far).cuda()
        kshape, vshape = (self.n_pages, hkv, page, d), (self.n_pages, hkv, d, page)
        self.ks = self.vs = None
        if store == "i8":
            self.kp = torch.randint(-127, 128, kshape, generator=g).to(torch.int8).cuda()
            self.vp = torch.randint(-127, 128, vshape, generator=g).to(torch.int8).cuda()
            self.ks = (torch.rand(kshape[:3], generator=g) * 0.01 + 0.01).cuda()
            self.vs = (torch.rand(kshape[:3], generator=g) * 0.01 + 0.01).cuda()
        else:
            self.kp = normal(*kshape).to(self.act).cuda()
            self.vp = normal(*vshape).to(self.act).cuda()
        self.cache = c2kv.Cache(self.kp, self.vp, self.ks, self.vs)

    def chunks(self, table=None, kv_len=None, tok_off=None, **kw):
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()
        return c2kv.Chunks(dev(self.tok_off if tok_off is None else tok_off),
                           dev(self.kv_len if kv_len is None else kv_len),
                           dev(self.table if table is None else table), self.n_tokens, **kw)

    def pages64(self):
        """Keys and values that the pages stand for, in float64."""
        k, v = f64(self.kp), f64(self.vp)
        if self.store == "i8":
            k, v = k * f64(self.ks)[..., None], v * f64(self.vs)[:, :, None]
        return k, v

    def copies(self):
        return [None if t is None else t.clone() for t in (self.kp, self.vp, self.ks, self.vs)]

    def out(self, fill=7.0):
        return torch.full((self.n_tokens, self.hq, self.d), fill, dtype=self.act, device="cuda")

    def lse(self, fill=7.0):
        return torch.full((self.n_tokens, self.hq), fill, dtype=torch.float32, device="cuda")
