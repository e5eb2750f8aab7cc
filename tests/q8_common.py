"""Caches in 8 bits for the GPU tests: the same slabs as numpy arrays per slab and as device buffers in either layout."""
import numpy as np
import torch

import oracle

DT = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
JUNK = {"e4m3": 0x7f, "int8": 0x80}                       # a NaN; a code that no store writes


class Cache:
    """Slabs with room for caps[b] rows; codes [slab] uint8 [cap][128], scales [slab] float64 [blocks].  Rows and scales that no slab holds are junk."""

    def __init__(self, B, lens, caps, hk, fmt, block, paged, seed, n_q=None, rows_before=0, d_model=0, window=1, max_sent=1, spare_pages=5):
        self.B, self.fmt, self.block, self.paged, self.hk, self.bt = B, fmt, block, paged, hk, len(caps)
        r = self.r = np.random.default_rng(seed)
        self.caps = np.asarray(caps, np.int64)
        if paged:
            self.caps = -(-self.caps // 128) * 128
        self.lens = np.asarray(lens, np.int32).reshape(self.bt, hk)
        self.slabs = self.bt * hk
        off = np.concatenate([[0], np.cumsum(self.caps)])
        self.rows16 = int(off[-1]) * hk
        self.max_cap = int(self.caps.max())
        self.row0 = [int(off[s // hk]) * hk + (s % hk) * int(self.caps[s // hk]) for s in range(self.slabs)]
        self.slab_off = torch.from_numpy(off[:-1].copy()).cuda()
        self.cap = torch.from_numpy(self.caps.astype(np.int32)).cuda()
        self.nblocks = -(-self.max_cap // block)
        if paged:
            per = self.caps // 128
            n = int(per.sum()) * hk
            self.pool = n + spare_pages
            ids = r.permutation(self.pool)[:n]
            self.max_pages = int(per.max())
            self.table = np.full((self.slabs, self.max_pages), -1, np.int32)
            k = 0
            for s in range(self.slabs):
                m = int(per[s // hk])
                self.table[s, :m] = ids[k:k + m]
                k += m
            self.rows = self.pool * 128
            self.block_table = torch.from_numpy(self.table.reshape(self.bt, hk, -1)).cuda()
            scale_shape = (self.pool, 128 // block)
        else:
            self.rows = self.rows16 + rows_before
            self.block_table = None
            scale_shape = (self.bt, hk, self.nblocks)
        self.K, self.V = (torch.full((self.rows, 128), JUNK[fmt], dtype=torch.uint8, device="cuda") for _ in range(2))
        self.ks, self.vs = (torch.full(scale_shape, float("nan"), device="cuda") for _ in range(2))
        self.shape = B.make_shape(self.bt, n_q or hk, hk, 128, window, d_model, max_sent, self.max_cap, self.slab_off, self.cap, self.rows16)
        self.ws = torch.empty(B.skipkv_workspace_bytes(self.shape), dtype=torch.uint8, device="cuda")
        B.skipkv_workspace_init(self.shape, self.ws)
        self.cache = B.make_q8_cache(self.K.view(DT[fmt]), self.V.view(DT[fmt]), self.ks, self.vs, block, self.block_table)
        self.kv_len = torch.from_numpy(self.lens).cuda()

    def places(self, s, n):
        """Rows of the buffers and places of the scales of slab s's first n rows."""
        t, i = np.arange(n), np.arange(-(-n // self.block))
        if not self.paged:
            return self.row0[s] + t, s * self.nblocks + i
        per = 128 // self.block
        return self.table[s][t // 128].astype(np.int64) * 128 + t % 128, self.table[s][i // per].astype(np.int64) * per + i % per

    def put(self, codes, scales):
        """codes, scales: (K, V) pairs of lists by slab; as many rows as a list entry has."""
        for buf, sc, c, f in ((self.K, self.ks, codes[0], scales[0]), (self.V, self.vs, codes[1], scales[1])):
            flat = sc.view(-1)
            for s in range(self.slabs):
                rows, at = self.places(s, len(c[s]))
                buf[torch.from_numpy(rows).cuda()] = torch.from_numpy(c[s]).cuda()
                flat[torch.from_numpy(at).cuda()] = torch.from_numpy(np.asarray(f[s][:len(at)], np.float32)).cuda()

    def get(self, s, n):
        """(codes, scales) of K and V of slab s's first n rows."""
        rows, at = self.places(s, n)
        rows, at = torch.from_numpy(rows).cuda(), torch.from_numpy(at).cuda()
        return [(buf[rows].cpu().numpy(), sc.view(-1)[at].double().cpu().numpy()) for buf, sc in ((self.K, self.ks), (self.V, self.vs))]

    def untouched(self, lens):
        """Rows and scales behind lens[slab] are the junk they were."""
        for buf, sc in ((self.K, self.ks), (self.V, self.vs)):
            rows, scales = torch.ones(self.rows, dtype=torch.bool), torch.ones(sc.numel(), dtype=torch.bool)
            for s in range(self.slabs):
                r, a = self.places(s, int(lens[s]))
                rows[torch.from_numpy(r)] = False
                scales[torch.from_numpy(a)] = False
            assert bool((buf[rows.cuda()] == JUNK[self.fmt]).all()) and bool(torch.isnan(sc.view(-1)[scales.cuda()]).all())

    def status(self):
        return self.B.skipkv_status(self.ws, raise_on_error=False)


def random_slab(r, n, block, fmt, sigma=1.0, general=False):
    """Codes of a slab with every code value, and scales that bring the rows to about sigma."""
    v = oracle.q8_values(fmt)
    good = np.array([c for c in range(256) if np.isfinite(v[c]) and abs(v[c]) <= oracle.Q8_TOP[fmt]], np.uint8)
    codes = oracle.q8_nearest(r.normal(0, oracle.Q8_TOP[fmt] / 5, (n, 128)).clip(-oracle.Q8_TOP[fmt], oracle.Q8_TOP[fmt]), fmt)
    if n:
        codes[r.integers(0, n, 64), r.integers(0, 128, 64)] = good[r.integers(0, len(good), 64)]
    blocks = -(-n // block)
    scale = 2.0 ** np.round(np.log2(5 * sigma / oracle.Q8_TOP[fmt]) + r.integers(-2, 3, blocks))
    if general:
        scale = np.asarray(scale * r.uniform(1, 2, blocks), np.float32).astype(np.float64)
    return codes, scale


def bf16(x):
    return torch.as_tensor(np.asarray(x, np.float32)).to(torch.bfloat16)
