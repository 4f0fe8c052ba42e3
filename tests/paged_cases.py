"""Paged-cache cases and their definitions in float64, shared by the paged tests."""
from __future__ import annotations

import numpy as np
import torch

QMAX = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}
MIN_AMAX = 2.0 ** -110


def quantise(x: torch.Tensor, dtype: torch.dtype):
    """x float32 [..., dh] -> (codes, scales) as the header defines them, in fp32."""
    bad = ~torch.isfinite(x).all(-1)
    x = torch.where(bad[..., None], torch.zeros_like(x), x)
    amax = x.abs().amax(-1).clamp_min(MIN_AMAX)
    y = x * torch.full_like(amax, QMAX[dtype]).div(amax)[..., None]  # (number / tensor would round twice)
    codes = (y.round().clamp(-127, 127) if dtype == torch.int8 else y.clamp(-448, 448)).to(dtype)
    scale = torch.where(bad, torch.full_like(amax, float("nan")), amax / QMAX[dtype])
    return codes, scale


class Case:
    """Sequences with rows[b] new tokens at the end of kv[b] cached positions.  What no sequence owns is poisoned: NaN
    in free pages and behind the last position of a page, page numbers far outside the pool behind a sequence's
    last page, and `pad` packed rows behind the last sequence."""

    def __init__(self, dtype, heads, kv_heads, dh, page, rows, kv, seed, pad=3, width_extra=2, strided=True):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.H, self.KV, self.dh, self.ps = dtype, heads, kv_heads, dh, page
        self.rows, self.kv = list(rows), list(kv)
        B = len(self.rows)
        need = [-(-k // page) for k in self.kv]
        n_pages = sum(need) + 2
        perm = torch.randperm(n_pages, generator=g)
        self.table = torch.full((B, max(max(need), 1) + width_extra), 1 << 29, dtype=torch.int32)
        x = [torch.full((n_pages, kv_heads, page, dh), float("nan")) for _ in range(2)]
        at = 0
        for b in range(B):
            self.table[b, :need[b]] = perm[at:at + need[b]].int()
            for p in range(need[b]):
                m = min(page, self.kv[b] - p * page)
                for t in x:
                    t[perm[at + p], :, :m] = torch.randn(kv_heads, m, dh, generator=g)
            at += need[b]
        x[0] *= 1.5  # keys: scores spread over several units
        self.set_pools(*[t.to(torch.bfloat16) for t in x])
        self.cu = np.concatenate([[0], np.cumsum(self.rows)]).astype(np.int32)
        self.n = int(self.cu[-1]) + pad
        w = (heads + 2 * kv_heads) * dh
        self.qkv = torch.randn(self.n, w + (8 if strided else 0), generator=g).to(torch.bfloat16)
        dq, dkv = heads * dh, kv_heads * dh
        self.q, self.k_new, self.v_new = self.qkv[:, :dq], self.qkv[:, dq:dq + dkv], self.qkv[:, dq + dkv:dq + 2 * dkv]
        self.max_rows = max(1, max(self.rows))

    def set_pools(self, k, v):
        self.k_scale = self.v_scale = None
        if self.dtype == torch.bfloat16:
            self.k, self.v = k, v
        else:
            self.k, self.k_scale = quantise(k.float(), self.dtype)
            self.v, self.v_scale = quantise(v.float(), self.dtype)

    def device(self, dev="cuda:0"):
        """(KVCache, PagedRows) on the device; q, k_new, v_new as slices of one packed matrix there."""
        from paper_2509_24257_b200 import binding as vb

        put = lambda t: None if t is None else t.to(dev)  # noqa: E731
        cache = vb.KVCache(put(self.k), put(self.v), put(self.k_scale), put(self.v_scale))
        rows = vb.PagedRows(put(self.table), torch.from_numpy(self.cu).to(dev), torch.tensor(self.kv, dtype=torch.int32, device=dev),
                            self.max_rows, torch.zeros(1, dtype=torch.int32, device=dev))
        m = self.qkv.to(dev)
        dq, dkv = self.H * self.dh, self.KV * self.dh
        self.dq, self.dk_new, self.dv_new = m[:, :dq], m[:, dq:dq + dkv], m[:, dq + dkv:dq + 2 * dkv]
        return cache, rows

    def positions(self, b):
        """float64 k, v [kv][KV][dh] of sequence b."""
        n = -(-self.kv[b] // self.ps)
        pages = self.table[b, :n].long()
        out = []
        for pool, scale in ((self.k, self.k_scale), (self.v, self.v_scale)):
            x = (pool.view(torch.uint8)[pages].view(pool.dtype) if pool.element_size() == 1 else pool[pages]).double()
            if scale is not None:
                x = x * scale[pages].double()[..., None]
            out.append(x.transpose(1, 2).reshape(n * self.ps, self.KV, self.dh)[:self.kv[b]])
        return out

    def attention(self):
        """(out [n][H][dh], tolerance of it, lse [n][H], tolerance of it) in float64; rows behind the last sequence 0.

        Tolerance: with u = 2^-8 the half step of bf16 and e = 2^-24 that of float32, the probabilities are rounded to
        bf16 (u of sum p |v|) and the output is (u of |out|).  A score is a float32 sum of dh products and up to
        three factors: off by at most d = (dh + 4) e sum |q_d k_d| / sqrt(dh), which changes a probability by a
        factor within 1 +- 2 d and its exponential by 2^-21 more (exp2 in float32 of an argument below 64 in size);
        the products and sums over L keys in float32 add at most (L + 64) e of sum p |v|.
        With 8-bit pools the products may run in float16, operands and probabilities scaled so that the largest lies near
        its top: a key or value entry is rounded to 11 bits (half = 2^-11), which adds half sum |q_d k_d| / sqrt(dh) to
        a score and half to the factor of sum p |v|, or is off by at most 2^-30 of the largest; a query row is scaled
        so that its largest entry lies in [1, 2), so an entry is off by at most 2^-25 of the largest; a probability is
        rounded to 11 bits (within u) or, for each key, off by 2^-31 where they sum to 1 or more."""
        n, H, dh = self.n, self.H, self.dh
        out, tol = torch.zeros(n, H, dh, dtype=torch.float64), torch.zeros(n, H, dh, dtype=torch.float64)
        lse, ltol = torch.full((n, H), -float("inf"), dtype=torch.float64), torch.zeros(n, H, dtype=torch.float64)
        u, e, half = 2.0 ** -8, 2.0 ** -24, 0.0 if self.dtype == torch.bfloat16 else 2.0 ** -11
        for b, nb in enumerate(self.rows):
            if nb == 0 or self.kv[b] == 0:
                continue
            k, v = self.positions(b)
            L, r0 = self.kv[b], int(self.cu[b])
            q = self.q[r0:r0 + nb].double().reshape(nb, H, dh)
            pos = torch.arange(L - nb, L)
            keep = torch.arange(L)[None, :] <= pos[:, None]
            for h in range(H):
                kh = h * self.KV // H
                s = (q[:, h] @ k[:, kh].T) / dh ** 0.5
                size = torch.where(keep, q[:, h].abs() @ k[:, kh].abs().T / dh ** 0.5, torch.zeros(()).double())
                d = (dh + 4) * e * size.nan_to_num(0, 0, 0).amax(-1)
                tiny = 0.0
                if self.dtype != torch.bfloat16:
                    row = torch.where(keep, k[:, kh].abs().sum(-1)[None].expand(nb, L), torch.zeros(()).double()).nan_to_num(0, 0, 0)
                    d = d + 2.0 ** -24 * q[:, h].abs().amax(-1) * row.amax(-1) / dh ** 0.5
                    d = d + half * size.nan_to_num(0, 0, 0).amax(-1)
                    vmax = v[:, kh].abs().nan_to_num(0, 0, 0).amax()
                    tiny = L * 2.0 ** -30 * float(vmax)
                s = torch.where(keep, s, torch.full((), -float("inf")).double())
                some = keep.any(-1)
                lse[r0:r0 + nb, h] = torch.logsumexp(s, -1)
                ltol[r0:r0 + nb, h] = d + 2.0 ** -20 + (L + 64) * e + lse[r0:r0 + nb, h].abs().nan_to_num(0, 0, 0) * 2.0 ** -21
                p = torch.where(some[:, None], torch.softmax(s, -1), torch.zeros(()).double())
                # a hidden key's value does not enter, whatever it is
                for cols, dst, x in ((slice(0, dh), out, v[:, kh]), (slice(0, dh), tol, v[:, kh].abs())):
                    clean = torch.isfinite(x).all()
                    y = p @ x if clean else torch.where(keep[:, :, None], p[:, :, None] * x[None], torch.zeros(()).double()).sum(1)
                    dst[r0:r0 + nb, h, cols] = torch.where(some[:, None], y, torch.zeros(()).double())
                tol[r0:r0 + nb, h] = tol[r0:r0 + nb, h] * (u + half + 2 * d[:, None] + 2.0 ** -21 + (L + 64) * e) * (1 + u) + u * out[r0:r0 + nb, h].abs() + tiny
        return out, tol, lse, ltol


def assert_within(got: torch.Tensor, ref: torch.Tensor, tol: torch.Tensor, what=""):
    """Finite entries within `tol` elementwise; infinities and NaN in the same places."""
    got, ref = got.double().cpu(), ref.double()
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), what + ": NaN elsewhere"
    inf = torch.isinf(ref)
    assert torch.equal(got[inf], ref[inf]), what + ": infinities differ"
    over = (got - ref).abs()[fine] - tol[fine]
    assert torch.isfinite(got[fine]).all() and (over.numel() == 0 or float(over.max()) <= 0.0), f"{what}: {float(over.max())} over the tolerance"
