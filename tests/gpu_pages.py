"""Pages on the device beside sequences that the host keeps as plain tensors: what the tests of the pages share."""

from __future__ import annotations

import math

import numpy as np
import torch

from paper_2607_15621_amd import fsx

BF16, F32, F64, FP8, U8 = torch.bfloat16, torch.float32, torch.float64, torch.float8_e4m3fn, torch.uint8
U = torch.finfo(BF16).eps / 2


def encode(x):
    """Codes and scales of fp8 rows [..., channels], in fp32 step by step."""
    x = x.to(F32)
    top = torch.where(torch.isfinite(x), x.abs(), torch.zeros(())).amax(-1).numpy()
    scale = np.maximum(top / np.float32(448.0), np.float32(2.0 ** -126)).astype(np.float32)
    scale = torch.from_numpy(np.where(top > 0, scale, np.float32(1.0)).astype(np.float32))
    with np.errstate(invalid="ignore"):
        q = torch.from_numpy(x.numpy() / scale.numpy()[..., None])  # one fp32 division, correctly rounded
    code = q.clamp(-448.0, 448.0).to(FP8).view(U8)
    return torch.where(q.isnan(), torch.where(torch.signbit(q), 0xFF, 0x7F).to(U8), code), scale


class Pool:
    """A pool whose rows all hold NaN, and what every sequence's rows should be: lists of (k, v, k_scale, v_scale) of a row, each
    [layers][heads](..)."""

    def __init__(self, pages=40, seqs=8, most=12, L=2, H=2, P=16, D=128, fp8=False):
        self.L, self.H, self.P, self.D, self.fp8, self.seqs = L, H, P, D, fp8, seqs
        shape = (L, pages, H, P, D)
        if fp8:
            self.k, self.v = (torch.full(shape, 0x7F, dtype=U8, device="cuda") for _ in "kv")
            self.ks, self.vs = (torch.full(shape[:4], math.nan, device="cuda") for _ in "kv")
        else:
            self.k, self.v = (torch.full(shape, math.nan, dtype=BF16, device="cuda") for _ in "kv")
            self.ks = self.vs = None
        self.pages = fsx.Pages(self.k, self.v, seqs, most, self.ks, self.vs)
        self.rows = [[] for _ in range(seqs)]
        self.g = torch.Generator().manual_seed(pages + seqs + P)

    def new(self, n, dtype=BF16, amp=1.0):
        """Packed rows [layers][n][heads][channels]."""
        return tuple((torch.randn(self.L, n, self.H, self.D, generator=self.g) * amp).to(dtype) for _ in "kv")

    def stored(self, k, v):
        """What pages hold of packed rows, a row at a time."""
        if not self.fp8:
            k, v = k.to(BF16), v.to(BF16)
            return [(k[:, r], v[:, r]) for r in range(k.shape[1])]
        (k, ks), (v, vs) = encode(k), encode(v)
        return [(k[:, r], v[:, r], ks[:, r], vs[:, r]) for r in range(k.shape[1])]

    def extend(self, seqs, counts, dtype=BF16, write=True, stream=None):
        self.pages.extend(seqs, counts, stream=stream)
        if write:
            k, v = self.new(sum(counts), dtype)
            self.pages.write(0, self.L, k.cuda(), v.cuda(), seqs, fsx.PackedRows(counts), stream=stream)
            at, stored = 0, self.stored(k, v)
            for s, n in zip(seqs, counts):
                self.rows[s] += stored[at:at + n]
                at += n

    def fork(self, src, dst, rows=None):
        self.pages.fork(src, dst, rows)
        for i, (a, b) in enumerate(zip(src, dst)):
            self.rows[b] = list(self.rows[a][:None if rows is None else rows[i]])

    def keep(self, seqs, ranges):
        self.pages.keep(seqs, ranges)
        for s, r in zip(seqs, ranges):
            self.rows[s] = [x for a, n in r for x in self.rows[s][a:a + n]]

    def free(self, seqs):
        self.pages.free(seqs)
        for s in seqs:
            self.rows[s] = []

    def check(self):
        """Every sequence's rows, bit for bit, and that no other row of the pool was written since it was last looked at."""
        table, length = self.pages.tables()
        tensors = [t.cpu() for t in (self.k, self.v, self.ks, self.vs) if t is not None]
        for s in range(self.seqs):
            assert length[s] == len(self.rows[s]), s
            for i, row in enumerate(self.rows[s]):
                page = int(table[s, i // self.P])
                for t, want in zip(tensors, row):
                    got = t[:, page, :, i % self.P].contiguous()
                    a, b = (x.view(torch.int16 if x.dtype is BF16 else torch.int32 if x.dtype is F32 else U8) for x in (got, want.contiguous()))
                    assert torch.equal(a, b), (s, i)

    def decoded(self, s, layer):
        """Keys and values of sequence s, [rows][heads][channels] in 64 bits."""
        if not self.rows[s]:
            return (torch.zeros(0, self.H, self.D, dtype=F64),) * 2
        parts = [torch.stack([r[i][layer] for r in self.rows[s]]) for i in range(len(self.rows[s][0]))]
        if self.fp8:
            return tuple(c.view(FP8).to(F64) * x.to(F64)[..., None] for c, x in ((parts[0], parts[2]), (parts[1], parts[3])))
        return parts[0].to(F64), parts[1].to(F64)


def attend(q, k, v, scale, weight=2.0 ** -15):
    """One token's attention in 64 bits: q [heads][channels], k, v [rows][key heads][channels]; output, its tolerance without the
    output's rounding, log sums and theirs.

    With A = sum_j P_j |v_j|: a weight is two bf16 values, the first cut off (at most a step, 2^-7, is left), the second what is left
    rounded by at most half a step, 2^-8 of that, so an output moves by at most 2^-15 A (fsx_prompt_attention rounds them once: `weight` is U there).  A score is a sum of D products in fp32, scaled (an fp8 row's scale among it) by two roundings more: off by at most
    ds = (D + 6) 2^-24 scale sum_c |q_c k_c|, which changes every weight by a factor within exp(+-2 ds); the exponentials are off by
    2^-22, and the statistics, sums and the merges of parts add (rows + 64) roundings of 2^-24."""
    q = q.to(BF16).to(F64)
    H, D = q.shape
    n, G = k.shape[0], H // k.shape[1]
    out, tol, lse, ltol = torch.zeros(H, D, dtype=F64), torch.zeros(H, D, dtype=F64), torch.full((H,), -math.inf, dtype=F64), torch.zeros(H, dtype=F64)
    if n == 0:
        return out, tol, lse, ltol
    for h in range(H):
        kh, vh = k[:, h // G], v[:, h // G]
        s, big = scale * (kh @ q[h]), (scale * (kh.abs() @ q[h].abs())).max()
        z = torch.logsumexp(s, 0)
        p = torch.exp(s - z)
        ds = (D + 6) * 2.0 ** -24 * big + (n + 64) * 2.0 ** -24 + 2.0 ** -22
        out[h], tol[h] = p @ vh, (p @ vh.abs()) * (weight + 4 * ds) + 1e-30
        lse[h], ltol[h] = z, 2 * ds + 2.0 ** -22 * z.abs() + 1e-7
    return out, tol, lse, ltol


def check_attention(pool, layer, q, out, lse, seqs, scale=0.0, what=""):
    for i, s in enumerate(seqs):
        k, v = pool.decoded(s, layer)
        o, tol, z, ztol = attend(q[i].cpu(), k, v, scale or 1 / math.sqrt(pool.D))
        if out.dtype is BF16:
            tol = tol + U * (o.abs() + tol)
        got = out[i].cpu().to(F64)
        near(got, o, tol, f"{what} entry {i} sequence {s}: output")
        if lse is not None:
            near(lse[i].cpu().to(F64), z, ztol, f"{what} entry {i} sequence {s}: log sums")


def near(got, want, tol, what):
    assert torch.equal(got.isnan(), want.isnan()), what
    ok = want.isnan() | (got == want) | ((got - want).abs() <= tol)
    assert bool(ok.all()), (what, int((~ok).sum()), float(((got - want).abs() / tol)[~ok].max()))
