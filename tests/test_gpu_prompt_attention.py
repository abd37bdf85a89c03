"""Causal attention of packed prompts (fsx_prompt_attention) against the formula in 64 bits.

Tolerances, per element of the output: with A = sum_j P_j |v_j| and half a bf16 step u = 2^-8, the probabilities' rounding moves
an output by at most u A and the output's own rounding by u |O| (0 for an fp32 output).  A score is a sum of D products in fp32,
scaled once: it is off by at most ds = (D + 4) 2^-24 scale sum_c |q_c k_c|, which changes every weight by a factor within
exp(+-2 ds), and the statistics add (keys + 16) roundings of 2^-24.  The log sum moves by ds and the same roundings.
"""

from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from paper_2607_15621_amd import fsx

pytestmark = pytest.mark.gpu

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
U = torch.finfo(BF16).eps / 2


def reference(q, k, v, scale):
    """Output, tolerance without the output's rounding, log sums and their tolerance of one sequence, on the CPU in 64 bits:
    [rows][heads][channels] and [rows][heads].  Masked keys take no part."""
    n, H, D = q.shape
    m, G = k.shape[0], H // k.shape[1]
    q = q.to(BF16).to(F64)
    out, tol = torch.zeros(n, H, D, dtype=F64), torch.zeros(n, H, D, dtype=F64)
    lse, ltol = torch.full((n, H), -math.inf, dtype=F64), torch.zeros(n, H, dtype=F64)
    for h in range(H):
        kh, vh = k[:, h // G].to(F64), v[:, h // G].to(F64)
        x, mag = scale * (q[:, h] @ kh.t()), scale * (q[:, h].abs() @ kh.abs().t())
        for t in range(n):
            seen = m - n + t + 1
            if seen <= 0:
                continue
            s, big = x[t, :seen], mag[t, :seen].max()
            z = torch.logsumexp(s, 0)
            p = torch.exp(s - z)
            ds = (D + 4) * 2.0 ** -24 * big + (seen + 16) * 2.0 ** -24
            a = p @ vh[:seen].abs()
            out[t, h], tol[t, h] = p @ vh[:seen], a * (U + 4 * ds) + 1e-30
            lse[t, h], ltol[t, h] = z, 2 * ds + 2.0 ** -22 * z.abs() + 1e-7
    return out, tol, lse, ltol


def check(got, want, tol, what):
    got = got.detach().cpu().to(F64)
    assert got.shape == want.shape
    assert torch.equal(got.isnan(), want.isnan()), what
    ok = want.isnan() | (got == want) | ((got - want).abs() <= tol)
    worst = ((got - want).abs() / tol)[~ok]
    assert bool(ok.all()), (what, int((~ok).sum()), float(worst.max()))


class Case:
    def __init__(self, q_len, k_len=None, heads=4, kv_heads=4, dim=128, q_dtype=BF16, out_dtype=BF16, layout="packed", seed=0,
                 amp=1.0, gap=0, scale=0.0, kernel=fsx.PROMPT_AUTO):
        g = torch.Generator().manual_seed(seed)
        self.q_len, self.k_len = list(q_len), list(q_len if k_len is None else k_len)
        self.H, self.Hk, self.D, self.scale, self.kernel = heads, kv_heads, dim, scale, kernel
        # the sequences lie in reverse order, `gap` rows apart
        self.q_rows, self.k_rows = (fsx.PackedRows(n, self._starts(n, gap)) for n in (self.q_len, self.k_len))
        nq, nk = (int((r.start + r.len).max(initial=0)) + gap for r in (self.q_rows, self.k_rows))
        # (what the host holds is exact in the types that the device gets)
        self.hq = (torch.randn(nq, heads, dim, generator=g) * amp).to(q_dtype)
        self.hk = (torch.randn(nk, kv_heads, dim, generator=g) * amp).to(BF16)
        self.hv = torch.randn(nk, kv_heads, dim, generator=g).to(BF16)
        self.layout, self.out_dtype = layout, out_dtype

    @staticmethod
    def _starts(lens, gap):
        starts, at = [], gap
        for n in reversed(lens):
            starts.append(at)
            at += n + gap
        return starts[::-1]

    def place(self, t, dtype=None):
        """The tensor on the device in the layout under test, as [rows][heads][channels]."""
        t = t.cuda()
        if self.layout == "packed":
            return t.contiguous()
        if self.layout == "head_major":
            return t.transpose(0, 1).contiguous().transpose(0, 1)
        wide = torch.full((t.shape[0], t.shape[1] + 3, t.shape[2] + 24), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, 1:1 + t.shape[1], 8:8 + t.shape[2]] = t  # rows of a wider projection, other columns between the heads
        return wide[:, 1:1 + t.shape[1], 8:8 + t.shape[2]]

    def run(self, workspace=True, stream=None):
        q, k, v = self.place(self.hq), self.place(self.hk), self.place(self.hv)
        out = self.place(torch.full(tuple(self.hq.shape), 7.0, dtype=self.out_dtype))
        lse = torch.full(tuple(self.hq.shape[:2]), 7.0, device="cuda")
        need = fsx.prompt_attention_workspace(q, k, self.q_rows, self.k_rows, self.kernel)
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if workspace and need else None
        torch.cuda.synchronize()
        fsx.prompt_attention(q, k, v, out, self.q_rows, self.k_rows, self.scale, lse, ws, stream, self.kernel)
        torch.cuda.synchronize()
        return out, lse

    def check(self, out, lse):
        touched = torch.zeros(self.hq.shape[0], dtype=torch.bool)
        for i in range(len(self.q_len)):
            a, n, b, m = self.q_rows.start[i], self.q_len[i], self.k_rows.start[i], self.k_len[i]
            touched[a:a + n] = True
            o, tol, z, ztol = reference(self.hq[a:a + n], self.hk[b:b + m], self.hv[b:b + m],
                                        self.scale or 1 / math.sqrt(self.D))
            if self.out_dtype is BF16:
                tol = tol + U * (o.abs() + tol)
            check(out[a:a + n], o, tol, f"sequence {i}: output")
            check(lse[a:a + n], z, ztol, f"sequence {i}: log sums")
        rest = out.cpu()[~touched]
        assert bool((rest == 7.0).all()) and bool((lse.cpu()[~touched] == 7.0).all()), "rows outside the sequences"


# (head width, kernel): each kernel at each width that it takes, whatever the sizes would choose
KERNELS = [(64, fsx.PROMPT_CHUNKS), (64, fsx.PROMPT_TILES), (128, fsx.PROMPT_CHUNKS), (128, fsx.PROMPT_TILES), (128, fsx.PROMPT_TURNS)]
every_kernel = pytest.mark.parametrize("dim,kernel", KERNELS, ids=["64-chunks", "64-tiles", "128-chunks", "128-tiles", "128-turns"])
LENGTHS = [(1,), (2,), (17,), (31, 33), (64,), (65, 1, 63), (127, 128, 129), (200, 5), (257,), (1, 1, 1, 300, 0, 12)]


@every_kernel
@pytest.mark.parametrize("lens", LENGTHS, ids=str)
def test_whole_prompts(lens, dim, kernel):
    c = Case(lens, dim=dim, kernel=kernel, seed=len(lens) + lens[0])
    c.check(*c.run())


@every_kernel
@pytest.mark.parametrize("q_len,k_len", [((1,), (1,)), ((1, 1, 1), (700, 3, 1025)), ((4, 64), (2100, 65)), ((33, 1), (34, 900)),
                                         ((5, 3, 80), (2, 0, 40)), ((130, 7), (1300, 7)), ((16,) * 20, tuple(range(20, 420, 20)))],
                         ids=str)
def test_new_rows_over_a_history(q_len, k_len, dim, kernel):
    """Fewer queries than keys, and more (rows before the first key see nothing), with and without a workspace."""
    c = Case(q_len, k_len, heads=4, kv_heads=2, dim=dim, kernel=kernel, seed=sum(k_len))
    c.check(*c.run())
    c.check(*c.run(workspace=False))


@every_kernel
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 1), (6, 2), (5, 5), (32, 8), (40, 2)])
def test_grouped_heads(heads, kv_heads, dim, kernel):
    c = Case((70, 9), (70, 400), heads=heads, kv_heads=kv_heads, dim=dim, kernel=kernel, seed=heads)
    c.check(*c.run())
    c = Case((1, 1), (333, 64), heads=heads, kv_heads=kv_heads, dim=dim, kernel=kernel, seed=heads)
    c.check(*c.run())


@pytest.mark.parametrize("kernel", [fsx.PROMPT_CHUNKS, fsx.PROMPT_TILES, fsx.PROMPT_TURNS])
@pytest.mark.parametrize("layout", ["packed", "head_major", "wide"])
@pytest.mark.parametrize("q_dtype,out_dtype", [(BF16, BF16), (F32, BF16), (BF16, F32), (F32, F32)], ids=str)
def test_layouts_and_types(layout, q_dtype, out_dtype, kernel):
    c = Case((90, 33, 2), (90, 200, 1000), heads=4, kv_heads=2, q_dtype=q_dtype, out_dtype=out_dtype, layout=layout, gap=3, seed=5,
             kernel=kernel)
    c.check(*c.run())


@every_kernel
@pytest.mark.parametrize("amp,scale", [(0.0, 0.0), (30.0, 0.0), (1.0, 2.5), (100.0, 1.0), (1e-20, 0.0)])
def test_flat_and_peaked_softmax(amp, scale, dim, kernel):
    c = Case((150, 1), (150, 600), heads=2, kv_heads=2, amp=amp, scale=scale, dim=dim, kernel=kernel, seed=9)
    c.check(*c.run())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@every_kernel
def test_masked_places_may_hold_anything(bad, dim, kernel):
    """Rows between and behind the sequences, and keys and values after a token's own place."""
    c = Case((100, 40, 1), (100, 170, 500), heads=4, kv_heads=2, dim=dim, kernel=kernel, gap=70, seed=21)
    inside = torch.zeros(c.hk.shape[0], dtype=torch.bool)
    for i in range(3):
        inside[c.k_rows.start[i]:c.k_rows.start[i] + c.k_len[i]] = True
    c.hk[~inside] = bad
    c.hv[~inside] = bad
    for i, t in ((0, 97), (0, 33), (1, 169), (1, 150)):
        c.hv[c.k_rows.start[i] + t, t % 2, 5] = bad  # a value that later rows see, and those before them do not
    out, lse = c.run()
    for i in range(3):
        a, n, b, m = c.q_rows.start[i], c.q_len[i], c.k_rows.start[i], c.k_len[i]
        v = c.hv[b:b + m].clone()
        hit = ~torch.isfinite(v.float())
        v[hit] = 0
        o, tol, z, ztol = reference(c.hq[a:a + n], c.hk[b:b + m], v, 1 / math.sqrt(dim))
        for t, h, ch in hit.nonzero().tolist():
            o[max(0, t - (m - n)):, 2 * h:2 * h + 2, ch] += bad  # the weight is positive
        check(out[a:a + n], o, tol + U * (o.nan_to_num(0, 0, 0).abs() + tol), f"sequence {i}: output")
        check(lse[a:a + n], z, ztol, f"sequence {i}: log sums")


@every_kernel
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_masked_keys_that_are_not_finite(bad, dim, kernel):
    """A key that is not finite spoils the rows that see it (here: to NaN, whose scores then have no maximum) and no other."""
    c = Case((120,), heads=2, kv_heads=2, dim=dim, kernel=kernel, seed=22)
    c.hk[100:, 1] = bad
    out, lse = c.run()
    o, tol, z, ztol = reference(c.hq[:100], c.hk[:100], c.hv[:100], 1 / math.sqrt(dim))
    check(out[:100], o, tol + U * (o.abs() + tol), "rows before")
    check(lse[:100], z, ztol, "rows before")
    if math.isnan(bad):
        assert bool(out[100:, 1].isnan().all())


@every_kernel
def test_the_same_bits_every_time_and_on_another_stream(dim, kernel):
    c = Case((130, 1, 64), (1300, 2000, 64), heads=8, kv_heads=2, dim=dim, kernel=kernel, seed=4)
    out, lse = c.run()
    for stream in (None, torch.cuda.Stream()):
        again, lse2 = c.run(stream=stream)
        assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse, lse2)


def test_captured_calls_are_replayed():
    """Two graphs with a workspace each, replayed in turn with other inputs between, against eager calls."""
    runs = []
    for seed in (1, 2):
        c = Case((60, 1, 1), (60, 900, 2000), heads=8, kv_heads=2, seed=seed)
        q, k, v = c.place(c.hq), c.place(c.hk), c.place(c.hv)
        out, need = torch.empty_like(q), fsx.prompt_attention_workspace(q, k, c.q_rows, c.k_rows)
        ws = torch.empty(max(16, need), dtype=torch.uint8, device="cuda")
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            fsx.prompt_attention(q, k, v, out, c.q_rows, c.k_rows, workspace=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            fsx.prompt_attention(q, k, v, out, c.q_rows, c.k_rows, workspace=ws)
        runs.append((c, q, k, v, out, ws, graph))
    for turn in range(3):
        for c, q, k, v, out, ws, graph in runs:
            q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(50 + turn)).to(BF16))
            out.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            got, want = out.clone(), torch.empty_like(out)
            fsx.prompt_attention(q, k, v, want, c.q_rows, c.k_rows, workspace=torch.empty_like(ws))
            torch.cuda.synchronize()
            assert torch.equal(got.view(torch.int16), want.view(torch.int16)), turn


def test_offsets_beyond_32_bits():
    """Keys and values of the last of many rings: more than 2^32 elements before them."""
    c = Case((3, 1), (70, 500), heads=2, kv_heads=1, seed=8)
    far = (1 << 25) + 11  # rows of 128 channels: 2^32 elements
    big = torch.empty(far + 600, 1, 128, dtype=BF16, device="cuda")
    big[far:far + c.hk.shape[0]] = c.hk.cuda()
    bigv = torch.empty(far + 600, 1, 128, dtype=BF16, device="cuda")
    bigv[far:far + c.hv.shape[0]] = c.hv.cuda()
    q, out = c.hq.cuda(), torch.full(tuple(c.hq.shape), 7.0, dtype=BF16, device="cuda")
    lse = torch.full(tuple(c.hq.shape[:2]), 7.0, device="cuda")
    rows = fsx.PackedRows(c.k_len, c.k_rows.start + far)
    for kernel in (fsx.PROMPT_CHUNKS, fsx.PROMPT_TILES, fsx.PROMPT_TURNS):
        out.fill_(7.0)
        lse.fill_(7.0)
        fsx.prompt_attention(q, big, bigv, out, c.q_rows, rows, lse=lse, kernel=kernel)
        torch.cuda.synchronize()
        c.check(out, lse)


@pytest.mark.parametrize("layout", [fsx.CACHE_HEAD_MAJOR, fsx.CACHE_TOKEN_MAJOR])
def test_keys_where_they_stand_in_a_cache(layout):
    """One layer of a bf16 cache whose rings have not wrapped, read in place: rows and heads are strides of the cache."""
    B, L, H, cap, D, layer = 3, 2, 4, 150, 128, 1
    c = Case((1, 9, 70), (100, 37, 150), heads=8, kv_heads=H, seed=3)
    shape = (B, L, cap, H, D) if layout == fsx.CACHE_TOKEN_MAJOR else (B, L, H, cap, D)
    k, v = (torch.full(shape, float("nan"), dtype=BF16, device="cuda") for _ in "kv")
    for b in range(B):
        for t, h in ((k, c.hk), (v, c.hv)):
            rows = h[c.k_rows.start[b]:c.k_rows.start[b] + c.k_len[b]].cuda()
            if layout == fsx.CACHE_TOKEN_MAJOR:
                t[b, layer, :c.k_len[b]] = rows
            else:
                t[b, layer, :, :c.k_len[b]] = rows.transpose(0, 1)
    if layout == fsx.CACHE_TOKEN_MAJOR:
        view = [t.view(B * L * cap, H, D) for t in (k, v)]
        starts = [(b * L + layer) * cap for b in range(B)]
    else:  # rows of one head; the heads lie cap rows apart
        n = B * L * H * cap - (H - 1) * cap
        view = [t.view(-1).as_strided((n, H, D), (D, cap * D, 1)) for t in (k, v)]
        starts = [(b * L + layer) * H * cap for b in range(B)]
    out = torch.full(tuple(c.hq.shape), 7.0, dtype=BF16, device="cuda")
    lse = torch.full(tuple(c.hq.shape[:2]), 7.0, device="cuda")
    fsx.prompt_attention(c.hq.cuda(), *view, out, c.q_rows, fsx.PackedRows(c.k_len, starts), lse=lse)
    torch.cuda.synchronize()
    c.check(out, lse)


def long_reference(q, k, v, scale, bad=()):
    """As reference(), vectorised on the GPU in 64 bits; bad: (key, key head, channel, value) of values that are not finite, 0 in
    v, added to the rows that see them."""
    n, H, D = q.shape
    m, G = k.shape[0], H // k.shape[1]
    out, tol = (torch.empty(n, H, D, dtype=F64, device="cuda") for _ in range(2))
    lse, ltol = (torch.empty(n, H, dtype=F64, device="cuda") for _ in range(2))
    for h in range(H):
        kh, vh = k[:, h // G].cuda().to(F64), v[:, h // G].cuda().to(F64)
        for a in range(0, n, 1024):
            x = q[a:a + 1024, h].cuda().to(BF16).to(F64)
            seen = torch.arange(m, device="cuda")[None] <= (m - n + a + torch.arange(len(x), device="cuda"))[:, None]
            s = torch.where(seen, scale * (x @ kh.t()), torch.full((), -math.inf, dtype=F64, device="cuda"))
            big = torch.where(seen, scale * (x.abs() @ kh.abs().t()), torch.zeros((), dtype=F64, device="cuda")).amax(1)
            z = torch.logsumexp(s, 1)
            p = torch.exp(s - z[:, None])
            ds = (D + 4) * 2.0 ** -24 * big + (m + 16) * 2.0 ** -24
            out[a:a + 1024, h], tol[a:a + 1024, h] = p @ vh, (p @ vh.abs()) * (U + 4 * ds)[:, None] + 1e-30
            lse[a:a + 1024, h], ltol[a:a + 1024, h] = z, 2 * ds + 2.0 ** -22 * z.abs() + 1e-7
    tol = tol + U * (out.abs() + tol)
    for j, hk, ch, x in bad:
        out[max(0, j - (m - n)):, hk * G:(hk + 1) * G, ch] += x
    return [t.cpu() for t in (out, tol, lse, ltol)]


@every_kernel
@pytest.mark.parametrize("q_len,k_len,heads,kv_heads", [((4500,), (4500,), 2, 2), ((4097, 700), (5000, 700), 6, 2), ((2049,), (9000,), 8, 1),
                                                        ((130, 1, 60), (9001, 6000, 6100), 40, 2)], ids=str)
def test_long_prompts(q_len, k_len, heads, kv_heads, dim, kernel):
    c = Case(q_len, k_len, heads=heads, kv_heads=kv_heads, dim=dim, kernel=kernel, seed=31)
    for spoilt in (False, True):
        bad = [[] for _ in q_len]
        if spoilt:  # values that are not finite, in tiles that all rows see, that some see, and the last key
            for i, m in enumerate(c.k_len):
                for j, ch, x in ((3, 0, math.inf), (m - q_len[i] // 2, 5, math.nan), (m - q_len[i] // 2 + 1, 9, -math.inf), (m - 1, 33, math.inf)):
                    if j < m:
                        c.hv[c.k_rows.start[i] + j, j % kv_heads, ch] = x
                        bad[i].append((j, j % kv_heads, ch, x))
        out, lse = c.run()
        for i, n in enumerate(q_len):
            a, b, m = c.q_rows.start[i], c.k_rows.start[i], k_len[i]
            v = c.hv[b:b + m].clone()
            v[~torch.isfinite(v.float())] = 0
            o, tol, z, ztol = long_reference(c.hq[a:a + n], c.hk[b:b + m], v, 1 / math.sqrt(dim), bad[i])
            check(out[a:a + n], o, tol, f"sequence {i}: output")
            check(lse[a:a + n], z, ztol, f"sequence {i}: log sums")


def test_as_many_sequences_as_there_may_be():
    """64 sequences, some without queries or keys, whole prompts among new rows over a history."""
    q_len = [(7 * i) % 40 for i in range(64)]
    k_len = [n if i % 3 else n + 50 * (i % 5) - 20 * (i % 2) for i, n in enumerate(q_len)]
    k_len = [max(0, n) for n in k_len]
    for dim, kernel in KERNELS + [(64, fsx.PROMPT_AUTO), (128, fsx.PROMPT_AUTO)]:
        c = Case(q_len, k_len, heads=2, kv_heads=1, dim=dim, kernel=kernel, gap=1, seed=77)
        c.check(*c.run())


def test_a_workspace_of_any_size_gives_the_output():
    c = Case((1, 3), (3000, 2000), heads=8, kv_heads=2, seed=13)
    q, k, v = c.place(c.hq), c.place(c.hk), c.place(c.hv)
    need = fsx.prompt_attention_workspace(q, k, c.q_rows, c.k_rows)
    assert need > 0
    for size in (0, 16, need // 7 * 16 // 16, need // 2, need, 2 * need):
        out, lse = torch.full(tuple(c.hq.shape), 7.0, dtype=BF16, device="cuda"), torch.full(tuple(c.hq.shape[:2]), 7.0, device="cuda")
        ws = torch.full((size + 64,), 0x7F, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        fsx.prompt_attention(q, k, v, out, c.q_rows, c.k_rows, lse=lse, workspace=ws[:size] if size else None)
        torch.cuda.synchronize()
        c.check(out, lse)
        assert bool((ws[size:] == 0x7F).all()), "behind the workspace"


def test_two_calls_at_once():
    """Calls on two streams, a workspace each, against the same calls one after the other."""
    calls = []
    for seed in (1, 2):
        c = Case((64, 1, 300), (900, 3000, 300), heads=8, kv_heads=2, seed=seed)
        t = [c.place(x) for x in (c.hq, c.hk, c.hv)]
        need = fsx.prompt_attention_workspace(t[0], t[1], c.q_rows, c.k_rows)
        calls.append((c, t, [torch.empty_like(t[0]) for _ in range(6)], torch.empty(max(16, need), dtype=torch.uint8, device="cuda"),
                      torch.cuda.Stream()))
    torch.cuda.synchronize()
    for i in range(6):
        for c, t, out, ws, stream in calls:
            fsx.prompt_attention(*t, out[i], c.q_rows, c.k_rows, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    for c, t, out, ws, stream in calls:
        want = torch.empty_like(t[0])
        fsx.prompt_attention(*t, want, c.q_rows, c.k_rows, workspace=ws)
        torch.cuda.synchronize()
        for o in out:
            assert torch.equal(o.view(torch.int16), want.view(torch.int16))
