"""Rows of a cache replaced by packed rows (fsx_cache_replace_rows: an fp8 cache's scales found from them) and read back
(fsx_cache_read_rows), bit for bit against the definitions computed on the CPU."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2607_15621_amd import fsx

pytestmark = pytest.mark.gpu

BF16, F32, FP8, U8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.uint8
TOKEN, HEAD = fsx.CACHE_TOKEN_MAJOR, fsx.CACHE_HEAD_MAJOR
BITS = {BF16: torch.int16, F32: torch.int32, U8: torch.uint8}


def bits(t):
    return t.contiguous().view(BITS[t.dtype]).cpu()


class Rings:
    """A device cache with every byte set to a pattern, and its descriptor."""

    def __init__(self, lengths, cap, L=2, H=3, D=128, dtype=U8, layout=HEAD, starts=None, agents=None):
        B = len(lengths)
        self.L, self.H, self.D, self.cap, self.layout, self.dtype = L, H, D, cap, layout, dtype
        shape = (agents or B, L, cap, H, D) if layout & TOKEN else (agents or B, L, H, cap, D)
        g = torch.Generator().manual_seed(7)
        if dtype is U8:
            host = [(torch.randn(shape, generator=g) * 60).clamp(-448, 448).to(FP8).view(U8) for _ in "kv"]
            sc = [torch.rand((agents or B, L, H), generator=g) + 0.01 for _ in "kv"]
        else:
            host, sc = [torch.randn(shape, generator=g).to(dtype) for _ in "kv"], [None, None]
        self.host, self.host_scale = host, sc
        self.k, self.v = (t.cuda() for t in host)
        self.scale = [t.cuda() if t is not None else None for t in sc]
        self.desc = fsx.CacheDesc(self.k, self.v, {U8: fsx.FP8_E4M3, BF16: fsx.BF16, F32: fsx.F32}[dtype], L, H, D, cap, lengths,
                                  starts=starts, k_scale=self.scale[0], v_scale=self.scale[1], layout=layout)
        torch.cuda.synchronize()

    def slots(self, host, b, l):
        """[slots][H][D] of a host copy."""
        return host[b, l] if self.layout & TOKEN else host[b, l].transpose(0, 1)


def scale_of(x, headroom):
    """Per head, from rows [n][H][D] fp32, in fp32 step by step."""
    a = x.abs()
    top = torch.where(torch.isfinite(a), a, torch.zeros(())).amax((0, 2)).numpy()
    s = np.maximum(top / np.float32(448.0) * np.float32(headroom), np.float32(2.0 ** -126)).astype(np.float32)
    return torch.from_numpy(np.where(top > 0, s, np.float32(1.0)).astype(np.float32))


def codes_of(x, scale):
    with np.errstate(invalid="ignore"):
        q = torch.from_numpy(x.numpy() / scale.numpy()[None, :, None])  # one fp32 division, correctly rounded
    code = q.clamp(-448.0, 448.0).to(FP8).view(U8)
    return torch.where(q.isnan(), torch.where(torch.signbit(q), 0xFF, 0x7F).to(U8), code)


def expect_replaced(r, layer, n_layers, rows, lens, starts, headroom):
    """The caches and scales that r holds after the call, on the host."""
    out, scales = [t.clone() for t in r.host], [t.clone() if t is not None else None for t in r.host_scale]
    for i in range(2):
        for b, n in enumerate(lens):
            kept = min(n, r.cap)
            if n == 0:
                continue
            for l in range(n_layers):
                x = rows[i][l, starts[b] + n - kept:starts[b] + n].float()
                if r.dtype is U8:
                    scales[i][b, layer + l] = scale_of(x, headroom)
                    x = codes_of(x, scales[i][b, layer + l])
                r.slots(out[i], b, layer + l)[:kept] = x.to(r.dtype)
    return out, scales


def replace_and_check(r, lens, rows, layer=0, n_layers=None, starts=None, headroom=1.0, stream=None):
    n_layers = n_layers or r.L
    packed = fsx.PackedRows(lens, starts)
    before = [list(x) for x in (r.desc.start, r.desc.len, r.desc.pos)]
    dev = [t.cuda() for t in rows]
    torch.cuda.synchronize()
    fsx.cache_replace_rows(r.desc, layer, n_layers, *dev, packed, headroom=headroom, stream=stream)
    torch.cuda.synchronize()
    want, scales = expect_replaced(r, layer, n_layers, rows, lens, packed.start, headroom)
    for i, t in enumerate((r.k, r.v)):
        if scales[i] is not None:
            assert torch.equal(r.scale[i].cpu(), scales[i]), "scales"
        assert torch.equal(bits(t), bits(want[i])), ("keys", "values")[i]
    for b, n in enumerate(lens):
        state = [int(x[b]) for x in (r.desc.start, r.desc.len, r.desc.pos)]
        assert state == ([0, min(n, r.cap), n] if n else [x[b] for x in before])
    r.host, r.host_scale = want, scales


def packed_rows(L, total, H, D, dtype, seed=0, amp=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(L, total, H, D, generator=g) * amp).to(dtype) for _ in "kv"]


@pytest.mark.parametrize("layout", [HEAD, TOKEN])
@pytest.mark.parametrize("source", [BF16, F32])
@pytest.mark.parametrize("lens", [(1, 1), (5, 0, 8), (37,), (224, 1, 300), (700, 1100), (2500,), (0, 5000, 3)], ids=str)
def test_fp8_rows_and_their_scales(lens, source, layout):
    r = Rings([0] * len(lens), max(lens) + 5, layout=layout)
    replace_and_check(r, lens, packed_rows(2, sum(lens), 3, 128, source, seed=sum(lens)), headroom=1.25)


@pytest.mark.parametrize("D", [16, 32, 48, 64, 80, 128, 256, 512])
@pytest.mark.parametrize("layout", [HEAD, TOKEN])
def test_head_widths(D, layout):
    r = Rings([3, 0], 40, L=1, H=5, D=D, layout=layout)
    replace_and_check(r, (33, 7), packed_rows(1, 40, 5, D, BF16, seed=D))


@pytest.mark.parametrize("layout", [HEAD, TOKEN])
@pytest.mark.parametrize("source,dtype", [(BF16, BF16), (F32, BF16), (BF16, F32), (F32, F32)], ids=str)
def test_other_caches_are_copied_or_rounded_once(source, dtype, layout):
    r = Rings([0, 4, 0], 70, dtype=dtype, layout=layout)
    rows = packed_rows(2, 150, 3, 128, source, seed=3)
    rows[0][0, 7, 1, 5:9] = torch.tensor([float("inf"), -float("inf"), -0.0, 1e-39]).to(source)
    replace_and_check(r, (64, 70, 3), rows, starts=(80, 9, 2))


def test_some_agents_and_some_layers():
    """What is not named keeps its bytes, scales and ring state; one layer at a time gives what one call gives."""
    r = Rings([5, 9, 3], 20, L=4, starts=[17, 2, 19])
    rows = packed_rows(2, 40, 3, 128, BF16, seed=1)
    replace_and_check(r, (0, 20, 11), rows, layer=1, n_layers=2, starts=(0, 3, 25))
    for l in range(4):
        replace_and_check(r, (7, 0, 11), [t[:1] for t in rows], layer=l, n_layers=1)


def test_longer_than_the_ring_keeps_the_newest():
    r = Rings([5, 0], 33)
    rows = packed_rows(2, 200, 3, 128, BF16, seed=2)
    rows[0][:, :100] *= 50  # not kept: no part in the scales
    replace_and_check(r, (150, 34), rows)


def test_rows_that_are_not_ordinary_numbers():
    """Zero rows, infinities, NaN of both signs, and magnitudes at both ends of fp32."""
    r = Rings([0] * 6, 24, L=1, H=2)
    rows = packed_rows(1, 6 * 24, 2, 128, F32, seed=5)
    for t in rows:
        t[0, 0:24] = 0.0
        t[0, 3, 0, 4] = -0.0
        t[0, 24:48, 0] = float("nan")
        t[0, 24 + 1, 1, 3:7] = torch.tensor([float("inf"), -float("inf"), float("nan"), -float("nan")])
        t[0, 48:72] *= 1e-42
        t[0, 72:96] *= 7e37
        t[0, 96:120] *= torch.logspace(-9, 0, 24)[:, None, None]  # every exponent of the codes
        t[0, 120:144] = torch.linspace(-448, 448, 24 * 2 * 128).reshape(24, 2, 128)
    replace_and_check(r, (24,) * 6, rows)
    replace_and_check(r, (24,) * 6, rows, headroom=64.0)


def test_every_finite_bf16_value_is_encoded_as_the_format_says():
    """All 65,536 bf16 patterns against a scale of exactly 1 (the largest finite magnitude that is left is 448)."""
    v = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(BF16).reshape(1, 256, 2, 128).clone()
    v[v.abs().float().nan_to_num(0) > 448] = 448.0
    r = Rings([0], 256, L=1, H=2)
    replace_and_check(r, (256,), [v, -v])


@pytest.mark.parametrize("top", [448.0, 1.0, 3.7e-5, 911.3, 2.3e-16, 5.1e-18, 1.7e-37, 3.1e38])
def test_quotients_next_to_a_border_of_two_codes(top):
    """Elements at the middle of two codes' values and a step of fp32 to either side, for scales that are not powers of two (and,
    by `top`, tiny and huge ones)."""
    codes = torch.arange(0, 0x7F, dtype=torch.uint8).view(FP8).double()
    middle = (codes[:-1] + codes[1:]) / 2
    r = Rings([0], 64, L=1, H=16)
    v = torch.zeros(1, 64, 16, 128)
    g = torch.Generator().manual_seed(3)
    for h in range(16):
        head = top * (0.5 + 0.5 * float(torch.rand((), generator=g)))
        v[0, 0, h, 0] = head
        scale = scale_of(v[0, :1], 1.0)[h].double()
        x = (middle * scale).float()
        up, down = (torch.nextafter(x, torch.full_like(x, s)) for s in (float("inf"), 0.0))
        rows = torch.cat([x, up, down, -x, -up, -down])
        flat = torch.zeros(63 * 128)
        flat[:len(rows)] = rows.clamp(-head, head)
        v[0, 1:, h] = flat.view(63, 128)
    replace_and_check(r, (64,), [v, -v])


@pytest.mark.parametrize("source", [BF16, F32])
@pytest.mark.parametrize("lens", [(60, 0, 64), (300, 0, 250), (700, 0, 1000)], ids=str)
def test_more_heads_than_workgroups(lens, source):
    """Workgroups go from one head's rows to the next; some of the rows hold what is not finite, some only zeros or tiny ones."""
    L, H, D = 3, 96, 64
    r = Rings([0] * 3, max(lens), L=L, H=H, D=D, layout=TOKEN)
    rows = packed_rows(L, sum(lens), H, D, source, seed=sum(lens))
    g = torch.Generator().manual_seed(1)
    for t in rows:
        for value in (float("nan"), float("inf"), -float("inf")):
            at = [torch.randint(0, n, (20,), generator=g) for n in t.shape]
            t[tuple(at)] = value
        t[1, :, 5:60:7] = 0
        t[2, :, 3:90:11] *= 1e-30
    replace_and_check(r, lens, rows)


@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 2, 3), (3, 1, 40), (16, 1, 5)])
def test_another_stream_and_again(shape):
    B, L, H = shape
    r = Rings([0] * B, 90, L=L, H=H)
    lens = tuple(1 + 11 * b % 90 for b in range(B))
    for seed, stream in ((1, None), (2, torch.cuda.Stream()), (3, None)):
        replace_and_check(r, lens, packed_rows(L, sum(lens), H, 128, BF16, seed=seed), stream=stream)


def test_captured_replace_and_read_are_replayed():
    lens = (70, 3000, 9)
    r = Rings([0] * 3, 3000, L=1)
    packed = fsx.PackedRows(lens)
    rows = [t.cuda() for t in packed_rows(1, sum(lens), 3, 128, BF16)]
    back = [torch.empty_like(t) for t in rows]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        fsx.cache_replace_rows(r.desc, 0, 1, *rows, packed)
        fsx.cache_read_rows(r.desc, 0, 1, *back, packed)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        fsx.cache_replace_rows(r.desc, 0, 1, *rows, packed)
        fsx.cache_read_rows(r.desc, 0, 1, *back, packed)
    for turn in range(3):
        host = packed_rows(1, sum(lens), 3, 128, BF16, seed=10 + turn, amp=0.1 + turn)
        for t, h in zip(rows, host):
            t.copy_(h)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want, scales = expect_replaced(r, 0, 1, host, lens, packed.start, 1.0)
        for i, t in enumerate((r.k, r.v)):
            assert torch.equal(bits(t), bits(want[i])) and torch.equal(r.scale[i].cpu(), scales[i])
            eager = torch.empty_like(back[i])
            fsx.cache_read_rows(r.desc, 0, 1, *((eager, None) if i == 0 else (None, eager)), packed)
            torch.cuda.synchronize()
            assert torch.equal(bits(eager), bits(back[i]))
        r.host, r.host_scale = want, scales


def read_and_check(r, lens, out, first=None, starts=None, layer=0, n_layers=None, agent=lambda b: b, which=(0, 1), stream=None):
    n_layers = n_layers or r.L
    packed = fsx.PackedRows(lens, starts)
    total = int((packed.start + packed.len).max()) + 3
    rows = [torch.full((n_layers, total, r.H, r.D), 3.0, dtype=out, device="cuda") for _ in "kv"]
    given = [rows[i] if i in which else None for i in range(2)]
    torch.cuda.synchronize()
    fsx.cache_read_rows(r.desc, layer, n_layers, *given, packed, first=first, stream=stream)
    torch.cuda.synchronize()
    for i in range(2):
        want = torch.full((n_layers, total, r.H, r.D), 3.0, dtype=out)
        if i in which:
            for b, n in enumerate(lens):
                at = (int(r.desc.start[b]) + (first[b] if first else 0) + np.arange(n)) % r.cap
                for l in range(n_layers):
                    x = r.slots(r.host[i], agent(b), layer + l)[torch.from_numpy(at)]
                    if r.dtype is U8:
                        x = x.view(FP8).float() * r.host_scale[i][agent(b), layer + l][None, :, None]
                    want[l, packed.start[b]:packed.start[b] + n] = x.to(out)
        assert torch.equal(bits(rows[i]), bits(want)), ("keys", "values")[i]


@pytest.mark.parametrize("layout", [HEAD, TOKEN])
@pytest.mark.parametrize("dtype", [U8, BF16, F32])
@pytest.mark.parametrize("out", [BF16, F32])
def test_read(dtype, out, layout):
    r = Rings([37, 0, 300, 1], 300, dtype=dtype, layout=layout, starts=[290, 0, 111, 299])
    read_and_check(r, (37, 0, 300, 1), out)
    read_and_check(r, (5, 0, 170, 0), out, first=(32, 0, 100, 0), starts=(200, 0, 3, 0), layer=1, n_layers=1)
    read_and_check(r, (37, 0, 300, 1), out, which=(1,))
    read_and_check(r, (37, 0, 299, 1), out, which=(0,), stream=torch.cuda.Stream())


@pytest.mark.parametrize("D", [16, 32, 48, 80, 256, 512])
def test_read_head_widths(D):
    r = Rings([33, 40], 40, L=1, H=5, D=D, starts=[20, 39])
    read_and_check(r, (33, 40), BF16)


@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("scale", [1.0, 0.037, 2.0 ** -126, 7e5])
def test_every_code_is_read_as_the_format_says(scale, out):
    """All 256 codes, the two that are not a number among them."""
    r = Rings([16], 16, L=1, H=1, D=16)
    codes = torch.arange(256).to(U8).view(16, 16)
    r.k.copy_(codes.view(1, 1, 1, 16, 16))
    r.scale[0].fill_(scale)
    got = torch.empty((1, 16, 1, 16), dtype=out, device="cuda")
    torch.cuda.synchronize()
    fsx.cache_read_rows(r.desc, 0, 1, got, None, fsx.PackedRows((16,)))
    torch.cuda.synchronize()
    want = (codes.view(FP8).float() * torch.tensor(scale)).to(out)
    got, nan = got.cpu().view(16, 16), want.isnan()
    assert int(nan.sum()) == 2 and torch.equal(got.isnan(), nan)
    assert torch.equal(bits(got)[~nan], bits(want)[~nan])


def test_read_a_shared_cache():
    """Agents of one set of rings, each through its own start and length."""
    r = Rings([10, 25, 3], 40, layout=HEAD | fsx.CACHE_SHARED, starts=[0, 30, 39], agents=1)
    read_and_check(r, (10, 25, 3), BF16, agent=lambda b: 0)


def test_rows_beyond_32_bits():
    """A cache of more than 2^32 codes per tensor: the last agent's rows."""
    B, L, H, D, cap = 2, 2, 32, 128, 1 << 18
    k = torch.zeros((B, L, H, cap, D), dtype=U8, device="cuda")
    sc = torch.ones((B, L, H), device="cuda")
    desc = fsx.CacheDesc(k, k, fsx.FP8_E4M3, L, H, D, cap, [0, 0], k_scale=sc, v_scale=sc)
    rows = packed_rows(1, 50, H, D, BF16, seed=1)
    dev = rows[0].cuda()
    fsx.cache_replace_rows(desc, 1, 1, dev, dev, fsx.PackedRows([0, 50]))
    back = torch.empty_like(dev)
    fsx.cache_read_rows(desc, 1, 1, back, None, fsx.PackedRows([0, 50]))
    torch.cuda.synchronize()
    scale = scale_of(rows[0][0].float(), 1.0)
    codes = codes_of(rows[0][0].float(), scale)
    assert torch.equal(k[1, 1, :, :50].transpose(0, 1).cpu(), codes)
    assert torch.equal(bits(back[0]), bits((codes.view(FP8).float() * scale[None, :, None]).to(BF16)))
    assert int(k[0].count_nonzero()) == 0 and int(k[1, 0].count_nonzero()) == 0 and int(k[1, 1, :, 50:].count_nonzero()) == 0


def test_appended_rows_take_the_found_scales():
    """Replace, append with the scales found (within the headroom: not clamped), and all rows back, each at most half a code
    step off: 2^-4 of its magnitude, or of the smallest normal code's (2^-6 scale) below that."""
    r = Rings([0, 0], 64)
    rows = packed_rows(2, 60, 3, 128, BF16, seed=8)
    replace_and_check(r, (20, 40), rows, headroom=2.0)
    new = [(t[:, :2 * 4] * 1.9).to(BF16) for t in packed_rows(2, 8, 3, 128, BF16, seed=8)]  # of 60 rows' distribution
    scale = [t.cpu() for t in r.scale]
    top = [torch.stack([s[b][:, None, :, None] * 448.0 for b in range(2)]) for s in scale]
    dev = [torch.minimum(torch.maximum(t.view(2, 2, 4, 3, 128).transpose(0, 1).float(), -c), c).to(BF16) for t, c in zip(new, top)]
    put = [t.permute(0, 1, 3, 2, 4).contiguous().cuda() for t in dev]  # [B][L][H][n][D]
    fsx.cache_append_rows_quantize(r.desc, *put, fsx.BF16, 4)
    assert list(r.desc.len) == [24, 44] and list(r.desc.pos) == [24, 44]
    back = [torch.empty(2, 68, 3, 128, dtype=F32, device="cuda") for _ in "kv"]
    fsx.cache_read_rows(r.desc, 0, 2, *back, fsx.PackedRows([24, 44]))
    torch.cuda.synchronize()
    for i in range(2):
        for b, (at, n, src) in enumerate(((0, 20, 0), (24, 40, 20))):
            want = torch.cat([rows[i][:, src:src + n].float(), dev[i][b].float()], 1)
            got, s = back[i].cpu()[:, at:at + n + 4], scale[i][b][:, None, :, None]
            assert bool(((got - want).abs() <= 2.0 ** -4 * want.abs().clamp_min(2.0 ** -6 * s) * (1 + 1e-6)).all())


@pytest.mark.parametrize("dtype,lens", [(BF16, (3,)), (U8, (3,)), (F32, (2, 1))], ids=str)
def test_more_than_65535_layers(dtype, lens):
    """The layers are a launch's second dimension."""
    L = 65_600
    r = Rings([0] * len(lens), 3, L=L, H=1, D=16, dtype=dtype, layout=TOKEN)
    rows = packed_rows(L, sum(lens), 1, 16, BF16, seed=3)
    dev, at = [t.cuda() for t in rows], fsx.PackedRows(lens)
    fsx.cache_replace_rows(r.desc, 0, L, *dev, at)
    back = [torch.empty_like(t) for t in dev]
    fsx.cache_read_rows(r.desc, 0, L, *back, at)
    torch.cuda.synchronize()
    for i in range(2):
        if dtype is not U8:
            assert torch.equal(bits(back[i]), bits(rows[i]))
            continue
        x = rows[i].float()
        top = x.abs().amax((1, 2, 3), keepdim=True).numpy()
        scale = torch.from_numpy(np.maximum(top / np.float32(448.0), np.float32(2.0 ** -126)))
        code = torch.from_numpy(x.numpy() / scale.numpy()).to(FP8)
        assert torch.equal(r.scale[i].cpu().flatten(), scale.flatten())
        assert torch.equal(bits(back[i]), bits((code.float() * scale).to(BF16)))


def test_more_rows_than_a_launch_has_threads_for():
    """17 agents' windows of one ring of 2^24 rows, 2^24 workgroups of 16 rows and more: a launch holds fewer than 2^32 threads."""
    n, agents = 1 << 24, 17
    k = torch.arange(n * 4, dtype=torch.int32, device="cuda").view(BF16).view(1, 1, n, 1, 8).repeat(1, 1, 1, 1, 2)
    cache = fsx.CacheDesc(k, k, fsx.BF16, 1, 1, 16, n, [n] * agents, starts=[5 * b for b in range(agents)],
                          layout=TOKEN | fsx.CACHE_SHARED)
    out = torch.zeros(1, n * agents, 1, 16, dtype=BF16, device="cuda")
    fsx.cache_read_rows(cache, 0, 1, out, None, fsx.PackedRows([n] * agents))
    torch.cuda.synchronize()
    want, got = k.view(n, 8, 2).view(torch.int32), out.view(agents, n, 8, 2).view(torch.int32)
    for b in range(agents):
        assert torch.equal(got[b], want.roll(-5 * b, 0)), b
