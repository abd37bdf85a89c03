"""A cache rebuilt from scratch on the GPU (fsx_backbone_rebuild): whole prompts of agents of different lengths in one call.

The rows and the hidden states of every layer match the oracle's forward over each prompt from an empty cache; agents with no
tokens keep everything; an fp8 cache gets scales found from the rows; and the operators run together as a deployment uses them:
rebuild, append, read back, attention over the rows read, the expert's tick.  The tolerance is the incremental forward's (the
same projections in bf16)."""

from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import oracle
import synth
from harness import Cache, Model, record, rel_err, run_forward, tokens_for
from paper_2607_15621_amd import fsx
from test_gpu_backbone import TOL, bb_workload

pytestmark = pytest.mark.gpu


class Rebuilder:
    def __init__(self, wl, max_batch=8, max_new_rows=64):
        self.wl = wl
        self.layers, _, _ = synth.make_weights(wl)
        dev = [{k: torch.from_numpy(v).to("cuda", torch.float32 if k in ("attn_norm", "ffn_norm") else torch.bfloat16)
                for k, v in lw.items()} for lw in self.layers]
        self.bb = fsx.Backbone(fsx.BackboneCfg(wl.n_layers, wl.d_model, wl.n_heads, wl.head_dim, wl.d_ffn, max_new_rows, max_batch,
                                               fsx.BF16, wl.rope_base, wl.rms_eps), dev)
        torch.cuda.synchronize()
        self.shape = oracle.BackboneShape(n_layers=wl.n_layers, d_model=wl.d_model, n_heads=wl.n_heads, head_dim=wl.head_dim,
                                          d_ffn=wl.d_ffn, rope_base=wl.rope_base, rms_eps=wl.rms_eps)

    def prompts(self, lens, seed=0):
        rng = np.random.default_rng([self.wl.wid, 77, seed])
        host = [synth.round_bf16(rng.standard_normal((n, self.wl.d_model), dtype=np.float32)) for n in lens]
        return host, torch.from_numpy(np.concatenate(host)).to("cuda", torch.bfloat16)

    def oracle(self, tokens, rows=None, pos=0):
        empty = np.zeros((0, self.wl.n_heads, self.wl.head_dim))
        return oracle.backbone_incremental_forward(self.shape, self.layers, tokens, rows or (lambda l: (empty, empty)), pos)


def rows_of(cache, b, n):
    """Decoded rows [layers][n][H][Dh] of agent b, the oldest first, by the library's own read and as the cache holds them."""
    wl = cache.wl
    lens = [n if x == b else 0 for x in range(len(cache.lengths))]
    out = [torch.empty(wl.n_layers, n, wl.n_heads, wl.head_dim, device="cuda") for _ in "kv"]
    fsx.cache_read_rows(cache.desc, 0, wl.n_layers, *out, fsx.PackedRows(lens))
    torch.cuda.synchronize()
    return [t.cpu().numpy() for t in out]


@pytest.mark.parametrize("layout", [fsx.CACHE_HEAD_MAJOR, fsx.CACHE_TOKEN_MAJOR])
@pytest.mark.parametrize("lens", [(224,), (37, 0, 150), (1, 2, 3), (300, 65)], ids=str)
def test_rebuild_matches_oracle(lens, layout):
    wl = bb_workload(810 + len(lens), lengths=(20,) * len(lens), n_new=4, capacity=320)
    r = Rebuilder(wl)
    cache = Cache(wl, starts=(310,) * len(lens), layout=layout)
    before = cache.k.clone()
    host, tok = r.prompts(lens)
    hid = torch.full((wl.n_layers, sum(lens), wl.d_model), float("nan"), device="cuda")
    r.bb.rebuild(cache.desc, tok, lens, hid)
    torch.cuda.synchronize()
    hid, at = hid.cpu().numpy(), 0
    for b, n in enumerate(lens):
        state = [int(x[b]) for x in (cache.desc.start, cache.desc.len, cache.desc.pos)]
        if n == 0:
            assert state == [310, 20, 20] and torch.equal(cache.k[b].view(torch.int16), before[b].view(torch.int16))
            continue
        assert state == [0, n, n]
        k_ref, v_ref, h_ref = r.oracle(host[b])
        k_got, v_got = rows_of(cache, b, n)
        record(b, rel_err(k_got, k_ref), TOL, what="rebuilt keys, max|d| / max|ref|")
        record(b, rel_err(v_got, v_ref), TOL, what="rebuilt values, max|d| / max|ref|")
        record(b, max(rel_err(hid[l, at:at + n], h_ref[l]) for l in range(wl.n_layers)), TOL, what="worst layer hidden, max|d| / max|ref|")
        at += n
    r.bb.close()


def test_rebuild_is_what_appends_from_empty_rings_give():
    wl = bb_workload(820, lengths=(0, 0), n_new=4, capacity=128)
    r = Rebuilder(wl)
    lens = (100, 64)
    host, tok = r.prompts(lens)
    whole, parts = Cache(wl), Cache(wl)
    r.bb.rebuild(whole.desc, tok, lens)
    one = fsx.CacheDesc(parts.k[:1], parts.v[:1], fsx.BF16, wl.n_layers, wl.n_heads, 128, 128, [0])
    r.bb.append(one, tok[:64].contiguous(), 1, 64)
    r.bb.append(one, tok[64:100].contiguous(), 1, 36)
    torch.cuda.synchronize()
    parts.desc.len[0] = 100
    for got, want in zip(rows_of(whole, 0, 100), rows_of(parts, 0, 100)):
        record(0, rel_err(got, want), TOL, what="rebuilt rows vs appended rows, max|d| / max|ref|")
    r.bb.close()


def test_rebuild_refuses_and_keeps_the_rings():
    wl = bb_workload(830, lengths=(5, 5), n_new=4, capacity=64)
    r = Rebuilder(wl, max_batch=2, max_new_rows=32)
    cache = Cache(wl)
    _, tok = r.prompts((64, 1))
    for lens, policy, code, word in (((60, 5), 0, 3, "64"), ((-1, 5), 0, 1, "n_tokens"), ((64, 0), 9, 1, "policy")):
        with pytest.raises(fsx.FsxError, match=word) as e:
            r.bb.rebuild(cache.desc, tok, lens, policy=policy)
        assert e.value.code == code
    small = Cache(wl, capacity=16)
    with pytest.raises(fsx.FsxError) as e:
        r.bb.rebuild(small.desc, tok, (17, 0), policy=fsx.APPEND_ERROR)
    assert e.value.code == 3
    with pytest.raises(fsx.FsxError, match="headroom"):
        r.bb.rebuild(cache.desc, tok, (5, 5), headroom=0.0)
    r.bb.rebuild(cache.desc, tok, (0, 0))
    assert list(cache.desc.len) == [5, 5]
    # more tokens than slots: the newest are kept, at their positions
    host, tok = r.prompts((40, 0))
    r.bb.rebuild(small.desc, tok, (40, 0))
    torch.cuda.synchronize()
    assert [int(x[0]) for x in (small.desc.start, small.desc.len, small.desc.pos)] == [0, 16, 40]
    k_ref, _, _ = r.oracle(host[0])
    record(0, rel_err(rows_of(small, 0, 16)[0], k_ref[:, 24:]), TOL, what="newest keys, max|d| / max|ref|")
    r.bb.close()


def test_captured_rebuild_is_replayed():
    wl = bb_workload(835, lengths=(0, 0), n_new=4, capacity=256, cache_dtype="fp8")
    r = Rebuilder(wl)
    cache, eager = Cache(wl), Cache(wl)
    lens = (130, 77)
    _, tok = r.prompts(lens)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        r.bb.rebuild(cache.desc, tok, lens)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        r.bb.rebuild(cache.desc, tok, lens)
    for turn in range(3):
        tok.copy_(r.prompts(lens, seed=turn + 1)[1])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        r.bb.rebuild(eager.desc, tok, lens)
        torch.cuda.synchronize()
        for x, y in ((cache.k, eager.k), (cache.v, eager.v)):
            assert torch.equal(x, y)
        assert torch.equal(cache.k_scale, eager.k_scale) and torch.equal(cache.v_scale, eager.v_scale)
    r.bb.close()


def test_rebuild_append_read_attend_and_tick():
    """The operators as a deployment runs them, over an fp8 cache: each step against the oracle over what the step before left."""
    lens = (120, 33)
    wl = bb_workload(840, lengths=(0, 0), n_new=4, capacity=192, cache_dtype="fp8")
    r = Rebuilder(wl)
    cache = Cache(wl)
    host, tok = r.prompts(lens)
    r.bb.rebuild(cache.desc, tok, lens, headroom=2.0)
    # 1. the rebuilt rows: half a code step, 2^-4 of a magnitude, on top of the projections' tolerance
    old = [rows_of(cache, b, n) for b, n in enumerate(lens)]
    for b, n in enumerate(lens):
        k_ref, v_ref, _ = r.oracle(host[b])
        for got, want, what in zip(old[b], (k_ref, v_ref), ("keys", "values")):
            top = np.abs(want).max()
            assert np.all(np.abs(got - want) <= 2.0 ** -4 * np.abs(want) + 1.07 * TOL * top), what
    # 2. a frame's four rows appended: encoded with the scales that the rebuild found
    scales = [t.clone() for t in (cache.k_scale, cache.v_scale)]
    new_host, new_tok = r.prompts((4, 4), seed=9)
    r.bb.append(cache.desc, new_tok.view(2, 4, wl.d_model), 2, 4)
    torch.cuda.synchronize()
    assert torch.equal(scales[0], cache.k_scale) and torch.equal(scales[1], cache.v_scale)
    assert list(cache.desc.len) == [124, 37]
    rows = [rows_of(cache, b, n + 4) for b, n in enumerate(lens)]
    for b, n in enumerate(lens):
        assert all(np.array_equal(x[:, :n], y) for x, y in zip(rows[b], old[b]))
        k_ref, _, _ = r.oracle(new_host[b], lambda l, b=b: (old[b][0][l].astype(np.float64), old[b][1][l].astype(np.float64)), n)
        record(b, rel_err(rows[b][0][:, n:], k_ref), 6e-2, what="appended keys (fp8 decoded), max|d| / max|ref|")
    # 3. attention of new queries over one layer's rows, read back in bf16
    total = sum(n + 4 for n in lens)
    kv = [torch.empty(1, total, wl.n_heads, 128, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    at = fsx.PackedRows([n + 4 for n in lens])
    fsx.cache_read_rows(cache.desc, 1, 1, *kv, at)
    q = torch.randn(6, wl.n_heads, 128, generator=torch.Generator().manual_seed(2)).to("cuda", torch.bfloat16)
    out = torch.empty(6, wl.n_heads, 128, device="cuda")
    fsx.prompt_attention(q, kv[0][0], kv[1][0], out, fsx.PackedRows([2, 4]), at)
    torch.cuda.synchronize()
    for b, (a, m) in enumerate(((0, 2), (2, 4))):
        n = lens[b] + 4
        k, v = (torch.from_numpy(x[1]).to(torch.bfloat16).double() for x in rows[b])
        for t in range(m):
            seen = n - m + t + 1
            p = torch.softmax(torch.einsum("hc,jhc->hj", q[a + t].double().cpu(), k[:seen]) / math.sqrt(128), 1)
            want, size = torch.einsum("hj,jhc->hc", p, v[:seen]), torch.einsum("hj,jhc->hc", p, v[:seen].abs())
            # the probabilities' rounding to bf16, and 1 % of it for the rest (scores of 128 products in fp32)
            assert bool(((out[a + t].cpu().double() - want).abs() <= 2.0 ** -8 * 1.01 * size).all()), (b, t)
    # 4. the expert's tick over the cache
    we = synth.Workload(name="tick", wid=841, n_layers=wl.n_layers, d_model=128, n_heads=wl.n_heads, head_dim=128, d_ffn=256,
                        n_expert_tokens=10, n_frame_tokens=0, batch=2, lengths=(124, 37), dtype="bf16", cache_dtype="fp8", capacity=192)
    model = Model(we)
    ex = model.create()
    cache.wl = we
    host_tok, etok = tokens_for(we)
    wp, _ = run_forward(ex, cache, etok, 2, 0)
    for b in range(2):
        ref, _ = model.oracle_agent(host_tok[b], lambda l, b=b: (rows[b][0][l].astype(np.float64), rows[b][1][l].astype(np.float64)),
                                    cache.desc.pos[b])
        record(b, rel_err(wp[b], ref), TOL)
    ex.close()
    r.bb.close()
