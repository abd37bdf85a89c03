"""Refusals of the prompt operators: every check runs on the host before any GPU work (the pointers below are never used)."""

import ctypes

import numpy as np
import pytest

from paper_2607_15621_amd import fsx

PTR = 1 << 20  # a 16-byte aligned address that no check dereferences
INVALID, UNSUPPORTED, CAPACITY = 1, 2, 3


def desc(**kw):
    d = dict(n_heads=4, n_kv_heads=2, head_dim=128, q_dtype=fsx.BF16, out_dtype=fsx.BF16, scale=0.0, kernel=0, q_rows=100, k_rows=200,
             q_row=512, q_head=128, k_row=256, k_head=128, v_row=256, v_head=128, out_row=512, out_head=128)
    d.update(kw)
    return fsx.PromptDesc(*(d[n] for n, _ in fsx.PromptDesc._fields_))


def attend(d=None, q=PTR, k=PTR, v=PTR, out=PTR, q_rows=((0, 30), (30, 70)), k_rows=((0, 30), (30, 170)), ws=0, ws_bytes=0,
           n=None):
    qr, kr = (fsx.PackedRows([x[1] for x in r], [x[0] for x in r]) if r is not None else None for r in (q_rows, k_rows))
    code = fsx.lib().fsx_prompt_attention(ctypes.byref(d if d is not None else desc()), q, k, v, out, None,
                                          qr.n if n is None else n, qr.c_start, qr.c_len, kr.c_start if kr else None,
                                          kr.c_len if kr else None, ws, ws_bytes, None)
    return code, fsx.last_error()


@pytest.mark.parametrize("change,code,word", [
    (dict(n_kv_heads=3), INVALID, "n_kv_heads"), (dict(n_heads=0), INVALID, "n_heads"), (dict(n_heads=2000), INVALID, "n_heads"),
    (dict(head_dim=96), UNSUPPORTED, "head_dim"), (dict(q_dtype=fsx.FP8_E4M3), UNSUPPORTED, "q and out"),
    (dict(out_dtype=7), UNSUPPORTED, "q and out"), (dict(scale=-1.0), INVALID, "scale"), (dict(scale=float("nan")), INVALID, "scale"),
    (dict(scale=float("inf")), INVALID, "scale"), (dict(kernel=4), INVALID, "kernel"), (dict(kernel=-1), INVALID, "kernel"),
    (dict(kernel=3, head_dim=64), UNSUPPORTED, "TURNS"), (dict(k_row=1 << 28), UNSUPPORTED, "2^27"), (dict(q_row=516), INVALID, "strides"), (dict(k_head=-8), INVALID, "strides"),
    (dict(v_row=1 << 62), INVALID, "strides"), (dict(out_head=64), INVALID, "overlap"), (dict(out_row=504), INVALID, "overlap"),
    (dict(out_row=128, out_head=12792), INVALID, "overlap"), (dict(out_row=0), INVALID, "overlap"), (dict(q_rows=-1), INVALID, "q_rows"),
    (dict(q_rows=99), INVALID, "queries"), (dict(k_rows=199), INVALID, "keys")])
def test_descriptor(change, code, word):
    got, msg = attend(desc(**change))
    assert got == code and word in msg, msg


def test_head_major_output_is_taken():
    got, msg = attend(desc(out_row=128, out_head=12800), q=0)
    assert got == INVALID and "non-NULL" in msg  # past the strides


@pytest.mark.parametrize("kw,word", [
    (dict(q=0), "non-NULL"), (dict(k=0), "non-NULL"), (dict(v=0), "non-NULL"), (dict(out=0), "non-NULL"), (dict(q=PTR + 8), "aligned"),
    (dict(v=PTR + 2), "aligned"), (dict(out=PTR + 4), "aligned"), (dict(n=0), "n_seq"), (dict(n=65), "n_seq"),
    (dict(q_rows=((0, 30), (29, 70))), "share rows"), (dict(q_rows=((0, 30), (10, 5))), "share rows"),
    (dict(q_rows=((-1, 30), (30, 70))), "queries"), (dict(k_rows=((0, -1), (30, 170))), "keys"),
    (dict(k_rows=((0, 30), (31, 170))), "keys"), (dict(ws=PTR + 8, ws_bytes=64), "workspace"), (dict(ws=0, ws_bytes=64), "workspace"),
    (dict(ws=PTR, ws_bytes=-1), "workspace")])
def test_arguments(kw, word):
    got, msg = attend(**kw)
    assert got == INVALID and word in msg, msg


def test_nulls():
    L, r = fsx.lib(), fsx.PackedRows([1])
    assert L.fsx_prompt_attention(None, PTR, PTR, PTR, PTR, None, 1, r.c_start, r.c_len, None, None, None, 0, None) == INVALID
    d = desc()
    assert L.fsx_prompt_attention(ctypes.byref(d), PTR, PTR, PTR, PTR, None, 1, None, r.c_len, None, None, None, 0, None) == INVALID
    assert L.fsx_prompt_attention(ctypes.byref(d), PTR, PTR, PTR, PTR, None, 1, r.c_start, r.c_len, r.c_start, None, None, 0,
                                  None) == INVALID
    assert L.fsx_prompt_attention_workspace(ctypes.byref(d), 1, r.c_len, None, None) == INVALID
    need = ctypes.c_int64(5)
    assert L.fsx_prompt_attention_workspace(None, 1, r.c_len, None, ctypes.byref(need)) == INVALID and need.value == 0
    assert L.fsx_prompt_attention_workspace(ctypes.byref(d), 1, None, None, ctypes.byref(need)) == INVALID
    assert L.fsx_prompt_attention_workspace(ctypes.byref(d), 65, r.c_len, None, ctypes.byref(need)) == INVALID
    bad = fsx.PackedRows([-1])
    assert L.fsx_prompt_attention_workspace(ctypes.byref(d), 1, bad.c_len, None, ctypes.byref(need)) == INVALID
    assert L.fsx_backbone_rebuild(None, None, None, None, None, 1.0, 0, None) == INVALID


def test_nothing_to_do_needs_no_gpu():
    assert attend(q_rows=((0, 0), (30, 0)), q=0, k=0, v=0, out=0)[0] == 0


def cache(dtype=fsx.FP8_E4M3, lengths=(5, 0, 8), cap=8, L=3, H=2, D=128, layout=0, k=PTR, scales=PTR):
    return fsx.CacheDesc(k, k, dtype, L, H, D, cap, list(lengths), k_scale=scales, v_scale=scales, layout=layout)


def replace(c, lens=(5, 0, 4), starts=None, layer=0, n_layers=3, k=PTR, v=PTR, dtype=fsx.BF16, total=9, headroom=1.0, policy=0):
    r = fsx.PackedRows(lens, starts)
    code = fsx.lib().fsx_cache_replace_rows(ctypes.byref(c.c), layer, n_layers, k, v, dtype, total, r.c_start, r.c_len, headroom,
                                            policy, None)
    return code, fsx.last_error()


@pytest.mark.parametrize("c,kw,code,word", [
    (dict(), dict(layer=1), INVALID, "layers"), (dict(), dict(layer=-1, n_layers=1), INVALID, "layers"),
    (dict(), dict(n_layers=0), INVALID, "layers"), (dict(), dict(dtype=fsx.FP8_E4M3), INVALID, "rows must be"),
    (dict(), dict(total=8), INVALID, "packed rows"), (dict(), dict(lens=(5, -1, 4)), INVALID, "packed rows"),
    (dict(), dict(starts=(-1, 0, 0)), INVALID, "packed rows"), (dict(), dict(headroom=0.5), INVALID, "headroom"),
    (dict(), dict(headroom=float("nan")), INVALID, "headroom"), (dict(), dict(headroom=65.0), INVALID, "headroom"),
    (dict(), dict(policy=2), INVALID, "policy"), (dict(), dict(k=0), INVALID, "row pointers"),
    (dict(), dict(v=PTR + 8), INVALID, "aligned"), (dict(k=PTR + 8, lengths=(0, 0, 0)), dict(), INVALID, "aligned"),
    (dict(k=0, lengths=(0, 0, 0)), dict(), INVALID, "NULL"), (dict(scales=0, lengths=(0, 0, 0)), dict(), INVALID, "scale"),
    (dict(), dict(lens=(5, 0, 9), total=14, policy=fsx.APPEND_ERROR), CAPACITY, "agent 2"),
    (dict(cap=0, lengths=(0, 0, 0)), dict(), CAPACITY, "no slots"), (dict(layout=fsx.CACHE_SHARED), dict(), UNSUPPORTED, "shared"),
    (dict(D=24), dict(), UNSUPPORTED, "head_dim"), (dict(D=1024), dict(), UNSUPPORTED, "head_dim"), (dict(H=0), dict(), INVALID, "geometry"),
    (dict(lengths=(5, 0, 9)), dict(), CAPACITY, "len")])
def test_replace_refuses(c, kw, code, word):
    desc_ = cache(**c)
    before = [list(x) for x in (desc_.start, desc_.len, desc_.pos)]
    got, msg = replace(desc_, **kw)
    assert got == code and word in msg, msg
    assert before == [list(x) for x in (desc_.start, desc_.len, desc_.pos)]


def test_replace_of_no_agent_changes_nothing():
    c = cache()
    assert replace(c, lens=(0, 0, 0), k=0, v=0)[0] == 0
    assert list(c.len) == [5, 0, 8]


def read(c, lens=(5, 0, 4), starts=None, layer=0, n_layers=3, k=PTR, v=PTR, dtype=fsx.BF16, total=9, first=None):
    r = fsx.PackedRows(lens, starts)
    f = np.array(first, np.int64) if first is not None else None
    code = fsx.lib().fsx_cache_read_rows(ctypes.byref(c.c), layer, n_layers,
                                         f.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)) if f is not None else None, k, v, dtype,
                                         total, r.c_start, r.c_len, None)
    return code, fsx.last_error()


@pytest.mark.parametrize("c,kw,code,word", [
    (dict(), dict(layer=3, n_layers=1), INVALID, "layers"), (dict(), dict(dtype=9), INVALID, "rows must be"),
    (dict(), dict(total=8), INVALID, "packed rows"), (dict(), dict(starts=(0, 0, 4)), INVALID, "share rows"),
    (dict(), dict(lens=(6, 0, 4), total=10), CAPACITY, "agent 0"), (dict(), dict(first=(1, 0, 0)), CAPACITY, "agent 0"),
    (dict(), dict(first=(0, 0, -1)), INVALID, "first"), (dict(), dict(lens=(0, 1, 0)), CAPACITY, "agent 1"),
    (dict(), dict(v=PTR + 8), INVALID, "aligned"), (dict(scales=0), dict(), INVALID, "scale"), (dict(D=24), dict(), UNSUPPORTED, "head_dim")])
def test_read_refuses(c, kw, code, word):
    got, msg = read(cache(**c), **kw)
    assert got == code and word in msg, msg


def test_read_of_nothing_needs_no_gpu():
    assert read(cache(), lens=(0, 0, 0), k=0, v=0)[0] == 0
    assert read(cache(), k=0, v=0)[0] == 0


def test_binding_checks_its_tensors():
    import torch

    q, k = torch.zeros(8, 4, 128, dtype=torch.bfloat16), torch.zeros(8, 2, 128, dtype=torch.bfloat16)
    r = fsx.PackedRows([8])
    with pytest.raises(ValueError):
        fsx.prompt_attention(q, k, k[:4], q, r)
    with pytest.raises(ValueError):
        fsx.prompt_attention(q, k.float(), k.float(), q, r)
    with pytest.raises(ValueError):
        fsx.prompt_attention(q, k, k, q.half(), r)
    with pytest.raises(ValueError):
        fsx.prompt_attention(q, k, k, q, r, lse=torch.zeros(8, 2))
    with pytest.raises(ValueError):
        fsx.prompt_attention(q, k, k, q, r, fsx.PackedRows([4, 4]))
    with pytest.raises(ValueError):
        fsx.PackedRows([1, 2], [0])
    c = cache()
    rows = torch.zeros(3, 9, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        fsx.cache_replace_rows(c, 0, 2, rows, rows, fsx.PackedRows([5, 0, 4]))
    with pytest.raises(ValueError):
        fsx.cache_replace_rows(c, 0, 3, rows, rows.transpose(1, 2), fsx.PackedRows([5, 0, 4]))
    with pytest.raises(ValueError):
        fsx.cache_read_rows(c, 0, 3, rows, rows, fsx.PackedRows([5, 4]))
    with pytest.raises(ValueError):
        fsx.cache_read_rows(c, 0, 3, rows, rows, fsx.PackedRows([5, 0, 4]), first=[0])


def backbone(d=256, layers=2):
    """A binding without a handle: calls that pass the binding's own checks are refused by the library."""
    bb = fsx.Backbone.__new__(fsx.Backbone)
    bb.handle, bb.cfg = 0, fsx.BackboneCfg(layers, d, 2, 128, 512, 4, 3, fsx.BF16, 10000.0, 1e-6)
    return bb


@pytest.mark.parametrize("tokens,hidden,word", [
    ((8, 256), None, "tokens"), ((9, 128), None, "tokens"), ((9, 2, 128), None, "tokens"), ((9, 256, "float32"), None, "tokens"),
    ((9, 256, "t"), None, "tokens"), ((9, 256), (2, 8, 256), "hidden"), ((9, 256), (1, 9, 256), "hidden"),
    ((9, 256), (2, 9, 256, "bfloat16"), "hidden"), ((9, 256), (2, 9, 256, "t"), "hidden")], ids=str)
def test_rebuild_checks_its_tensors(tokens, hidden, word):
    import torch

    def make(shape, dtype):
        sizes, how = [n for n in shape if not isinstance(n, str)], [n for n in shape if isinstance(n, str)]
        if how == ["t"]:
            return torch.zeros(sizes[:-2] + sizes[:-3:-1], dtype=dtype).transpose(-1, -2)
        return torch.zeros(sizes, dtype=getattr(torch, how[0]) if how else dtype)

    with pytest.raises(ValueError, match=word):
        backbone().rebuild(cache(), make(tokens, torch.bfloat16), (5, 0, 4),
                           make(hidden, torch.float32) if hidden else None, stream=0)


def test_workspace_must_be_dense():
    import torch

    q, k = torch.zeros(8, 4, 128, dtype=torch.bfloat16), torch.zeros(8, 2, 128, dtype=torch.bfloat16)
    for ws in (torch.zeros(64, 2)[:, 0], torch.zeros(1).expand(1 << 20)):
        with pytest.raises(ValueError, match="workspace"):
            fsx.prompt_attention(q, k, k, q, fsx.PackedRows([8]), workspace=ws, stream=0)


def test_host_tensors_are_refused():
    """Tensors of the host, or of a device that is not the current one, would be read by the wrong device."""
    import torch

    q, k = torch.zeros(8, 4, 128, dtype=torch.bfloat16), torch.zeros(8, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current device"):
        fsx.prompt_attention(q, k, k, q, fsx.PackedRows([8]), stream=0)
    rows = torch.zeros(3, 9, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current device"):
        fsx.cache_replace_rows(cache(), 0, 3, rows, rows, fsx.PackedRows([5, 0, 4]), stream=0)
    with pytest.raises(ValueError, match="current device"):
        fsx.cache_read_rows(cache(), 0, 3, None, rows, fsx.PackedRows([5, 0, 4]), stream=0)
    with pytest.raises(ValueError, match="current device"):
        backbone().rebuild(cache(), torch.zeros(9, 256, dtype=torch.bfloat16), (5, 0, 4), stream=0)


def workspace_of(d, lens):
    need, r = ctypes.c_int64(5), fsx.PackedRows(lens)
    return fsx.lib().fsx_prompt_attention_workspace(ctypes.byref(d), r.n, r.c_len, None, ctypes.byref(need)), need.value


@pytest.mark.parametrize("heads,lens,kernel,code", [
    (1024, [1 << 24] * 64, fsx.PROMPT_AUTO, UNSUPPORTED), (1024, [1 << 24] * 64, fsx.PROMPT_CHUNKS, UNSUPPORTED),
    (1024, [1 << 24] * 64, fsx.PROMPT_TURNS, UNSUPPORTED), (1024, [(1 << 20) + 1], fsx.PROMPT_TILES, UNSUPPORTED),
    (1024, [1 << 20], fsx.PROMPT_TILES, 0), (1024, [1 << 20], fsx.PROMPT_AUTO, 0),
    # a workgroup of two waves per 32 rows and head: a launch holds fewer than 2^32 threads
    (1024, [(1 << 19) + 1], fsx.PROMPT_CHUNKS, UNSUPPORTED), (1024, [1 << 19], fsx.PROMPT_CHUNKS, 0),
    (32, [1 << 24, 1], fsx.PROMPT_CHUNKS, UNSUPPORTED), (32, [1 << 24, 1], fsx.PROMPT_AUTO, 0)])
def test_sizes_that_a_call_refuses_have_no_workspace(heads, lens, kernel, code):
    d = desc(n_heads=heads, n_kv_heads=heads, kernel=kernel, q_rows=1 << 31, k_rows=1 << 31, q_row=128 * heads, out_row=128 * heads)
    got, need = workspace_of(d, lens)
    assert got == code and need >= 0
    if code:
        assert need == 0 and "2^" in fsx.last_error()
        r = [(i << 24, n) for i, n in enumerate(lens)]
        got, msg = attend(d, q_rows=r, k_rows=None)
        assert got == code and "2^" in msg, msg


@pytest.mark.parametrize("rows,heads,code", [(-1, 2, INVALID), ((1 << 20) + 1, 2, INVALID), (1 << 20, 2048, UNSUPPORTED)])
def test_rows_of_a_rebuild_are_limited_at_create(rows, heads, code):
    cfg = fsx.BackboneCfg(1, 256, heads, 128, 512, 4, 1, fsx.BF16, 10000.0, 1e-6, rows)
    out = ctypes.c_void_p(1)
    assert fsx.lib().fsx_backbone_create(ctypes.byref(cfg), None, None, ctypes.byref(out)) == code
    assert out.value is None and "max_prompt_rows" in fsx.last_error()


@pytest.mark.parametrize("H,L", [(1 << 20, 1 << 10), (1 << 16, 1 << 16)])
def test_caches_with_more_scales_than_an_index_holds_are_refused(H, L):
    c = cache(H=H, L=L, D=16, cap=1, lengths=(0, 0, 0))
    for code, msg in (replace(c, lens=(1, 0, 0), total=1, n_layers=L), read(cache(H=H, L=L, D=16, cap=1, lengths=(1, 0, 0)), lens=(1, 0, 0),
                                                                            total=1, n_layers=L)):
        assert code == UNSUPPORTED and "2^29" in msg, msg
