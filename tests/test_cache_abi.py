"""CPU-side checks of the cache operators' and sampling's C ABI: bad arguments are refused before anything is
launched (none of these calls reaches the GPU)."""
import ctypes

import pytest

import paper_2512_21911_amd as S


def good(**kw):
    base = dict(B=2, Hq=8, Hkv=2, d=128, dtype="bf16", max_seq_len=1000, max_new=16, n_rows=32, n_pages=200, page_size=16,
                max_pages_per_seq=63, kv_strides=(16 * 2 * 128, 2 * 128, 128), rotary_dim=64)
    base.update(kw)
    return S.make_chunk_shape(**base)


OK, NULL = ctypes.c_void_p(0x10000), None


def append(sh, **kw):
    names = ["k_new", "v_new", "table", "seq_lens", "new_rows", "new_lens", "K", "V", "q", "q_out", "inv_freq", "positions"]
    return S.lib().svf_append_kv(ctypes.byref(sh) if sh else None, *[kw.get(n, OK) for n in names], None)


def attend(sh, ws_bytes=1 << 40, **kw):
    names = ["q", "K", "V", "table", "seq_lens", "new_rows", "new_lens", "out", "lse", "ws"]
    return S.lib().svf_chunk_attn(ctypes.byref(sh) if sh else None, *[kw.get(n, OK) for n in names], ws_bytes, None)


def both(sh):
    assert S.svf_chunk_workspace_bytes(sh) == 0
    a, b = append(sh), attend(sh)
    assert a == b
    return a


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=7), -3), (dict(dtype=-1), -3),
    (dict(B=0), -2), (dict(B=4097), -2), (dict(Hq=7), -2), (dict(Hkv=0), -2), (dict(Hq=0), -2), (dict(Hq=514, Hkv=2), -2), (dict(d=96), -2), (dict(d=256), -2),
    (dict(page_size=-1), -2), (dict(n_pages=0), -2), (dict(max_seq_len=0), -2), (dict(max_seq_len=(1 << 30) + 1), -2),
    (dict(max_new=0), -2), (dict(max_new=(1 << 24) + 1), -2), (dict(n_rows=0), -2), (dict(window=-1), -2),
    (dict(kv_strides=(4096, 100, 128)), -2), (dict(kv_strides=(4096, 256, 64)), -2), (dict(kv_strides=(4097, 256, 128)), -2),
    (dict(q_stride=1016), -2), (dict(q_stride=1028), -2), (dict(k_stride=248), -2), (dict(v_stride=260), -2), (dict(out_stride=-1024), -2),
    (dict(sm_scale=float("nan")), -2), (dict(sm_scale=float("inf")), -2), (dict(rotary_scale=float("nan")), -2),
    (dict(rotary_dim=8), -2), (dict(rotary_dim=144), -2), (dict(rotary_dim=-16), -2), (dict(rotary_interleaved=2), -2),
    (dict(max_pages_per_seq=62), -4), (dict(max_pages_per_seq=0), -4), (dict(page_size=0, n_pages=1), -4),
])
def test_shapes_are_refused(kw, code):
    assert both(good(**kw)) == code


def test_workspace_bytes():
    for kw in ({}, dict(dtype="f32", kv_strides=(16 * 256, 256, 128)), dict(d=64), dict(max_new=4000, n_rows=8000), dict(page_size=0, n_pages=2)):
        n = S.svf_chunk_workspace_bytes(good(**kw))
        assert n > 0 and n % 256 == 0
        assert attend(good(**kw), ws_bytes=n - 1) == -6
    assert S.lib().svf_chunk_workspace_bytes(None) == 0
    with pytest.raises(S.SvfError):
        S.new_chunk_workspace(good(d=96))


def test_append_null_and_alignment():
    sh = good()
    assert append(None) == -1
    for n in ("k_new", "v_new", "table", "seq_lens", "new_rows", "new_lens", "K", "V", "q", "q_out", "inv_freq"):
        assert append(sh, **{n: NULL}) == -1, n
    assert append(good(dtype=5), q=NULL) == -3             # the shape comes first
    for n in ("k_new", "v_new", "K", "V", "q", "q_out"):
        assert append(sh, **{n: ctypes.c_void_p(0x10008)}) == -2, n
    assert append(sh, inv_freq=ctypes.c_void_p(0x10004)) == -2
    for n in ("table", "seq_lens", "new_rows", "new_lens", "positions"):
        assert append(sh, **{n: ctypes.c_void_p(0x10002)}) == -2, n


def test_attention_null_alignment_and_workspace():
    sh = good()
    assert attend(None) == -1
    for n in ("q", "K", "V", "table", "seq_lens", "new_rows", "new_lens", "out"):
        assert attend(sh, **{n: NULL}) == -1, n
    for n in ("q", "K", "V", "out"):
        assert attend(sh, **{n: ctypes.c_void_p(0x10008)}) == -2, n
    for n in ("table", "seq_lens", "new_rows", "new_lens", "lse"):
        assert attend(sh, **{n: ctypes.c_void_p(0x10001)}) == -2, n
    assert attend(sh, ws=NULL) == -6
    assert attend(sh, ws=ctypes.c_void_p(0x10010)) == -6
    # a contiguous cache needs no table: the checks go on to the workspace
    flat = good(page_size=0, max_pages_per_seq=0, n_pages=2, kv_strides=(1000 * 256, 256, 128))
    assert attend(flat, table=NULL, ws_bytes=0) == -6


def sample(logits=OK, dtype=1, stride=0, rows=4, V=1000, u=OK, tokens=OK, probs=OK, ws=OK, ws_bytes=1 << 40, settings=OK):
    return S.lib().svf_sample(logits, dtype, stride, rows, V, settings, settings, settings, settings, u, tokens, probs, ws, ws_bytes, None)


def test_sampling_refusals():
    assert sample(dtype=2) == -3 and sample(dtype=-1) == -3
    assert sample(logits=NULL) == -1
    assert sample(u=NULL) == -1 and sample(tokens=NULL) == -1
    assert sample(u=NULL, tokens=NULL, probs=NULL) == -1
    for kw in (dict(rows=0), dict(rows=-1), dict(V=0), dict(V=524289), dict(stride=999), dict(stride=-1000)):
        assert sample(**kw) == -2, kw
    assert sample(logits=ctypes.c_void_p(0x10001)) == -2
    assert sample(dtype=0, logits=ctypes.c_void_p(0x10002)) == -2
    for n in ("u", "tokens", "probs", "settings"):
        assert sample(**{n: ctypes.c_void_p(0x10002)}) == -2, n
    assert sample(ws=NULL) == -6 and sample(ws=ctypes.c_void_p(0x10080)) == -6
    n = S.svf_sample_workspace_bytes(4, 1000)
    assert n > 0 and n % 256 == 0 and sample(ws_bytes=n - 1) == -6
    assert S.svf_sample_workspace_bytes(0, 1000) == 0 and S.svf_sample_workspace_bytes(4, 524289) == 0
    with pytest.raises(S.SvfError):
        S.new_sample_workspace(1, 0)


def test_python_arguments():
    """The binding's own refusals (CPU tensors stand in for device memory: nothing is launched)."""
    import torch
    ws = torch.empty(0)
    with pytest.raises((AttributeError, TypeError)):       # (no data_ptr())
        S.svf_sample("logits", None, None, ws)
    with pytest.raises(ValueError):
        S.svf_sample(torch.zeros(8), None, None, ws)
    with pytest.raises(ValueError):
        S.svf_sample(torch.zeros(4, 8).t(), None, None, ws)
    with pytest.raises(ValueError):
        S.svf_sample(torch.zeros(8).expand(4, 8), None, None, ws)
    with pytest.raises(TypeError):
        S.svf_chunk_attn(S.make_shape(B=1, gamma=1, Hq=1, Hkv=1, d=64, dtype="bf16", block_size=16, max_seq_len=16, k_blocks=1,
                                      kv_strides=(64, 64, 64)), *[None] * 9)
    with pytest.raises(TypeError):
        S.svf_append_kv(good(), None)


def test_sampling_arguments_have_the_types_and_sizes_that_are_read():
    """(CPU tensors: every call is refused by the binding.)"""
    import torch
    R, V = 4, 9
    good = dict(logits=torch.zeros(R, V), u=torch.zeros(R), tokens=torch.zeros(R, dtype=torch.int32), temperature=torch.ones(R),
                top_k=torch.ones(R, dtype=torch.int32), top_p=torch.ones(R), min_p=torch.ones(R), probs=torch.zeros(R, V))

    def call(**kw):
        S.svf_sample(**{**good, **kw}, ws=torch.empty(0, dtype=torch.uint8))
    for n in ("u", "temperature", "top_p", "min_p", "probs"):
        for dt in (torch.float64, torch.bfloat16, torch.int32):
            with pytest.raises(TypeError, match=n):
                call(**{n: good[n].to(dt)})
    for n in ("tokens", "top_k"):
        for dt in (torch.int64, torch.float32, torch.int16):
            with pytest.raises(TypeError, match=n):
                call(**{n: good[n].to(dt)})
    for n, x in good.items():
        if n != "logits":
            with pytest.raises(ValueError, match=n):
                call(**{n: x[:R - 1]})
            with pytest.raises(ValueError, match=n):
                call(**{n: torch.stack((x, x), -1)[..., 0]})
    with pytest.raises(ValueError, match="probs"):
        call(probs=torch.zeros(R, V - 1))


def test_shapes_at_the_limits():
    for kw in (dict(max_new=1 << 22), dict(n_rows=1 << 28), dict(max_seq_len=1 << 30, page_size=0, n_pages=2), dict(Hq=4096, Hkv=4096), dict(B=4096),
               dict(Hq=512, Hkv=2), dict(kv_strides=((1 << 34) - 8, 256, 128)), dict(kv_strides=(4096, (1 << 34) - 8, 128)),
               dict(kv_strides=(4096, 256, (1 << 34) - 8)), dict(window=(1 << 31) - 1), dict(rotary_dim=128)):
        assert S.svf_chunk_workspace_bytes(good(**kw)) > 0, kw
    for kw in (dict(max_new=(1 << 22) + 1), dict(n_rows=(1 << 28) + 1), dict(Hq=4100, Hkv=4100), dict(kv_strides=(1 << 34, 256, 128)),
               dict(kv_strides=(4096, 1 << 34, 128)), dict(kv_strides=(4096, 256, 1 << 34))):
        assert both(good(**kw)) == -2, kw
