"""svf_chunk_attn against the fp64 oracle.

Bars, from the arithmetic.  A logit is a sum of d exact products in fp32, scaled: off by at most
e = (d + 64) 2^-24 times the scaled sum of |q_c k_c| (the 64 for the scaling, the maximum and the exponential of
an argument of that size) + 1e-6.  A weight is then off by that relative, in bf16 by another half step
(2^-8), and every sum of n terms in fp32 by n 2^-24: the output by at most
A (2 e + 2^-8 + 2 n 2^-24), A the weighted sum of |V|, plus half a step of its own; the log-sum-exp by
e + n 2^-24 and two of its own steps."""
import math

import numpy as np
import pytest
import torch

import paper_2512_21911_amd as S
from oracle import cache_oracle as O

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def build(lens, news, *, dtype=torch.bfloat16, Hq=8, Hkv=2, d=128, page=16, window=0, gaps=0, head_major=False, seed=0, gain=1.0,
          max_new=None, max_seq_len=None, scale=0.0, q_pad=0):
    g = torch.Generator().manual_seed(seed)
    B = len(lens)
    rows, at = [], 0
    for n in news:
        rows.append(at + gaps)
        at += gaps + n
    n_rows = max(at + gaps, 1)
    T = max_seq_len or max(max(max(L, 0) + n for L, n in zip(lens, news)), 1)
    if page:
        per = -(-T // page)
        n_pages = B * per + 1
        table = torch.randperm(n_pages - 1, generator=g)[:B * per].reshape(B, per).to(torch.int32) + 1
        slots = page
    else:
        table, n_pages, slots, per = None, B, T, 0
    shape = (n_pages, Hkv, slots, d) if head_major else (n_pages, slots, Hkv, d)
    K, V = (torch.randn(shape, generator=g).to(dtype) for _ in range(2))
    if head_major:
        K, V = K.permute(0, 2, 1, 3), V.permute(0, 2, 1, 3)
    # places that no new token sees hold NaN
    seen = torch.zeros(n_pages, slots, dtype=torch.bool)
    for b, (L, n) in enumerate(zip(lens, news)):
        if n:
            for t in range(max(0, L + 1 - window) if window else 0, L + n):
                seen[O.place(t, b, table, page)] = True
    K[~seen], V[~seen] = float("nan"), float("nan")
    q = (gain * torch.randn(n_rows, Hq + q_pad, d, generator=g)).to(dtype)[:, :Hq]
    x = dict(q=q, K=K, V=V, table=table, seq_lens=torch.tensor(lens, dtype=torch.int32),
             new_rows=torch.tensor(rows, dtype=torch.int32), new_lens=torch.tensor(news, dtype=torch.int32))
    sh = S.make_chunk_shape(B=B, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, max_seq_len=T, max_new=max_new or max(1, max(news)), n_rows=n_rows,
                            n_pages=n_pages, page_size=page, max_pages_per_seq=per, k_pool=K, window=window,
                            q_stride=(Hq + q_pad) * d, out_stride=(Hq + q_pad) * d, sm_scale=scale)
    return sh, x


def to_gpu(x):
    out = {}
    for n, t in x.items():
        if t is None:
            out[n] = None
            continue
        c = torch.empty(t.stride(0) * t.shape[0] if t.dim() > 1 else t.numel(), dtype=t.dtype, device="cuda")
        out[n] = c.as_strided(t.shape, t.stride())
        out[n].copy_(t)
    return out


def call(sh, g, ws=None, fill=3.0):
    out = torch.full_like(g["q"], fill) if g["q"].is_contiguous() else \
        torch.full((g["q"].stride(0) * g["q"].shape[0],), fill, dtype=g["q"].dtype, device="cuda").as_strided(g["q"].shape, g["q"].stride())
    lse = torch.full((sh.n_rows, sh.Hq), fill, device="cuda")
    if ws is None:
        ws = S.new_chunk_workspace(sh)
    S.svf_chunk_attn(sh, g["q"], g["K"], g["V"], g["table"], g["seq_lens"], g["new_rows"], g["new_lens"], out, ws, lse=lse)
    torch.cuda.synchronize()
    return out, lse


def verify(sh, x, out, lse, fill=3.0):
    seqs = O.sequences(x["seq_lens"].tolist(), x["new_rows"].tolist(), x["new_lens"].tolist(), sh.max_seq_len, sh.max_new, sh.n_rows)
    scale = sh.sm_scale if sh.sm_scale > 0 else 1 / math.sqrt(sh.d)
    ref, ref_lse, mag, size = O.attend(x["q"].double().numpy(), x["K"].double().numpy(), x["V"].double().numpy(), x["table"], sh.page_size, seqs,
                                       sh.Hq // sh.Hkv, scale, sh.window)
    dt = x["q"].dtype
    live = np.zeros(sh.n_rows, dtype=bool)
    keys = np.ones(sh.n_rows)
    for _, L, r, n in seqs:
        live[r:r + n] = True
        keys[r:r + n] = min(L + n, sh.window) if sh.window else L + n
    got, got_lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
    assert (got[~live] == fill).all() and (got_lse[~live] == fill).all(), "rows of no sequence were written"
    e = (sh.d + 64) * 2.0 ** -24 * size + 1e-6
    n = keys[:, None] * 2.0 ** -24
    weights = HALF[dt] if dt == torch.bfloat16 else 0.0
    tol = mag * (2 * e + weights + 2 * n)[..., None] + HALF[dt] * np.abs(ref)
    off = (np.abs(got - ref) - tol)[live]
    assert not np.isnan(got[live]).any() and (off <= 0).all(), f"out off by {np.nanmax(off):.3e} more than allowed"
    off = (np.abs(got_lse - ref_lse) - (e + n + 2.0 ** -22 * np.abs(ref_lse)))[live]
    assert (off <= 0).all(), f"lse off by {off.max():.3e} more than allowed"


def check(sh, x):
    g = to_gpu(x)
    out, lse = call(sh, g)
    verify(sh, x, out, lse)
    return g, out, lse


DTYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("L,n", [(0, 1), (0, 2), (1, 1), (62, 1), (63, 1), (64, 1), (0, 63), (0, 64), (0, 65), (31, 33), (500, 7), (1000, 1)])
def test_lengths(dtype, d, L, n):
    check(*build([L], [n], dtype=dtype, d=d))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 1), (4, 4), (32, 8), (32, 4), (10, 2), (64, 1)])
def test_head_groups(dtype, Hq, Hkv):
    check(*build([5, 130], [70, 3], dtype=dtype, Hq=Hq, Hkv=Hkv, d=64))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page,head_major", [(0, False), (0, True), (1, False), (7, False), (16, True), (24, False), (64, False), (100, True)])
def test_pages(dtype, page, head_major):
    check(*build([0, 77, 200], [40, 1, 30], dtype=dtype, page=page, head_major=head_major))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window", [1, 2, 50, 64, 65, 200, 5000])
def test_windows(dtype, d, window):
    check(*build([0, 300, 129], [90, 1, 70], dtype=dtype, d=d, window=window, Hq=4, Hkv=1))


@pytest.mark.parametrize("dtype", DTYPES)
def test_mixed_batches_gaps_and_empty_sequences(dtype):
    check(*build([0, 400, 33, 0, 64, 10, 7], [0, 1, 130, 1, 0, 64, 0], dtype=dtype, gaps=2, q_pad=4))
    check(*build([9], [0], dtype=dtype))                   # nothing at all
    check(*build([b * 13 % 90 for b in range(150)], [b % 3 for b in range(150)], dtype=dtype, Hq=2, Hkv=1, d=64))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens,news", [([3000], [1]), ([2900, 10], [1, 200]), ([5, 1500, 0], [3, 260, 300])])
def test_work_cut_anywhere(dtype, lens, news):
    """Long and short sequences side by side, so that ranges of work begin and end inside of items."""
    check(*build(lens, news, dtype=dtype, Hq=4, Hkv=2, d=128, page=32))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("gain", [0.0, 30.0])
def test_flat_and_peaked_weights(dtype, gain):
    check(*build([300, 1], [40, 64], dtype=dtype, gain=gain))


@pytest.mark.parametrize("dtype", DTYPES)
def test_rising_logits_move_the_maximum(dtype):
    """Keys that grow along the sequence: every tile raises the maximum, by little and by much."""
    for step in (0.002, 0.05):
        sh, x = build([700], [40], dtype=dtype, Hq=2, Hkv=1, d=64, page=0)
        x["K"] = x["K"] * 0.1 + step * torch.arange(x["K"].shape[1])[None, :, None, None]
        x["K"] = x["K"].to(dtype)
        x["q"] = (x["q"].abs() * 0.3).to(dtype)
        check(sh, x)


def test_scale_and_shape_limits():
    check(*build([100], [5], scale=0.5, gain=0.2))
    # lengths that the shape has no room for
    sh, x = build([90, 100, 30], [9, 9, 9], max_seq_len=100, max_new=6)
    x["seq_lens"] = torch.tensor([97, 100, -4], dtype=torch.int32)
    x["K"], x["V"] = torch.nan_to_num(x["K"]), torch.nan_to_num(x["V"])
    check(sh, x)
    x["seq_lens"] = torch.tensor([2, 3, 4], dtype=torch.int32)
    x["new_rows"] = torch.tensor([0, 24, -1], dtype=torch.int32)
    check(sh, x)


@pytest.mark.parametrize("dtype", DTYPES)
def test_pages_outside_the_pool_stay_in_bounds(dtype):
    """Bad entries are read as page 0; rows that do not see them keep their results."""
    sh, x = build([0, 100], [60, 5], dtype=dtype, page=16)
    good = to_gpu(x)
    want, want_lse = call(sh, good)
    bad = to_gpu(x)
    bad["K"][0], bad["V"][0] = 1.0, 1.0
    bad["table"][0, 3], bad["table"][1, 0] = sh.n_pages, -7
    out, lse = call(sh, bad)
    assert torch.equal(out[:48], want[:48]) and torch.equal(lse[:48], want_lse[:48])
    assert not torch.isnan(out).any()


@pytest.mark.parametrize("dtype", DTYPES)
def test_same_bits_from_call_to_call_and_under_capture(dtype):
    sh, x = build([2000, 30, 0], [1, 140, 77], dtype=dtype, Hq=8, Hkv=2)
    g, out, lse = check(sh, x)
    ws = S.new_chunk_workspace(sh)
    for _ in range(3):
        o, l = call(sh, g, ws)
        assert torch.equal(o, out) and torch.equal(l, lse)
    st = torch.cuda.Stream()
    o, l = torch.empty_like(out), torch.empty_like(lse)
    # two graphs that share the workspace, replayed in turn with other shapes' work in between
    sh2, x2 = build([100, 900], [200, 1], dtype=dtype, Hq=8, Hkv=2, seed=5)
    g2, out2, lse2 = check(sh2, x2)
    big = torch.zeros(max(ws.numel(), S.svf_chunk_workspace_bytes(sh2)), dtype=torch.uint8, device="cuda")
    o2, l2 = torch.empty_like(out2), torch.empty_like(lse2)
    graphs = []
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        for s, y, a, b in ((sh, g, o, l), (sh2, g2, o2, l2)):
            gr = torch.cuda.CUDAGraph()
            with torch.cuda.graph(gr, stream=st):
                S.svf_chunk_attn(s, y["q"], y["K"], y["V"], y["table"], y["seq_lens"], y["new_rows"], y["new_lens"], a, big, lse=b)
            graphs.append(gr)
    for _ in range(3):
        for t in (o, l, o2, l2):
            t.fill_(3.0)
        torch.cuda.synchronize()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert torch.equal(o, out) and torch.equal(l, lse) and torch.equal(o2, out2) and torch.equal(l2, lse2)


@pytest.mark.parametrize("d", [64, 128])
def test_single_tokens_of_many_batches_share_a_workspace(d):
    """The kernel for few rows joins the parts of its items by counters in the workspace: batches of every kind behind one another, each
    twice, with the same bits."""
    ws = None
    for i, (lens, news) in enumerate([([3000], [1]), ([0], [1]), ([63, 64, 65], [1, 1, 1]), ([5000, 3, 0, 900], [1, 0, 1, 1]),
                                      ([40] * 130, [1] * 130), ([1000] * 9, [1] * 9), ([31], [4]), ([2500, 700], [4, 2])]):
        sh, x = build(lens, news, Hq=16, Hkv=4 if i % 2 else 2, d=d, page=16, seed=i)
        sh.max_new = 2 if max(news) < 3 else 4
        if ws is None:
            ws = S.new_chunk_workspace(sh)
        assert S.svf_chunk_workspace_bytes(sh) <= ws.numel()
        g = to_gpu(x)
        out, lse = call(sh, g, ws)
        verify(sh, x, out, lse)
        again, lse2 = call(sh, g, ws)
        assert torch.equal(again, out) and torch.equal(lse2, lse)


def test_lengths_change_under_a_captured_call():
    """A graph of a shape's upper bounds serves every batch within them."""
    sh, x = build([600, 600], [100, 100], page=32)
    x["K"], x["V"] = torch.nan_to_num(x["K"]), torch.nan_to_num(x["V"])
    g = to_gpu(x)
    ws = S.new_chunk_workspace(sh)
    out, lse = torch.empty_like(g["q"]), torch.empty(sh.n_rows, sh.Hq, device="cuda")
    call(sh, g, ws)
    st = torch.cuda.Stream()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.stream(st), torch.cuda.graph(gr, stream=st):
        S.svf_chunk_attn(sh, g["q"], g["K"], g["V"], g["table"], g["seq_lens"], g["new_rows"], g["new_lens"], out, ws, lse=lse)
    for lens, news in (([600, 600], [100, 100]), ([0, 599], [1, 2]), ([17, 0], [0, 0]), ([300, 64], [64, 1])):
        x["seq_lens"], x["new_lens"] = torch.tensor(lens, dtype=torch.int32), torch.tensor(news, dtype=torch.int32)
        g["seq_lens"].copy_(x["seq_lens"])
        g["new_lens"].copy_(x["new_lens"])
        out.fill_(3.0)
        lse.fill_(3.0)
        gr.replay()
        torch.cuda.synchronize()
        verify(sh, x, out, lse)


def test_offsets_past_32_bits():
    """A pool of more than 2^32 bytes, its last pages in use."""
    d, Hkv, page = 128, 8, 64
    n_pages = (1 << 32) // (page * Hkv * d * 2) + 40       # bytes; elements pass 2^31 on the way
    K = torch.empty(n_pages, page, Hkv, d, dtype=torch.bfloat16, device="cuda")
    V = torch.empty(n_pages, page, Hkv, d, dtype=torch.bfloat16, device="cuda")
    sh, x = build([150], [20], Hq=8, Hkv=Hkv, d=d, page=page)
    used = x["table"].reshape(-1).long()
    far = n_pages - 1 - torch.arange(used.numel())
    K[far.cuda()], V[far.cuda()] = x["K"][used].cuda(), x["V"][used].cuda()
    g = to_gpu({n: x[n] for n in ("q", "seq_lens", "new_rows", "new_lens")})
    g.update(K=K, V=V, table=far.to(torch.int32).reshape(x["table"].shape).cuda())
    sh.n_pages = n_pages
    out, lse = call(sh, g)
    verify(sh, x, out, lse)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,Hkv,L,n", [(32, 8, 300, 1), (31, 8, 300, 1), (3, 2, 700, 130), (6, 2, 400, 200)])
def test_items_of_like_size_are_not_cut(dtype, B, Hkv, L, n):
    # no more items than workgroups, all about as large: each has a workgroup of its own; one far longer sequence among them, and they are cut
    for longest in (L, 6000):
        lens = [L + 3 * i for i in range(B)]
        lens[B // 2] = longest
        check(*build(lens, [max(1, n - 5 * i) for i in range(B)], dtype=dtype, Hq=4 * Hkv, Hkv=Hkv, d=64))


def test_shapes_of_both_kernels_share_a_workspace():
    cases = [build([300, 20], [200, 130], Hq=8, Hkv=2, d=128, seed=1), build([3000, 5], [1, 1], Hq=8, Hkv=2, d=128, seed=2),
             build([900], [40], Hq=4, Hkv=1, d=64, dtype=torch.float32, seed=3), build([2000, 70, 0], [1, 3, 2], Hq=8, Hkv=2, d=64, seed=4)]
    alone = [call(sh, to_gpu(x)) for sh, x in cases]
    ws = max((S.new_chunk_workspace(sh) for sh, _ in cases), key=lambda w: w.numel())
    for i in (0, 1, 2, 3, 1, 0, 3, 2, 0, 1):
        sh, x = cases[i]
        out, lse = call(sh, to_gpu(x), ws=ws)
        assert torch.equal(out, alone[i][0]) and torch.equal(lse, alone[i][1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,news,window", [([0], [64], 0), ([0, 70], [200, 65], 1), ([3, 300], [130, 90], 50), ([0, 1500], [260, 300], 0),
                                              ([0, 63, 5], [1, 2, 1], 0)])
@pytest.mark.parametrize("level", [7.0, 30.0])
def test_scores_far_below_zero(dtype, d, lens, news, window, level):
    """The first keys that a row sees score -100 and less: what it has summed until then, nothing, stays nothing."""
    sh, x = build(lens, news, dtype=dtype, d=d, window=window)
    x["K"] = (x["K"] * 0.125 + 2.0).to(dtype)
    x["q"] = (x["q"].abs() * 0.25 - level).to(dtype)       # scores of -2 (level - 0.2) sqrt(d)
    check(sh, x)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rise", [0.1, 0.3, 1.0])
def test_large_values_under_rising_scores(dtype, d, rise):
    """Values of up to 2^125 / (tokens + 64), scores that rise by 0.1 to 1 a key: weights relative to an early key stay small enough."""
    sh, x = build([900] * 6, [40] * 6, dtype=dtype, Hq=8, Hkv=8, d=d, page=0)   # (items that are not cut)
    slots = x["K"].shape[1]
    x["K"] = (x["K"] * 0.01 + rise * d ** -0.5 * torch.arange(slots)[None, :, None, None]).to(dtype)
    x["q"] = torch.ones_like(x["q"])
    x["V"] = (x["V"].clamp(-4, 4) * 2.0 ** 112).to(dtype)  # 4 x 2^112 x (940 + 64) < 2^125
    check(sh, x)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window", [(1 << 31) - 1, (1 << 31) - 2, (1 << 31) - 200, 1 << 30])
def test_windows_of_any_size(dtype, window):
    """A window that no sequence fills is none."""
    for lens, news, Hq, Hkv in (([0], [300], 8, 2), ([50, 0], [700, 3], 2, 2), ([0, 900, 7], [1, 1, 1], 8, 2)):
        sh, x = build(lens, news, dtype=dtype, Hq=Hq, Hkv=Hkv, d=64)
        g = to_gpu(x)
        want, want_lse = call(sh, g)
        sh.window = window
        out, lse = call(sh, g)
        verify(sh, x, out, lse)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
