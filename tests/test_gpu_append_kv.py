"""svf_append_kv against the fp64 oracle.

Bars.  Copied channels and everything the call must not touch: the same bits.  Rotated channels: the
fp32 rotation is off by at most 2^-24 for each of its two products and its sum and 2^-22 for sine and
cosine (two steps of the fp32 function, and its argument's rounding: pi 2^-25), i.e. 2^-21 (|x| + |y|), then
half a step of the element type."""
import numpy as np
import pytest
import torch

import paper_2512_21911_amd as S
from oracle import cache_oracle as O

pytestmark = pytest.mark.gpu

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def build(lens, news, *, dtype=torch.bfloat16, Hq=8, Hkv=2, d=128, page=16, rotary=128, interleaved=False, gaps=0, head_major=False,
          packed=True, seed=0, max_seq_len=None, max_new=None):
    """A batch with `gaps` rows in front of every sequence's, caches full of a pattern, pages in random order."""
    g = torch.Generator().manual_seed(seed)
    B = len(lens)
    rows, at = [], 0
    for n in news:
        rows.append(at + gaps)
        at += gaps + n
    n_rows = max(at + gaps, 1)
    need = [max(L, 0) + max(n, 0) for L, n in zip(lens, news)]
    T = max_seq_len or max(max(need), 1)
    if page:
        per = -(-T // page)
        n_pages = B * per + 2
        table = torch.randperm(n_pages, generator=g)[:B * per].reshape(B, per).to(torch.int32)
        slots = page
    else:
        table, n_pages, slots, per = None, B, T, 0
    shape = (n_pages, Hkv, slots, d) if head_major else (n_pages, slots, Hkv, d)
    K, V = (torch.randn(shape, generator=g).to(dtype) for _ in range(2))
    if head_major:
        K, V = K.permute(0, 2, 1, 3), V.permute(0, 2, 1, 3)
    heads = Hq + 2 * Hkv
    qkv = torch.randn(n_rows, heads, d, generator=g).to(dtype)
    x = dict(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:], K=K, V=V, table=table,
             seq_lens=torch.tensor(lens, dtype=torch.int32), new_rows=torch.tensor(rows, dtype=torch.int32),
             new_lens=torch.tensor(news, dtype=torch.int32),
             inv_freq=10000.0 ** (-torch.arange(rotary // 2, dtype=torch.float64) / max(1, rotary // 2)))
    stride = heads * d
    if not packed:
        x.update({n: x[n].contiguous() for n in "qkv"})
        stride = 0
    sh = S.make_chunk_shape(B=B, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, max_seq_len=T, max_new=max_new or max(1, max(news)), n_rows=n_rows,
                            n_pages=n_pages, page_size=page, max_pages_per_seq=per, k_pool=K, q_stride=stride, k_stride=stride,
                            v_stride=stride, rotary_dim=rotary, rotary_interleaved=interleaved)
    return sh, x


def gpu(x):
    def move(t):
        if t is None:
            return None
        c = torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda")
        c.copy_(t)
        return c
    flat = {n: move(t) for n, t in x.items()}
    if x["q"].stride(0) != x["q"].shape[1] * x["q"].shape[2]:          # side by side, as they came
        heads = sum(x[n].shape[1] for n in "qkv")
        qkv = torch.empty(x["q"].shape[0], heads, x["q"].shape[2], dtype=x["q"].dtype, device="cuda")
        at = 0
        for n in "qkv":
            h = x[n].shape[1]
            qkv[:, at:at + h] = x[n].cuda()
            flat[n] = qkv[:, at:at + h]
            at += h
    return flat


def like(q, fill):
    """A tensor with the rows of q as far apart as they are (the shape has one stride for both)."""
    out = torch.empty_strided(q.shape, q.stride(), dtype=q.dtype, device="cuda")
    return out.fill_(fill)


def check(sh, x, positions=None, with_q=True, in_place=False):
    g = gpu(x)
    q_out = None
    if with_q:
        q_out = g["q"] if in_place else like(g["q"], 7.0)
    before = q_out.clone() if with_q else None
    S.svf_append_kv(sh, g["k"], g["v"], g["table"], g["seq_lens"], g["new_rows"], g["new_lens"], g["K"], g["V"],
                    q=g["q"] if with_q else None, q_out=q_out, inv_freq=g["inv_freq"] if sh.rotary_dim else None,
                    positions=None if positions is None else positions.cuda())
    torch.cuda.synchronize()
    dt = x["q"].dtype
    K, V, Q = x["K"].clone(), x["V"].clone(), before.cpu() if with_q else None
    rot = sh.rotary_dim
    inv = x["inv_freq"].numpy()
    scale = sh.rotary_scale if sh.rotary_scale > 0 else 1.0
    tolK = torch.zeros(K.shape, dtype=torch.float64)
    tolQ = torch.zeros(Q.shape, dtype=torch.float64) if with_q else None
    refK, refQ = K.double(), Q.double() if with_q else None
    for b, L, r, n in O.sequences(x["seq_lens"].tolist(), x["new_rows"].tolist(), x["new_lens"].tolist(), sh.max_seq_len,
                                  sh.max_new, sh.n_rows):
        for j in range(n):
            pg, sl = O.place(L + j, b, x["table"], sh.page_size)
            V[pg, sl] = x["v"][r + j]
            pos = L + j if positions is None else int(positions[r + j])

            def turned(t):
                y = t.double().numpy()
                ref = O.rotate(y, pos, inv, sh.rotary_interleaved, scale) if rot else y
                ones = np.abs(y)
                half = rot // 2
                i = np.arange(half)
                a, c = (2 * i, 2 * i + 1) if sh.rotary_interleaved else (i, i + half)
                tol = np.zeros_like(y)
                both = ones[..., a] + ones[..., c]
                for k in (a, c):
                    tol[..., k] = scale * both * 2.0 ** -21 + np.abs(ref[..., k]) * HALF_STEP[dt]
                return torch.from_numpy(ref), torch.from_numpy(tol)
            refK[pg, sl], tolK[pg, sl] = turned(x["k"][r + j])
            if with_q:
                refQ[r + j], tolQ[r + j] = turned(x["q"][r + j])
    assert torch.equal(g["V"].cpu(), V)
    for got, ref, tol in ((g["K"].cpu(), refK, tolK),) + (((q_out.cpu(), refQ, tolQ),) if with_q else ()):
        off = (got.double() - ref).abs() - tol
        assert (off <= 0).all(), f"off by {off.max():.3e} more than allowed"
    return g, q_out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,rotary,interleaved", [(128, 128, False), (128, 128, True), (128, 32, False), (64, 64, False), (64, 16, True),
                                                  (64, 48, False), (128, 112, True), (64, 0, False), (128, 0, True)])
def test_styles_and_partial_rotation(dtype, d, rotary, interleaved):
    check(*build([0, 5, 40], [3, 1, 18], dtype=dtype, d=d, rotary=rotary, interleaved=interleaved))


@pytest.mark.parametrize("page,head_major", [(0, False), (1, False), (16, True), (24, False), (64, True), (7, False)])
@pytest.mark.parametrize("gaps", [0, 3])
def test_pages_orders_and_gaps(page, head_major, gaps):
    check(*build([0, 31, 16, 7], [5, 0, 1, 33], page=page, head_major=head_major, gaps=gaps, Hq=12, Hkv=4, packed=gaps == 0))


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 1), (32, 8), (5, 5), (48, 4)])
def test_head_counts(Hq, Hkv):
    check(*build([3, 100], [2, 9], Hq=Hq, Hkv=Hkv, d=64, rotary=64))


def test_many_rows_take_the_kernel_of_four():
    sh, x = build([0, 17, 2], [700, 3, 401], Hq=2, Hkv=1, d=64, rotary=32, gaps=1)
    assert sh.n_rows > 1024
    check(sh, x)
    check(*build([0, 17, 2], [700, 3, 401], Hq=2, Hkv=2, d=128, rotary=128, interleaved=True, dtype=torch.float32, page=0))


def test_many_sequences():
    lens = [(7 * b) % 50 for b in range(200)]
    check(*build(lens, [1 if b % 5 else 0 for b in range(200)], Hq=2, Hkv=1, d=64, rotary=64))


def test_in_place_and_without_queries():
    check(*build([4, 9], [3, 6]), in_place=True)
    check(*build([4, 9], [3, 6]), with_q=False)
    check(*build([4, 9], [3, 6], rotary=0), with_q=False)


def test_positions_of_their_own_far_out():
    sh, x = build([0, 5], [6, 4])
    sh.rotary_scale = 1.25
    check(sh, x, positions=torch.tensor([0, 1, 1, 2, 2, 2, 131071, 1048575, 2 ** 30 + 1, 3], dtype=torch.int32))


def test_what_the_shape_has_no_room_for_is_left_out():
    sh, x = build([10, 20, -1, 5, 9], [8, 8, 8, 8, 8], max_seq_len=28, max_new=6)
    x["seq_lens"] = torch.tensor([25, 28, -1, 5, 9], dtype=torch.int32)
    x["new_rows"] = torch.tensor([0, 8, 16, 35, -3], dtype=torch.int32)
    x["new_lens"] = torch.tensor([8, 8, 8, 100, 8], dtype=torch.int32)
    check(sh, x)


def test_pages_outside_the_pool_are_not_written():
    sh, x = build([0, 0], [40, 40], page=16)
    bad = x["table"].clone()
    x["table"] = bad.clone()
    g = gpu(x)
    g["table"][0, 1], g["table"][1, 2] = sh.n_pages, -5
    q_out = like(g["q"], 0.0)
    before = g["K"].clone(), g["V"].clone()
    S.svf_append_kv(sh, g["k"], g["v"], g["table"], g["seq_lens"], g["new_rows"], g["new_lens"], g["K"], g["V"], q=g["q"], q_out=q_out,
                    inv_freq=g["inv_freq"])
    torch.cuda.synchronize()
    skipped = [int(bad[0, 1]), int(bad[1, 2])]
    written = [int(bad[0, 0]), int(bad[0, 2]), int(bad[1, 0]), int(bad[1, 1])]
    for now, then in zip((g["K"], g["V"]), before):
        for p in range(sh.n_pages):
            same = torch.equal(now[p], then[p])
            assert same if p in skipped or p not in written else not same


def test_captured_and_replayed_on_another_stream():
    sh, x = build([0, 33], [4, 1])
    g, q_out = check(sh, x)
    want = g["K"].clone(), q_out.clone()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        g["K"].zero_()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            S.svf_append_kv(sh, g["k"], g["v"], g["table"], g["seq_lens"], g["new_rows"], g["new_lens"], g["K"], g["V"], q=g["q"],
                            q_out=q_out, inv_freq=g["inv_freq"])
    for _ in range(3):
        q_out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q_out, want[1])
        written = g["K"].abs().sum(-1) > 0
        assert torch.equal(g["K"][written], want[0][written]) and int(written.sum()) == 5 * sh.Hkv


def test_more_rows_than_a_grid_has_threads_in_x():
    # (workgroups of 256 threads, one to four rows each; one sequence, in the last rows)
    n_rows, n = (1 << 26) + 7, 6
    sh, x = build([3], [n], Hq=1, Hkv=1, d=64, rotary=64, packed=False)
    K, V = x["K"].cuda(), x["V"].cuda()
    big = [torch.empty(n_rows, 1, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for b, name in zip(big, "kv"):
        b[-n:] = x[name].cuda()
    sh.n_rows = n_rows
    S.svf_append_kv(sh, big[0], big[1], x["table"].cuda(), x["seq_lens"].cuda(), torch.tensor([n_rows - n], dtype=torch.int32, device="cuda"),
                    x["new_lens"].cuda(), K, V, inv_freq=x["inv_freq"].cuda())
    small = dict(K=x["K"].cuda(), V=x["V"].cuda())
    sh.n_rows = n
    S.svf_append_kv(sh, x["k"].cuda(), x["v"].cuda(), x["table"].cuda(), x["seq_lens"].cuda(), x["new_rows"].cuda(), x["new_lens"].cuda(),
                    small["K"], small["V"], inv_freq=x["inv_freq"].cuda())
    torch.cuda.synchronize()
    assert torch.equal(K, small["K"]) and torch.equal(V, small["V"]) and not torch.equal(K, x["K"].cuda())
