"""A prompt, two verification steps and the tokens in between, as a server makes the calls: prompts are appended
and attended in chunks (svf_append_kv, svf_chunk_attn), the first token is sampled (svf_sample), drafts are verified over
the cache that was built (svf_block_reps, svf_verify_step), accepted (svf_accept_resample) and appended.

Bars.  The cache is the one that the oracle's rotation gives; attention over it is checked by its own bars in
test_gpu_chunk_attn; with a budget of all blocks the drafts' attention is the attention of a chunk: both are within
their bar of the exact result (2^-7 A and half a step of the output, A the weighted sum of |V| <= max |V|)."""
import numpy as np
import pytest
import torch

import paper_2512_21911_amd as S
from oracle import cache_oracle as O
from test_gpu_chunk_attn import verify

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_prompts_then_verification_steps(dtype):
    torch.manual_seed(3)
    B, Hq, Hkv, d, page, T, block, gamma = 3, 8, 2, 128, 16, 512, 64, 5
    G, per = Hq // Hkv, T // page
    prompts = [200, 77, 131]
    table = torch.randperm(B * per)[:B * per].reshape(B, per).to(torch.int32)
    K = torch.zeros(B * per, page, Hkv, d, dtype=dtype, device="cuda")
    V = torch.zeros_like(K)
    dev_table = table.cuda()
    inv = 10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))
    heads = Hq + 2 * Hkv
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    mirror_k = [np.zeros((0, Hkv, d))] * B                  # fp64: unrotated keys, values in order

    def shape(n_rows, max_new, **kw):
        return S.make_chunk_shape(B=B, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, max_seq_len=T, max_new=max_new, n_rows=n_rows, n_pages=B * per,
                                  page_size=page, max_pages_per_seq=per, k_pool=K, rotary_dim=d, **kw)

    def cache_of(b, n):
        t = np.arange(n)
        pg = table[b].numpy()[t // page]
        return K.cpu()[pg, t % page].double().numpy()

    # prompts in chunks of 64 tokens
    done = [0] * B
    while any(x < p for x, p in zip(done, prompts)):
        new = [min(64, p - x) for x, p in zip(done, prompts)]
        rows = np.cumsum([0] + new)
        n_rows = int(rows[-1])
        qkv = torch.randn(n_rows, heads, d).to(dtype)
        x = qkv.cuda()
        sh = shape(n_rows, 64, q_stride=heads * d, k_stride=heads * d, v_stride=heads * d)
        r32 = torch.tensor(rows[:-1], dtype=torch.int32, device="cuda")
        n32 = torch.tensor(new, dtype=torch.int32, device="cuda")
        S.svf_append_kv(sh, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], dev_table, lens, r32, n32, K, V, q=x[:, :Hq], q_out=x[:, :Hq],
                        inv_freq=inv.cuda())
        out = torch.full((n_rows, Hq, d), 3.0, dtype=dtype, device="cuda")
        lse = torch.empty(n_rows, Hq, device="cuda")
        S.svf_chunk_attn(sh, x, K, V, dev_table, lens, r32, n32, out, S.new_chunk_workspace(sh), lse=lse)
        torch.cuda.synchronize()
        verify(sh, dict(q=x[:, :Hq].cpu(), K=K.cpu(), V=V.cpu(), table=table, seq_lens=lens.cpu(), new_rows=r32.cpu(), new_lens=n32.cpu()),
               out, lse)
        for b in range(B):
            mirror_k[b] = np.concatenate([mirror_k[b], qkv[rows[b]:rows[b + 1], Hq:Hq + Hkv].double().numpy()])
            done[b] += new[b]
        lens += n32
    for b in range(B):
        want = np.stack([O.rotate(mirror_k[b][t], t, inv.numpy(), False) for t in range(prompts[b])])
        step = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
        assert (np.abs(cache_of(b, prompts[b]) - want) <= step * np.abs(want) + 2.0 ** -19 * 6).all()

    for step in range(2):
        # the next token of every sequence, then drafts behind it, all rotated to their places
        Vocab = 4000
        logits = torch.randn(B, Vocab, device="cuda") * 3
        u = torch.rand(B, device="cuda")
        tokens = torch.empty(B, dtype=torch.int32, device="cuda")
        S.svf_sample(logits, u, tokens, S.new_sample_workspace(B, Vocab), top_p=torch.full((B,), 0.9, device="cuda"))
        assert ((tokens >= 0) & (tokens < Vocab)).all()
        q = torch.randn(B, gamma, Hq, d, device="cuda").to(dtype)
        kd, vd = (torch.randn(B, gamma, Hkv, d, device="cuda").to(dtype) for _ in range(2))
        vs = S.make_shape(B=B, gamma=gamma, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, block_size=block, max_seq_len=T, k_blocks=T // block, k_pool=K,
                          page_size=page, max_pages_per_seq=per)
        ws = S.new_workspace(vs)
        reps = torch.empty(B, Hkv, T // block, d, device="cuda")
        S.svf_block_reps(vs, K, dev_table, lens, reps)
        idx, cnt = torch.empty(B, Hkv, T // block, dtype=torch.int32, device="cuda"), torch.empty(B, Hkv, dtype=torch.int32, device="cuda")
        out_v = torch.empty_like(q)
        S.svf_verify_step(vs, S.SVF_STEP_ANCHOR, q, reps, K, V, dev_table, lens, kd, vd, None, idx, cnt, out_v, ws)
        # the same tokens as a chunk of the cache
        sh = shape(B * gamma, gamma)
        r32 = torch.arange(0, B * gamma, gamma, dtype=torch.int32, device="cuda")
        all_new = torch.full((B,), gamma, dtype=torch.int32, device="cuda")
        plain = S.make_chunk_shape(B=B, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, max_seq_len=T, max_new=gamma, n_rows=B * gamma, n_pages=B * per,
                                   page_size=page, max_pages_per_seq=per, k_pool=K)
        K2, V2 = K.clone(), V.clone()
        S.svf_append_kv(plain, kd, vd, dev_table, lens, r32, all_new, K2, V2)
        out_c = torch.empty_like(q)
        S.svf_chunk_attn(plain, q, K2, V2, dev_table, lens, r32, all_new, out_c, S.new_chunk_workspace(plain))
        eps = 2.0 ** -6 if dtype == torch.bfloat16 else 2.0 ** -14
        assert (out_v.float() - out_c.float()).abs().max() <= 2 * eps * float(V2.float().abs().max())
        # the accepted ones join the cache; rejected rows stay out of it
        n_acc = torch.tensor([gamma, 0, 2 + step], dtype=torch.int32, device="cuda")
        before = K.clone()
        S.svf_append_kv(plain, kd, vd, dev_table, lens, r32, n_acc, K, V)
        torch.cuda.synchronize()
        for b in range(B):
            L, n = int(lens[b]), int(n_acc[b])
            got = torch.from_numpy(cache_of(b, L + n)[L:])
            assert torch.equal(got, kd[b, :n].double().cpu())
        assert int(((K != before).flatten(2).any(-1)).sum()) == int(n_acc.sum())
        lens += n_acc
