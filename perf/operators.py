"""Performance cases of the operators that fill the cache and answer from it: what a speculative-decoding
server does around a verification step.

Kinds of pass (the field "kind" of a case):

  append   svf_append_kv: the keys and values of new tokens are rotated to their positions and written into
           the (paged) cache of their sequences; their queries are rotated on the way.
  chunk    svf_chunk_attn: attention of new tokens over all cached tokens in front of them and over
           themselves: a prompt read in chunks, single tokens, and batches that mix both.
  sample   svf_sample: tokens drawn from logits with temperature, top-k, top-p and min-p from given random
           numbers, with the distributions they were drawn from where acceptance needs those.

With `own` false, `run` computes the operators from elementary torch operations.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ROPE_BASE = 500000.0


# ---- the cases -------------------------------------------------------------------------------------

def _append(name=None, *, dtype="bf16", B, Hq=32, Hkv=8, d=128, page=16, head_major=False, prefix, new, slots=0,
            rotary=128, interleaved=False):
    """prefix, new: (least, most) per sequence.  slots: rows that a sequence has in the batch (0: as many as it has
    tokens).  rotary: channels that are rotated (0: none, and no queries come along)."""
    c = dict(kind="append", dtype=dtype, B=B, Hq=Hq, Hkv=Hkv, d=d, page=page, head_major=head_major, prefix_min=prefix[0],
             prefix_max=prefix[1], new_min=new[0], new_max=new[1], slots=slots, rotary=rotary, interleaved=interleaved)
    return dict(c, name=name) if name else c


def _chunk(name=None, *, dtype="bf16", B, Hq=32, Hkv=8, d=128, page=16, head_major=False, prefix, new, window=0, lse=False):
    c = dict(kind="chunk", dtype=dtype, B=B, Hq=Hq, Hkv=Hkv, d=d, page=page, head_major=head_major, prefix_min=prefix[0],
             prefix_max=prefix[1], new_min=new[0], new_max=new[1], slots=0, window=window, lse=lse)
    return dict(c, name=name) if name else c


def _sample(name=None, *, rows, V, dtype="f32", filters="mixed", probs=False):
    """filters: "none" (temperature alone), "usual" (top-k 50, top-p 0.9) or "mixed" (every row its own)."""
    c = dict(kind="sample", rows=rows, V=V, dtype=dtype, filters=filters, probs=probs)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decoding step of 64 users: one new token each, pages of 16; latency is all there is
        _append("append_step_b64", B=64, prefix=(100, 1000), new=(1, 1)),
        # after a verification step: of eight drafts per sequence the accepted ones (none to all) go from the draft
        # buffers, rotated already, into an fp32 cache of head dimension 64
        _append("append_accepted_f32", dtype="f32", B=32, Hq=8, Hkv=8, d=64, page=64, prefix=(300, 2000), new=(0, 8), slots=8,
                rotary=0),
        # four prompts of odd lengths, read whole: half of the channels rotated, neighbours paired, head-major pages
        _append("append_prompts_8k", B=4, page=64, head_major=True, prefix=(0, 700), new=(1801, 2301), rotary=64,
                interleaved=True),
        # a tiny fp32 model: one chunk into an empty contiguous cache
        _chunk("chunk_1k_f32", dtype="f32", B=1, Hq=8, Hkv=2, d=64, page=0, prefix=(0, 0), new=(1024, 1024), lse=True),
        # one user with an 8k context, one new token: few workgroups' worth of work, split over the keys
        _chunk("chunk_token_8k", B=1, page=0, prefix=(8191, 8191), new=(1, 1)),
        # four users with 32k contexts, one new token each: the cache goes by once
        _chunk("chunk_token_32k_b4", B=4, prefix=(32767, 32767), new=(1, 1), lse=True),
        # a running batch: eight sequences over four KV heads, single tokens beside chunks of up to 500
        _chunk("chunk_mixed_b8", B=8, Hkv=4, prefix=(900, 12000), new=(1, 500)),
        # head dimension 64, layers that look back 1024 tokens, odd lengths, head-major pages
        _chunk("chunk_window_d64", B=3, d=64, page=32, head_major=True, prefix=(1500, 7001), new=(333, 1111), window=1024),
        # the last chunk of a 32k prompt: the largest, bound by the matrix cores
        _chunk("chunk_prompt_32k", B=1, prefix=(30720, 30720), new=(2048, 2048)),
        # one user: the next token out of 32 000; latency again
        _sample("sample_one_32k", rows=1, V=32000, filters="usual"),
        # 64 users with settings of their own, a 129 280-token vocabulary
        _sample("sample_b64", rows=64, V=129280),
        # the distributions of 64 sequences with four drafts each, from bf16 logits, as acceptance takes them
        _sample("sample_probs_b64x4", rows=256, V=129280, dtype="bf16", probs=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _range(rng, lo, hi):
    a, b = _log_int(rng, lo, hi), _log_int(rng, lo, hi)
    return min(a, b), max(a, b)


def _draw_append(rng):
    d = rng.choice((64, 128))
    rotary = rng.choice((0, d, d, d // 2))
    B = _log_int(rng, 1, 96)
    most = max(1, 9000 // B)
    slots = rng.choice((0, rng.randint(1, 16))) if most >= 16 else 0
    new = (0, slots) if slots else _range(rng, 1, min(most, 2400))
    Hq, Hkv = rng.choice(((32, 8), (32, 4), (8, 8), (8, 2)))
    return _append(dtype=rng.choice(("bf16", "bf16", "f32")), B=B, Hq=Hq, Hkv=Hkv, d=d, page=rng.choice((0, 16, 24, 64)),
                   head_major=rng.random() < 0.3, prefix=_range(rng, 1, 1500), new=new, slots=slots, rotary=rotary,
                   interleaved=rng.random() < 0.5)


def _draw_chunk(rng):
    Hq, Hkv = rng.choice(((32, 8), (32, 8), (32, 4), (8, 8)))
    page, head_major, lse, d = rng.choice((0, 16, 24, 64)), rng.random() < 0.3, rng.random() < 0.5, rng.choice((64, 128, 128))
    window = rng.choice((0, 0, 0, _log_int(rng, 100, 4000)))
    how = rng.random()
    if how < 0.2:                                        # fp32: small models and correctness runs
        Hq, Hkv = rng.choice(((8, 2), (4, 4)))
        return _chunk(dtype="f32", B=rng.choice((1, 2)), Hq=Hq, Hkv=Hkv, d=d, page=page, head_major=head_major,
                      prefix=_range(rng, 1, 4000), new=_range(rng, 1, 1000), window=window, lse=lse)
    if how < 0.5:                                        # single tokens
        B = _log_int(rng, 1, 32)
        return _chunk(B=B, Hq=Hq, Hkv=Hkv, d=d, page=page, head_major=head_major,
                      prefix=_range(rng, 500, min(32000, 130000 // B)), new=(1, rng.choice((1, 1, 4))), window=window, lse=lse)
    B = _log_int(rng, 1, 8)                              # chunks and mixed batches
    return _chunk(B=B, Hq=Hq, Hkv=Hkv, d=d, page=page, head_major=head_major, prefix=_range(rng, 1, 16000 // B),
                  new=_range(rng, 1, 2048 // B), window=window, lse=lse)


def draw(rng: random.Random):
    kind = rng.choice(("append", "chunk", "chunk", "sample"))
    if kind == "append":
        return _draw_append(rng)
    if kind == "chunk":
        return _draw_chunk(rng)
    V = _log_int(rng, 1000, 130000)
    return _sample(rows=_log_int(rng, 1, max(1, min(256, 16000000 // V))), V=V, dtype=rng.choice(("f32", "bf16")),
                   filters=rng.choice(("none", "usual", "mixed", "mixed")), probs=rng.random() < 0.4)


# ---- sizes that follow from a case -----------------------------------------------------------------

def _spread(lo, hi, B, step):
    """B lengths from lo to hi, both among them, in an order without a trend."""
    return [lo + (hi - lo) * ((b * step + B - 1) % B) // max(1, B - 1) for b in range(B)]


def _step(B, from_):
    return next(s for s in range(from_, from_ + B + 1) if math.gcd(s, B) == 1)


def _lengths(c):
    """(prefix lengths, new tokens) of the sequences."""
    B = c["B"]
    return _spread(c["prefix_min"], c["prefix_max"], B, _step(B, 3)), _spread(c["new_min"], c["new_max"], B, _step(B, 2))


def _visible(c, L, j):
    """Cached tokens that new token j of a sequence with L tokens in front attends."""
    return min(L + j + 1, c["window"]) if c["window"] else L + j + 1


def work(c):
    if c["kind"] == "sample":
        e = 4 if c["dtype"] == "f32" else 2
        n = c["rows"] * c["V"]
        return {"bytes": n * e + (4 * n if c["probs"] else 0) + 24 * c["rows"], "flops": 4 * n}
    e, d, Hq, Hkv = (4 if c["dtype"] == "f32" else 2), c["d"], c["Hq"], c["Hkv"]
    prefix, new = _lengths(c)
    if c["kind"] == "append":
        rows = sum(new)
        heads = 2 * Hkv + (Hq if c["rotary"] else 0)
        return {"bytes": rows * (2 * heads * d * e + 8), "flops": rows * 3 * c["rotary"] * (Hq + Hkv)}
    keys = sum(_visible(c, L, j) for L, n in zip(prefix, new) for j in range(n))
    held = sum(min(L + n, _visible(c, L, 0) + n - 1) for L, n in zip(prefix, new) if n)
    rows = sum(new)
    return {"bytes": 2 * held * Hkv * d * e + 2 * rows * Hq * d * e + (4 * rows * Hq if c["lse"] else 0),
            "flops": 4 * d * Hq * keys}


# ---- inputs ----------------------------------------------------------------------------------------

def _prepare_sample(c, g):
    R, V = c["rows"], c["V"]
    logits = (3.0 * torch.randn(R, V, generator=g, device="cuda")).to(DT[c["dtype"]])
    s = {"c": c, "logits": logits, "u": torch.rand(R, generator=g, device="cuda")}
    r = torch.rand(4, R, generator=g, device="cuda")
    if c["filters"] == "none":
        s.update(temperature=0.6 + 0.6 * r[0], top_k=None, top_p=None, min_p=None)
    elif c["filters"] == "usual":
        s.update(temperature=torch.full((R,), 0.8, device="cuda"), top_k=torch.full((R,), 50, device="cuda", dtype=torch.int32),
                 top_p=torch.full((R,), 0.9, device="cuda"), min_p=None)
    else:                                                # greedy rows, and every filter on and off
        i = torch.arange(R, device="cuda")
        s.update(temperature=torch.where(i % 7 == 3, 0.0, 0.6 + 0.6 * r[0]),
                 top_k=torch.where(i % 3 == 1, 1 + (r[1] * 200).int(), 0).to(torch.int32),
                 top_p=torch.where(i % 4 == 2, 1.0, 0.7 + 0.29 * r[2]),
                 min_p=torch.where(i % 5 == 4, 0.1 * r[3], 0.0))
    if own:
        import paper_2512_21911_amd as S
        s.update(ws=S.new_sample_workspace(R, V), tokens=torch.empty(R, device="cuda", dtype=torch.int32),
                 out=torch.empty(R, V, device="cuda") if c["probs"] else None)
    return s


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(251221911 + 7907 * seed)
    if c["kind"] == "sample":
        return _prepare_sample(c, g)
    B, Hq, Hkv, d, dt, page = c["B"], c["Hq"], c["Hkv"], c["d"], DT[c["dtype"]], c["page"]
    prefix, new = _lengths(c)
    rows_of = [c["slots"] or n for n in new]
    n_rows = sum(rows_of)
    total = [L + n for L, n in zip(prefix, new)]
    T = max(max(total), 1)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    if page:
        per_seq = -(-T // page)
        n_pages = sum(-(-t // page) for t in total) + 1
        ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        table = torch.zeros(B, per_seq, device="cuda", dtype=torch.int32)
        off = 0
        for b, t in enumerate(total):
            u = -(-t // page)
            table[b, :u] = ids[off:off + u]
            off += u
        slots = page
    else:
        per_seq, n_pages, slots, table = 0, B, T, None
    K, V = ((randn(n_pages, Hkv, slots, d).to(dt).permute(0, 2, 1, 3) if c["head_major"] else
             randn(n_pages, slots, Hkv, d).to(dt)) for _ in range(2))
    first = [sum(rows_of[:b]) for b in range(B)]
    i32 = dict(device="cuda", dtype=torch.int32)
    s = {"c": c, "K": K, "V": V, "table": table, "T": T, "n_rows": n_rows, "n_tokens": sum(new), "n_pages": n_pages,
         "seq_lens": torch.tensor(prefix, **i32), "new_rows": torch.tensor(first, **i32), "new_lens": torch.tensor(new, **i32)}
    heads = Hq + 2 * Hkv
    if c["kind"] == "append":
        # what a fused projection leaves: queries, keys and values of a token side by side
        qkv = randn(max(1, n_rows), heads, d).to(dt)
        s.update(q=qkv[:, :Hq] if c["rotary"] else None, k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:])
        half = c["rotary"] // 2
        s["inv_freq"] = (ROPE_BASE ** (-torch.arange(half, device="cuda", dtype=torch.float64) / max(1, half))) if half else None
    else:
        # keys and queries as after a rotation; some heads look at few tokens, others at many
        gain = torch.linspace(0.5, 2.0, Hq, device="cuda")[:, None]
        s["q"] = (gain * randn(max(1, n_rows), Hq, d)).to(dt)
    if own:
        import paper_2512_21911_amd as S
        stride = heads * d if c["kind"] == "append" else 0
        s["shape"] = S.make_chunk_shape(
            B=B, Hq=Hq, Hkv=Hkv, d=d, dtype=dt, max_seq_len=T, max_new=max(1, max(new)), n_rows=max(1, n_rows), n_pages=n_pages,
            page_size=page, max_pages_per_seq=per_seq, k_pool=K, window=c.get("window", 0), q_stride=stride, k_stride=stride,
            v_stride=stride, rotary_dim=c.get("rotary", 0), rotary_interleaved=c.get("interleaved", False))
        if c["kind"] == "append":
            s["q_out"] = torch.empty_strided(s["q"].shape, s["q"].stride(), dtype=dt, device="cuda") if c["rotary"] else None
        else:
            s["ws"] = S.new_chunk_workspace(s["shape"])
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty(max(1, n_rows), Hq, device="cuda") if c["lse"] else None
    return s


# ---- one pass --------------------------------------------------------------------------------------

def _tokens(s):
    """(sequence, place among its new tokens, row) of every new token."""
    B = s["c"]["B"]
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), s["new_lens"].long(), output_size=s["n_tokens"])
    before = torch.cumsum(s["new_lens"], 0) - s["new_lens"]
    j = torch.arange(s["n_tokens"], device="cuda") - before[seq]
    return seq, j, s["new_rows"].long()[seq] + j


def _rotate(x, angle, c):
    """x fp32 [n][heads][d], angle fp64 [n][rotary / 2]."""
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    r = c["rotary"]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((ra, rb), -1).flatten(-2) if c["interleaved"] else torch.cat((ra, rb), -1)
    return torch.cat((turned, x[..., r:]), -1)


def _plain_append(s):
    c, dt = s["c"], DT[s["c"]["dtype"]]
    seq, j, row = _tokens(s)
    at = s["seq_lens"].long()[seq] + j
    k, v = s["k"][row], s["v"][row]
    q_out = None
    if c["rotary"]:
        angle = at.double()[:, None] * s["inv_freq"][None]
        k = _rotate(k.float(), angle, c).to(dt)
        q_out = _rotate(s["q"][row].float(), angle, c).to(dt)
    where = (s["table"].long()[seq, at // c["page"]], at % c["page"]) if c["page"] else (seq, at)
    s["K"][where] = k
    s["V"][where] = v
    return {"K": s["K"], "V": s["V"], "q": q_out}


def _plain_chunk(s):
    c = s["c"]
    B, Hq, Hkv, d, T = c["B"], c["Hq"], c["Hkv"], c["d"], s["T"]
    N, G = max(1, c["new_max"]), Hq // Hkv
    if c["page"]:
        k, v = (x[s["table"].long()].reshape(B, -1, Hkv, d)[:, :T] for x in (s["K"], s["V"]))
    else:
        k, v = s["K"], s["V"]
    k, v = (x.permute(0, 2, 1, 3).float() for x in (k, v))                                       # [B][Hkv][T][d]
    rows = (s["new_rows"].long()[:, None] + torch.arange(N, device="cuda")).clamp(max=s["n_rows"] - 1)
    q = s["q"][rows].float().view(B, N, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, d)
    x = torch.matmul(q, k.transpose(2, 3)).view(B, Hkv, N, G, T) / math.sqrt(d)
    last = s["seq_lens"].long()[:, None] + torch.arange(N, device="cuda")                         # [B][N]
    t = torch.arange(T, device="cuda")
    seen = t <= last[..., None]
    if c["window"]:
        seen = seen & (t > last[..., None] - c["window"])
    x = x.masked_fill(~seen[:, None, :, None, :], float("-inf"))
    m = x.amax(-1, keepdim=True)
    x = (x - m).exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x.view(B, Hkv, N * G, T), v).view(B, Hkv, N, G, d) / total
    lse = (m + total.log()).squeeze(-1)
    seq, j, _ = _tokens(s)
    out = out.permute(0, 2, 1, 3, 4).reshape(B, N, Hq, d)[seq, j].to(DT[c["dtype"]])
    lse = lse.permute(0, 2, 1, 3).reshape(B, N, Hq)[seq, j]
    return {"out": out, "lse": lse if c["lse"] else None}


def _plain_sample(s):
    c, V = s["c"], s["c"]["V"]
    x = s["logits"].double()
    warm = s["temperature"].double()[:, None]
    greedy = warm <= 0
    warm = torch.where(greedy, 1.0, warm)
    top = x.amax(-1, keepdim=True)
    w = ((x - top) / warm).exp()
    order = torch.sort(x, dim=-1, descending=True, stable=True)
    ranked = w.gather(-1, order.indices)
    most = s["top_k"].long()[:, None] if s["top_k"] is not None else torch.zeros_like(greedy, dtype=torch.long)
    most = torch.where(greedy, 1, torch.where(most <= 0, V, most))
    keep = torch.arange(V, device="cuda")[None] < most
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        ranked = ranked * keep
        mass = ranked.cumsum(-1)
        keep = keep & ((mass - ranked < p * mass[:, -1:]) | (p >= 1))
    if s["min_p"] is not None:
        keep = keep & (order.values >= top + warm * s["min_p"].double()[:, None].log())
    w = w * torch.zeros_like(keep).scatter_(-1, order.indices, keep)
    mass = w.cumsum(-1)
    token = (mass <= s["u"].double()[:, None] * mass[:, -1:]).sum(-1).clamp(max=V - 1).to(torch.int32)
    return {"tokens": token, "probs": (w / mass[:, -1:]).float() if c["probs"] else None}


def run(s):
    kind = s["c"]["kind"]
    if not own:
        return {"append": _plain_append, "chunk": _plain_chunk, "sample": _plain_sample}[kind](s)
    import paper_2512_21911_amd as S
    if kind == "append":
        S.svf_append_kv(s["shape"], s["k"], s["v"], s["table"], s["seq_lens"], s["new_rows"], s["new_lens"], s["K"], s["V"],
                        q=s["q"], q_out=s["q_out"], inv_freq=s["inv_freq"])
        return {"K": s["K"], "V": s["V"], "q": s["q_out"]}
    if kind == "chunk":
        S.svf_chunk_attn(s["shape"], s["q"], s["K"], s["V"], s["table"], s["seq_lens"], s["new_rows"], s["new_lens"], s["out"],
                         s["ws"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    S.svf_sample(s["logits"], s["u"], s["tokens"], s["ws"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                 min_p=s["min_p"], probs=s["out"])
    return {"tokens": s["tokens"], "probs": s["out"]}


# ---- the definitions in 64 bits --------------------------------------------------------------------

def _exact_append(c, s):
    prefix, new = _lengths(c)
    K, V = s["K"].double(), s["V"].double()
    q = s["q"].double() if c["rotary"] else None
    first = 0
    for b, (L, n) in enumerate(zip(prefix, new)):
        r = slice(first, first + n)
        first += c["slots"] or n
        pos = torch.arange(L, L + n, device="cuda")
        k, v = s["k"][r].double(), s["v"][r].double()
        for h in range(c["rotary"] // 2):
            i, j = (2 * h, 2 * h + 1) if c["interleaved"] else (h, h + c["rotary"] // 2)
            a = (pos.double() * s["inv_freq"][h])[:, None]
            for x in (k, q[r]):
                x[..., i], x[..., j] = x[..., i] * a.cos() - x[..., j] * a.sin(), x[..., j] * a.cos() + x[..., i] * a.sin()
        page = s["table"][b].long()[pos // c["page"]] if c["page"] else torch.full_like(pos, b)
        slot = pos % c["page"] if c["page"] else pos
        K[page, slot], V[page, slot] = k, v
    return {"K": K, "V": V, "q": q}


def _exact_chunk(c, s):
    prefix, new = _lengths(c)
    G, d = c["Hq"] // c["Hkv"], c["d"]
    out = torch.zeros(s["n_rows"], c["Hq"], d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["n_rows"], c["Hq"], dtype=torch.float64, device="cuda")
    first = 0
    for b, (L, n) in enumerate(zip(prefix, new)):
        pos = torch.arange(L + n, device="cuda")
        page = s["table"][b].long()[pos // c["page"]] if c["page"] else torch.full_like(pos, b)
        slot = pos % c["page"] if c["page"] else pos
        hidden = torch.zeros(n, L + n, dtype=torch.bool, device="cuda")
        me = torch.arange(L, L + n, device="cuda")[:, None]
        hidden |= pos[None] > me
        if c["window"]:
            hidden |= pos[None] <= me - c["window"]
        for h in range(c["Hkv"]):
            k, v = s["K"][page, slot, h].double(), s["V"][page, slot, h].double()
            for g in range(h * G, (h + 1) * G):
                x = s["q"][first:first + n, g].double() @ k.T / d ** 0.5
                x[hidden] = -math.inf
                lse[first:first + n, g] = torch.logsumexp(x, -1)
                out[first:first + n, g] = torch.exp(x - lse[first:first + n, g, None]) @ v
        first += n
    return {"out": out, "lse": lse if c["lse"] else None}


def _exact_sample(c, s):
    tokens, probs = [], []
    for r in range(c["rows"]):
        x = s["logits"][r].double()
        T = float(s["temperature"][r])
        k = 1 if T <= 0 else int(s["top_k"][r]) if s["top_k"] is not None else 0
        z = x / (T if T > 0 else 1.0)
        by = torch.argsort(x, descending=True, stable=True)
        if k > 0:
            by = by[:k]
        p = torch.softmax(z[by], 0)
        if s["top_p"] is not None and float(s["top_p"][r]) < 1:
            p = p[torch.cumsum(p, 0) - p < s["top_p"][r].double()]
        if s["min_p"] is not None:
            p = p[z[by[:p.numel()]] >= z[by[0]] + s["min_p"][r].double().log()]
        full = torch.zeros(c["V"], dtype=torch.float64, device="cuda")
        full[by[:p.numel()]] = p / p.sum()
        cdf = torch.cumsum(full, 0)
        tokens.append(torch.searchsorted(cdf, (s["u"][r].double() * cdf[-1]).reshape(1), right=True).clamp(max=c["V"] - 1))
        if c["probs"]:
            probs.append(full)
    return {"tokens": torch.cat(tokens).to(torch.int32), "probs": torch.stack(probs) if c["probs"] else None}


def exact(c, seed):
    s = prepare(c, seed)
    return {"append": _exact_append, "chunk": _exact_chunk, "sample": _exact_sample}[c["kind"]](c, s)
