"""The operators around an update and around serving that are measured against their plain forms.

A case is a dict of plain values. `prepare` makes what a program holds before the call, `run` is one pass:
where `own` is false in elementary torch operations in float32, where it is true through the library's
entry points. `exact` is the same result from the definitions in float64.

Kinds:
  prompt    causal attention over whole prompts, packed episodes, grouped heads: o and lse
  train     the same forward and the backward that reads what it saved: o, lse, dq, dk, dv
  append    new tokens' keys and values into a paged 4-bit cache: the values it then stands for
  cached    append, then attention of the new tokens over the cache (one token each: a decoding step)
  logprobs  log-probability and entropy of given tokens through the LM head, and the top alternatives

The 4-bit cache: pages of 128 tokens, per page and key/value head one record of 17152 bytes.
  keys      e2m1 codes [128 tokens][64 bytes] (low nibble first along the head dimension); every 32
            elements share a power of two 2^(b - 127), bytes b at [block of 32][token % 16][token / 16]
  values    e2m1 codes [128 elements][64 bytes] along the tokens, in the order of `_POS`; every token has one
            scale (bfloat16 with 6 significant bits), in the same order
"""
import math

import torch

own = False

DH = 128
PAGE = 128
REC = 2 * PAGE * DH // 2 + PAGE * 4 + PAGE * 2
DEV = "cuda"


# ---- the cases ---------------------------------------------------------------------------------
def listed():
    return [
        # three short prompts of a small model: launch and latency count
        dict(name="prompt_small", kind="prompt", E=3, N=300, heads=16, kv=4),
        # one long prompt, the Llama-8B attention block
        dict(name="prompt_llama8b", kind="prompt", E=1, N=8192, heads=32, kv=8),
        # sixteen ragged prompts in one batch, the shortest a single token
        dict(name="prompt_packed16", kind="prompt", E=16, N=7001, heads=32, kv=8),
        # the attention block of a small model's update, forward and backward
        dict(name="train_small", kind="train", E=1, N=2048, heads=16, kv=4),
        # the Llama-8B attention block of a long update
        dict(name="train_llama8b", kind="train", E=1, N=8192, heads=32, kv=8),
        # a prompt of 512 tokens for each of sixteen episodes into the cache
        dict(name="append_prompt16", kind="append", E=16, rows=512, ctx=1024, heads=32, kv=8, idle=False),
        # one decoding step of sixteen episodes, the last slot of the batch idle
        dict(name="decode16", kind="cached", E=16, rows=1, ctx=4000, heads=32, kv=8, idle=True),
        # one decoding step over long histories: a gigabyte of cache
        dict(name="decode_long", kind="cached", E=8, rows=1, ctx=131072, heads=32, kv=8, idle=False),
        # the next 64 tokens of four episodes against their caches
        dict(name="chunk64", kind="cached", E=4, rows=64, ctx=8200, heads=32, kv=8, idle=False),
        # the small float32 head: 512 tokens scored
        dict(name="logprobs_tiny_f32", kind="logprobs", dtype="f32", N=512, d=256, V=4096, top=4),
        # the tokens of one decoding step of sixteen episodes, with alternatives
        dict(name="logprobs_decode16", kind="logprobs", dtype="bf16", N=16, d=4096, V=128256, top=8),
        # a whole update text scored through the Llama-8B head: the largest product
        dict(name="logprobs_llama8b", kind="logprobs", dtype="bf16", N=8192, d=4096, V=128256, top=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    kv = rng.choice([1, 2, 4, 8])
    return dict(heads=kv * rng.randint(1, 8), kv=kv)


def draw(rng):
    kind = rng.choice(["prompt", "train", "append", "cached", "cached", "logprobs", "logprobs"])
    if kind in ("prompt", "train"):
        while True:
            c = dict(kind=kind, E=rng.randint(1, 16), N=_log(rng, 1, 8192), **_heads(rng))
            if c["N"] ** 2 * c["heads"] <= 8192 ** 2 * 32:
                return c
    if kind in ("append", "cached"):
        while True:
            rows = 1 if rng.random() < 0.5 else _log(rng, 2, 1024 if kind == "append" else 64)
            c = dict(kind=kind, E=rng.randint(1, 16), rows=rows, ctx=rows - 1 + _log(rng, 1, 131072), idle=rng.random() < 0.3,
                     **_heads(rng))
            if c["E"] * c["ctx"] * c["kv"] <= 8 * 131072 * 8 and c["E"] * c["ctx"] * c["rows"] * c["heads"] <= 2 ** 30:
                return c
    if rng.random() < 0.3:
        return dict(kind=kind, dtype="f32", N=_log(rng, 1, 1024), d=8 * _log(rng, 8, 64), V=_log(rng, 100, 8192),
                    top=rng.randint(0, 20))
    while True:
        c = dict(kind=kind, dtype="bf16", N=_log(rng, 1, 8192), d=8 * _log(rng, 64, 640), V=_log(rng, 1000, 152000),
                 top=rng.randint(0, 20))
        if c["N"] * c["d"] * c["V"] <= 8192 * 4096 * 128256:
            return c


# ---- inputs ------------------------------------------------------------------------------------
def _randn(g, shape, std=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _row_offsets(case):
    """Ragged episodes of N rows in all: weights 3, 2, 4, 1, 3, ...; of many rows, the last has one."""
    E, N = case["E"], case["N"]
    one = 1 if E > 1 and N >= 4 * E else 0
    w = [(3, 2, 4, 1)[e % 4] for e in range(E - one)]
    off, s = [0], 0
    for x in w:
        s += x
        off.append((N - one) * s // sum(w))
    return off + [N] * one


def _lengths(case):
    """Tokens of every sequence, the new rows among them; an idle slot has none."""
    L = [max(case["rows"], case["ctx"] * f // 16) for e in range(case["E"]) for f in [(16, 6, 13, 1)[e % 4]]]
    if case["idle"] and case["E"] > 1:
        L[-1] = 0
    return L


# Positions along a value row: position 32 a + 4 b + c holds token 16 b + 4 a + c (a, c < 4, b < 8).
_POS = [16 * ((p >> 2) & 7) + 4 * (p >> 5) + (p & 3) for p in range(PAGE)]
_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def _codes(x):
    """e2m1 codes of float32 x: to nearest, ties to the even code, 6 at most."""
    a = x.abs()
    mag = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)).to(torch.uint8)
    return mag + 8 * torch.signbit(x).to(torch.uint8)


def _quant_k(x):
    """Keys [..., 128] -> (codes, exponent bytes [..., 4]): the power of two that keeps the largest of 32
    below 7 times itself."""
    b = x.float().view(*x.shape[:-1], 4, 32)
    top = b.abs().amax(-1)
    e = ((top.view(torch.int32) + 0x200000) >> 23).sub(2).clamp_(27, 252)
    e = torch.where(torch.isfinite(top), e, torch.full_like(e, 255))
    return _codes(b * torch.exp2(127.0 - e)[..., None]).view(x.shape), e.to(torch.uint8)


def _quant_v(x):
    """Values [..., 128] -> (codes, scale [...]): a sixth of the largest, rounded up to 6 significant bits."""
    top = x.float().abs().amax(-1)
    s = (((top / 6.0).view(torch.int32) + 0x3FFFF) & ~0x3FFFF).view(torch.float32).clamp(2.0 ** -100, 1.3125 * 2.0 ** 125)
    s = torch.where(torch.isfinite(top), s, torch.full_like(s, math.nan))
    return _codes(x.float() / s[..., None]), s


def _pairs(c):
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _write_pages(cache, pages, k, v):
    """Whole sequences' keys and values [tokens, kv, 128] into their pages; the rest of a page stays."""
    T, kv, _ = k.shape
    P = (T + PAGE - 1) // PAGE
    (kc, ke), (vc, vs) = _quant_k(k), _quant_v(v)
    new = cache[pages].view(P, kv, REC)
    at = torch.arange(T, device=DEV)
    p, t = at // PAGE, at % PAGE
    codes = new[..., :8192].clone().view(P, kv, PAGE, 64)
    codes[p, :, t] = _pairs(kc)
    new[..., :8192] = codes.view(P, kv, 8192)
    exps = new[..., 16384:16896].clone().view(P, kv, 4, 16, 8)
    exps[p, :, :, t % 16, t // 16] = ke
    new[..., 16384:16896] = exps.view(P, kv, 512)
    pos = torch.empty(PAGE, dtype=torch.long, device=DEV)
    pos[torch.tensor(_POS, device=DEV)] = torch.arange(PAGE, device=DEV)
    vn = torch.zeros(P, kv, DH, PAGE, dtype=torch.uint8, device=DEV)
    vn[p, :, :, pos[t]] = vc
    new[..., 8192:16384] = _pairs(vn).view(P, kv, 8192)
    sc = new[..., 16896:].clone().view(torch.bfloat16).view(P, kv, PAGE)
    sc[p, :, pos[t]] = vs.to(torch.bfloat16)
    new[..., 16896:] = sc.view(torch.uint8).view(P, kv, 256)
    cache[pages] = new


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    kind = case["kind"]
    s = dict(case=case)
    if kind in ("prompt", "train"):
        N, H, kv = case["N"], case["heads"], case["kv"]
        s.update(q=_randn(g, (N, H, DH)), k=_randn(g, (N, kv, DH)), v=_randn(g, (N, kv, DH)), off=_row_offsets(case))
        if kind == "train":
            s["do"] = _randn(g, (N, H, DH), 0.05)
    if kind in ("append", "cached"):
        E, n, H, kv = case["E"], case["rows"], case["heads"], case["kv"]
        L = _lengths(case)
        used = [(x + PAGE - 1) // PAGE for x in L]
        total = sum(used) + 3
        order = torch.randperm(total, generator=g, device=DEV)
        cache = torch.full((total, kv, REC), 255, dtype=torch.uint8, device=DEV)  # what no token was written to is not read
        table = torch.full((E, max(1, max(used))), -1, dtype=torch.int32, device=DEV)
        a = 0
        for e in range(E):
            table[e, :used[e]] = order[a:a + used[e]].int()
            had = max(0, L[e] - n)
            if had:
                pages = order[a:a + (had + PAGE - 1) // PAGE]
                _write_pages(cache, pages, _randn(g, (had, kv, DH)), _randn(g, (had, kv, DH)))
            a += used[e]
        s.update(cache=cache, table=table, lengths=torch.tensor(L, dtype=torch.int32, device=DEV), max_length=max(L),
                 off=[n * e for e in range(E + 1)], q=_randn(g, (E * n, H, DH)), k=_randn(g, (E * n, kv, DH)),
                 v=_randn(g, (E * n, kv, DH)))
    if kind == "logprobs":
        # The alternatives are whole numbers and have to agree, so two logits may not swap by how a sum is
        # rounded: hidden states are multiples of 2^-4, head weights of 2^-9, and every sum of their products
        # is exact in float32 in any order. Equal logits do occur, and the lowest id wins. Every other row's
        # hidden state leans to its token, as a trained model's does.
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        N, d, V = case["N"], case["d"], case["V"]
        W = torch.randn((V, d), generator=g, device=DEV).mul_(0.02 * 512).round_().div_(512)
        y = torch.randint(0, V, (N,), generator=g, device=DEV)
        h = torch.randn((N, d), generator=g, device=DEV)
        h[::2] += 8.0 * W[y[::2]]
        s.update(h=h.mul_(16).round_().div_(16).to(dt), W=W.to(dt), y=y.int())
    return s


# ---- one pass ----------------------------------------------------------------------------------
def run(s):
    case, kind = s["case"], s["case"]["kind"]
    if own:
        import paper_2607_03441_amd as attt
        if kind == "prompt":
            o, lse = attt.attention_fwd(s["q"], s["k"], s["v"], row_offsets=s["off"])
            return dict(o=o, lse=lse)
        if kind == "train":
            o, lse = attt.attention_fwd(s["q"], s["k"], s["v"], row_offsets=s["off"])
            dq, dk, dv, _ = attt.attention_bwd_saved(s["q"], s["k"], s["v"], o, lse, s["do"], row_offsets=s["off"])
            return dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv)
        if kind in ("append", "cached"):
            kh, vh = attt.kv4_append(s["cache"], s["k"], s["v"], s["table"], s["lengths"], row_offsets=s["off"], want_held=True)
            if kind == "append":
                return dict(k=kh, v=vh)
            o, lse = attt.kv4_attention(s["q"], s["cache"], s["table"], s["lengths"], row_offsets=s["off"],
                                        max_length=s["max_length"])
            return dict(k=kh, v=vh, o=o, lse=lse)
        logp, entropy, ids, top = attt.token_logprobs(s["h"], s["W"], s["y"], top=case["top"])
        return dict(logp=logp, entropy=entropy, **(dict(ids=ids, top=top) if case["top"] else {}))
    if kind == "prompt":
        o, lse, _ = _plain_forward(s)
        return dict(o=o.transpose(0, 1).to(torch.bfloat16), lse=lse)
    if kind == "train":
        return _plain_train(s)
    if kind in ("append", "cached"):
        return _plain_cached(s)
    return _plain_logprobs(s)


def _plain_forward(s):
    """o [H, N, 128] and lse [H, N] of every head at once, over the mask of all episodes; and P."""
    case = s["case"]
    N, g = case["N"], case["heads"] // case["kv"]
    ep = torch.bucketize(torch.arange(N, device=DEV), torch.tensor(s["off"][1:], device=DEV), right=True)
    allowed = (ep[:, None] == ep[None, :]).tril()
    q = s["q"].float().transpose(0, 1)
    k, v = (s[n].float().transpose(0, 1).repeat_interleave(g, 0) for n in "kv")
    S = (q @ k.transpose(1, 2).contiguous()).mul_(1.0 / math.sqrt(DH)).masked_fill_(~allowed, -math.inf)
    lse = torch.logsumexp(S, 2)
    P = S.sub_(lse[..., None]).exp_()
    return P @ v, lse, (P, q, k, v)


def _plain_train(s):
    o, lse, (P, q, k, v) = _plain_forward(s)
    case = s["case"]
    N, kv = case["N"], case["kv"]
    do = s["do"].float().transpose(0, 1).contiguous()
    D = (do * o).sum(2, keepdim=True)
    dv = P.transpose(1, 2).contiguous() @ do
    dS = (do @ v.transpose(1, 2).contiguous()).sub_(D).mul_(P).mul_(1.0 / math.sqrt(DH))
    dq, dk = dS @ k, dS.transpose(1, 2).contiguous() @ q
    shared = lambda t: t.view(kv, -1, N, DH).sum(1)  # noqa: E731  the query heads of a key/value head
    rows = lambda t: t.transpose(0, 1).to(torch.bfloat16)  # noqa: E731
    return dict(o=rows(o), lse=lse, dq=rows(dq), dk=rows(shared(dk)), dv=rows(shared(dv)))


def _values(codes):
    lut = torch.tensor(_E2M1, device=DEV)
    return lut[codes.int()]


def _split(b):
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)


def _plain_cached(s):
    case = s["case"]
    E, n, H, kv = case["E"], case["rows"], case["heads"], case["kv"]
    (kc, ke), (vc, vs) = _quant_k(s["k"]), _quant_v(s["v"])
    pos = s["lengths"].long()[:, None] - n + torch.arange(n, device=DEV)  # of the new tokens
    here = (pos >= 0).view(E * n, 1, 1)
    kh = (_values(kc).view(E * n, kv, 4, 32) * torch.exp2(ke.float() - 127.0)[..., None]).view(E * n, kv, DH)
    vh = _values(vc) * vs[..., None]
    kh, vh = torch.where(here, kh, torch.zeros_like(kh)), torch.where(here, vh, torch.zeros_like(vh))
    out = dict(k=kh.to(torch.bfloat16), v=vh.to(torch.bfloat16))
    if case["kind"] == "append":
        return out
    # what the pages stand for, then the new tokens in their places
    P = s["table"].shape[1]
    rec = s["cache"][s["table"].clamp(min=0).long()].view(E, P, kv, REC)
    ks = rec[..., 16384:16896].reshape(E, P, kv, 4, 16, 8).permute(0, 1, 2, 5, 4, 3).reshape(E, P, kv, PAGE, 4, 1)
    K = _values(_split(rec[..., :8192].reshape(E, P, kv, PAGE, 64))).view(E, P, kv, PAGE, 4, 32)
    K = (K * torch.exp2(ks.float() - 127.0)).view(E, P, kv, PAGE, DH).transpose(1, 2).reshape(E, kv, P * PAGE, DH)
    V = _values(_split(rec[..., 8192:16384].reshape(E, P, kv, DH, 64)))
    V = V * rec[..., 16896:].contiguous().view(torch.bfloat16).float()[..., None, :]
    back = torch.empty(PAGE, dtype=torch.long, device=DEV)
    back[torch.tensor(_POS, device=DEV)] = torch.arange(PAGE, device=DEV)
    V = V[..., back].permute(0, 2, 1, 4, 3).reshape(E, kv, P * PAGE, DH)
    at = torch.arange(P * PAGE, device=DEV)
    kept = (at < s["lengths"].long()[:, None] - n)[:, None, :, None]
    K, V = K.masked_fill_(~kept, 0.0), V.masked_fill_(~kept, 0.0)
    e, i = (pos >= 0).nonzero(as_tuple=True)
    K[e, :, pos[e, i]] = kh.view(E, n, kv, DH)[e, i]
    V[e, :, pos[e, i]] = vh.view(E, n, kv, DH)[e, i]
    q = s["q"].float().view(E, n, kv, H // kv, DH).permute(0, 2, 3, 1, 4).reshape(E, kv, -1, DH)
    S = (q @ K.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(DH)).view(E, kv, H // kv, n, P * PAGE)
    S.masked_fill_((at > pos[..., None])[:, None, None], -math.inf)
    lse = torch.logsumexp(S, 4)
    none = (lse == -math.inf)[..., None]
    w = S.sub_(lse[..., None]).exp_().masked_fill_(none, 0.0)
    o = (w.view(E, kv, -1, P * PAGE) @ V).view(E, H, n, DH).transpose(1, 2).reshape(E * n, H, DH)
    return dict(out, o=o.to(torch.bfloat16), lse=lse.view(E, H, n).transpose(0, 1).reshape(H, E * n))


def _plain_logprobs(s):
    z = s["h"].float() @ s["W"].float().t() + 0.0
    V, top = z.shape[1], s["case"]["top"]
    lse = torch.logsumexp(z, 1, keepdim=True)
    out = dict(logp=(z.gather(1, s["y"].long()[:, None]) - lse)[:, 0])
    lp = z - lse
    out["entropy"] = -(lp.exp() * lp).sum(1)
    if top:
        # one key per logit, larger for the larger logit and among equal ones for the lower id
        b = z.view(torch.int32)
        key = ((b ^ ((b >> 31) & 0x7FFFFFFF)).long() << 32) + torch.arange(V - 1, -1, -1, device=DEV)
        ids = V - 1 - (torch.topk(key, top, 1)[0] & 0xFFFFFFFF)
        out.update(ids=ids.int(), top=lp.gather(1, ids))
    return out


# ---- what a pass cannot do without --------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind in ("prompt", "train"):
        off, N, H, kv = _row_offsets(case), case["N"], case["heads"], case["kv"]
        pairs = sum((b - a) * (b - a + 1) / 2 for a, b in zip(off, off[1:]))
        nbytes = 2.0 * DH * N * (2 * H + 2 * kv) + 4.0 * N * H
        if kind == "prompt":
            return dict(bytes=nbytes, flops=4.0 * DH * H * pairs)
        return dict(bytes=nbytes + 2.0 * DH * N * (2 * H + 2 * kv), flops=14.0 * DH * H * pairs)
    if kind in ("append", "cached"):
        E, n, H, kv = case["E"], case["rows"], case["heads"], case["kv"]
        L = _lengths(case)
        new = n * sum(x > 0 for x in L)
        nbytes = new * kv * (8.0 * DH + REC / PAGE)  # keys and values in, what they stand for and their codes out
        flops = 8.0 * DH * kv * new
        if kind == "cached":
            nbytes += sum(L) * kv * REC / PAGE + 4.0 * E * n * H * (DH + 1)
            flops += 4.0 * DH * H * sum(n * x - n * (n - 1) / 2 for x in L if x)
        return dict(bytes=nbytes, flops=flops)
    N, d, V, size = case["N"], case["d"], case["V"], 2 if case["dtype"] == "bf16" else 4
    return dict(bytes=size * d * (float(N) + V) + N * (12.0 + 8.0 * case["top"]), flops=2.0 * N * d * V)


# ---- the same in 64 bits --------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("prompt", "train"):
        return _exact_attention(s)
    if kind in ("append", "cached"):
        return _exact_cached(s)
    h, W, y = s["h"].double(), s["W"].double().t(), s["y"].long()
    out = dict(logp=[], entropy=[], top=[])
    step = max(1, (1 << 29) // case["V"])
    for a in range(0, case["N"], step):
        lp = torch.log_softmax(h[a:a + step] @ W, 1)
        out["logp"].append(lp[torch.arange(lp.shape[0], device=DEV), y[a:a + step]])
        out["entropy"].append(torch.special.entr(lp.exp()).sum(1))
        out["top"].append(torch.topk(lp, case["top"], 1)[0] if case["top"] else lp[:, :0])
    out = {n: torch.cat(t) for n, t in out.items()}
    if not case["top"]:
        del out["top"]
    return dict(out, ids=None)


def _exact_attention(s):
    q, k, v = (s[n].double() for n in "qkv")
    do = s["do"].double() if "do" in s else None
    N, H = q.shape[:2]
    g, scale = H // k.shape[1], DH ** -0.5
    o, lse = torch.zeros_like(q), torch.zeros(H, N, dtype=torch.float64, device=DEV)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for a, b in zip(s["off"], s["off"][1:]):
        later = torch.ones(b - a, b - a, dtype=torch.bool, device=DEV).triu(1)
        for h in range(H):
            Q, K, V = q[a:b, h], k[a:b, h // g], v[a:b, h // g]
            P = torch.softmax((scale * (Q @ K.t())).masked_fill_(later, -math.inf), 1)
            lse[h, a:b] = torch.logsumexp((scale * (Q @ K.t())).masked_fill_(later, -math.inf), 1)
            o[a:b, h] = P @ V
            if do is not None:
                dO = do[a:b, h]
                dP = dO @ V.t()
                dS = scale * P * (dP - (P * dP).sum(1, keepdim=True))
                dq[a:b, h] = dS @ K
                dk[a:b, h // g] += dS.t() @ Q
                dv[a:b, h // g] += P.t() @ dO
    return dict(o=o, lse=lse) if do is None else dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv)


def _exact_nearest(x):
    """The e2m1 value nearest to each of x (float64); ties to the even code."""
    grid = torch.tensor(_E2M1[:8], dtype=torch.float64, device=DEV)
    a = x.abs().clamp(max=6.0)
    i = torch.searchsorted(grid, a).clamp(min=1)
    lo, hi = grid[i - 1], grid[i]
    up = (a - lo > hi - a) | ((a - lo == hi - a) & (i % 2 == 0))
    return torch.where(up, hi, lo) * torch.sign(x)


def _exact_cached(s):
    case = s["case"]
    E, n, H, kv = case["E"], case["rows"], case["heads"], case["kv"]
    L = s["lengths"].tolist()
    kx = s["k"].double().view(E * n, kv, 4, 32)
    m, e = torch.frexp(kx.abs().amax(-1, keepdim=True))  # m in [1/2, 1): at 7/8 the next power
    ks = torch.ldexp(torch.ones_like(m), (e - 3 + (m >= 0.875)).clamp(min=-100))
    kh = (_exact_nearest(kx / ks) * ks).view(E * n, kv, DH)
    vx = s["v"].double()
    m, e = torch.frexp(vx.abs().amax(-1, keepdim=True) / 6.0)
    vs = torch.ldexp(torch.ceil(m * 64.0), e - 6).clamp(min=2.0 ** -100)
    vh = _exact_nearest(vx / vs) * vs
    for i in range(E):
        if L[i] < n:
            kh[i * n:i * n + n - L[i]] = 0.0
            vh[i * n:i * n + n - L[i]] = 0.0
    out = dict(k=kh, v=vh)
    if case["kind"] == "append":
        return out
    value = torch.tensor(_E2M1, dtype=torch.float64, device=DEV)
    token = torch.arange(PAGE, device=DEV)
    place = 32 * (token // 4 % 4) + 4 * (token // 16) + token % 4  # of a token along a value row
    q = s["q"].double().view(E, n, H, DH)
    o = torch.zeros(E, n, H, DH, dtype=torch.float64, device=DEV)
    lse = torch.full((H, E, n), -math.inf, dtype=torch.float64, device=DEV)
    for i in range(E):
        if not L[i]:
            continue
        pages = s["cache"][s["table"][i, :(L[i] + PAGE - 1) // PAGE].long()]
        new = min(n, L[i])
        for c in range(kv):
            rec = pages[:, c]
            b = rec[:, :8192].view(-1, PAGE, 64, 1)
            K = value[torch.cat([b % 16, b // 16], -1).long()].view(-1, PAGE, 4, 32)
            x = rec[:, 16384:16896].view(-1, 4, 16, 8)[:, :, token % 16, token // 16].transpose(1, 2)
            K = (K * torch.exp2(x.double() - 127.0)[..., None]).reshape(-1, DH)[:L[i]]
            b = rec[:, 8192:16384].view(-1, DH, 64, 1)
            V = value[torch.cat([b % 16, b // 16], -1).long()].view(-1, DH, PAGE)[:, :, place].transpose(1, 2)
            x = rec[:, 16896:].contiguous().view(torch.bfloat16)[:, place].double()
            V = (V * x[..., None]).reshape(-1, DH)[:L[i]]
            K[L[i] - new:] = kh[i * n + n - new:(i + 1) * n, c]
            V[L[i] - new:] = vh[i * n + n - new:(i + 1) * n, c]
            at = L[i] - new + torch.arange(new, device=DEV)[:, None]
            later = torch.arange(L[i], device=DEV) > at
            for h in range(c * (H // kv), (c + 1) * (H // kv)):
                S = (q[i, n - new:, h] @ K.t() * DH ** -0.5).masked_fill_(later, -math.inf)
                lse[h, i, n - new:] = torch.logsumexp(S, 1)
                o[i, n - new:, h] = torch.softmax(S, 1) @ V
    return dict(out, o=o.view(E * n, H, DH), lse=lse.reshape(H, E * n))
