"""Performance cases of the static-pattern attention and of the paged 8-bit cache, with their plain forms.

A case is a dict of plain values.  Its ``kind`` names the calls of one pass:

  fwd      window_fwd: attention with a sliding window and a few first tokens (sinks) that stay visible
  step     window_fwd and window_bwd, as a training layer makes them
  append   cache_append: keys and values rotated, quantised to 8 bits and written into their pages, queries rotated
  attn     cache_attn: attention of the newest tokens over the paged 8-bit cache

A row at position i of its sequence sees the keys j <= i with i - j < W (W = 0: all of them) or j < S.
The cache holds blocks (pages) of 64 tokens: K codes [pages, Hkv, 64, d] and V codes [pages, Hkv, d, 64] in e4m3,
and a scale (a power of two) per page and head for each.
"""
import math

import torch

own = False
DEV = "cuda"
PAGE = 64


def listed():
    return [
        # the smallest training call: one short document of odd length, where launches and latency count
        dict(name="fwd_777_d64", kind="fwd", B=1, Hq=4, Hkv=2, N=777, d=64, W=256, S=4, packed=False),
        # prefill of a 32K layer's heads with the static pattern
        dict(name="fwd_32k", kind="fwd", B=1, Hq=16, Hkv=2, N=32768, d=128, W=4096, S=64, packed=False),
        # an ordinary training layer at head dim 64
        dict(name="step_16k_d64", kind="step", B=1, Hq=12, Hkv=4, N=16384, d=64, W=1024, S=16, packed=False),
        # packed documents of ragged, odd lengths in one 20K-token row
        dict(name="step_packed_20k", kind="step", B=7, Hq=28, Hkv=4, N=20011, d=128, W=1024, S=4, packed=True),
        # a long training layer: 128K tokens, GQA 4
        dict(name="step_128k", kind="step", B=1, Hq=32, Hkv=8, N=131072, d=128, W=4096, S=64, packed=False),
        # one decoded token for each of 64 sequences
        dict(name="append_b64_t1", kind="append", B=64, Hq=28, Hkv=4, T=1, d=128, L=20000, ragged=False),
        # ragged chunks that start and end inside pages, head dim 64
        dict(name="append_b6_t501_d64", kind="append", B=6, Hq=12, Hkv=4, T=501, d=64, L=3000, ragged=True),
        # the prompt of a 128K prefill into its pages
        dict(name="append_128k", kind="append", B=1, Hq=28, Hkv=4, T=131072, d=128, L=0, ragged=False),
        # one sequence, one token, a short context: latency
        dict(name="attn_b1_4k_d64", kind="attn", B=1, Hq=4, Hkv=1, T=1, d=64, L=4097, W=0, S=0),
        # a serving batch of ragged contexts, one token each
        dict(name="attn_b32_16k", kind="attn", B=32, Hq=28, Hkv=4, T=1, d=128, L=16384, W=0, S=0),
        # long contexts, one token each: the cache's bytes
        dict(name="attn_b8_128k", kind="attn", B=8, Hq=32, Hkv=8, T=1, d=128, L=131072, W=0, S=0),
        # a prefill chunk over a cached context in the static pattern
        dict(name="attn_chunk_200_window", kind="attn", B=4, Hq=16, Hkv=2, T=200, d=128, L=32768, W=4096, S=64),
    ]


def _log(rng, a, b):
    return max(a, min(b, int(math.exp(rng.uniform(math.log(a), math.log(b + 1))))))


def draw(rng):
    kind = rng.choice(["fwd", "step", "append", "attn"])
    Hq, Hkv = rng.choice([(1, 1), (4, 1), (8, 8), (8, 2), (12, 4), (16, 2), (28, 4), (32, 8)])
    c = dict(kind=kind, Hq=Hq, Hkv=Hkv, d=rng.choice([64, 128, 128]))
    if kind in ("fwd", "step"):
        c["packed"] = rng.random() < 0.5
        c["N"] = _log(rng, 20, 65536)
        c["B"] = _log(rng, 2, 12) if c["packed"] else (rng.choice([1, 1, 2, 3]) if c["N"] < 16384 else 1)
        c["W"] = _log(rng, 16, min(4096, c["N"])) if rng.random() < 0.9 or c["N"] > 8192 else 0
        c["S"] = rng.choice([0, 1, 4, 16, 64, 100])
        return c
    if kind == "append":
        c["B"] = _log(rng, 1, 128)
        c["T"] = 1 if rng.random() < 0.3 else _log(rng, 1, 65536 // c["B"])
        c["L"] = rng.choice([0, _log(rng, 1, min(32768, 524288 // c["B"]))])
        c["ragged"] = rng.random() < 0.5
        return c
    c["T"] = rng.choice([1, 1, _log(rng, 2, 8), _log(rng, 9, 300)])
    c["L"] = max(c["T"], _log(rng, 64, 65536))
    c["B"] = _log(rng, 1, max(1, min(64, 524288 // c["L"], (1 << 31) // (c["L"] * c["T"] * Hq))))
    c["W"], c["S"] = rng.choice([(0, 0), (0, 0), (_log(rng, 64, 4096), rng.choice([0, 4, 64, 130]))])
    return c


# ---------------------------------------------------------------- inputs
def _lengths(total, parts, g):
    """`parts` ragged positive lengths that add up to `total`."""
    if parts >= total:
        return [1] * total
    w = (torch.rand(parts, generator=g, dtype=torch.float64) + 0.1).tolist()
    n = [max(1, int(x / sum(w) * total)) for x in w]
    n[n.index(max(n))] += total - sum(n)
    return n


def _pow2_scale(amax):
    """The smallest power of two s >= 2^-126 with amax <= 448 s (448 = 0.875 * 2^9 is e4m3's largest value)."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    one = torch.ones_like(amax)
    return torch.ldexp(one, torch.where(amax > 0, e, torch.full_like(e, -126)).clamp(min=-126))


def _randn(shape, g):
    return torch.randn(shape, generator=g, device=DEV)


def prepare(case, seed):
    c, kind = case, case["kind"]
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    h = torch.Generator()
    h.manual_seed(seed)
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    bf = torch.bfloat16
    s = dict(c=c)
    if kind in ("fwd", "step"):
        rows = 1 if c["packed"] else c["B"]
        s["lens"] = _lengths(c["N"], c["B"], h) if c["packed"] else [c["N"]] * c["B"]
        q = _randn((rows, Hq, c["N"], d), g)
        k = _randn((rows, Hkv, c["N"], d), g)
        # the first tokens draw weight from every row, as they do in trained models
        lift = 1.5 * q.mean((1, 2), keepdim=True) / q.mean((1, 2), keepdim=True).norm(dim=-1, keepdim=True)
        q += lift
        at = 0
        for n in s["lens"] if c["packed"] else [c["N"]]:
            k[:, :, at:at + min(4, n)] += 1.5 * lift
            at += n
        s["q"], s["k"], s["v"] = q.to(bf), k.to(bf), _randn((rows, Hkv, c["N"], d), g).to(bf)
        s["do"] = _randn((rows, Hq, c["N"], d), g).to(bf) if kind == "step" else None
        starts = torch.tensor([0] + s["lens"]).cumsum(0).to(torch.int32)
        s["starts"] = starts.to(DEV) if c["packed"] else None
        return s
    B, T, L = c["B"], c["T"], c["L"]
    if kind == "append":
        lens = [L] * B if B == 1 else [int(L * (0.2 + 0.8 * x)) for x in torch.rand(B, generator=h).tolist()]
        counts = [max(0, int(T * (1.1 * x - 0.05))) for x in torch.rand(B, generator=h).tolist()]
        counts = [min(T, x) for x in counts] if c["ragged"] else [T] * B
        need = [(n + T + PAGE) // PAGE + 1 for n in lens]
    else:
        lens = [L] if B == 1 else [max(T, int(L * (0.1 + 0.9 * x))) for x in torch.rand(B, generator=h).tolist()]
        lens[0] = L
        need = [(n + PAGE - 1) // PAGE for n in lens]
    width = (L + T + PAGE) // PAGE + 1
    pages = B * width
    order = torch.randperm(pages, generator=h).tolist()
    table = torch.zeros((B, width), dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    s["table"] = table.to(DEV)
    s["lens"] = torch.tensor(lens, dtype=torch.int32).to(DEV)
    s["host_lens"] = lens
    # pages in use hold keys with a few large channels and ordinary values; unused slots hold an older sequence's
    f8 = torch.float8_e4m3fn
    chan = 1.0 + 3.0 * (torch.rand(d, generator=g, device=DEV) < 0.05)
    s["k"] = torch.empty((pages, Hkv, PAGE, d), dtype=f8, device=DEV)
    s["v"] = torch.empty((pages, Hkv, d, PAGE), dtype=f8, device=DEV)
    s["ks"], s["vs"] = (torch.empty((pages, Hkv), device=DEV) for _ in range(2))
    step = max(1, (1 << 27) // (Hkv * PAGE * d))
    for p in range(0, pages, step):
        e = min(pages, p + step)
        for x, codes, scale in ((_randn((e - p, Hkv, PAGE, d), g) * chan, s["k"], s["ks"]),
                                (_randn((e - p, Hkv, d, PAGE), g), s["v"], s["vs"])):
            sc = _pow2_scale(x.abs().amax((2, 3)))
            codes[p:e] = (x / sc[:, :, None, None]).to(f8)
            scale[p:e] = sc
    s["q"] = _randn((B, Hq, T, d), g).to(bf)
    if kind == "append":
        s["knew"] = (_randn((B, Hkv, T, d), g) * chan).to(bf)
        s["vnew"] = _randn((B, Hkv, T, d), g).to(bf)
        s["counts"] = torch.tensor(counts, dtype=torch.int32).to(DEV) if c["ragged"] else None
        s["freq"] = (500000.0 ** (-torch.arange(d // 2, dtype=torch.float64) * 2 / d)).float().to(DEV)
    return s


# ---------------------------------------------------------------- plain forms
ROWS = 1024  # query rows of a chunk: bounds the memory of the plain form's logits


def _plain_window(c, q, k, v, do):
    """One document or one batch of equal lengths: q [B, Hq, n, d], all in 32 bits."""
    B, Hq, n, d = q.shape
    Hkv, W, S = c["Hkv"], c["W"] or n, c["S"]
    G, scale = Hq // Hkv, 1 / math.sqrt(d)
    q5, lse = q.view(B, Hkv, G, n, d), torch.empty((B, Hkv, G, n), device=q.device)
    out = torch.empty_like(q5)
    if do is not None:
        do5, dq, dk, dv = do.view(B, Hkv, G, n, d), torch.empty_like(q5), torch.zeros_like(k), torch.zeros_like(v)
    pos = torch.arange(n, device=q.device)
    for r0 in range(0, n, ROWS):
        r1 = min(n, r0 + ROWS)
        lo = max(0, r0 - W + 1)
        s1 = min(S, lo)
        m, i = torch.cat([pos[:s1], pos[lo:r1]]), pos[r0:r1, None]
        hidden = (m > i) | ((i - m >= W) & (m >= S))
        kk, vv = torch.cat([k[:, :, :s1], k[:, :, lo:r1]], 2), torch.cat([v[:, :, :s1], v[:, :, lo:r1]], 2)
        qq = q5[:, :, :, r0:r1].reshape(B, Hkv, -1, d)
        z = (qq @ kk.transpose(-1, -2).contiguous()).mul_(scale).view(B, Hkv, G, r1 - r0, -1)
        z.masked_fill_(hidden, -math.inf)
        top = z.amax(-1, keepdim=True)
        p = z.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        p = p.div_(total).view(B, Hkv, G * (r1 - r0), -1)
        o = p @ vv
        out[:, :, :, r0:r1] = o.view(B, Hkv, G, r1 - r0, d)
        lse[:, :, :, r0:r1] = (top + total.log()).squeeze(-1)
        if do is None:
            continue
        gg = do5[:, :, :, r0:r1].reshape(B, Hkv, -1, d)
        dvs = p.transpose(-1, -2) @ gg
        dz = (gg @ vv.transpose(-1, -2).contiguous()).sub_((gg * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
        dq[:, :, :, r0:r1] = (dz @ kk).view(B, Hkv, G, r1 - r0, d)
        dks = dz.transpose(-1, -2) @ qq
        for acc, part in ((dk, dks), (dv, dvs)):
            acc[:, :, :s1] += part[:, :, :s1]
            acc[:, :, lo:r1] += part[:, :, s1:]
    got = [out.view(B, Hq, n, d), lse.view(B, Hq, n)]
    return got if do is None else got + [dq.view(B, Hq, n, d), dk, dv]


def _window(s):
    c, bf = s["c"], torch.bfloat16
    x = [None if t is None else t.float() for t in (s["q"], s["k"], s["v"], s["do"])]
    if c["packed"]:
        docs = zip(*(([None] * len(s["lens"])) if t is None else t.split(s["lens"], 2) for t in x))
        got = [_plain_window(c, *(None if t is None else t.contiguous() for t in doc)) for doc in docs]
        got = [torch.cat(parts, 2) for parts in zip(*got)]
    else:
        got = _plain_window(c, *x)
    names = ("out", "lse", "dq", "dk", "dv")
    return {n: t if n == "lse" else t.to(bf) for n, t in zip(names, got)}


def _rotate(x, cos, sin):
    """x [B, H, T, d], halves paired (i, i + d / 2)."""
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _angles(s, T):
    pos = s["lens"].double()[:, None] + torch.arange(T, device=DEV, dtype=torch.float64)
    ang = pos[:, None, :, None] * s["freq"].double()
    return ang.cos().float(), ang.sin().float()


def _append(s):
    c = s["c"]
    B, T, Hkv, d = c["B"], c["T"], c["Hkv"], c["d"]
    cos, sin = _angles(s, T)
    q_rot = _rotate(s["q"].float(), cos, sin).to(torch.bfloat16)
    lens = s["lens"].long()[:, None, None]
    counts = T if s["counts"] is None else s["counts"].long()[:, None, None]
    P = (T + PAGE - 1 + PAGE - 1) // PAGE
    slot = (lens // PAGE + torch.arange(P, device=DEV)[:, None]) * PAGE + torch.arange(PAGE, device=DEV)  # [B, P, 64]
    old, new = slot < lens, (slot >= lens) & (slot < lens + counts)
    t = (slot - lens).clamp(0, T - 1).view(B, 1, P * PAGE, 1).expand(B, Hkv, P * PAGE, d)
    page = s["table"].gather(1, (lens.view(B, 1) // PAGE + torch.arange(P, device=DEV)).clamp(
        max=s["table"].shape[1] - 1)).long()  # [B, P]
    old, new = old[:, :, None, :, None], new[:, :, None, :, None]
    for x, codes, scale, turned in ((_rotate(s["knew"].float(), cos, sin), s["k"], s["ks"], False),
                                    (s["vnew"].float(), s["v"], s["vs"], True)):
        x = x.gather(2, t).view(B, Hkv, P, PAGE, d).transpose(1, 2) * new  # [B, P, Hkv, 64, d]
        held = codes.view(torch.uint8)[page].view(codes.dtype).float()
        held = held.transpose(-1, -2) if turned else held
        was, has = scale[page], old.any(3, keepdim=True).view(B, P, 1)
        need = _pow2_scale(x.abs().amax((3, 4)))
        now = torch.where(has, torch.maximum(need, was), need)
        now = torch.where(new.any(3, keepdim=True).view(B, P, 1), now, was)
        ratio = (was / now)[..., None, None]
        value = torch.where(new, x / now[..., None, None], torch.where(old, held * ratio, held))
        value = (value.transpose(-1, -2) if turned else value).to(codes.dtype)
        codes.view(torch.uint8)[page] = value.contiguous().view(torch.uint8)
        scale[page] = now
    return dict(q=q_rot, k=s["k"], v=s["v"], ks=s["ks"], vs=s["vs"])


def _attn(s):
    c = s["c"]
    B, T, Hq, Hkv, d = c["B"], c["T"], c["Hq"], c["Hkv"], c["d"]
    G, table = Hq // Hkv, s["table"].long()
    L = table.shape[1] * PAGE
    k = s["k"].view(torch.uint8)[table].view(s["k"].dtype).float().mul_(s["ks"][table][..., None, None])
    k = k.permute(0, 2, 4, 1, 3).reshape(B, Hkv, d, L)  # [B, Hkv, d, L]
    z = (s["q"].float().view(B, Hkv, G * T, d) @ k).mul_(1 / math.sqrt(d)).view(B, Hkv, G, T, L)
    del k
    i = (s["lens"].long()[:, None] - T + torch.arange(T, device=DEV))[:, None, None, :, None]
    m = torch.arange(L, device=DEV)
    hidden = (m > i) | ((i - m >= (c["W"] or L + T)) & (m >= c["S"]))
    z.masked_fill_(hidden, -math.inf)
    top = z.amax(-1, keepdim=True)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(total).view(B, Hkv, G * T, L)
    v = s["v"].view(torch.uint8)[table].view(s["v"].dtype).float().mul_(s["vs"][table][..., None, None])
    v = v.permute(0, 2, 1, 4, 3).reshape(B, Hkv, L, d)
    return dict(out=(p @ v).view(B, Hq, T, d).to(torch.bfloat16),
                lse=(top + total.log()).view(B, Hq, T))


# ---------------------------------------------------------------- one pass
def run(s):
    c, kind = s["c"], s["c"]["kind"]
    if not own:
        return {"fwd": _window, "step": _window, "append": _append, "attn": _attn}[kind](s)
    import paper_2510_18830_amd as ms
    if kind in ("fwd", "step"):
        q, k, v = s["q"], s["k"], s["v"]
        win = ms.make_window(c["B"], max(s["lens"]), c["Hq"], c["Hkv"], c["d"], window=c["W"], sinks=c["S"],
                             tokens=c["N"] if c["packed"] else 0)
        out, lse = ms.window_fwd(win, q, k, v, starts=s["starts"])
        if kind == "fwd":
            return dict(out=out, lse=lse)
        dq, dk, dv = ms.window_bwd(win, q, k, v, out, s["do"], lse, starts=s["starts"])
        return dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv)
    cache = ms.Cache(s["k"], s["v"], s["ks"], s["vs"])
    if kind == "append":
        q = ms.cache_append(cache, s["table"], s["lens"], s["knew"], s["vnew"], q=s["q"], inv_freq=s["freq"],
                            counts=s["counts"])
        return dict(q=q, k=s["k"], v=s["v"], ks=s["ks"], vs=s["vs"])
    out, lse = ms.cache_attn(cache, s["table"], s["lens"], s["q"], window=c["W"], sinks=c["S"])
    return dict(out=out, lse=lse)


# ---------------------------------------------------------------- floors
def _visible(first, last, W, S):
    """Keys that the rows at the positions first .. last - 1 see, added up."""
    def upto(n):  # rows 0 .. n - 1
        if not W or n <= W:
            return n * (n + 1) / 2
        far = n - W  # rows W .. n - 1: the window and min(S, i + 1 - W) first tokens
        sinks = far * (far + 1) / 2 if far <= S else S * (S + 1) / 2 + (far - S) * S
        return W * (W + 1) / 2 + far * W + sinks
    return upto(last) - upto(first)


def _even_lengths(c):
    return [c["N"] / c["B"]] * c["B"] if c["packed"] else [c["N"]] * c["B"]


def work(case):
    c, kind = case, case["kind"]
    B, Hq, Hkv, d = c["B"], c["Hq"], c["Hkv"], c["d"]
    if kind in ("fwd", "step"):
        rows = c["N"] * (1 if c["packed"] else B)
        qb, kb = 2.0 * Hq * rows * d, 2.0 * Hkv * rows * d
        fwd = 4.0 * d * Hq * sum(_visible(0, n, c["W"], c["S"]) for n in _even_lengths(c))
        b = 2 * qb + 2 * kb + 4.0 * Hq * rows
        if kind == "fwd":
            return dict(bytes=b, flops=fwd)
        return dict(bytes=b + 2 * qb + 2 * kb, flops=3.5 * fwd)
    T = c["T"]
    if kind == "append":
        tokens = B * T * (0.5 if c["ragged"] else 1.0)
        return dict(bytes=tokens * d * (6.0 * Hkv + 4.0 * Hq), flops=tokens * d * 3.0 * (Hkv + Hq))
    lens = [c["L"]] if B == 1 else [max(T, 0.55 * c["L"])] * B
    read = [min(n, c["W"] + T - 1 + min(c["S"], n)) if c["W"] else n for n in lens]
    seen = sum(_visible(n - T, n, c["W"], c["S"]) for n in lens)
    return dict(bytes=2.0 * Hkv * d * sum(read) + B * T * Hq * (4.0 * d + 4), flops=4.0 * d * Hq * seen)


# ---------------------------------------------------------------- exact results
def _exact_rows(c, q, k, v, do, i, m):
    """One head, rows at the positions i over the keys at the positions m; 64 bits."""
    scale, W = 1 / math.sqrt(c["d"]), c["W"]
    seen = m[None] <= i[:, None]
    if W:
        seen &= (m[None] > i[:, None] - W) | (m[None] < c["S"])
    z = (q @ k.T * scale).masked_fill_(~seen, -math.inf)
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    o = p @ v
    if do is None:
        return o, lse
    dz = p * (do @ v.T - (do * o).sum(1, keepdim=True))
    return o, lse, scale * (dz @ k), scale * (dz.T @ q), p.T @ do


def _exact_window(c, s):
    names = ("q", "k", "v", "do") if c["kind"] == "step" else ("q", "k", "v")
    f64 = dict(dtype=torch.float64, device=DEV)
    shape, kshape, G = s["q"].shape, s["k"].shape, c["Hq"] // c["Hkv"]
    r = dict(out=torch.empty(shape, **f64), lse=torch.empty(shape[:3], **f64), dq=torch.empty(shape, **f64),
             dk=torch.zeros(kshape, **f64), dv=torch.zeros(kshape, **f64))
    docs, at = [], 0
    for n in s["lens"] if c["packed"] else [c["N"]]:
        docs.append((at, n))
        at += n
    for b in range(shape[0]):
        for h in range(c["Hq"]):
            for at, n in docs:
                x = dict((name, s[name][b, h if name in ("q", "do") else h // G, at:at + n].double()) for name in names)
                for r0 in range(0, n, 2048):
                    r1 = min(n, r0 + 2048)
                    pos = torch.arange(r1, device=DEV)
                    if c["W"]:
                        pos = pos[(pos < c["S"]) | (pos > r0 - c["W"])]
                    got = _exact_rows(c, x["q"][r0:r1], x["k"][pos], x["v"][pos],
                                      x["do"][r0:r1] if "do" in x else None, torch.arange(r0, r1, device=DEV), pos)
                    r["out"][b, h, at + r0:at + r1], r["lse"][b, h, at + r0:at + r1] = got[:2]
                    if "do" in x:
                        r["dq"][b, h, at + r0:at + r1] = got[2]
                        r["dk"][b, h // G].index_add_(0, at + pos, got[3])
                        r["dv"][b, h // G].index_add_(0, at + pos, got[4])
    if c["kind"] == "fwd":
        return dict(out=r["out"], lse=r["lse"])
    return r


def _to_e4m3(x):
    """The nearest e4m3 value (ties to even) of 64-bit values of magnitude up to 448."""
    e = torch.frexp(x)[1].clamp(min=-5) - 1
    step = torch.ldexp(torch.ones_like(x), e - 3)
    return torch.round(x / step) * step


def _exact_append(c, s):
    T, d = c["T"], c["d"]
    at = torch.tensor(s["host_lens"], device=DEV)[:, None] + torch.arange(T, device=DEV)
    spin = at.double()[:, None, :, None] * s["freq"].double()
    spin = torch.polar(torch.ones_like(spin), spin)

    def turn(x):
        x = torch.complex(x[..., :d // 2].double(), x[..., d // 2:].double()) * spin
        return torch.cat([x.real, x.imag], -1)

    r = dict(q=turn(s["q"]), ks=s["ks"].double(), vs=s["vs"].double())
    codes = dict(k=s["k"].double(), v=s["v"].double().transpose(-1, -2).contiguous())
    counts = [T] * c["B"] if s["counts"] is None else s["counts"].tolist()
    new = dict(k=turn(s["knew"]), v=s["vnew"].double())
    table = s["table"].tolist()
    for b, (at, n) in enumerate(zip(s["host_lens"], counts)):
        end, t = at + n, 0
        while at < end:
            page, o = table[b][at // PAGE], at % PAGE
            m = min(PAGE - o, end - at)
            for name, scale in (("k", r["ks"]), ("v", r["vs"])):
                x = new[name][b, :, t:t + m]  # [Hkv, m, d]
                top = x.abs().amax((1, 2))
                need = torch.exp2(torch.ceil(torch.log2(top / 448.0)).clamp(min=-126.0))
                need = torch.where(top > 448.0 * need, 2 * need, torch.where(top <= 224.0 * need, need / 2, need))
                was = scale[page].clone()
                now = torch.maximum(need, was) if o else need
                if o:
                    codes[name][page, :, :o] = _to_e4m3(codes[name][page, :, :o] * (was / now)[:, None, None])
                codes[name][page, :, o:o + m] = _to_e4m3(x / now[:, None, None])
                scale[page] = now
            at, t = at + m, t + m
    return dict(q=r["q"], k=codes["k"], v=codes["v"].transpose(-1, -2).contiguous(), ks=r["ks"], vs=r["vs"])


def _exact_attn(c, s):
    B, T, G = c["B"], c["T"], c["Hq"] // c["Hkv"]
    out = torch.empty((B, c["Hq"], T, c["d"]), dtype=torch.float64, device=DEV)
    lse = torch.empty((B, c["Hq"], T), dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["host_lens"]):
        pos = torch.arange(n, device=DEV)
        if c["W"]:
            pos = pos[(pos < c["S"]) | (pos > n - T - c["W"])]
        page, slot = s["table"][b].long()[pos // PAGE], pos % PAGE
        for hk in range(c["Hkv"]):
            k = s["k"].view(torch.uint8)[page, hk, slot].view(s["k"].dtype).double() * s["ks"][page, hk, None].double()
            v = s["v"].view(torch.uint8)[page, hk, :, slot].view(s["v"].dtype).double() * s["vs"][page, hk, None].double()
            for h in range(hk * G, hk * G + G):
                out[b, h], lse[b, h] = _exact_rows(c, s["q"][b, h].double(), k, v, None,
                                                   torch.arange(n - T, n, device=DEV), pos)
    return dict(out=out, lse=lse)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "append":
        return _exact_append(c, s)
    if c["kind"] == "attn":
        return _exact_attn(c, s)
    return _exact_window(c, s)
