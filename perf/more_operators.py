"""Performance cases of positions with several axes, of drafted trees over the paged 8-bit cache and of the operations
that rearrange its pages, with their plain forms.

A case is a dict of plain values.  Its ``kind`` names the calls of one pass:

  rotate   rotate of q and k, and the inverse one of their gradients: a training layer whose tokens have a position on
           each of several axes (time, row, column)
  append   cache_append at given positions of several axes: a prompt with images
  draft    tree_mask and cache_append at its positions: the nodes of a drafted tree enter the cache
  tree     cache_tree_attn: the nodes' attention over the cached context and their ancestors
  keep     cache_keep: the accepted path's tokens move to the places behind the context
  fork     cache_fork: sequences continue others; full pages shared, the last one copied, pages allotted and given back

Pair i of a head's columns (i, i + d / 2) turns by positions[axis[i]] * inv_freq[i].
A tree's node t has the parent parents[t] < t (-1: the context's last token) and lies in the cache behind the context, in
the order of the nodes, at the position context + depth.  It sees the context's tokens as any token at its position does
(the last W, the first S), its ancestors likewise, and itself.
The cache holds blocks (pages) of 64 tokens: K codes [pages, Hkv, 64, d] and V codes [pages, Hkv, d, 64] in e4m3,
and a scale (a power of two) per page and head for each.
"""
import math

import torch

own = False
DEV = "cuda"
PAGE = 64
F8, BF = torch.float8_e4m3fn, torch.bfloat16


def listed():
    return [
        # the smallest training call: a short sequence of odd length with the positions of an image; bf16 gradients
        dict(name="rotate_777_d64", kind="rotate", B=1, Hq=4, Hkv=2, N=777, d=64, axes=2, grads="bf16"),
        # a 128K layer with video positions, whose sparse attention gives gradients in 32 bits
        dict(name="rotate_128k", kind="rotate", B=1, Hq=32, Hkv=8, N=131072, d=128, axes=3, grads="fp32"),
        # two prompts of text and images into their pages, odd length
        dict(name="append_b2_20k", kind="append", B=2, Hq=28, Hkv=4, T=20011, d=128, L=0, axes=3, ragged=False),
        # a drafted tree for each sequence of a serving batch
        dict(name="draft_b64_t16", kind="draft", B=64, Hq=28, Hkv=4, T=16, d=128, L=4000, ragged=False),
        # few larger trees of ragged size at head dim 64
        dict(name="draft_b5_t61_d64", kind="draft", B=5, Hq=12, Hkv=4, T=61, d=64, L=1500, ragged=True),
        # one sequence, a small tree, a short context: latency
        dict(name="tree_b1_t8_4k_d64", kind="tree", B=1, Hq=4, Hkv=1, T=8, d=64, L=4097, W=0, S=0, ragged=False),
        # a serving batch of ragged contexts with a tree each
        dict(name="tree_b32_t16_16k", kind="tree", B=32, Hq=28, Hkv=4, T=16, d=128, L=16384, W=0, S=0, ragged=False),
        # long contexts and large trees: the matrix cores' work
        dict(name="tree_b8_t64_64k", kind="tree", B=8, Hq=32, Hkv=8, T=64, d=128, L=65536, W=0, S=0, ragged=False),
        # the accepted paths of a serving batch
        dict(name="keep_b64_t16", kind="keep", B=64, Hkv=8, T=16, d=128, L=1000),
        # long paths of large trees, over several pages
        dict(name="keep_b7_t200_d64", kind="keep", B=7, Hkv=2, T=200, d=64, L=700),
        # one step of a beam search: eight beams, the better ones forked, the others' pages given back
        dict(name="fork_b8_d64", kind="fork", B=8, N=8, Hkv=2, d=64, L=1000, more=1),
        # four continuations of each of 64 prompts, with room for the tokens to come
        dict(name="fork_b64_n256", kind="fork", B=64, N=256, Hkv=8, d=128, L=8192, more=200),
    ]


def _log(rng, a, b):
    return max(a, min(b, int(math.exp(rng.uniform(math.log(a), math.log(b + 1))))))


def draw(rng):
    kind = rng.choice(["rotate", "append", "draft", "tree", "tree", "keep", "fork"])
    Hq, Hkv = rng.choice([(1, 1), (4, 1), (8, 8), (8, 2), (12, 4), (16, 2), (28, 4), (32, 8)])
    c = dict(kind=kind, Hkv=Hkv, d=rng.choice([64, 128, 128]))
    if kind in ("keep", "fork"):
        c["B"] = _log(rng, 1, 128)
        c["L"] = _log(rng, 1, 2000 if kind == "keep" else 8192)
        if kind == "keep":
            c["T"] = _log(rng, 2, 256)
        else:
            c["N"] = _log(rng, 1, 256)
            c["more"] = _log(rng, 1, 300)
        return c
    c["Hq"] = Hq
    if kind == "rotate":
        c["N"] = _log(rng, 20, 65536)
        c["B"] = rng.choice([1, 1, 2, 3]) if c["N"] < 16384 else 1
        c["axes"], c["grads"] = rng.choice([1, 2, 3, 4]), rng.choice(["bf16", "fp32"])
        return c
    c["ragged"] = rng.random() < 0.5
    if kind == "append":
        c["B"] = _log(rng, 1, 16)
        c["T"] = _log(rng, 2, 32768 // c["B"])
        c["L"] = rng.choice([0, _log(rng, 1, 8192)])
        c["axes"] = rng.choice([1, 2, 3, 4])
    elif kind == "draft":
        c["B"], c["T"], c["L"] = _log(rng, 1, 128), _log(rng, 2, 256), _log(rng, 1, 4096)
    else:
        c["T"] = rng.choice([_log(rng, 2, 8), _log(rng, 9, 64), _log(rng, 65, 256)])
        c["L"] = max(c["T"], _log(rng, 64, 65536))
        c["B"] = _log(rng, 1, max(1, min(64, 524288 // c["L"], (1 << 29) // (c["L"] * c["T"] * Hq))))
        c["W"], c["S"] = rng.choice([(0, 0), (0, 0), (_log(rng, 64, 4096), rng.choice([0, 4, 64, 130]))])
    return c


# ---------------------------------------------------------------- inputs
def _pow2_scale(amax):
    """The smallest power of two s >= 2^-126 with amax <= 448 s (448 = 0.875 * 2^9 is e4m3's largest value)."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    one = torch.ones_like(amax)
    return torch.ldexp(one, torch.where(amax > 0, e, torch.full_like(e, -126)).clamp(min=-126))


def _randn(shape, g):
    return torch.randn(shape, generator=g, device=DEV)


def _freq(d):
    return (500000.0 ** (-torch.arange(d // 2, dtype=torch.float64) * 2 / d)).float().to(DEV)


def _grid(axes, B, n, first, g):
    """Positions [axes, B, n] of text with images or video between it: a line of text counts up on every axis, a patch has
    the time of its frame and its own row and column."""
    t = torch.arange(n, device=DEV)
    rows, columns = torch.randint(6, 30, (2, B, 1), generator=g, device=DEV)
    text = 40
    chunk = text + rows * columns
    turn, at = t // chunk, t % chunk                                  # [B, n]
    patch = (at - text).clamp(min=0)
    image = at >= text
    base = first[:, None] + turn * (text + 30)
    whole = [base + torch.where(image, torch.full_like(at, text), at),
             base + torch.where(image, text + patch // columns, at),
             base + torch.where(image, text + patch % columns, at),
             base + at]
    return torch.stack(whole[:axes]).to(torch.int32).contiguous()


def _axis(d, axes):
    """The axis of each pair of columns: the first takes a share of the slow ones too, the others take turns."""
    i = torch.arange(d // 2)
    return torch.where(i < d // 8, torch.zeros_like(i), i % axes).to(torch.int32).to(DEV)


def _pool(pages, Hkv, d, g, s):
    """Pages hold keys with a few large channels and ordinary values; unused slots hold an older sequence's."""
    chan = 1.0 + 3.0 * (torch.rand(d, generator=g, device=DEV) < 0.05)
    s["k"] = torch.empty((pages, Hkv, PAGE, d), dtype=F8, device=DEV)
    s["v"] = torch.empty((pages, Hkv, d, PAGE), dtype=F8, device=DEV)
    s["ks"], s["vs"] = (torch.empty((pages, Hkv), device=DEV) for _ in range(2))
    step = max(1, (1 << 27) // (Hkv * PAGE * d))
    for p in range(0, pages, step):
        e = min(pages, p + step)
        for x, codes, scale in ((_randn((e - p, Hkv, PAGE, d), g) * chan, s["k"], s["ks"]),
                                (_randn((e - p, Hkv, d, PAGE), g), s["v"], s["vs"])):
            sc = _pow2_scale(x.abs().amax((2, 3)))
            codes[p:e] = (x / sc[:, :, None, None]).to(F8)
            scale[p:e] = sc
    return chan


def _table(need, width, pages, h):
    """Table [B, width] with `need` pages of each sequence, in no order; -1 where there is none."""
    order = torch.randperm(pages, generator=h).tolist()
    table = torch.full((len(need), width), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    return table


def _parents(B, T, h):
    """Trees whose nodes follow any earlier one, later ones more often (paths of some length among them)."""
    u = torch.rand((B, T), generator=h, dtype=torch.float64) ** 0.5
    return ((u * (torch.arange(T) + 1)).long() - 1).to(torch.int32)


def prepare(case, seed):
    c, kind = case, case["kind"]
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    h = torch.Generator()
    h.manual_seed(seed)
    Hq, Hkv, d, B = c.get("Hq"), c["Hkv"], c["d"], c["B"]
    s = dict(c=c)
    if kind == "rotate":
        N, to = c["N"], torch.float32 if c["grads"] == "fp32" else BF
        for name, heads, t in (("q", Hq, BF), ("kk", Hkv, BF), ("dq", Hq, to), ("dk", Hkv, to)):
            s[name] = _randn((B, heads, N, d), g).to(t)
        s["positions"] = _grid(c["axes"], B, N, torch.zeros(B, dtype=torch.int64, device=DEV), g)
        s["axis"], s["freq"] = _axis(d, c["axes"]), _freq(d)
        return s
    L = c["L"]
    lens = [L] if B == 1 else [max(1, int(L * (0.2 + 0.8 * x))) for x in torch.rand(B, generator=h).tolist()]
    lens = [0] * B if L == 0 else lens
    if kind == "fork":
        N, more = c["N"], c["more"]
        width = (L + max(more, 2 * PAGE) + PAGE - 1) // PAGE + 1
        held = [min(width, (n + PAGE - 1) // PAGE + x) for n, x in zip(lens, torch.randint(0, 2, (B,), generator=h).tolist())]
        # a few pages hold a prefix that other tables share, and some room is left
        pages = B * width + N * (more // PAGE + 2) + 37
        table = _table(held, width, pages, h)
        refs = torch.zeros(pages, dtype=torch.int32)
        refs[table[table >= 0].long()] = 1
        refs[torch.randperm(pages, generator=h)[:max(1, pages // 50)]] += 1
        src = torch.randint(0, B, (N,), generator=h)
        src[torch.rand(N, generator=h) < 0.02] = -1
        src = src.to(torch.int32)
        s["src"], s["table"], s["refs"] = src.to(DEV), table.to(DEV), refs.to(DEV)
        s["lens"] = torch.tensor(lens, dtype=torch.int32).to(DEV)
        s["room"] = torch.where(src >= 0, torch.tensor(lens)[src.clamp(min=0).long()] + more, 0).to(torch.int32).to(DEV)
        _pool(pages, Hkv, d, g, s)
        return s
    T = c["T"]
    counts = [max(1, int(T * x)) for x in torch.rand(B, generator=h).tolist()] if c.get("ragged") else [T] * B
    s["counts"] = torch.tensor(counts, dtype=torch.int32).to(DEV) if c.get("ragged") else None
    width = (L + T + PAGE) // PAGE + 1
    pages = B * width
    s["table"] = _table([(n + T + PAGE) // PAGE + 1 for n in lens], width, pages, h).to(DEV)
    chan = _pool(pages, Hkv, d, g, s)
    s["host_lens"], s["host_counts"] = lens, counts
    before = torch.tensor(lens, dtype=torch.int32).to(DEV)
    if kind in ("draft", "tree"):
        parents = _parents(B, T, h)
        s["host_parents"], s["parents"] = parents.tolist(), parents.to(DEV)
    if kind == "append":
        s["positions"] = _grid(c["axes"], B, T, before.long(), g)
        s["axis"] = _axis(d, c["axes"])
    if kind in ("append", "draft"):
        s["lens"], s["freq"] = before, _freq(d)
        s["q"] = _randn((B, Hq, T, d), g).to(BF)
        s["knew"] = (_randn((B, Hkv, T, d), g) * chan).to(BF)
        s["vnew"] = _randn((B, Hkv, T, d), g).to(BF)
        return s
    s["lens"] = before + (T if s["counts"] is None else s["counts"])
    if kind == "tree":
        # the masks are made once for all layers of a step, so that a layer's call finds them there
        s["at"], s["seen"] = _plain_mask(s["parents"], before, s["counts"], c["W"], c["S"])
        s["q"] = _randn((B, Hq, T, d), g).to(BF)
        return s
    # accepted paths: one in five nodes or so, ascending
    path, kept = torch.zeros((B, T), dtype=torch.int32), []
    for b in range(B):
        take = (torch.rand(T, generator=h) < 0.2).nonzero().flatten()
        path[b, :take.numel()] = take.to(torch.int32)
        kept.append(take.numel())
    s["host_path"], s["host_kept"] = path.tolist(), kept
    s["path"], s["kept"] = path.to(DEV), torch.tensor(kept, dtype=torch.int32).to(DEV)
    return s


# ---------------------------------------------------------------- plain forms
def _angles(s, positions):
    """cos and sin [B, 1, T, d / 2] of every pair's angle."""
    half = s["freq"].numel()
    axis = s["axis"].long() if "axis" in s else torch.zeros(half, dtype=torch.int64, device=DEV)
    ang = positions.double()[axis].permute(1, 2, 0)[:, None] * s["freq"].double()
    return ang.cos().float(), ang.sin().float()


def _turn(x, cos, sin):
    """x [B, H, T, d] in 32 bits."""
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _rotate(s):
    cos, sin = _angles(s, s["positions"])
    q, k = (_turn(s[n].float(), cos, sin).to(BF) for n in ("q", "kk"))
    dq, dk = (_turn(s[n].float(), cos, -sin).to(s[n].dtype) for n in ("dq", "dk"))
    return dict(q=q, k=k, dq=dq, dk=dk)


def _plain_mask(parents, before, counts, W, S):
    """Positions [B, T] and words [B, T, (T + 31) / 32] whose bit u says whether node t sees node u."""
    B, T = parents.shape
    t = torch.arange(T, device=DEV)
    live = torch.ones((B, T), dtype=torch.bool, device=DEV) if counts is None else t < counts[:, None]
    up = ((parents[:, :, None] == t) & (parents[:, :, None] < t[:, None])).float() + torch.eye(T, device=DEV)
    for _ in range((T - 1).bit_length()):  # ancestors 1, 2, 4, .. steps up
        up = (up @ up > 0).float()
    depth = up.sum(-1).to(torch.int32) - 1
    at = torch.where(live, before[:, None] + depth, before[:, None])
    sees = (up > 0) & live[:, :, None] & live[:, None, :]
    if W:
        sees &= (at[:, :, None] - at[:, None, :] < W) | (at[:, None, :] < S)
    words = (T + 31) // 32
    sees = torch.nn.functional.pad(sees, (0, 32 * words - T)).view(B, T, words, 32)
    bits = (sees.long() << torch.arange(32, device=DEV)).sum(-1)
    return at.to(torch.int32), ((bits ^ (1 << 31)) - (1 << 31)).to(torch.int32)


def _append(s):
    c = s["c"]
    B, T, Hkv, d = c["B"], c["T"], c["Hkv"], c["d"]
    more = {}
    if c["kind"] == "draft":
        more["at"], more["seen"] = _plain_mask(s["parents"], s["lens"], s["counts"], 0, 0)
    cos, sin = _angles(s, more["at"][None] if more else s["positions"])
    q_rot = _turn(s["q"].float(), cos, sin).to(BF)
    lens = s["lens"].long()[:, None, None]
    counts = T if s["counts"] is None else s["counts"].long()[:, None, None]
    P = (T + PAGE - 1 + PAGE - 1) // PAGE
    slot = (lens // PAGE + torch.arange(P, device=DEV)[:, None]) * PAGE + torch.arange(PAGE, device=DEV)  # [B, P, 64]
    old, new = slot < lens, (slot >= lens) & (slot < lens + counts)
    t = (slot - lens).clamp(0, T - 1).view(B, 1, P * PAGE, 1).expand(B, Hkv, P * PAGE, d)
    page = s["table"].gather(1, (lens.view(B, 1) // PAGE + torch.arange(P, device=DEV)).clamp(
        max=s["table"].shape[1] - 1)).long()  # [B, P]
    old, new = old[:, :, None, :, None], new[:, :, None, :, None]
    for x, codes, scale, turned in ((_turn(s["knew"].float(), cos, sin), s["k"], s["ks"], False),
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
    return dict(q=q_rot, k=s["k"], v=s["v"], ks=s["ks"], vs=s["vs"], **more)


def _tree(s):
    c = s["c"]
    B, T, Hq, Hkv, d = c["B"], c["T"], c["Hq"], c["Hkv"], c["d"]
    G, table = Hq // Hkv, s["table"].clamp(min=0).long()
    L = table.shape[1] * PAGE
    counts = torch.full((B,), T, device=DEV) if s["counts"] is None else s["counts"].long()
    before = (s["lens"].long() - counts)[:, None, None]
    # which tokens a node sees: of the context by its position, of the tree by its bits
    j, at, live = torch.arange(L, device=DEV), s["at"].long()[:, :, None], (torch.arange(T, device=DEV) < counts[:, None])
    context = (j < before) & (((at - j < c["W"]) | (j < c["S"])) if c["W"] else (j >= 0)) & live[:, :, None]
    bits = (s["seen"].long()[..., None] >> torch.arange(32, device=DEV)) & 1
    bits = bits.reshape(B, T, -1)[:, :, :T]
    sees = context | ((j >= before) & (j < before + T) & (bits.gather(2, (j - before).clamp(0, T - 1).expand(B, T, L)) > 0))
    k = s["k"].view(torch.uint8)[table].view(F8).float().mul_(s["ks"][table][..., None, None])
    k = k.permute(0, 2, 4, 1, 3).reshape(B, Hkv, d, L)
    z = (s["q"].float().view(B, Hkv, G * T, d) @ k).mul_(1 / math.sqrt(d)).view(B, Hkv, G, T, L)
    del k
    z.masked_fill_(~sees[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    p = z.sub_(top.clamp(min=-3e38)).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(total.clamp(min=1e-38)).view(B, Hkv, G * T, L)
    v = s["v"].view(torch.uint8)[table].view(F8).float().mul_(s["vs"][table][..., None, None])
    v = v.permute(0, 2, 1, 4, 3).reshape(B, Hkv, L, d)
    return dict(out=(p @ v).view(B, Hq, T, d).to(BF), lse=(top + total.log()).view(B, Hq, T))


def _keep(s):
    c = s["c"]
    B, T, Hkv, d = c["B"], c["T"], c["Hkv"], c["d"]
    before = s["lens"].long()[:, None] - T  # [B, 1]
    P = (T + PAGE - 1 + PAGE - 1) // PAGE
    first = before // PAGE
    slot = first * PAGE + torch.arange(P * PAGE, device=DEV)  # [B, P 64]
    i = slot - before
    moves = (i >= 0) & (i < s["kept"].long()[:, None])
    come = torch.where(moves, before + s["path"].long().gather(1, i.clamp(0, T - 1)), slot) - first * PAGE
    live = slot < before + s["kept"].long()[:, None]
    other = (moves & (come // PAGE != torch.arange(P * PAGE, device=DEV) // PAGE))[:, None, :, None]
    page = s["table"].gather(1, first + torch.arange(P, device=DEV)).long()
    wide = come[:, None, :, None].expand(B, Hkv, P * PAGE, d)
    for codes, scale, turned in ((s["k"], s["ks"], False), (s["v"], s["vs"], True)):
        raw = codes.view(torch.uint8)[page].view(F8).float()  # [B, P, Hkv, 64, d]
        raw = (raw.transpose(-1, -2) if turned else raw).transpose(1, 2).reshape(B, Hkv, P * PAGE, d)
        was = scale[page].transpose(1, 2)  # [B, Hkv, P]
        x = (raw * was.repeat_interleave(PAGE, 2)[..., None]).gather(2, wide)
        need = _pow2_scale((x.abs() * other).view(B, Hkv, P, -1).amax(-1))
        now = torch.where(other.view(B, 1, P, PAGE).any(-1), torch.maximum(need, was), was)
        x = torch.where(live[:, None, :, None], x / now.repeat_interleave(PAGE, 2)[..., None], raw)
        x = x.view(B, Hkv, P, PAGE, d).transpose(1, 2)
        x = (x.transpose(-1, -2) if turned else x).to(F8)
        codes.view(torch.uint8)[page] = x.contiguous().view(torch.uint8)
        scale[page] = now.transpose(1, 2)
    return dict(k=s["k"], v=s["v"], ks=s["ks"], vs=s["vs"])


def _fork(s):
    table, src, refs = s["table"].long(), s["src"].long(), s["refs"].long()
    B, width = table.shape
    N, pages = src.numel(), refs.numel()
    n, i = torch.arange(N, device=DEV), torch.arange(width, device=DEV)
    real, from_ = src >= 0, src.clamp(min=0)
    length = torch.where(real, s["lens"].long()[from_], 0)
    R = ((torch.maximum(s["room"].long(), length) + PAGE - 1) // PAGE).clamp(max=width)[:, None]
    full, held = (length // PAGE)[:, None], ((length + PAGE - 1) // PAGE)[:, None]
    first = torch.where(src[:, None] == torch.arange(B, device=DEV), n[:, None], N).amin(0)  # the first taker of each
    leads = (real & (first[from_] == n))[:, None]
    old = torch.where(real[:, None], table[from_], -1)
    there = old >= 0
    stays = there & (i < R) & (leads | (i < full))
    lost = (i < held) & ~there                                     # tokens without a page stay without one
    fresh = (i < R) & ~stays & ~lost
    out = torch.where(stays, old, -1)
    end = torch.full((), pages, device=DEV)
    count = lambda t: torch.zeros(pages + 1, dtype=torch.int64, device=DEV).index_add_(  # noqa: E731
        0, torch.where(t >= 0, t, end).flatten(), torch.ones(t.numel(), dtype=torch.int64, device=DEV))[:pages]
    mid = refs - count(table) + count(out)
    free = mid == 0
    rank = free.long().cumsum(0) - 1
    order = torch.full((pages + 1,), -1, dtype=torch.int64, device=DEV)
    order.scatter_(0, torch.where(free, rank, end), torch.arange(pages, device=DEV))
    order[pages] = -1
    ask = fresh.flatten().long().cumsum(0).view(N, width) - 1
    given = torch.where(ask < free.sum(), order[ask.clamp(0, pages)], -1)
    out = torch.where(fresh, given, out)
    copies = fresh & (i == full) & (i < held) & (out >= 0)
    to, of = out[copies], old[copies]
    for t in (s["k"].view(torch.uint8), s["v"].view(torch.uint8), s["ks"], s["vs"]):
        t[to] = t[of]
    short = (fresh & (out < 0)).sum(1)
    cut = (fresh & (i < held) & (out < 0)).any(1)
    return dict(table=out.to(torch.int32), refs=(mid + count(torch.where(fresh, out, -1))).to(torch.int32),
                lens=torch.where(cut, full[:, 0] * PAGE, length).to(torch.int32), missing=short.to(torch.int32),
                k=s["k"], v=s["v"], ks=s["ks"], vs=s["vs"])


# ---------------------------------------------------------------- one pass
def run(s):
    c, kind = s["c"], s["c"]["kind"]
    if not own:
        return {"rotate": _rotate, "append": _append, "draft": _append, "tree": _tree, "keep": _keep, "fork": _fork}[kind](s)
    import paper_2510_18830_amd as ms
    if kind == "rotate":
        q, k = ms.rotate(s["q"], s["kk"], s["positions"], s["freq"], axis=s["axis"])
        dq, dk = ms.rotate(s["dq"], s["dk"], s["positions"], s["freq"], axis=s["axis"], inverse=True)
        return dict(q=q, k=k, dq=dq, dk=dk)
    cache = ms.Cache(s["k"], s["v"], s["ks"], s["vs"])
    pool = dict(k=s["k"], v=s["v"], ks=s["ks"], vs=s["vs"])
    if kind == "append":
        q = ms.cache_append(cache, s["table"], s["lens"], s["knew"], s["vnew"], q=s["q"], inv_freq=s["freq"],
                            counts=s["counts"], positions=s["positions"], axis=s["axis"])
        return dict(q=q, **pool)
    if kind == "draft":
        at, seen = ms.tree_mask(s["parents"], s["lens"], counts=s["counts"])
        q = ms.cache_append(cache, s["table"], s["lens"], s["knew"], s["vnew"], q=s["q"], inv_freq=s["freq"],
                            counts=s["counts"], positions=at)
        return dict(q=q, at=at, seen=seen, **pool)
    if kind == "tree":
        out, lse = ms.cache_tree_attn(cache, s["table"], s["lens"], s["q"], s["seen"], positions=s["at"],
                                      counts=s["counts"], window=c["W"], sinks=c["S"])
        return dict(out=out, lse=lse)
    if kind == "keep":
        ms.cache_keep(cache, s["table"], s["lens"], s["path"], s["kept"])
        return pool
    table, lens, refs, missing = ms.cache_fork(cache, s["table"], s["lens"], s["refs"], s["src"], room=s["room"])
    return dict(table=table, lens=lens, refs=refs, missing=missing, **pool)


# ---------------------------------------------------------------- floors
def work(case):
    c, kind = case, case["kind"]
    B, Hkv, d = c["B"], c["Hkv"], c["d"]
    if kind == "rotate":
        rows = float(c["N"]) * B * (c["Hq"] + Hkv)
        return dict(bytes=rows * d * (4 + (4 if c["grads"] == "bf16" else 8)) + 4.0 * c["axes"] * B * c["N"],
                    flops=rows * d * 6.0)
    some = 0.5 if c.get("ragged") else 1.0
    if kind in ("append", "draft"):
        T = c["T"]
        b = B * T * d * (some * 6.0 * Hkv + 4.0 * c["Hq"]) + 4.0 * B * T * c.get("axes", 1)
        if kind == "draft":
            b += B * T * (4.0 + (T + 31) // 32 * 4.0)
        return dict(bytes=b, flops=B * T * d * 3.0 * (some * Hkv + c["Hq"]))
    if kind == "tree":
        T, Hq = c["T"], c["Hq"]
        n = (c["L"] if B == 1 else 0.6 * c["L"])
        sees = min(n, c["W"] + min(c["S"], n)) if c["W"] else n
        nodes = T * some
        return dict(bytes=2.0 * Hkv * d * B * (sees + nodes) + B * T * Hq * (4.0 * d + 4) + 4.0 * B * T * ((T + 31) // 32),
                    flops=4.0 * d * Hq * B * nodes * (sees + math.log(T + 1.0) + 1))
    if kind == "keep":
        moved = 0.2 * c["T"] * B
        return dict(bytes=moved * Hkv * d * 4.0 + 4.0 * B * (c["T"] + 2), flops=moved * Hkv * d * 2.0)
    N, L = c["N"], (c["L"] if B == 1 else 0.6 * c["L"])
    width = (c["L"] + max(c["more"], 2 * PAGE) + PAGE - 1) // PAGE + 1
    pages = B * width + N * (c["more"] // PAGE + 2) + 37
    copies = max(0, N - B * (1 - math.exp(-N / B)))
    return dict(bytes=4.0 * (B + N) * width + 8.0 * pages + copies * 4.0 * PAGE * Hkv * d, flops=0.0)


# ---------------------------------------------------------------- exact results
def _exact_turn(s, positions, x, sign=1.0):
    """x turned by complex factors; positions a list of [B, T] tensors, one for each axis."""
    half = x.shape[-1] // 2
    axis = s["axis"].tolist() if "axis" in s else [0] * half
    ang = torch.stack([positions[a].double() * float(f) for a, f in zip(axis, s["freq"].double().tolist())], -1)
    z = torch.complex(x[..., :half].double(), x[..., half:].double())
    z *= torch.polar(torch.ones_like(ang), sign * ang)[:, None]
    return torch.cat([z.real, z.imag], -1)


def _to_e4m3(x):
    """The nearest e4m3 value (ties to even) of 64-bit values of magnitude up to 448."""
    e = torch.frexp(x)[1].clamp(min=-5) - 1
    step = torch.ldexp(torch.ones_like(x), e - 3)
    return torch.round(x / step) * step


def _scale_for(top):
    need = torch.exp2(torch.ceil(torch.log2(top / 448.0)).clamp(min=-126.0))
    return torch.where(top > 448.0 * need, 2 * need, torch.where(top <= 224.0 * need, need / 2, need)).clamp(min=2.0 ** -126)


def _ancestors(parents):
    """For each node the list of its ancestors, itself first."""
    up = []
    for t, p in enumerate(parents):
        up.append([t] + (up[p] if 0 <= p < t else []))
    return up


def _codes(s):
    """The pool in 64 bits, values [.., token, column] of K and V."""
    return dict(k=s["k"].double(), v=s["v"].double().transpose(-1, -2).contiguous(), ks=s["ks"].double(), vs=s["vs"].double())


def _pool_of(r):
    return dict(k=r["k"], v=r["v"].transpose(-1, -2).contiguous(), ks=r["ks"], vs=r["vs"])


def _exact_append(c, s):
    B, T = c["B"], c["T"]
    r = _codes(s)
    counts, table = s["host_counts"], s["table"].tolist()
    if c["kind"] == "draft":
        at = [[n + (len(up) - 1 if t < m else 0) for t, up in enumerate(_ancestors(p))]
              for n, m, p in zip(s["host_lens"], counts, s["host_parents"])]
        positions = [torch.tensor(at, device=DEV)]
    else:
        positions = list(s["positions"])
    new = dict(k=_exact_turn(s, positions, s["knew"]), v=s["vnew"].double())
    for b, (at, n) in enumerate(zip(s["host_lens"], counts)):
        end, t = at + n, 0
        while at < end:
            page, o = table[b][at // PAGE], at % PAGE
            m = min(PAGE - o, end - at)
            for name in ("k", "v"):
                x, scale = new[name][b, :, t:t + m], r[name + "s"]  # [Hkv, m, d]
                need = _scale_for(x.abs().amax((1, 2)))
                was = scale[page].clone()
                now = torch.maximum(need, was) if o else need
                if o:
                    r[name][page, :, :o] = _to_e4m3(r[name][page, :, :o] * (was / now)[:, None, None])
                r[name][page, :, o:o + m] = _to_e4m3(x / now[:, None, None])
                scale[page] = now
            at, t = at + m, t + m
    more = dict(at=None, seen=None) if c["kind"] == "draft" else {}
    return dict(q=_exact_turn(s, positions, s["q"]), **_pool_of(r), **more)


def _exact_tree(c, s):
    B, T, G = c["B"], c["T"], c["Hq"] // c["Hkv"]
    out = torch.zeros((B, c["Hq"], T, c["d"]), dtype=torch.float64, device=DEV)
    lse = torch.full((B, c["Hq"], T), -math.inf, dtype=torch.float64, device=DEV)
    for b, (n, m) in enumerate(zip(s["host_lens"], s["host_counts"])):
        up = _ancestors(s["host_parents"][b])[:m]
        sees = torch.zeros((m, n + m), dtype=torch.bool)
        j = torch.arange(n)
        for t, line in enumerate(up):
            at = n + len(line) - 1
            sees[t, :n] = (j > at - c["W"]) | (j < c["S"]) if c["W"] else True
            for u in line:
                there = n + len(up[u]) - 1
                sees[t, n + u] = not c["W"] or at - there < c["W"] or there < c["S"]
        sees = sees.to(DEV)
        pos = torch.arange(n + m, device=DEV)
        pos = pos[sees.any(0)]
        sees = sees[:, pos]
        page, slot = s["table"][b].long()[pos // PAGE], pos % PAGE
        for hk in range(c["Hkv"]):
            k = s["k"].view(torch.uint8)[page, hk, slot].view(F8).double() * s["ks"][page, hk, None].double()
            v = s["v"].view(torch.uint8)[page, hk, :, slot].view(F8).double() * s["vs"][page, hk, None].double()
            z = s["q"][b, hk * G:(hk + 1) * G, :m].double() @ k.T.contiguous() / math.sqrt(c["d"])
            z = z.masked_fill(~sees, -math.inf)
            lse[b, hk * G:(hk + 1) * G, :m] = torch.logsumexp(z, -1)
            out[b, hk * G:(hk + 1) * G, :m] = torch.softmax(z, -1) @ v
    return dict(out=out, lse=lse)


def _exact_keep(c, s):
    r, table = _codes(s), s["table"].tolist()
    for b, (n, kept, path) in enumerate(zip(s["host_lens"], s["host_kept"], s["host_path"])):
        for name in ("k", "v"):
            x, scale = r[name], r[name + "s"]
            i = 0
            while i < kept:
                lp = (n + i) // PAGE
                page, m = table[b][lp], min(kept, (lp + 1) * PAGE - n)
                come = [(n + path[y], (n + y) % PAGE) for y in range(i, m)]
                moved = [(x[table[b][f // PAGE], :, f % PAGE] * scale[table[b][f // PAGE], :, None], f // PAGE, o) for f, o in come]
                was, now = scale[page].clone(), scale[page].clone()
                strange = [t for t, of, _ in moved if of != lp]
                if strange:
                    now = torch.maximum(was, _scale_for(torch.stack(strange).abs().amax((0, 2))))
                o = (n + i) % PAGE
                x[page, :, :o] = _to_e4m3(x[page, :, :o] * (was / now)[:, None, None])
                for t, _, o in moved:
                    x[page, :, o] = _to_e4m3(t / now[:, None])
                scale[page] = now
                i = m
    return _pool_of(r)


def _exact_fork(s):
    """Only the copied pages have values that are not whole numbers."""
    table, src, room, lens = (s[n].tolist() for n in ("table", "src", "room", "lens"))
    refs, width, first, rows, asked = s["refs"].tolist(), len(table[0]), {}, [], []
    for row in table:
        for p in row:
            if p >= 0:
                refs[p] -= 1
    for n, b in enumerate(src):
        length = lens[b] if b >= 0 else 0
        R = min(width, (max(room[n], length) + PAGE - 1) // PAGE)
        leads = b >= 0 and first.setdefault(b, n) == n
        row = [-1] * width
        for i in range(R):
            p = table[b][i] if b >= 0 else -1
            if p >= 0 and (leads or i < length // PAGE):
                row[i] = p
                refs[p] += 1
            elif p >= 0 or PAGE * i >= length:
                asked.append((n, i, p if PAGE * i < length else -1))
        rows.append(row)
    free = [p for p, x in enumerate(refs) if x == 0]
    r = dict(k=s["k"].double(), v=s["v"].double(), ks=s["ks"].double(), vs=s["vs"].double())
    for (n, i, p), to in zip(asked, free):
        if p >= 0:
            for x in r.values():
                x[to] = x[p]
    return dict(table=None, refs=None, lens=None, missing=None, **r)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rotate":
        positions = list(s["positions"])
        return dict(q=_exact_turn(s, positions, s["q"]), k=_exact_turn(s, positions, s["kk"]),
                    dq=_exact_turn(s, positions, s["dq"], -1.0), dk=_exact_turn(s, positions, s["dk"], -1.0))
    if kind in ("append", "draft"):
        return _exact_append(case, s)
    if kind == "tree":
        return _exact_tree(case, s)
    return _exact_keep(case, s) if kind == "keep" else _exact_fork(s)
