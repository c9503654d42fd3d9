"""What a serving loop does with more than one new token per sequence: prompts filled chunk by
chunk into a Hard-KV Cascade Cache, and drafted tokens tested and taken back.

A case is one of four kinds of call, through the package's pipeline classes:

  append   ChunkDecoder.append: slots for the new tokens of every sequence (tables, masks, page
           stack, slot map), then their K and V rows into the pool through that map
  attend   ChunkDecoder.attend: causal attention of the new tokens over the paged cache
  verify   Verifier.verify: drafted tokens against the target's probabilities
  trim     ChunkDecoder.trim: the newest slots of every head go back to the pool

Calls that change the cache first put its metadata (tables, masks, counts, allocator: one
buffer) back, so that every pass does the same work.  With `own` false the same results come from
elementary torch operations over padded batches.
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 16
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
ONE = 1 << 40                                   # a probability of 1 as a whole number


def _case(name, kind, NS, Hq, Hkv, D, dtype, N, n_new, **more):
    """NS sequences of the batch, L layers; N: the longest context in tokens before the new ones;
    lo: the shortest as a share of it (spread evenly, per head with `ragged`, as a head-adaptive
    budget leaves them); holes: share of masked slots in the context (a sparse tier); n_new: the
    longest chunk; new: "same" for all, "spread" from 1 to n_new, "mixed" one of n_new and one
    token for every other sequence; pad: rows behind the last sequence; table: page-table width in
    tokens; tau: queries sharpened or flattened per head by up to this factor; V: vocabulary;
    drafts: whether the drafts come with their own distributions."""
    c = dict(name=name, kind=kind, NS=NS, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, N=N, n_new=n_new, L=1, lo=1.0,
             ragged=False, holes=0.0, new="same", pad=0, table=0, tau=1.0, V=0, drafts=True)
    c.update(more)
    return c


def listed():
    return [
        # one user's drafts over a compressed context: the launch-latency end
        _case("attend_drafts_one_sequence", "attend", 1, 32, 8, 128, "bf16", 1999, 5, lo=0.6, ragged=True,
              holes=0.2, table=12288),
        # a batch of drafts in a steady decode loop: compressed rows of every length
        _case("attend_drafts_batch", "attend", 64, 32, 8, 128, "bf16", 5600, 8, new="spread", lo=0.14,
              ragged=True, holes=0.1, table=12288),
        # one prompt arriving while the rest of the batch decodes single tokens
        _case("attend_mixed_batch", "attend", 32, 32, 8, 128, "bf16", 4001, 500, new="mixed", lo=0.3,
              ragged=True, pad=37, table=12288),
        # the last chunk of one long prompt, 7 query heads per KV head
        _case("attend_long_chunk_g7", "attend", 1, 28, 4, 128, "bf16", 28671, 2048, tau=10.0, table=32768),
        # a batch of whole prompts: the largest plain amount of arithmetic
        _case("attend_prompts", "attend", 8, 32, 8, 128, "bf16", 0, 4096, tau=10.0),
        # an fp32 cache of two heads
        _case("attend_small_f32", "attend", 2, 8, 2, 64, "f32", 301, 203, new="spread"),
        # drafts of a whole batch, 32 layers at once
        _case("append_drafts_all_layers", "append", 64, 32, 8, 128, "bf16", 300, 5, L=32, lo=0.3, ragged=True,
              table=1024),
        # a batch of whole prompts of one layer, cut out of a longer token buffer
        _case("append_prompts", "append", 8, 32, 8, 128, "bf16", 0, 4096, new="spread", pad=100),
        # one user's four drafts
        _case("verify_one_sequence", "verify", 1, 1, 1, 64, "f32", 0, 5, V=32000),
        # a batch of drafts with a large vocabulary
        _case("verify_batch", "verify", 64, 1, 1, 64, "f32", 0, 8, new="spread", V=131072),
        # the rejected drafts of one user's layer
        _case("trim_one_layer", "trim", 1, 32, 8, 128, "bf16", 1999, 5, lo=0.6, ragged=True, holes=0.2, table=12288),
        # the rejected drafts of a whole batch, 32 layers at once
        _case("trim_all_layers", "trim", 64, 32, 8, 128, "bf16", 300, 8, L=32, lo=0.3, ragged=True, new="spread",
              table=1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend"] * 6 + ["append"] * 2 + ["verify"] * 2 + ["trim"])
    if kind == "verify":
        V = _log(rng, 1000, 131072)
        return _case("", kind, _log(rng, 1, 64), 1, 1, 64, "f32" if rng.random() < 0.6 else "bf16", 0, rng.randint(2, 8),
                     new=rng.choice(["same", "spread"]), V=V, drafts=rng.random() < 0.7, pad=rng.choice([0, 3]))
    dtype = "bf16" if rng.random() < 0.8 else "f32"
    D = 128 if rng.random() < 0.75 else 64
    G, Hkv = rng.choice([1, 2, 3, 4, 4, 6, 7, 8]), rng.choice([1, 2, 4, 8])
    new = rng.choice(["same", "spread", "mixed"])
    more = dict(new=new, lo=round(rng.uniform(0.1, 1.0), 2), ragged=rng.random() < 0.5, pad=rng.choice([0, 0, 9]),
                holes=rng.choice([0.0, 0.0, 0.3]), table=rng.choice([0, 0, 12288]), tau=rng.choice([1.0, 10.0]))
    if kind == "attend":
        # rows x columns of the padded scores: at most those of the largest listed case
        n_new = _log(rng, 1, 4096) if dtype == "bf16" else _log(rng, 1, 700)
        N = _log(rng, 1, 32768) if rng.random() < 0.85 else 0
        most = (1 << 31) // (n_new * G * (N + n_new))
        most = min(most, (1 << 22) // (N + n_new))
        most = most >> 2 if dtype == "f32" else most
        Hkv = min(Hkv, max(1, most))
        NS = max(1, min(_log(rng, 1, 64), most // Hkv))
    else:
        n_new, N = _log(rng, 1, 4096) if kind == "append" else rng.randint(1, 40), _log(rng, 1, 2000)
        more.update(L=rng.choice([1, 1, 2, 8]))
        NS = max(1, min(_log(rng, 1, 64), (1 << 19) // ((n_new + N) * Hkv * more["L"])))
    more["table"] = more["table"] if N + n_new <= more["table"] else 0
    return _case("", kind, NS, Hkv * G, Hkv, D, dtype, N, n_new, **more)


# ---------------------------------------------------------------------------------- inputs
def _spread(i):
    return (i * 0.6180339887498949) % 1.0


def _news(case):
    """Chunk lengths, one per sequence."""
    B, n = case["NS"], case["n_new"]
    if case["new"] == "spread":
        return [n - int((n - 1) * _spread(i) + 0.5) for i in range(B)]
    if case["new"] == "mixed":
        return [1] * (B // 2) + [n] + [1] * (B - B // 2 - 1)
    return [n] * B


def _context(case):
    """Context lengths, one per head (layer, sequence, KV head), in golden-ratio order."""
    NS, Hkv, N, lo = case["NS"] * case["L"], case["Hkv"], case["N"], case["lo"]
    n = NS * Hkv if case["ragged"] else NS
    at = [N - int((1.0 - lo) * N * _spread(i)) for i in range(n)]
    return at if case["ragged"] else [x for x in at for _ in range(Hkv)]


def _randn(shape, gen, dtype):
    """N(0, 1) draws, made in pieces so that the fp32 draw of a large pool is never whole."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 28):
        piece = flat[i:i + (1 << 28)]
        piece.copy_(torch.randn(piece.shape, generator=gen, device="cuda"))
    return out


def _cache(case, gen, news, holding):
    """A paged cache whose pages lie scattered over a pool, with its allocator: the contexts, and
    with `holding` the new tokens behind them too."""
    dev, L, Hkv = "cuda", case["L"], case["Hkv"]
    ctx = torch.tensor(_context(case), dtype=torch.int64, device=dev)
    H = ctx.numel()
    new = torch.tensor(news, dtype=torch.int64, device=dev).repeat(L).repeat_interleave(Hkv)
    lens = ctx + new if holding else ctx
    n_pages = (lens + PAGE - 1) // PAGE
    longest = int(((ctx + new + PAGE - 1) // PAGE).max())
    width = max(longest, -(-case["table"] // PAGE))
    width += width % 2
    used = int(n_pages.sum())
    pool = used + int(((ctx + new + PAGE - 1) // PAGE).sum()) - used + used // 8 + H + 16
    perm = torch.randperm(pool, generator=gen, device=dev).to(torch.int32)
    slot = torch.arange(width, device=dev)[None, :]
    live = slot < n_pages[:, None]
    table = torch.full((H, width), -1, dtype=torch.int32, device=dev)
    table[live] = perm[:used]
    at = torch.arange(width * PAGE, device=dev)[None, :]
    bits = at < lens[:, None]
    if case["holes"]:
        drop = torch.rand((H, width * PAGE), generator=gen, device=dev) < case["holes"]
        newest = at >= (n_pages[:, None] - 1) * PAGE
        bits &= ~drop | (at >= ctx[:, None]) | newest
    mask = (bits.view(H, width, PAGE).to(torch.int32) << torch.arange(PAGE, device=dev, dtype=torch.int32)).sum(-1)
    free = torch.zeros(pool, dtype=torch.int32, device=dev)
    free[:pool - used] = torch.sort(perm[used:]).values
    top = torch.tensor([pool - used], dtype=torch.int32, device=dev)
    parts = [table, mask.to(torch.int16), n_pages.to(torch.int32), free, top]
    off, total = [], 0
    for t in parts:
        off.append(total)
        total += -(-t.numel() * t.element_size() // 256) * 256
    meta = torch.zeros(total, dtype=torch.uint8, device=dev)
    names = ("page_table", "page_mask", "n_pages", "free_ids", "free_top")
    st = {}
    for name, t, o in zip(names, parts, off):
        st[name] = meta[o:o + t.numel() * t.element_size()].view(t.dtype).view(t.shape)
        st[name].copy_(t)
    dt = DTYPE[case["dtype"]]
    st["k_pool"] = _randn((pool, PAGE, case["D"]), gen, dt)
    st["v_pool"] = _randn((pool, PAGE, case["D"]), gen, dt)
    return dict(st, meta=meta, meta0=meta.clone(), longest=longest)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 29)
    kind, B, L, Hq, Hkv, D = (case[k] for k in ("kind", "NS", "L", "Hq", "Hkv", "D"))
    news = _news(case)
    T = sum(news) + case["pad"]
    at = [0]
    for n in news:
        at.append(at[-1] + n)
    start = torch.tensor(at, dtype=torch.int32, device="cuda")
    st = dict(kind=kind, start=start, T=T, most=case["n_new"], Hkv=Hkv, G=Hq // Hkv, B=B, L=L)
    dt = DTYPE[case["dtype"]]
    if kind == "verify":
        V = case["V"]
        st["tokens"] = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
        z = torch.randn((T, V), generator=gen, device="cuda") * 3.0
        st["p"] = torch.softmax(z, 1).to(dt)
        st["q"] = None
        if case["drafts"]:
            # row t: the distribution that token t was drafted from, near the target's of row t - 1
            z = z.roll(1, 0) + torch.randn((T, V), generator=gen, device="cuda") * 0.7
            q = torch.softmax(z, 1)
            st["q"] = q.to(dt)
            u = torch.rand((T, 1), generator=gen, device="cuda")
            st["tokens"].copy_((torch.cumsum(q, 1) < u * 0.99).sum(1).clamp_(max=V - 1))
        else:
            # drafts of a table: often the target's own first choice
            st["tokens"][1:] = torch.where(torch.rand((T - 1,), generator=gen, device="cuda") < 0.7,
                                           st["p"][:-1].argmax(1).to(torch.int32), st["tokens"][1:])
        st["u"] = torch.rand((T,), generator=gen, device="cuda")
        st["n_accept"], st["next_token"], st["n_drop"] = (torch.empty(B, dtype=torch.int32, device="cuda") for _ in range(3))
        if own:
            from paper_2606_28831_amd import Chunks
            from paper_2606_28831_amd.pipeline import Verifier
            st["chunks"] = Chunks(start, T, case["n_new"])
            st["verifier"] = Verifier(B, V, "cuda")
        return st
    st.update(_cache(case, gen, news, kind != "append"))
    if kind == "attend":
        q = torch.randn((T, Hq, D), generator=gen, device="cuda")
        if case["tau"] > 1.0:
            u = torch.rand((Hkv,), generator=gen, device="cuda") * 2.0 - 1.0
            q /= torch.pow(torch.tensor(case["tau"], device="cuda"), u).repeat_interleave(Hq // Hkv)[None, :, None]
        st["q"] = q.to(dt)
        st["o"] = torch.zeros((T, Hq, D), dtype=dt, device="cuda")
        st["lse"] = torch.zeros((T, Hq), dtype=torch.float32, device="cuda")
    elif kind == "append":
        # K and V as they leave one projection: the rows of a token side by side
        kvs = torch.randn((L, T, 2 * Hkv, D), generator=gen, device="cuda").to(dt)
        st["k_new"], st["v_new"] = kvs[:, :, :Hkv], kvs[:, :, Hkv:]
        st["slot_map"] = torch.empty((L, T, Hkv), dtype=torch.int64, device="cuda")
    else:
        r = torch.rand((B,), generator=gen, device="cuda")
        st["n_drop"] = torch.floor(r * (start[1:] - start[:-1] + 1)).to(torch.int32)
    if own:
        from paper_2606_28831_amd import Allocator, Chunks, PagedKV
        from paper_2606_28831_amd.pipeline import ChunkDecoder
        kv = PagedKV(st["k_pool"], st["v_pool"], st["page_table"], st["page_mask"], st["n_pages"])
        st["chunks"] = Chunks(start, T, case["n_new"])
        st["dec"] = ChunkDecoder(B, Hq, Hkv, D, kv, Allocator(st["free_ids"], st["free_top"]), T, case["n_new"], layers=L)
    return st


# ------------------------------------------------------------------------ the plain forms
def _bits(mask):
    """[H, 16 * width] truth values of page masks."""
    m = mask.to(torch.int32)[:, :, None] >> torch.arange(PAGE, device=mask.device, dtype=torch.int32)
    return (m & 1).bool().reshape(mask.shape[0], -1)


def _ends(st):
    """One past the highest valid slot of every head's newest page (its first slot if it has none)."""
    n = st["n_pages"].long()
    newest = st["page_mask"].gather(1, (n - 1).clamp(min=0)[:, None])
    top = (_bits(newest) * torch.arange(1, PAGE + 1, device=n.device)).amax(1)
    return torch.where(n > 0, (n - 1) * PAGE + top, 0)


def _rows_of(st):
    """(sequence, position in its chunk, whether it belongs to one) of every row."""
    t = torch.arange(st["T"], device="cuda")
    s = (torch.searchsorted(st["start"].long(), t, right=True) - 1).clamp(max=st["B"] - 1)
    return s, t - st["start"].long()[s], t < st["start"][-1]


def _plain_attend(st):
    B, Hkv, G, P, n = st["B"], st["Hkv"], st["G"], st["longest"], st["most"]
    T, Hq, D = st["q"].shape
    H, S = B * Hkv, P * PAGE
    pages = st["page_table"][:, :P].long().clamp(min=0)
    valid = _bits(st["page_mask"][:, :P])
    k = st["k_pool"][pages].float().view(H, S, D)
    v = st["v_pool"][pages].float().view(H, S, D).masked_fill(~valid[:, :, None], 0.0)
    first, lens = st["start"][:-1].long(), (st["start"][1:] - st["start"][:-1]).long()
    i = torch.arange(n, device="cuda")
    rows = (first[:, None] + i).clamp(max=T - 1)
    q = st["q"][rows].view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(H, n * G, D).float()
    z = torch.matmul(q, k.transpose(1, 2)).mul_(1.0 / math.sqrt(D)).view(H, n, G, S)
    # the new tokens are the row's newest slots: token i of len sees the slots before end - len + i + 1
    upto = _ends(st)[:, None] - lens.repeat_interleave(Hkv)[:, None] + i + 1
    seen = valid[:, None, :] & (torch.arange(S, device="cuda") < upto[:, :, None])
    z.masked_fill_(~seen[:, :, None, :], -math.inf)
    m = z.amax(3, keepdim=True)
    m.masked_fill_(torch.isinf(m), 0.0)
    e = z.sub_(m).exp_()
    l = e.sum(3, keepdim=True)
    o = torch.matmul(e.view(H, n * G, S), v).view(H, n, G, D) / torch.where(l > 0, l, 1.0)
    lse = (m + torch.log(l)).view(B, Hkv, n, G).permute(0, 2, 1, 3).reshape(B, n, Hq)
    o = o.view(B, Hkv, n, G, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D)
    s, i, live = _rows_of(st)
    i = i.clamp(max=n - 1)
    st["o"].copy_(torch.where(live[:, None, None], o[s, i].to(st["o"].dtype), st["o"]))
    st["lse"].copy_(torch.where(live[:, None], lse[s, i], st["lse"]))


def _plain_append(st):
    L, Hkv, B = st["L"], st["Hkv"], st["B"]
    H, width = st["page_table"].shape
    end, n, top = _ends(st), st["n_pages"].long(), st["free_top"].long()
    lens = (st["start"][1:] - st["start"][:-1]).long().repeat(L).repeat_interleave(Hkv)
    need = ((end + lens + PAGE - 1) // PAGE - n).clamp(min=0)
    before = torch.cumsum(need, 0) - need
    ok = (need.sum() <= top) & ((n + need) <= width).all()
    page = torch.arange(width, device="cuda")
    fresh = (page >= n[:, None]) & (page < (n + need)[:, None]) & ok
    pops = (top - need.sum() + before)[:, None] + page - n[:, None]
    st["page_table"].copy_(torch.where(fresh, st["free_ids"][pops.clamp(0, st["free_ids"].numel() - 1)], st["page_table"]))
    lo, hi = (end[:, None] - page * PAGE).clamp(0, PAGE), ((end + lens)[:, None] - page * PAGE).clamp(0, PAGE)
    bits = torch.where(ok, (1 << hi) - (1 << lo), 0)
    st["page_mask"].copy_((st["page_mask"].long() | bits).to(torch.int16))
    st["n_pages"].copy_(torch.where(ok, n + need, n))
    st["free_top"].copy_(torch.where(ok, top - need.sum(), top))
    s, i, live = _rows_of(st)
    head = ((torch.arange(L, device="cuda")[:, None] * B + s)[:, :, None] * Hkv + torch.arange(Hkv, device="cuda"))
    slot = end[head] + i[None, :, None]
    where = st["page_table"].view(-1)[(head * width + slot // PAGE).clamp(max=H * width - 1)].long() * PAGE + slot % PAGE
    st["slot_map"].copy_(torch.where((live & ok)[None, :, None], where, -1))
    # rows without a slot write the first row once more
    at = torch.where(live[None, :, None], where, where[:, :1])
    for_rows = torch.where(live, torch.arange(st["T"], device="cuda"), 0)
    D = st["k_pool"].shape[2]
    st["k_pool"].view(-1, D)[at] = st["k_new"][:, for_rows]
    st["v_pool"].view(-1, D)[at] = st["v_new"][:, for_rows]


def _whole(x):
    return torch.floor(x.double().nan_to_num(nan=0.0).clamp(0.0, 1.0) * ONE).long()


def _plain_verify(st):
    B, T, n = st["B"], st["T"], st["most"]
    first, lens = st["start"][:-1].long(), (st["start"][1:] - st["start"][:-1]).long()
    u = torch.floor(st["u"].double() * (1 << 24)).long().clamp(0, (1 << 24) - 1)
    tok = st["tokens"].long()
    row = (first[:, None] + 1 + torch.arange(n - 1, device="cuda")).clamp(max=T - 1)      # [B, n - 1] drafts
    x = tok[row]
    target = _whole(st["p"][row - 1, x])
    draft = _whole(st["q"][row, x]) if st["q"] is not None else torch.full_like(target, ONE)
    # u * draft < 2^24 * target, in two parts
    high = u[row] * (draft >> 20) + ((u[row] * (draft & 0xfffff)) >> 20)
    good = (high < (target << 4)) & (torch.arange(1, n, device="cuda") < lens[:, None])
    took = torch.cumprod(good.long(), 1).sum(1)
    at = (first + took).clamp(max=T - 1)
    p = _whole(st["p"][at])
    nxt = (at + 1).clamp(max=T - 1)
    if st["q"] is not None:
        less = _whole(st["q"][nxt])
    else:
        less = torch.where(torch.arange(p.shape[1], device="cuda") == tok[nxt][:, None], ONE, 0)
    w = torch.where((took < lens - 1)[:, None], (p - less).clamp(min=0), p)
    w = torch.where(w.sum(1, keepdim=True) > 0, w, p)
    total, u0 = w.sum(1), u[first.clamp(max=T - 1)]
    goal = u0 * (total >> 24) + ((u0 * (total & 0xffffff)) >> 24)
    token = (torch.cumsum(w, 1) <= goal[:, None]).sum(1)
    st["n_accept"].copy_(torch.where(lens > 0, took, 0))
    st["next_token"].copy_(torch.where((lens > 0) & (total > 0), token, -1))
    st["n_drop"].copy_((lens - 1 - took).clamp(min=0))


def _plain_trim(st):
    H, width = st["page_table"].shape
    n, end, top = st["n_pages"].long(), _ends(st), st["free_top"].long()
    drop = st["n_drop"].long().clamp(min=0).repeat(st["L"]).repeat_interleave(st["Hkv"])
    end = (end - drop).clamp(min=0)
    keep = torch.where(drop > 0, (end + PAGE - 1) // PAGE, n)
    gone = n - keep
    before = torch.cumsum(gone, 0) - gone
    page = torch.arange(width, device="cuda")
    freed = (page >= keep[:, None]) & (page < n[:, None])
    free = st["free_ids"]
    to = torch.where(freed, (top + before)[:, None] + page - keep[:, None], free.numel())
    room = torch.cat([free, free[:1]])            # one more place, for the pages that stay
    room[to] = st["page_table"]
    free.copy_(room[:-1])
    left = (end[:, None] - page * PAGE).clamp(0, PAGE)
    bits = torch.where((drop > 0)[:, None], (1 << left) - 1, (1 << PAGE) - 1)
    st["page_mask"].copy_((st["page_mask"].long() & bits & 0xffff).to(torch.int16))
    st["page_table"].copy_(torch.where(freed, -1, st["page_table"]))
    st["n_pages"].copy_(keep)
    st["free_top"].copy_(top + gone.sum())


def run(st):
    kind = st["kind"]
    if kind in ("append", "trim"):
        st["meta"].copy_(st["meta0"])
    if own:
        if kind == "verify":
            st["verifier"].verify(st["chunks"], st["tokens"], st["p"], st["u"], st["n_accept"], st["next_token"],
                                  st["n_drop"], q=st["q"])
        elif kind == "attend":
            st["dec"].attend(st["chunks"], st["q"], st["o"], st["lse"])
        elif kind == "append":
            st["dec"].append(st["chunks"], st["k_new"], st["v_new"], st["slot_map"])
        else:
            st["dec"].trim(st["n_drop"])
    else:
        {"attend": _plain_attend, "append": _plain_append, "verify": _plain_verify, "trim": _plain_trim}[kind](st)
    if kind == "attend":
        return dict(o=st["o"], lse=st["lse"])
    if kind == "verify":
        return dict(n_accept=st["n_accept"], next_token=st["next_token"], n_drop=st["n_drop"])
    out = {k: st[k] for k in ("page_table", "page_mask", "n_pages", "free_ids", "free_top")}
    if kind == "append":
        out.update(slot_map=st["slot_map"], k_pool=st["k_pool"], v_pool=st["v_pool"])
    return out


# ------------------------------------------------------------------------- what it must cost
def work(case):
    kind, B, L, Hq, Hkv, D = (case[k] for k in ("kind", "NS", "L", "Hq", "Hkv", "D"))
    e = 4 if case["dtype"] == "f32" else 2
    news = _news(case)
    T = sum(news)
    if kind == "verify":
        rows = 2 if case["drafts"] else 1
        return dict(bytes=rows * B * case["V"] * e + T * (8 + rows * e) + 12 * B, flops=0)
    ctx = _context(case)
    heads = [(c, news[(h // Hkv) % B]) for h, c in enumerate(ctx)]
    pages = lambda x: -(-x // PAGE)  # noqa: E731
    if kind == "trim":
        # count and newest mask of every head read, what the mean drop changes written
        gone = sum(n / 2 for _, n in heads)
        return dict(bytes=len(heads) * (4 + 2 + 2 + 4) + 4 * B + gone / PAGE * (4 + 4 + 4 + 2), flops=0)
    if kind == "append":
        fresh = sum(pages(c + n) - pages(c) for c, n in heads)
        return dict(bytes=T * L * Hkv * (4 * D * e + 8) + len(heads) * 12 + fresh * (4 + 4 + 2), flops=0)
    keep = 1.0 - case["holes"]
    slots = sum(c * keep + n for c, n in heads)
    pairs = sum(n * c * keep + n * (n + 1) / 2 for c, n in heads)
    tables = 6 * sum(pages(c + n) for c, n in heads)
    return dict(bytes=2 * slots * D * e + T * Hq * (2 * D * e + 4) + tables, flops=4 * D * pairs * (Hq // Hkv))


# ------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    kind, B, Hq, Hkv, D = (case[k] for k in ("kind", "NS", "Hq", "Hkv", "D"))
    if kind != "attend":
        return None                               # whole numbers, and rows copied as they are
    st = prepare(case, seed)
    d, G = torch.float64, Hq // Hkv
    o = torch.zeros(st["o"].shape, dtype=d, device="cuda")
    lse = torch.zeros(st["lse"].shape, dtype=d, device="cuda")
    start, n_pages = st["start"].tolist(), st["n_pages"].tolist()
    masks, table = st["page_mask"].to(torch.int32).tolist(), st["page_table"]
    for h in range(B * Hkv):
        s, g = h // Hkv, (h % Hkv) * G
        a, b = start[s], start[s + 1]
        held = [16 * j + t for j in range(n_pages[h]) for t in range(16) if masks[h][j] >> t & 1]
        end = held[-1] + 1 if held else 0
        at = torch.tensor(held, device="cuda")
        where = table[h][at // 16].long() * 16 + at % 16
        k, v = st["k_pool"].view(-1, D)[where].to(d), st["v_pool"].view(-1, D)[where].to(d)
        for x in range(a, b, 512):                # a few hundred tokens of the head at a time
            y = min(x + 512, b)
            z = st["q"][x:y, g:g + G].to(d) @ k.t() / math.sqrt(D)
            last = end - (b - a) + torch.arange(x - a, y - a, device="cuda")
            z.masked_fill_((at[None, :] > last[:, None])[:, None, :], -math.inf)
            lse[x:y, g:g + G] = torch.logsumexp(z, 2)
            o[x:y, g:g + G] = torch.softmax(z, 2) @ v
    return dict(o=o, lse=lse)
