"""What a serving loop does with a Cascade Cache held in 8 bits: K and V rows quantised as they are
written, read back, attended to as they lie, and rewritten under a selection.

A row of D codes (int8, or the 8-bit float e4m3) has one fp32 scale.  A case is one of five kinds:

  write    hk_write_kv8: new rows into the pool through a slot map, each with its scale; the pass
           reads them back through the same map (hk_read_kv8), so that its result is their values
  read     hk_read_kv8: cached rows back to bf16 or fp32, as scoring takes them
  decode   hk_decode_attn8: attention of one new token per sequence over the 8-bit pages
  attend   hk_chunk_attn8: causal attention of several new tokens per sequence over them
  compact  hk_compact8: the rewrite of codes and scales under a selection

A rewrite first puts the cache's metadata (tables, masks, counts, allocator: one buffer) back, so that
every pass does the same work.  With `own` false the same results come from elementary torch operations
over padded batches.
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 16
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}
MOST = {"i8": 127.0, "e4m3": 448.0}             # the largest code
LEAST = 2.0 ** -100                             # a row whose largest value is below it counts as one of it


def _case(name, kind, NS, Hq, Hkv, D, fmt, dtype, N, n_new, **more):
    """NS sequences of the batch, L layers; fmt: of the codes; dtype: of rows, queries and results; N:
    the longest context in tokens before the new ones; lo: the shortest as a share of it (spread
    evenly, per head with `ragged`, as a head-adaptive budget leaves them); holes: share of masked
    slots in the context (a sparse tier); n_new: the longest chunk; new: "same" for all, "spread" from
    1 to n_new, "mixed" one of n_new and one token for every other sequence; pad: rows behind the last
    sequence; table: page-table width in tokens; tau: queries sharpened or flattened per head by up to
    this factor; keep: share of the slots that a rewrite keeps; dense, sparse: its tiers in tokens."""
    c = dict(name=name, kind=kind, NS=NS, Hq=Hq, Hkv=Hkv, D=D, fmt=fmt, dtype=dtype, N=N, n_new=n_new, L=1, lo=1.0,
             ragged=False, holes=0.0, new="same", pad=0, table=0, tau=1.0, keep=0.0, dense=0, sparse=0)
    c.update(more)
    return c


def listed():
    return [
        # one user's token in every layer: the launch-latency end
        _case("write_token_all_layers", "write", 1, 32, 8, 128, "i8", "bf16", 0, 1, L=32),
        # a batch of whole prompts of one layer, cut out of a longer token buffer
        _case("write_prompts", "write", 8, 32, 8, 128, "e4m3", "bf16", 0, 4096, new="spread", pad=100),
        # a short fp32 cache of two sequences
        _case("read_short_f32", "read", 2, 8, 2, 64, "i8", "f32", 301, 0, lo=0.5, holes=0.2),
        # one layer of a batch back to bf16, to be scored
        _case("read_layer", "read", 32, 28, 4, 128, "e4m3", "bf16", 8192, 0, lo=0.5, ragged=True),
        # one user's next token
        _case("decode_one_sequence", "decode", 1, 32, 8, 128, "i8", "bf16", 4097, 1, table=12288),
        # a batch over compressed rows of every length
        _case("decode_batch", "decode", 64, 32, 8, 128, "e4m3", "bf16", 5600, 1, lo=0.14, ragged=True, holes=0.1,
              table=12288),
        # one very long fp32 conversation, a query head per KV head
        _case("decode_long_f32", "decode", 1, 8, 8, 64, "i8", "f32", 131071, 1),
        # a batch of drafts over compressed rows
        _case("attend_drafts_batch", "attend", 64, 32, 8, 128, "i8", "bf16", 5600, 8, new="spread", lo=0.14, ragged=True,
              holes=0.1, table=12288),
        # an fp32 model of two heads, prompts of any length
        _case("attend_small_f32", "attend", 2, 8, 2, 64, "e4m3", "f32", 301, 203, new="spread"),
        # a batch of whole prompts: the largest amount of arithmetic
        _case("attend_prompts", "attend", 8, 32, 8, 128, "i8", "bf16", 0, 4096, tau=10.0),
        # one user's layer
        _case("compact_one_layer", "compact", 1, 32, 8, 128, "e4m3", "bf16", 1999, 0, lo=0.6, ragged=True, holes=0.2,
              keep=0.5, dense=128, sparse=256),
        # a batch at the end of long contexts
        _case("compact_batch", "compact", 32, 28, 4, 128, "i8", "bf16", 32768, 0, keep=0.6),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "write", "read", "decode", "decode", "decode", "attend", "attend", "attend", "compact"])
    fmt = rng.choice(["i8", "e4m3"])
    dtype = "bf16" if rng.random() < 0.75 else "f32"
    D = 128 if rng.random() < 0.7 else 64
    G, Hkv = rng.choice([1, 2, 3, 4, 4, 5, 6, 7, 8, 8, 12, 16]), rng.choice([1, 2, 3, 4, 8])
    new = rng.choice(["same", "spread", "mixed"])
    more = dict(lo=round(rng.uniform(0.1, 1.0), 2), ragged=rng.random() < 0.5, pad=rng.choice([0, 0, 9]),
                holes=rng.choice([0.0, 0.0, 0.3]), tau=rng.choice([1.0, 10.0]))
    if kind == "write":
        more.update(L=rng.choice([1, 1, 4, 32]), new=new)
        n_new = _log(rng, 1, 4096)
        most = (1 << 18) // (Hkv * more["L"] * n_new)
        return _case("", kind, max(1, min(_log(rng, 1, 64), most)), Hkv * G, Hkv, D, fmt, dtype, 0, n_new, **more)
    if kind in ("read", "compact"):
        N = _log(rng, 1, 32768)
        NS = max(1, min(_log(rng, 1, 64), (1 << 20) // (N * Hkv)))
        if kind == "compact":
            more.update(keep=round(rng.uniform(0.02, 0.98), 2), dense=rng.choice([0, 0, 100, 512]),
                        sparse=rng.choice([0, 0, 100, 2048]))
        return _case("", kind, NS, Hkv * G, Hkv, D, fmt, dtype, N, 0, **more)
    if kind == "decode":
        n_new, N = 1, _log(rng, 1, 131072)
        NS = max(1, min(_log(rng, 1, 64), (1 << 20) // (N * Hkv)))
        more["table"] = rng.choice([0, 0, 12288])
    else:
        # rows x columns of the padded scores: at most those of the largest listed case
        n_new = _log(rng, 1, 4096) if dtype == "bf16" else _log(rng, 1, 700)
        N = _log(rng, 1, 32768) if rng.random() < 0.85 else 0
        most = min((1 << 31) // (n_new * G * (N + n_new)), (1 << 22) // (N + n_new))
        most = most >> 2 if dtype == "f32" else most
        Hkv = min(Hkv, max(1, most))
        NS = max(1, min(_log(rng, 1, 64), most // Hkv))
        more.update(new=new, table=rng.choice([0, 0, 12288]))
    more["table"] = more["table"] if N + n_new <= more["table"] else 0
    return _case("", kind, NS, Hkv * G, Hkv, D, fmt, dtype, N, n_new, **more)


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
    """Context lengths, one per head (sequence, KV head), in golden-ratio order."""
    NS, Hkv, N, lo = case["NS"], case["Hkv"], case["N"], case["lo"]
    n = NS * Hkv if case["ragged"] else NS
    at = [N - int((1.0 - lo) * N * _spread(i)) for i in range(n)]
    return at if case["ragged"] else [x for x in at for _ in range(Hkv)]


def _round_up(x):
    return -(-x // PAGE)


def _quantise(x, fmt):
    """Codes and scales of rows, and the rows' values: elementary fp32 operations, each rounded."""
    x = x.float()
    most = MOST[fmt]
    a = x.abs().amax(-1, keepdim=True).clamp(min=LEAST)
    fine = torch.isfinite(a)
    top = torch.full_like(a, most)                # (a plain number in its place would be divided by its inverse)
    scale = torch.where(fine, a / top, math.nan)
    y = torch.where(fine, x * (top / a), 0.0)
    codes = torch.round(y).to(torch.int8) if fmt == "i8" else y.to(torch.float8_e4m3fn)
    return codes, scale.squeeze(-1)


def _rows(shape, gen, fmt):
    """Codes and scales of cached rows: some channels larger than the others, rows of differing size."""
    n, D = math.prod(shape[:-1]), shape[-1]
    codes = torch.empty((n, D), dtype=CODE[fmt], device="cuda")
    scales = torch.empty(n, dtype=torch.float32, device="cuda")
    channel = 1.0 + 3.0 * (torch.rand(D, generator=gen, device="cuda") < 0.05)
    for i in range(0, n, 1 << 20):
        m = min(n - i, 1 << 20)
        x = torch.randn((m, D), generator=gen, device="cuda") * channel
        x *= 0.5 + torch.rand((m, 1), generator=gen, device="cuda")
        codes[i:i + m], scales[i:i + m] = _quantise(x, fmt)
    return codes.view(shape), scales.view(shape[:-1])


def _cache(case, gen, news):
    """An 8-bit paged cache whose pages lie scattered over a pool, the new tokens behind the contexts,
    with its allocator."""
    dev, Hkv, fmt = "cuda", case["Hkv"], case["fmt"]
    ctx = torch.tensor(_context(case), dtype=torch.int64, device=dev)
    H = ctx.numel()
    lens = ctx + torch.tensor(news, dtype=torch.int64, device=dev).repeat_interleave(Hkv)
    n_pages = (lens + PAGE - 1) // PAGE
    longest = int(n_pages.max())
    width = max(longest, _round_up(case["table"]), 1)
    width += width % 2
    used = int(n_pages.sum())
    pool = used + used // 8 + H + 16
    if case["kind"] == "compact":
        pool += used
    perm = torch.randperm(pool, generator=gen, device=dev).to(torch.int32)
    live = torch.arange(width, device=dev)[None, :] < n_pages[:, None]
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
    st = {}
    for name, t, o in zip(("page_table", "page_mask", "n_pages", "free_ids", "free_top"), parts, off):
        st[name] = meta[o:o + t.numel() * t.element_size()].view(t.dtype).view(t.shape)
        st[name].copy_(t)
    st["k_pool"], st["k_scale"] = _rows((pool, PAGE, case["D"]), gen, fmt)
    st["v_pool"], st["v_scale"] = _rows((pool, PAGE, case["D"]), gen, fmt)
    return dict(st, meta=meta, meta0=meta.clone(), longest=longest)


def _own_cache(st):
    from paper_2606_28831_amd import PagedKV8
    return PagedKV8(st["k_pool"], st["v_pool"], st["k_scale"], st["v_scale"], st["page_table"], st["page_mask"],
                    st["n_pages"])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 31)
    kind, B, L, Hq, Hkv, D, fmt = (case[k] for k in ("kind", "NS", "L", "Hq", "Hkv", "D", "fmt"))
    dev, dt = "cuda", DTYPE[case["dtype"]]
    news = _news(case)
    T = sum(news) + case["pad"] * (kind in ("write", "attend"))
    at = [0]
    for n in news:
        at.append(at[-1] + n)
    start = torch.tensor(at, dtype=torch.int32, device=dev)
    st = dict(kind=kind, start=start, T=T, most=case["n_new"], Hkv=Hkv, G=Hq // Hkv, B=B, L=L, D=D, fmt=fmt, dt=dt)
    if kind == "write":
        # the slots that hk_reserve_slots gave: a row's in order in its pages, the pages scattered
        pages = [_round_up(n) for n in news]
        first = [0]
        for p in pages:
            first.append(first[-1] + p)
        pool = first[-1] * L * Hkv
        perm = torch.randperm(pool, generator=gen, device=dev)
        t = torch.arange(T, device=dev)
        s = (torch.searchsorted(start.long(), t, right=True) - 1).clamp(max=B - 1)
        i = t - start.long()[s]
        page = torch.tensor(first[:-1], device=dev)[s] + i // PAGE
        row = torch.arange(L, device=dev)[:, None, None] * Hkv + torch.arange(Hkv, device=dev)
        slot = perm[(row * first[-1] + page[None, :, None]).clamp(max=pool - 1)] * PAGE + (i % PAGE)[None, :, None]
        st["slot_map"] = torch.where((t < start[-1])[None, :, None], slot, -1).contiguous()
        # K and V as they leave one projection: the rows of a token side by side
        kvs = torch.empty((L, T, 2 * Hkv, D), dtype=dt, device=dev)
        for l in range(L):
            x = torch.randn((T, 2 * Hkv, D), generator=gen, device=dev)
            kvs[l] = x * torch.exp(torch.randn((T, 2 * Hkv, 1), generator=gen, device=dev))
        st["k_new"], st["v_new"] = kvs[:, :, :Hkv], kvs[:, :, Hkv:]
        for x in ("k", "v"):
            st[x + "_pool"] = torch.zeros((pool, PAGE, D), dtype=torch.uint8, device=dev).view(CODE[fmt])
            st[x + "_scale"] = torch.zeros((pool, PAGE), dtype=torch.float32, device=dev)
            st[x + "_out"] = torch.zeros((L, T, Hkv, D), dtype=dt, device=dev)
        st["page_table"], st["page_mask"], st["n_pages"] = (torch.zeros(x, dtype=y, device=dev) for x, y in (
            ((Hkv, 2), torch.int32), ((Hkv, 2), torch.int16), (Hkv, torch.int32)))
        if own:
            from paper_2606_28831_amd import dims
            st["kv"], st["d"] = _own_cache(st), dims(B, Hq, Hkv, D)
        return st
    st.update(_cache(case, gen, news))
    if kind == "read":
        # every slot of the longest rows' width, -1 where nothing lies
        P = st["longest"]
        slot = st["page_table"][:, :P].long()[:, :, None] * PAGE + torch.arange(PAGE, device=dev)
        valid = _bits(st["page_mask"][:, :P])
        st["slot_map"] = torch.where(valid, slot.reshape(B * Hkv, P * PAGE), -1).reshape(1, -1, 1).contiguous()
        n = st["slot_map"].numel()
        st["k_out"], st["v_out"] = (torch.zeros((1, n, 1, D), dtype=dt, device=dev) for _ in range(2))
    elif kind in ("decode", "attend"):
        q = torch.randn((T, Hq, D), generator=gen, device=dev)
        if case["tau"] > 1.0:
            u = torch.rand((Hkv,), generator=gen, device=dev) * 2.0 - 1.0
            q /= torch.pow(torch.tensor(case["tau"], device=dev), u).repeat_interleave(Hq // Hkv)[None, :, None]
        st["q"] = q.to(dt)
        st["o"] = torch.zeros((T, Hq, D), dtype=torch.float32 if kind == "decode" else dt, device=dev)
        st["lse"] = torch.zeros((T, Hq), dtype=torch.float32, device=dev)
    else:
        H, width = st["page_table"].shape
        bits = torch.rand((H, width * PAGE), generator=gen, device=dev)
        bits = (bits < case["keep"]).view(H, -1, 32).long() << torch.arange(32, device=dev)
        st["sel_bits"] = bits.sum(-1).to(torch.int32)
        st["dense"], st["sparse"] = case["dense"], case["sparse"]
        st["status"] = torch.zeros(1, dtype=torch.int32, device=dev)
    if own:
        from paper_2606_28831_amd import OP_COMPACT, Allocator, Chunks, dims, workspace
        from paper_2606_28831_amd.pipeline import ChunkDecoder, Decoder
        kv, al = _own_cache(st), Allocator(st["free_ids"], st["free_top"])
        st["kv"], st["alloc"], st["d"] = kv, al, dims(B, Hq, Hkv, D)
        if kind == "read":
            st["d"] = dims(1, 1, 1, D)
        elif kind == "decode":
            st["dec"] = Decoder(B, Hq, Hkv, D, kv, al)
        elif kind == "attend":
            st["chunks"] = Chunks(start, T, case["n_new"])
            st["dec"] = ChunkDecoder(B, Hq, Hkv, D, kv, al, T, case["n_new"])
        else:
            st["ws"] = workspace(OP_COMPACT, st["d"], kv.max_pages, dev)
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


def _read(st):
    """Rows of the pool through the slot map; rows without a slot stay as they are."""
    at = st["slot_map"].clamp(min=0)
    live = (st["slot_map"] >= 0)[..., None]
    for x in ("k", "v"):
        codes, scale = st[x + "_pool"].view(-1, st["D"]).view(torch.uint8)[at], st[x + "_scale"].view(-1)[at]
        y = codes.view(CODE[st["fmt"]]).float() * scale[..., None]
        st[x + "_out"].copy_(torch.where(live, y.to(st["dt"]), st[x + "_out"]))


def _plain_write(st):
    # rows without a slot write the first row once more
    live = st["slot_map"][:, :, :1] >= 0
    at = torch.where(st["slot_map"] >= 0, st["slot_map"], st["slot_map"][:, :1])
    for x in ("k", "v"):
        codes, scale = _quantise(torch.where(live[..., None], st[x + "_new"], st[x + "_new"][:, :1]), st["fmt"])
        st[x + "_pool"].view(-1, st["D"]).view(torch.uint8)[at] = codes.view(torch.uint8)
        st[x + "_scale"].view(-1)[at] = scale
    _read(st)


def _plain_attend(st):
    B, Hkv, G, P, n = st["B"], st["Hkv"], st["G"], st["longest"], st["most"]
    T, Hq, D = st["q"].shape
    H, S = B * Hkv, P * PAGE
    pages = st["page_table"][:, :P].long().clamp(min=0)
    valid = _bits(st["page_mask"][:, :P])
    values = lambda x: st[x + "_pool"].view(torch.uint8)[pages].view(CODE[st["fmt"]]).float().view(H, S, D).mul_(  # noqa: E731
        st[x + "_scale"][pages].view(H, S, 1))
    k, v = values("k"), values("v").masked_fill_(~valid[:, :, None], 0.0)
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
    t = torch.arange(T, device="cuda")
    s = (torch.searchsorted(st["start"].long(), t, right=True) - 1).clamp(max=B - 1)
    i, live = (t - st["start"].long()[s]).clamp(max=n - 1), t < st["start"][-1]
    st["o"].copy_(torch.where(live[:, None, None], o[s, i].to(st["o"].dtype), st["o"]))
    st["lse"].copy_(torch.where(live[:, None], lse[s, i], st["lse"]))


def _plain_compact(st):
    H, width = st["page_table"].shape
    n, top, free = st["n_pages"].long(), st["free_top"].long(), st["free_ids"]
    page = torch.arange(width, device="cuda")
    nd = n.clamp(max=_round_up(st["dense"]))
    ns = (n - nd).clamp(max=st["sparse"] // PAGE)
    nc = (n - nd - ns)[:, None]
    sel = ((st["sel_bits"].long()[:, :, None] >> torch.arange(32, device="cuda")) & 1).bool().view(H, -1)
    kept = _bits(st["page_mask"]) & sel                                      # [H, S]
    moved = kept & (page < nc).repeat_interleave(PAGE, 1)
    rank = torch.cumsum(moved, 1) - 1
    count = moved.sum(1)
    npc = (count + PAGE - 1) // PAGE
    base = top - npc.sum()
    begin = base + torch.cumsum(npc, 0) - npc                                # a head's first popped page
    # rows into their new pages
    h, j = torch.nonzero(moved, as_tuple=True)
    to = free[begin[h] + rank[h, j] // PAGE].long() * PAGE + rank[h, j] % PAGE
    at = st["page_table"][h, j // PAGE].long() * PAGE + j % PAGE
    for x in ("k", "v"):
        rows, scale = st[x + "_pool"].view(-1, st["D"]).view(torch.uint8), st[x + "_scale"].view(-1)
        rows[to] = rows[at]
        scale[to] = scale[at]
    # the sparse pages that keep a slot stay, in order, the dense ones behind them
    in_sparse = (page >= nc) & (page < nc + ns[:, None])
    in_dense = (page >= nc + ns[:, None]) & (page < n[:, None])
    left = (kept.view(H, width, PAGE).long() << torch.arange(PAGE, device="cuda")).sum(-1)
    stays = in_sparse & (left > 0) | in_dense
    new_at = torch.where(stays, npc[:, None] + torch.cumsum(stays, 1) - 1, width)
    fresh = page < npc[:, None]
    ids = torch.where(fresh, free[(begin[:, None] + page).clamp(max=free.numel() - 1)], -1)
    last = count[:, None] - page * PAGE
    bits = torch.where(fresh, (1 << last.clamp(0, PAGE)) - 1, 0)
    room = torch.cat([ids, ids[:, :1]], 1).scatter_(1, new_at, st["page_table"])[:, :width]
    kind = torch.where(in_sparse, left, st["page_mask"].long())
    masks = torch.cat([bits, bits[:, :1]], 1).scatter_(1, new_at, kind)[:, :width]
    # pages that leave, in row order
    gone = (page < n[:, None]) & ~stays
    where = base + torch.cumsum(gone.view(-1), 0) - 1
    stack = torch.cat([free, free[:1]])                                      # one more place, for the pages that stay
    stack[torch.where(gone.view(-1), where, free.numel())] = st["page_table"].view(-1)
    free.copy_(stack[:-1])
    st["free_top"].copy_(base + gone.sum())
    st["page_table"].copy_(room)
    st["page_mask"].copy_(masks.to(torch.int16))
    st["n_pages"].copy_(npc + stays.sum(1))


def run(st):
    kind = st["kind"]
    if kind == "compact":
        st["meta"].copy_(st["meta0"])
    if not own:
        {"write": _plain_write, "read": _read, "decode": _plain_attend, "attend": _plain_attend,
         "compact": _plain_compact}[kind](st)
    elif kind in ("write", "read"):
        from paper_2606_28831_amd import hk_read_kv8, hk_write_kv8
        n = st["slot_map"].shape[1]
        if kind == "write":
            hk_write_kv8(st["d"], st["kv"], n, st["slot_map"], st["k_new"], st["v_new"])
        hk_read_kv8(st["d"], st["kv"], n, st["slot_map"], st["k_out"], st["v_out"])
    elif kind == "decode":
        st["dec"].attend(st["q"], st["o"], st["lse"])
    elif kind == "attend":
        st["dec"].attend(st["chunks"], st["q"], st["o"], st["lse"])
    else:
        from paper_2606_28831_amd import hk_compact8
        hk_compact8(st["d"], st["kv"], st["sel_bits"], st["dense"], st["sparse"], st["alloc"], st["status"], st["ws"])
    if kind in ("write", "read"):
        return dict(k=st["k_out"], v=st["v_out"])
    if kind in ("decode", "attend"):
        return dict(o=st["o"], lse=st["lse"])
    out = {k: st[k] for k in ("page_table", "page_mask", "n_pages", "free_ids", "free_top", "k_scale", "v_scale")}
    # rows move as they are: their codes, one after the other as bytes
    return dict(out, k_pool=st["k_pool"].view(torch.uint8), v_pool=st["v_pool"].view(torch.uint8))


# ------------------------------------------------------------------------- what it must cost
def work(case):
    kind, B, L, Hq, Hkv, D = (case[k] for k in ("kind", "NS", "L", "Hq", "Hkv", "D"))
    e = 4 if case["dtype"] == "f32" else 2
    news, ctx = _news(case), _context(case)
    row = D + 4                                   # codes and scale
    if kind == "write":
        # rows read, codes written and read, values written, the map
        rows = sum(news) * L * Hkv
        return dict(bytes=rows * (2 * (2 * D * e + 2 * row) + 8), flops=0)
    slots = sum(c * (1.0 - case["holes"]) for c in ctx)
    if kind == "read":
        return dict(bytes=slots * 2 * (row + D * e) + 8 * len(ctx) * PAGE * _round_up(max(ctx)), flops=0)
    tables = 6 * sum(_round_up(c) for c in ctx)
    if kind == "compact":
        older = sum(max(0, c - case["dense"] - case["sparse"]) * (1.0 - case["holes"]) for c in ctx)
        moved = older * case["keep"]
        return dict(bytes=moved * 4 * row + sum(c / 8 for c in ctx) + 2 * tables + 4 * sum(c / PAGE for c in ctx), flops=0)
    heads = [(c, news[h // Hkv]) for h, c in enumerate(ctx)]
    keep = 1.0 - case["holes"]
    slots = sum(c * keep + n for c, n in heads)
    pairs = sum(n * c * keep + n * (n + 1) / 2 for c, n in heads)
    oe = 4 if kind == "decode" else e
    return dict(bytes=2 * slots * row + sum(news) * Hq * (D * (e + oe) + 4) + tables, flops=4 * D * pairs * (Hq // Hkv))


# ------------------------------------------------------------------------- in 64 bits
def _value(codes):
    """Codes as what they stand for, from their bits."""
    if codes.dtype == torch.int8:
        return codes.double()
    b = codes.view(torch.uint8).long()
    exp, man = b >> 3 & 15, b & 7
    size = torch.where(exp == 0, man.double() * 2.0 ** -9, torch.ldexp((man + 8).double(), (exp - 10).double()))
    return torch.where(b >> 7 == 1, -size, size)


def _exact_rows(x, fmt):
    """The values that rows have once they are written: the rule's fp32 steps, in 64 bits."""
    x, most = x.double(), MOST[fmt]
    fp32 = lambda y: y.float().double()  # noqa: E731
    a = x.abs().amax(-1, keepdim=True).clamp(min=LEAST)
    y = fp32(x * fp32(most / a))
    if fmt == "i8":
        codes = torch.round(y)
    else:
        step = torch.ldexp(torch.ones_like(y), (torch.frexp(y.abs()).exponent - 1).clamp(min=-6) - 3)
        codes = torch.round(y / step) * step
    return codes * fp32(a / most)


def exact(case, seed):
    kind, B, Hq, Hkv, D = (case[k] for k in ("kind", "NS", "Hq", "Hkv", "D"))
    if kind == "compact":
        return None                               # whole numbers, and rows and scales copied as they are
    st = prepare(case, seed)
    d, G = torch.float64, Hq // Hkv
    if kind in ("write", "read"):
        out = {}
        for x in ("k", "v"):
            y = torch.zeros(st[x + "_out"].shape, dtype=d, device="cuda")
            live = st["slot_map"] >= 0
            if kind == "write":
                y[live] = _exact_rows(st[x + "_new"], case["fmt"])[live]
            else:
                at = st["slot_map"][live]
                y[live] = (_value(st[x + "_pool"].view(-1, D).view(torch.uint8)[at].view(CODE[case["fmt"]]))
                           * st[x + "_scale"].view(-1)[at][:, None].double())
            out[x] = y
        return out
    o = torch.zeros(st["o"].shape, dtype=d, device="cuda")
    lse = torch.zeros(st["lse"].shape, dtype=d, device="cuda")
    start, n_pages = st["start"].tolist(), st["n_pages"].tolist()
    masks, table = st["page_mask"].to(torch.int32).tolist(), st["page_table"]
    rows = lambda x, where: (_value(st[x + "_pool"].view(-1, D).view(torch.uint8)[where].view(CODE[case["fmt"]]))  # noqa: E731
                             * st[x + "_scale"].view(-1)[where][:, None].double())
    for h in range(B * Hkv):
        s, g = h // Hkv, (h % Hkv) * G
        a, b = start[s], start[s + 1]
        held = [16 * j + t for j in range(n_pages[h]) for t in range(16) if masks[h][j] >> t & 1]
        end = held[-1] + 1 if held else 0
        at = torch.tensor(held, device="cuda", dtype=torch.int64)
        where = table[h][at // 16].long() * 16 + at % 16
        k, v = rows("k", where), rows("v", where)
        for x in range(a, b, 512):                # a few hundred tokens of the head at a time
            y = min(x + 512, b)
            z = st["q"][x:y, g:g + G].to(d) @ k.t() / math.sqrt(D)
            last = end - (b - a) + torch.arange(x - a, y - a, device="cuda")
            z.masked_fill_((at[None, :] > last[:, None])[:, None, :], -math.inf)
            lse[x:y, g:g + G] = torch.logsumexp(z, 2)
            o[x:y, g:g + G] = torch.softmax(z, 2) @ v
    return dict(o=o, lse=lse)
