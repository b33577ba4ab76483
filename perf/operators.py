"""Cases and plain forms of the serving operators around an ISD step: attention over a cache held in 4 bits, writing
prompts into that cache and reading them back, admission of requests (page tables and slot maps), and log
probabilities of emitted tokens.

`run` computes an operator in elementary torch operations, or, where `own` is true, through the library.

Layout of the 4-bit cache, kv_pool [pages, kv heads, 2176] bytes: per (page, head)
  [0, 1024)     K codes, words [4 chunks of 32 dims][16 tokens][4]; a word holds 8 consecutive dims of a token
  [1024, 2048)  V codes, words [128 dims][2]; a word holds 8 consecutive tokens of a dim
  [2048, 2176)  bf16 K scale[16], K zero[16], V scale[16], V zero[16]; "zero" holds 128 + z
in a word, element 2i sits at bits 4i and element 2i + 1 at bits 16 + 4i.  A vector x of 128 values is held as
  s = bf16((max(0, max x) - min(0, min x)) / 15),  z = clamp(rint(-min(0, min x) / s), 0, 15),
  c = clamp(rint(x / s) + z, 0, 15),  standing for s (c - z)        (quotients and differences in 32 bits).
"""
import math

import torch

own = False

PAGE, D, TILE = 16, 128, 2176
SHIFTS = (0, 16, 4, 20, 8, 24, 12, 28)


def listed():
    return [
        # one request in flight, a short context: the call's own latency
        {"name": "attn one request", "op": "attn", "batch": 1, "stride": 4, "hq": 8, "hkv": 2, "ctx_min": 256, "ctx_max": 256},
        # plain decoding (one row a slot) of a few long conversations: a long axis and few rows
        {"name": "attn decode 8 x 32k", "op": "attn", "batch": 8, "stride": 1, "hq": 32, "hkv": 8, "ctx_min": 16000, "ctx_max": 32768},
        # a moderate ragged batch, five query heads to a kv head
        {"name": "attn batch 64, stride 4", "op": "attn", "batch": 64, "stride": 4, "hq": 40, "hkv": 8, "ctx_min": 0, "ctx_max": 4096},
        # the stationary batch of the step benchmark
        {"name": "attn batch 256, stride 8", "op": "attn", "batch": 256, "stride": 8, "hq": 32, "hkv": 8, "ctx_min": 1024, "ctx_max": 8192},
        # one short prompt enters the cache
        {"name": "prompt of 127", "op": "kv", "requests": 1, "hkv": 8, "len_min": 127, "len_max": 127, "pad": 1, "fused": True},
        # a prefill batch of ragged prompts, K and V as slices of a fused projection, padded at its end
        {"name": "prompts 24 x 512..4096", "op": "kv", "requests": 24, "hkv": 8, "len_min": 512, "len_max": 4096, "pad": 37, "fused": True},
        # one request joins a running batch
        {"name": "admit one", "op": "admit", "batch": 64, "requests": 1, "stride": 4, "len_min": 700, "len_max": 700, "share": 1.0},
        # a whole batch is admitted, and the pool cannot serve the last requests
        {"name": "admit 256", "op": "admit", "batch": 256, "requests": 256, "stride": 8, "len_min": 1024, "len_max": 8192, "share": 0.9},
        # the tokens of one slot's step, a small vocabulary
        {"name": "logprobs one slot", "op": "logprobs", "rows": 4, "vocab": 4096, "dtype": "f32", "top": 0, "skip": 0.0},
        # the tokens a batch of eight emitted in a step
        {"name": "logprobs batch 8", "op": "logprobs", "rows": 64, "vocab": 151936, "dtype": "bf16", "top": 5, "skip": 0.4},
        # the tokens of the stationary batch, many positions of which emitted nothing
        {"name": "logprobs batch 256", "op": "logprobs", "rows": 2048, "vocab": 151936, "dtype": "bf16", "top": 20, "skip": 0.49},
        # scoring a prompt
        {"name": "logprobs prompt", "op": "logprobs", "rows": 777, "vocab": 50008, "dtype": "f32", "top": 32, "skip": 0.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "kv", "admit", "logprobs", "logprobs"])
    if op == "attn":
        hq, hkv = rng.choice([(8, 2), (32, 8), (40, 8), (16, 16), (24, 8), (28, 4)])
        stride = rng.randint(1, min(16, (128 // (hq // hkv) + 1) // 2))
        batch = _log(rng, 1, 256)
        most = min(32768, (256 * 8192 * 8 // (batch * hkv)), (256 * 8192 * 480) // (batch * hq * (2 * stride - 1)))
        ctx_max = _log(rng, 1, most)
        return {"op": op, "batch": batch, "stride": stride, "hq": hq, "hkv": hkv, "ctx_min": rng.choice([0, ctx_max // 3, ctx_max]), "ctx_max": ctx_max}
    if op == "kv":
        requests = _log(rng, 1, 64)
        len_max = _log(rng, 1, 65536 // requests)
        return {"op": op, "requests": requests, "hkv": rng.choice([1, 2, 4, 8]), "len_min": rng.choice([0, len_max // 2, len_max]), "len_max": len_max,
                "pad": rng.randint(0, 40), "fused": rng.random() < 0.5}
    if op == "admit":
        batch = _log(rng, 1, 512)
        len_max = _log(rng, 1, min(16384, (256 * 8192) // batch))
        return {"op": op, "batch": batch, "requests": rng.randint(1, batch), "stride": rng.randint(1, 16), "len_min": rng.choice([0, len_max // 3, len_max]),
                "len_max": len_max, "share": rng.choice([1.0, 1.0, 0.7])}
    vocab = 8 * _log(rng, 1, 19000)
    return {"op": op, "rows": _log(rng, 1, min(3000, 2048 * 151936 // (2 * vocab))), "vocab": vocab, "dtype": rng.choice(["f32", "bf16"]),
            "top": min(rng.choice([0, 1, 5, 20, 32]), vocab), "skip": rng.choice([0.0, 0.3])}


def _lens(case, lo, hi, n):
    """Ragged lengths of a case: the same for every seed, so that its work is known."""
    g = torch.Generator().manual_seed(1000003 * lo + 1009 * hi + n)
    return torch.randint(lo, hi + 1, (n,), generator=g)


def _n_ver(case):
    """Proposals under verification: full blocks after a step that accepted all, none after a rejection."""
    g = torch.Generator().manual_seed(7 * case["batch"] + case["stride"])
    return torch.where(torch.rand(case["batch"], generator=g) < 0.55, case["stride"] - 1, 0)


def work(case):
    if case["op"] == "attn":
        n, ctx = _n_ver(case).tolist(), _lens(case, case["ctx_min"], case["ctx_max"], case["batch"]).tolist()
        rows = [a + case["stride"] for a in n]
        keys = sum(c + r for c, r in zip(ctx, rows))
        pairs = sum((c + r) * r for c, r in zip(ctx, rows))
        # the cache once, q and the output, the block's rows in, their tiles out and back as values
        return {"bytes": keys * case["hkv"] * 136 + sum(rows) * (case["hq"] * D * 4 + case["hq"] * 4 + case["hkv"] * (512 + 136 + 136 + 512)),
                "flops": 4 * pairs * case["hq"] * D}
    if case["op"] == "kv":
        t = int(_lens(case, case["len_min"], case["len_max"], case["requests"]).sum())
        return {"bytes": t * (case["hkv"] * 2 * (512 + 136) + 16) + 8, "flops": t * case["hkv"] * 2 * D * 6}
    if case["op"] == "admit":
        lens = _lens(case, case["len_min"], case["len_max"], case["requests"])
        want = (lens + 2 * case["stride"] - 1 + PAGE - 1) // PAGE
        ok = torch.cumsum(want, 0) <= _free_pages(case, want)
        t, p = int(lens[ok].sum()), int(want[ok].sum())
        return {"bytes": t * 16 + p * 8 + case["requests"] * 40, "flops": 0}
    read = int(_given(case).sum())
    return {"bytes": read * case["vocab"] * (4 if case["dtype"] == "f32" else 2) + case["rows"] * (16 + 8 * case["top"]), "flops": read * case["vocab"] * 6}


def _free_pages(case, want):
    return max(1, int(int(want.sum()) * case["share"])) + (3 if case["share"] == 1.0 else 0)


def _given(case):
    g = torch.Generator().manual_seed(case["rows"])
    return torch.rand(case["rows"], generator=g) >= case["skip"]


# ---------------------------------------------------------------------------------------------------------- the codec
def _encode(x):
    """x [..., 128] -> codes int32 [..., 128], scale f32 [...], z f32 [...] (the definition above, step by step)."""
    x = x.float()
    lo, hi = x.amin(-1).clamp(max=0.0), x.amax(-1).clamp(min=0.0)
    s = torch.div(hi - lo, torch.full_like(lo, 15.0)).bfloat16().float()
    bad = ~torch.isfinite(s)
    live = (s > 0) & ~bad
    d = torch.where(live, s, torch.ones_like(s))
    z = torch.where(live, torch.round(-lo / d).clamp(0, 15), torch.zeros_like(s))
    c = (torch.round(x / d[..., None]) + z[..., None]).clamp(0, 15)
    c = torch.where(live[..., None], c, torch.zeros_like(c)).to(torch.int32)
    return c, torch.where(bad, torch.full_like(s, math.nan), s), z


def _words(c):
    """codes [..., 8] -> int32 words [...]"""
    return (c << torch.tensor(SHIFTS, device=c.device, dtype=torch.int32)).sum(-1, dtype=torch.int32)


def _codes(w):
    return (w[..., None] >> torch.tensor(SHIFTS, device=w.device, dtype=torch.int32)) & 15


def _unpack(tiles):
    """tiles uint8 [..., 2176] -> K codes, V codes [..., 16, 128] and [..., 4, 16] bf16 (K scale, K zero, V scale, V zero)"""
    head = tiles.shape[:-1]
    k = _codes(tiles[..., :1024].contiguous().view(torch.int32).view(*head, 4, 16, 4)).transpose(-4, -3).reshape(*head, 16, D)
    v = _codes(tiles[..., 1024:2048].contiguous().view(torch.int32).view(*head, D, 2)).reshape(*head, D, 16).transpose(-1, -2)
    return k, v, tiles[..., 2048:].contiguous().view(torch.bfloat16).view(*head, 4, 16)


def _pack(k, v, meta):
    head = k.shape[:-2]
    kw = _words(k.reshape(*head, 16, 4, 4, 8).transpose(-4, -3)).reshape(*head, 256)
    vw = _words(v.transpose(-1, -2).reshape(*head, D, 2, 8)).reshape(*head, 256)
    return torch.cat([kw.contiguous().view(torch.uint8), vw.contiguous().view(torch.uint8), meta.reshape(*head, 64).contiguous().view(torch.uint8)], -1)


def _values(c, scale, zero):
    """codes [..., 16, 128], scale and zero [..., 16] -> f32 values"""
    return scale.float()[..., None] * (c.float() - (zero.float()[..., None] - 128.0))


def _store_pages(pool, pages, rows, hit, zero_tail):
    """Rewrites whole pages: pages [P] ids (a page may occur twice with the same contents), rows = (k codes, v codes [P, 16, Hkv, 128], meta
    [P, 4, 16, Hkv]) of the tokens where hit [P, 16]; the tokens where zero_tail [P, 16] become zeros, the others stay."""
    k, v, meta = _unpack(pool[pages])  # [P, Hkv, 16, 128], [P, Hkv, 4, 16]
    nk, nv, nm = rows
    h = hit[:, None, :, None]
    k, v = torch.where(h, nk.transpose(1, 2), k), torch.where(h, nv.transpose(1, 2), v)
    m = torch.where(hit[:, None, None, :], nm.permute(0, 3, 1, 2), meta)
    empty = torch.tensor([0.0, 128.0, 0.0, 128.0], device=pool.device, dtype=torch.bfloat16)[None, None, :, None]
    m = torch.where(zero_tail[:, None, None, :], empty, m)
    pool[pages] = _pack(k, v, m)


# -------------------------------------------------------------------------------------------------------------- inputs
def _gen(seed, salt=0):
    return torch.Generator(device="cuda").manual_seed(seed * 64 + salt)


def _normal(shape, g, sigma=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * sigma).bfloat16()


def _new_pool(pages, hkv, g):
    """A cache that earlier steps filled: normal keys with a few loud channels and normal values, held by the codec."""
    pool = torch.empty(pages, hkv, TILE, dtype=torch.uint8, device="cuda")
    loud = 1.0 + 3.0 * (torch.rand(hkv, 1, D, generator=g, device="cuda") < 0.03)
    step = max(1, (1 << 26) // (hkv * 16 * D))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        kc, ks, kz = _encode((torch.randn(n, hkv, 16, D, generator=g, device="cuda") * 0.5 * loud).bfloat16())
        vc, vs, vz = _encode((torch.randn(n, hkv, 16, D, generator=g, device="cuda") * 0.5).bfloat16())
        pool[p:p + n] = _pack(kc, vc, torch.stack([ks, kz + 128, vs, vz + 128], 2).bfloat16())
    return pool


def _handle(case, **kw):
    from paper_2604_11035_b200 import Isd
    args = dict(batch=1, stride=1, n_q_heads=8, n_kv_heads=case.get("hkv", 8), vocab=64, max_pages_per_slot=8, num_pages=8, logits_dtype="bf16")
    return Isd(**{**args, **kw})


def prepare(case, seed):
    make = {"attn": _prepare_attn, "kv": _prepare_kv, "admit": _prepare_admit, "logprobs": _prepare_logprobs}
    return make[case["op"]](case, seed)


def _prepare_attn(case, seed):
    B, N, hq, hkv = case["batch"], case["stride"], case["hq"], case["hkv"]
    Q = 2 * N - 1
    ctx, n_ver = _lens(case, case["ctx_min"], case["ctx_max"], B), _n_ver(case)
    g, gc = _gen(seed), torch.Generator().manual_seed(seed)
    have = (ctx + Q + PAGE - 1) // PAGE
    width = int(have.max())
    pages = int(have.sum()) + 5
    order = torch.randperm(pages, generator=gc)
    table = torch.full((B, width), -1, dtype=torch.int64)
    start = torch.cumsum(have, 0) - have
    col = torch.arange(width)[None]
    table = torch.where(col < have[:, None], order[(start[:, None] + col).clamp(max=pages - 1)], table)
    pos = ctx[:, None] + torch.arange(Q)[None]
    block_map = torch.gather(table, 1, pos // PAGE) * PAGE + pos % PAGE
    block_map = torch.where(torch.arange(Q)[None] < (n_ver + N)[:, None], block_map, -1)
    i32 = dict(dtype=torch.int32, device="cuda")
    st = dict(ctx_len=ctx.to(**i32), n_ver=n_ver.to(**i32), block_tok=torch.zeros(B, Q, **i32), q_row0=torch.zeros(B, **i32),
              q_stats=torch.zeros(B, N - 1, 2, device="cuda"), page_table=table.to(**i32), free_stack=torch.zeros(pages, **i32),
              free_top=torch.zeros(1, **i32), active=torch.ones(B, dtype=torch.uint8, device="cuda"), slot_status=torch.zeros(B, **i32))
    s = dict(case=case, st=st, kv_pool=_new_pool(pages, hkv, g), q=_normal((B, Q, hq, D), g), k_new=_normal((B, Q, hkv, D), g, 0.5),
             v_new=_normal((B, Q, hkv, D), g, 0.5), block_map=block_map.reshape(-1).cuda(),
             out=torch.zeros(B, Q, hq, D, dtype=torch.bfloat16, device="cuda"), lse=torch.zeros(B, Q, hq, device="cuda"),
             k_back=torch.zeros(B * Q, hkv, D, dtype=torch.bfloat16, device="cuda"), v_back=torch.zeros(B * Q, hkv, D, dtype=torch.bfloat16, device="cuda"))
    if own:
        s["isd"] = _handle(case, batch=B, stride=N, n_q_heads=hq, n_kv_heads=hkv, max_pages_per_slot=width, num_pages=pages)
    return s


def _prepare_kv(case, seed):
    hkv, lens = case["hkv"], _lens(case, case["len_min"], case["len_max"], case["requests"])
    g, gc = _gen(seed, 1), torch.Generator().manual_seed(seed)
    have = (lens + PAGE - 1) // PAGE
    pages = int(have.sum()) + 2
    order = torch.randperm(pages, generator=gc)
    total = int(lens.sum())
    T = total + case["pad"]
    req = torch.repeat_interleave(torch.arange(len(lens)), lens)
    pos = torch.arange(total) - (torch.cumsum(lens, 0) - lens)[req]
    slot = torch.full((T,), -1, dtype=torch.int64)
    slot[:total] = order[(torch.cumsum(have, 0) - have)[req] + pos // PAGE] * PAGE + pos % PAGE
    rows = torch.cat([_normal((T, hkv, D), g), _normal((T, hkv, D), g, 0.5), _normal((T, hkv, D), g, 0.5)], 1)  # q | k | v of a fused projection
    k, v = rows[:, hkv:2 * hkv], rows[:, 2 * hkv:]
    if not case["fused"]:
        k, v = k.contiguous(), v.contiguous()
    s = dict(case=case, k=k, v=v, slot_map=slot.cuda(), kv_pool=torch.zeros(pages, hkv, TILE, dtype=torch.uint8, device="cuda"),
             k_back=torch.zeros(T, hkv, D, dtype=torch.bfloat16, device="cuda"), v_back=torch.zeros(T, hkv, D, dtype=torch.bfloat16, device="cuda"))
    if own:
        s["isd"] = _handle(case, n_q_heads=hkv, num_pages=pages)
    return s


def _prepare_admit(case, seed):
    B, n, N = case["batch"], case["requests"], case["stride"]
    Q = 2 * N - 1
    lens = _lens(case, case["len_min"], case["len_max"], n)
    gc = torch.Generator().manual_seed(seed)
    want = (lens + Q + PAGE - 1) // PAGE
    free = _free_pages(case, want)
    pages = free + 40
    width = (case["len_max"] + Q + PAGE - 1) // PAGE + 2
    cap = int(lens.sum())
    i32 = dict(dtype=torch.int32, device="cuda")
    stack = torch.full((pages,), -1, dtype=torch.int64)
    stack[:free] = torch.randperm(pages, generator=gc)[:free]
    # `active` and `free_top` share a buffer that one copy sets back to what it was before the admission
    pad = -(-B // 16) * 16
    held = torch.zeros(pad + 16, dtype=torch.uint8, device="cuda")
    held[pad:pad + 4].view(torch.int32).fill_(free)
    now = held.clone()
    st = dict(ctx_len=torch.zeros(B, **i32), n_ver=torch.zeros(B, **i32), block_tok=torch.zeros(B, Q, **i32), q_row0=torch.zeros(B, **i32),
              q_stats=torch.zeros(B, N - 1, 2, device="cuda"), page_table=torch.full((B, width), -1, **i32), free_stack=stack.to(**i32),
              free_top=now[pad:pad + 4].view(torch.int32), active=now[:B], slot_status=torch.zeros(B, **i32))
    s = dict(case=case, st=st, now=now, held=held, lens=lens.to(**i32), slots=torch.randperm(B, generator=gc)[:n].to(**i32),
             anchors=torch.randint(0, 50000, (n,), generator=gc).to(**i32), mask=63,
             maps=dict(result=torch.zeros(n, **i32), cu_len=torch.zeros(n + 1, **i32), slot_map=torch.full((cap,), -1, dtype=torch.int64, device="cuda"),
                       tok_req=torch.full((cap,), -1, **i32), tok_pos=torch.full((cap,), -1, **i32)))
    if own:
        s["isd"] = _handle(case, batch=B, stride=N, n_kv_heads=8, max_pages_per_slot=width, num_pages=pages)
    return s


def _prepare_logprobs(case, seed):
    n, V, top = case["rows"], case["vocab"], case["top"]
    g = _gen(seed, 3)
    total = n + n // 8 + 1  # the step's logits: more rows than are asked for
    logits = torch.empty(total, V, dtype=torch.float32 if case["dtype"] == "f32" else torch.bfloat16, device="cuda")
    for r in range(0, total, 256):
        x = torch.randn(min(256, total - r), V, generator=g, device="cuda") * 3.0
        peaked = torch.rand(x.shape[0], generator=g, device="cuda") < 0.6
        at = torch.randint(0, V, (x.shape[0], 1), generator=g, device="cuda")
        x.scatter_(1, at, torch.where(peaked[:, None], x.amax(1, keepdim=True) + 8.0, x.gather(1, at)))
        logits[r:r + 256] = x.to(logits.dtype)
    rows = torch.randperm(total, generator=g, device="cuda")[:n].to(torch.int32)
    best = logits.argmax(1)[rows.long()]
    tokens = torch.where(torch.rand(n, generator=g, device="cuda") < 0.6, best, torch.randint(0, V, (n,), generator=g, device="cuda"))
    tokens = torch.where(_given(case).cuda(), tokens, -1).to(torch.int32)
    s = dict(case=case, logits=logits, rows=rows, tokens=tokens,
             out=dict(logprob=torch.zeros(n, device="cuda"), entropy=torch.zeros(n, device="cuda"), top_id=torch.zeros(n, top, dtype=torch.int32, device="cuda"),
                      top_logprob=torch.zeros(n, top, device="cuda")))
    if own:
        s["isd"] = _handle(case, vocab=V, logits_dtype=case["dtype"])
    return s


# ----------------------------------------------------------------------------------------------------------------- run
def run(s):
    return {"attn": _run_attn, "kv": _run_kv, "admit": _run_admit, "logprobs": _run_logprobs}[s["case"]["op"]](s)


def _run_attn(s):
    if own:
        s["isd"].isd_attn_quant(s["st"], s["q"], s["k_new"], s["v_new"], s["kv_pool"], s["out"], s["lse"])
        s["isd"].isd_kv_read_quant(s["kv_pool"], s["block_map"], s["k_back"], s["v_back"])
    else:
        _plain_attn(s)
        _plain_read(s["kv_pool"], s["block_map"], s["k_back"], s["v_back"])
    return s["out"], s["lse"], s["k_back"], s["v_back"]


def _plain_attn(s):
    st, pool, q = s["st"], s["kv_pool"], s["q"]
    B, Q, hq, _ = q.shape
    hkv = pool.shape[1]
    G, N = hq // hkv, (Q + 1) // 2
    table, ctx, q_len = st["page_table"].long(), st["ctx_len"].long(), st["n_ver"].long() + N
    kv_len = ctx + q_len
    # the block's rows enter the pages from the one that holds position ctx on; the rest of the last page is emptied
    span = (Q + 14) // PAGE + 1
    first, last = ctx // PAGE, (kv_len - 1) // PAGE
    lp = torch.minimum(first[:, None] + torch.arange(span, device=q.device), last[:, None])  # logical pages [B, span]
    row = lp[..., None] * PAGE + torch.arange(PAGE, device=q.device) - ctx[:, None, None]  # [B, span, 16]
    at = row.clamp(0, Q - 1).reshape(B, span * PAGE, 1, 1).expand(-1, -1, hkv, D)
    new = []
    for x in (s["k_new"], s["v_new"]):
        c, sc, z = _encode(x)
        new.append((c.gather(1, at).view(B * span, PAGE, hkv, D), sc.gather(1, at[..., 0]), (z + 128).gather(1, at[..., 0])))
    meta = torch.stack([x.view(B * span, PAGE, hkv) for _, sc, z in new for x in (sc, z)], 1).bfloat16()
    hit = ((row >= 0) & (row < q_len[:, None, None])).view(-1, PAGE)
    _store_pages(pool, table.gather(1, lp).reshape(-1), (new[0][0], new[1][0], meta), hit, (row >= q_len[:, None, None]).view(-1, PAGE))
    # scores of every row against every key of the padded batch
    k, v, meta = _unpack(pool[table.clamp(min=0)])  # [B, W, Hkv, 16, 128], [B, W, Hkv, 4, 16]
    W = table.shape[1]
    k = _values(k, meta[..., 0, :], meta[..., 1, :]).transpose(1, 2).reshape(B, hkv, W * PAGE, D)
    qg = q.float().view(B, Q, hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, hkv, Q * G, D)
    score = (qg @ k.transpose(-1, -2)).view(B, hkv, Q, G, W * PAGE) * (1.0 / math.sqrt(D))
    del k
    r = torch.arange(Q, device=q.device)
    seen = torch.arange(W * PAGE, device=q.device) <= (ctx[:, None] + r)[..., None]  # [B, Q, keys]
    score = score.masked_fill(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - top)
    del score
    total = p.sum(-1, keepdim=True)
    v = _values(v, meta[..., 2, :], meta[..., 3, :])
    v = torch.where(torch.arange(W * PAGE, device=q.device).view(1, W, 1, PAGE, 1) < kv_len.view(-1, 1, 1, 1, 1), v, torch.zeros((), device=q.device))
    v = v.transpose(1, 2).reshape(B, hkv, W * PAGE, D)
    o = (p.view(B, hkv, Q * G, W * PAGE) @ v).view(B, hkv, Q, G, D) / total
    o = o.permute(0, 2, 1, 3, 4).reshape(B, Q, hq, D)
    lse = (top + torch.log(total))[..., 0].permute(0, 2, 1, 3).reshape(B, Q, hq)
    valid = (r < q_len[:, None])[..., None]
    s["out"].copy_(torch.where(valid[..., None], o.bfloat16(), s["out"]))
    s["lse"].copy_(torch.where(valid, lse, s["lse"]))


def _plain_read(pool, slot_map, k_back, v_back):
    """The tokens of a slot map as bf16 values; rows of negative entries stay as they are."""
    ok = slot_map >= 0
    page, off = slot_map.clamp(min=0) // PAGE, slot_map.clamp(min=0) % PAGE
    k, v, meta = _unpack(pool[page])  # [T, Hkv, 16, 128], [T, Hkv, 4, 16]
    at = off[:, None, None, None]
    for back, c, m in ((k_back, k, 0), (v_back, v, 2)):
        c = c.gather(2, at.expand(-1, c.shape[1], 1, D))
        sc, z = (meta[:, :, m + i].gather(2, at[..., 0].expand(-1, c.shape[1], 1)) for i in (0, 1))
        back.copy_(torch.where(ok[:, None, None], _values(c, sc, z)[:, :, 0].bfloat16(), back))


def _plain_write(k, v, slot_map, pool):
    """Byte by byte: the codes of K are whole bytes of their token's words, those of V are added into emptied nibbles."""
    P, hkv, _ = pool.shape
    T = slot_map.shape[0]
    dev = pool.device
    ok = slot_map >= 0
    page, off = torch.where(ok, slot_map // PAGE, P), slot_map.clamp(min=0) % PAGE  # padding goes to a page behind the last
    (kc, ks, kz), (vc, vs, vz) = _encode(k), _encode(v)
    held = torch.cat([pool, torch.zeros(1, hkv, TILE, dtype=torch.uint8, device=dev)])
    h = torch.arange(hkv, device=dev)
    w32 = held[:, :, :1024].contiguous().view(torch.int32).view(P + 1, hkv, 4, 16, 4)
    w32[page[:, None, None], h[None, :, None], torch.arange(4, device=dev)[None, None, :], off[:, None, None]] = _words(kc.view(T, hkv, 4, 4, 8))
    codes = _codes(held[:, :, 1024:2048].contiguous().view(torch.int32).view(P + 1, hkv, D, 2)).view(P + 1, hkv, D, 16)
    codes[page[:, None, None], h[None, :, None], torch.arange(D, device=dev)[None, None, :], off[:, None, None]] = vc
    meta = held[:, :, 2048:].contiguous().view(torch.bfloat16).view(P + 1, hkv, 4, 16)
    meta[page[:, None, None], h[None, :, None], torch.arange(4, device=dev)[None, None, :], off[:, None, None]] = torch.stack([ks, kz + 128, vs, vz + 128], 2).bfloat16()
    pool[:, :, :1024] = w32[:P].reshape(P, hkv, 256).contiguous().view(torch.uint8)
    pool[:, :, 1024:2048] = _words(codes[:P].view(P, hkv, D, 2, 8)).reshape(P, hkv, 256).view(torch.uint8)
    pool[:, :, 2048:] = meta[:P].reshape(P, hkv, 64).view(torch.uint8)


def _run_kv(s):
    if own:
        s["isd"].isd_kv_write_quant(s["k"], s["v"], s["slot_map"], s["kv_pool"])
        s["isd"].isd_kv_read_quant(s["kv_pool"], s["slot_map"], s["k_back"], s["v_back"])
    else:
        _plain_write(s["k"], s["v"], s["slot_map"], s["kv_pool"])
        _plain_read(s["kv_pool"], s["slot_map"], s["k_back"], s["v_back"])
    return s["k_back"], s["v_back"]


def _run_admit(s):
    s["now"].copy_(s["held"])  # the requests of the pass before are gone
    st, m = s["st"], s["maps"]
    if own:
        s["isd"].isd_admit(st, s["slots"], s["lens"], s["anchors"], m)
    else:
        _plain_admit(s)
    return [m["result"], m["cu_len"], m["slot_map"], m["tok_req"], m["tok_pos"]] + [
        st[k] for k in ("page_table", "ctx_len", "n_ver", "block_tok", "q_row0", "active", "slot_status", "free_top")]


def _plain_admit(s):
    st, m, lens, slots = s["st"], s["maps"], s["lens"].long(), s["slots"].long()
    Q, cap, dev = st["block_tok"].shape[1], m["slot_map"].shape[0], lens.device
    want = (lens + Q + PAGE - 1) // PAGE
    top = st["free_top"].long()
    upto = torch.cumsum(want, 0)
    before, ok = upto - want, upto <= top
    m["result"].copy_(torch.where(ok, 0, 1))
    m["cu_len"][1:] = torch.cumsum(torch.where(ok, lens, 0), 0)
    m["cu_len"][0].zero_()
    cu = m["cu_len"].long()
    t = torch.arange(cap, device=dev)
    req = torch.searchsorted(cu[1:].contiguous(), t, right=True).clamp(max=lens.shape[0] - 1)
    pos = t - cu[req]
    inside = t < cu[-1]
    stack = st["free_stack"].long()
    page = stack[(top - 1 - before[req] - torch.where(inside, pos, 0) // PAGE).clamp(min=0)]
    m["slot_map"].copy_(torch.where(inside, page * PAGE + pos % PAGE, m["slot_map"]))
    m["tok_req"].copy_(torch.where(inside, req, m["tok_req"]))
    m["tok_pos"].copy_(torch.where(inside, pos, m["tok_pos"]))
    j = torch.arange(st["page_table"].shape[1], device=dev)[None]
    entry = stack[(top - 1 - before[:, None] - j).clamp(min=0)]
    st["page_table"][slots] = torch.where(ok[:, None] & (j < want[:, None]), entry, st["page_table"][slots].long()).int()
    block = torch.full((lens.shape[0], Q), s["mask"], device=dev)
    block[:, 0] = s["anchors"]
    st["block_tok"][slots] = torch.where(ok[:, None], block, st["block_tok"][slots].long()).int()
    st["ctx_len"][slots] = torch.where(ok, lens, st["ctx_len"][slots].long()).int()
    for name in ("n_ver", "q_row0", "slot_status"):
        st[name][slots] = torch.where(ok, 0, st[name][slots])
    st["active"][slots] = torch.where(ok, 1, st["active"][slots]).to(torch.uint8)
    st["free_top"].copy_(top - torch.where(ok, want, 0).sum())


def _run_logprobs(s):
    out, top = s["out"], s["case"]["top"]
    if own:
        s["isd"].isd_logprobs(s["logits"], s["tokens"], rows=s["rows"], top_n=top, out=out)
    else:
        x = s["logits"][s["rows"].long()].float()
        given = s["tokens"] >= 0
        x = x - x.amax(1, keepdim=True)
        e = torch.exp(x)
        total = e.sum(1, keepdim=True)
        log_total = torch.log(total)
        none = torch.full((), math.nan, device=x.device)
        out["logprob"].copy_(torch.where(given, (x.gather(1, s["tokens"].long().clamp(min=0)[:, None]) - log_total)[:, 0], none))
        out["entropy"].copy_(torch.where(given, log_total[:, 0] - (e * x).sum(1) / total[:, 0], none))
        if top:
            del e
            value, index = torch.sort(x, dim=1, descending=True, stable=True)  # equal values: the lowest index first
            out["top_id"].copy_(torch.where(given[:, None], index[:, :top].int(), -1))
            out["top_logprob"].copy_(torch.where(given[:, None], value[:, :top] - log_total, none))
    return out


# -------------------------------------------------------------------------------------------------- values in 64 bits
def _exact_codec(x):
    """(codes, scale, zero) of the codec's definition; x [..., 128] bf16.  Scale and z go by the stated 32-bit steps, x / s is taken in 64."""
    x = x.double()
    lo, hi = torch.clamp(x.min(-1).values, max=0), torch.clamp(x.max(-1).values, min=0)
    s = torch.div(hi.float() - lo.float(), torch.full_like(lo, 15, dtype=torch.float32)).bfloat16().double()
    safe = torch.where(s > 0, s, 1.0)
    z = torch.clamp(torch.round(-lo / safe), 0, 15) * (s > 0)
    c = torch.clamp(torch.round(x / safe[..., None]) + z[..., None], 0, 15) * (s > 0)[..., None]
    return c, s, z


def _exact_tables(device):
    """Byte and shift of the code of (token, dim), for K and V."""
    tok, dim = torch.arange(16)[:, None], torch.arange(D)[None]
    place = []
    for word, e in ((dim // 32 * 64 + tok * 4 + dim % 32 // 8, dim % 8 + 0 * tok), (256 + dim * 2 + tok // 8, tok % 8 + 0 * dim)):
        bit = e // 2 * 4 + e % 2 * 16
        place.append(((word * 4 + bit // 8).to(device), (bit % 8).to(device)))
    return place


def _exact_values(tiles):
    """tiles [n, Hkv, 2176] -> K, V [Hkv, n * 16, 128] in 64 bits"""
    got = []
    for (byte, shift), m in zip(_exact_tables(tiles.device), (0, 2)):
        c = (tiles[..., byte].int() >> shift.int()) & 15
        meta = tiles[..., 2048 + 32 * m:2048 + 32 * m + 64].contiguous().view(torch.bfloat16).double()
        x = meta[..., :16, None] * (c.double() - (meta[..., 16:, None] - 128))
        got.append(x.transpose(0, 1).reshape(tiles.shape[1], -1, D))
    return got


def exact(case, seed):
    if case["op"] == "admit":
        return None
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"attn": _exact_attn, "kv": _exact_kv, "logprobs": _exact_logprobs}[case["op"]](s)


def _exact_attn(s):
    st, q = s["st"], s["q"].double()
    B, Q, hq, _ = q.shape
    hkv, N = s["kv_pool"].shape[1], (Q + 1) // 2
    out, lse = torch.zeros(q.shape, dtype=torch.float64, device=q.device), torch.zeros(B, Q, hq, dtype=torch.float64, device=q.device)
    back = [torch.zeros(B, Q, hkv, D, dtype=torch.float64, device=q.device) for _ in range(2)]
    for b, (ctx, nv) in enumerate(zip(st["ctx_len"].tolist(), st["n_ver"].tolist())):
        n = nv + N
        old = _exact_values(s["kv_pool"][st["page_table"][b, :(ctx + 15) // 16].long()])
        full = []
        for i, x in enumerate((s["k_new"], s["v_new"])):
            c, sc, z = _exact_codec(x[b, :n])
            back[i][b, :n] = sc[..., None] * (c - z[..., None])
            full.append(torch.cat([old[i][:, :ctx], back[i][b, :n].transpose(0, 1)], 1))  # [Hkv, ctx + n, 128]
        qb = q[b, :n].view(n, hkv, hq // hkv, D).permute(1, 2, 0, 3).reshape(hkv, -1, D)  # [Hkv, G * n, 128]
        a = torch.einsum("hmd,hkd->hmk", qb, full[0]).view(hkv, -1, n, ctx + n) / math.sqrt(D)
        hidden = torch.arange(ctx + n, device=q.device)[None] > ctx + torch.arange(n, device=q.device)[:, None]
        a = a.masked_fill(hidden, -math.inf)
        lse[b, :n] = torch.logsumexp(a, -1).permute(2, 0, 1).reshape(n, hq)
        o = torch.einsum("hgnk,hkd->nhgd", torch.softmax(a, -1), full[1])
        out[b, :n] = o.reshape(n, hq, D)
    return out, lse, back[0].view(B * Q, hkv, D), back[1].view(B * Q, hkv, D)


def _exact_kv(s):
    got = []
    for x in (s["k"], s["v"]):
        c, sc, z = _exact_codec(x)
        got.append(torch.where((s["slot_map"] >= 0)[:, None, None], sc[..., None] * (c - z[..., None]), 0.0))
    return tuple(got)


def _exact_logprobs(s):
    n, top = s["tokens"].shape[0], s["case"]["top"]
    got = dict(logprob=[], entropy=[], top_id=None, top_logprob=[])
    for r in range(0, n, 64):
        tok = s["tokens"][r:r + 64].long()
        lp = torch.log_softmax(s["logits"][s["rows"][r:r + 64].long()].double(), 1)
        none = torch.where(tok >= 0, 0.0, math.nan).double()
        got["logprob"].append(lp.gather(1, tok.clamp(min=0)[:, None])[:, 0] + none)
        got["entropy"].append(-torch.special.xlogy(lp.exp(), lp.exp()).sum(1) + none)
        got["top_logprob"].append(torch.sort(lp, 1, descending=True).values[:, :top] + none[:, None])
    return {k: torch.cat(v) if v else v for k, v in got.items()}
