"""What the operators around the paged K/V cache are measured by: page tables and slot maps from request lengths, the
cache in 4 bits (rows in and out, attention over it) and attention with a sliding window and sinks.

A case is a dict of plain values; `kind` says which operator it goes through:

  table    tidar_table_extend       page table entries and slots for the new rows of every sequence
  store    tidar_kv4_store + _load  rows of K and V into 4-bit pages, and back as the values they are held as
  kv4      tidar_kv4_attention      hybrid-mask attention over 4-bit pages (window 0: over the whole prefix)
  window   tidar_window_attention   hybrid-mask attention over exact pages with a sliding window and sinks

Rows of an attention call: `nc` causal rows, then `nb` blocks of `bl` mask rows, block j conditioned on the first
`cond0` + j causal rows (one-token step: 1, 0; decode step: k, k, k, 1; prefill: prompt rows and one block behind them).
"""
import math

import torch

own = False

DEV = "cuda:0"
PAGE = 16
HEADS = {"8b": (32, 8, 128), "1p5b": (12, 2, 128), "small": (4, 2, 128), "tiny": (4, 4, 32)}   # q heads, kv heads, head_dim


def _case(name, kind, **more):
    c = {"kind": kind}
    if kind == "table":
        c.update(batch=1, prefix=0, new=1, short=False)
    else:
        c.update(heads="8b", dtype="bf16")
        if kind == "store":
            c.update(rows=1)
        else:
            c.update(batch=1, prefix=0, ragged=False, nc=1, nb=0, bl=1, cond0=1, window=0, sinks=0)
    c.update(more)
    if name:
        c["name"] = name
    return c


def _step(k):
    return {"nc": k, "nb": k, "bl": k, "cond0": 1}


def _prefill(nc, k):
    return {"nc": nc, "nb": 1, "bl": k, "cond0": nc}


def listed():
    return [
        # one new token for each of six sequences: a decode loop's bookkeeping, nothing but latency
        _case("table_decode_b6", "table", batch=6, prefix=1500, new=1),
        # a full serving batch, prompts and decodes mixed, and the pool runs out towards its end
        _case("table_serve_b2048", "table", batch=2048, prefix=8192, new=300, short=True),
        # the sixteen drafts of one decode step go into the cache
        _case("kv4_store_step", "store", rows=16),
        # the prompts of a batch, packed
        _case("kv4_store_prompts", "store", rows=16000),
        # plain decoding of one sequence: few bytes, the split over the keys decides
        _case("kv4_ar_8b_b1", "kv4", prefix=8000),
        # a serving batch on long contexts, one token each: the 4-bit cache streams
        _case("kv4_ar_8b_b32", "kv4", batch=32, prefix=8192, ragged=True),
        # a decode step of eight sequences, sixteen drafts each: the matrix cores decide
        _case("kv4_step_8b_b8_k16", "kv4", batch=8, prefix=8192, ragged=True, **_step(16)),
        # the second half of a long prompt on the small model, with its first mask block
        _case("kv4_prefill_1p5b", "kv4", heads="1p5b", prefix=1000, **_prefill(1999, 16)),
        # one token each over a window of a long text
        _case("window_ar_8b_b16", "window", batch=16, prefix=8192, ragged=True, window=1024, sinks=4),
        # a decode step of the small model, the window not a multiple of anything
        _case("window_step_1p5b_k16", "window", heads="1p5b", prefix=4096, window=1000, sinks=4, **_step(16)),
        # a pass of a long prompt
        _case("window_prefill_8b", "window", prefix=2048, window=1024, sinks=16, **_prefill(2048, 16)),
        # the small fp32 model's step
        _case("window_step_tiny_f32", "window", heads="tiny", dtype="f32", prefix=200, window=64, sinks=3, **_step(4)),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["table", "store", "kv4", "kv4", "kv4", "window", "window", "window"])
    if kind == "table":
        return _case(None, kind, batch=_log_int(rng, 1, 2048), prefix=_log_int(rng, 1, 8192), new=_log_int(rng, 1, 300),
                     short=rng.random() < 0.3)
    heads = rng.choice(["8b", "8b", "1p5b", "1p5b", "small", "tiny"])
    dtype = "f32" if heads == "tiny" or (heads == "small" and rng.random() < 0.5) else "bf16"
    if kind == "store":
        return _case(None, kind, heads=heads, dtype=dtype, rows=_log_int(rng, 1, 16000))
    f32 = dtype == "f32"
    prefix = _log_int(rng, 1, 1024 if f32 else 8192)
    window = _log_int(rng, 1, 4096) if kind == "window" or rng.random() < 0.3 else 0
    sinks = rng.choice([0, 1, 4, 4, 16, 37]) if window else 0
    rows = rng.choice(["ar", "ar", "step", "step", "prefill"])
    c = {"heads": heads, "dtype": dtype, "prefix": prefix, "window": window, "sinks": sinks}
    if rows == "ar":
        c.update(batch=_log_int(rng, 1, 32))
    elif rows == "step":
        k = rng.choice([1, 2, 3, 4, 8, 11, 16])
        c.update(batch=_log_int(rng, 1, 4 if f32 else 8), **_step(k))
    else:
        c.update(batch=rng.randint(1, 2), **_prefill(_log_int(rng, 5, 300 if f32 else 1500), rng.choice([4, 8, 16])))
    c["ragged"] = c["batch"] > 1
    return _case(None, kind, **c)


# ---------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _lengths(case):
    """Prefix of every sequence: all alike, or spread from a half to the whole of it."""
    B, P = case["batch"], case["prefix"]
    if not case["ragged"] or B == 1:
        return [P] * B
    return [max(1, P - i * P // (2 * B)) for i in range(B)]


def _normal(g, shape, dtype):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(generator=g).to(dtype)


def _pages(pool, nb):
    """The four parts of the 4-bit pages [page][kv head][bytes]: K codes by block, token and byte, V codes by token
    quad, group of eight elements, token and byte, and the scales of both by block and token."""
    a, s = 256 * nb, 16 * nb
    return (pool[..., :a].unflatten(-1, (nb, 16, 16)), pool[..., a:2 * a].unflatten(-1, (4, 4 * nb, 4, 4)),
            pool[..., 2 * a:2 * a + s].unflatten(-1, (nb, 16)), pool[..., 2 * a + s:].unflatten(-1, (nb, 16)))


def _quantise(x):
    """x [..., head_dim] fp32 -> (codes [..., nb, 32] uint8, scale bytes [..., nb]).  A block's exponent is the smallest
    that keeps its largest magnitude within 7 (half a step above the largest code, 6); codes go to the nearest, ties to even."""
    b = x.unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1)
    bits = amax.view(torch.int32)
    byte = ((bits >> 23) - 2 + ((bits & 0x7fffff) > 0x600000).int()).clamp(2, 252)
    y = b.abs() * torch.exp2((127 - byte).float()).unsqueeze(-1)
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=x.device)
    code = (y > edges[0]).int() + (y >= edges[1]).int() + (y > edges[2]).int() + (y >= edges[3]).int()
    code = code + (y > edges[4]).int() + (y >= edges[5]).int() + (y > edges[6]).int()
    return (code + 8 * torch.signbit(b).int()).to(torch.uint8), byte.to(torch.uint8)


def _put(pool, nb, page, slot, k, v):
    """Rows k, v [n][kv head][head_dim] fp32 into the pages, row i at slot[i] of page[i]."""
    kc, vc, ks, vs = _pages(pool, nb)
    for x, codes, scales, in_k in ((k, kc, ks, True), (v, vc, vs, False)):
        code, byte = _quantise(x)
        pair = (code[..., 0::2] | (code[..., 1::2] << 4)).flatten(-2)          # [n][kv head][head_dim / 2]
        if in_k:
            codes[page, :, :, slot, :] = pair.unflatten(-1, (nb, 16))
        else:
            codes[page, :, slot // 4, :, slot % 4, :] = pair.unflatten(-1, (4 * nb, 4))
        scales[page, :, :, slot] = byte


def _get(pool, nb, page, slot):
    """The values that page and slot (of any one shape) hold: K and V, [...][kv head][head_dim] fp32."""
    kc, vc, ks, vs = _pages(pool, nb)
    level = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=pool.device)
    shape = page.shape
    page, slot = page.reshape(-1), slot.reshape(-1)
    got = []
    for byte, scale in ((kc[page, :, :, slot, :], ks[page, :, :, slot]),
                        (vc[page, :, slot // 4, :, slot % 4, :], vs[page, :, :, slot])):
        byte = byte.flatten(-2)
        x = level[torch.stack((byte & 15, byte >> 4), -1).flatten(-2).int()].unflatten(-1, (nb, 32))
        got.append((x * torch.exp2(scale.float() - 127).unsqueeze(-1)).flatten(-2).unflatten(0, shape))
    return got


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    st = {"case": case}
    if kind == "table":
        return _prepare_table(case, g, st)
    n_q, n_kv, hd = HEADS[case["heads"]]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    nb = hd // 32
    if kind == "store":
        rows = case["rows"]
        n_pages = rows // PAGE + 9
        slots = torch.randperm(n_pages * PAGE, generator=g, device=DEV)[:rows].to(torch.int32)
        if rows > 8:
            slots[rows // 2] = -1                          # a padded row
        spread = torch.empty(rows, n_kv, 1, device=DEV).normal_(generator=g).exp()      # tokens differ in size
        st.update(slots=slots, n_pages=n_pages, k=(_normal(g, (rows, n_kv, hd), torch.float32) * spread).to(dt),
                  v=_normal(g, (rows, n_kv, hd), dt),
                  pool=torch.zeros(n_pages + 1, n_kv, 544 * nb, dtype=torch.uint8, device=DEV),
                  k_out=torch.empty(rows, n_kv, hd, dtype=dt, device=DEV), v_out=torch.empty(rows, n_kv, hd, dtype=dt, device=DEV))
    else:
        lens = _lengths(case)
        B, nc, nm = case["batch"], case["nc"], case["nb"] * case["bl"]
        R = nc + nm
        pps = -(-(max(lens) + nc) // PAGE)
        n_pages = B * pps + 3
        st.update(lens=torch.tensor(lens, dtype=torch.int32, device=DEV), n_pages=n_pages, pps=pps, hint=max(lens),
                  table=torch.randperm(n_pages, generator=g, device=DEV)[:B * pps].view(B, pps).to(torch.int32),
                  q=_normal(g, (B, R, n_q, hd), dt), out=torch.empty(B, R, n_q, hd, dtype=dt, device=DEV))
        new = nm if kind == "kv4" else R                   # over 4 bits the causal rows are in the cache already
        st.update(k_new=_normal(g, (B, new, n_kv, hd), dt), v_new=_normal(g, (B, new, n_kv, hd), dt))
        if kind == "kv4":
            st["pool"] = torch.zeros(n_pages + 1, n_kv, 544 * nb, dtype=torch.uint8, device=DEV)
            for p0 in range(0, n_pages, 2048):
                p = torch.arange(p0, min(n_pages, p0 + 2048), device=DEV).repeat_interleave(PAGE)
                s = torch.arange(p.numel(), device=DEV) % PAGE
                _put(st["pool"], nb, p, s, _normal(g, (p.numel(), n_kv, hd), torch.float32),
                     _normal(g, (p.numel(), n_kv, hd), torch.float32))
        else:
            st["k_pages"] = _normal(g, (n_pages, n_kv, PAGE, hd), dt)
            st["v_pages"] = _normal(g, (n_pages, n_kv, hd, PAGE), dt)
    if own:                                                # the handle and the workspace that a program keeps
        import paper_2511_08923_amd as T
        code = T.TIDAR_BF16 if case["dtype"] == "bf16" else T.TIDAR_F32
        cfg = T.tidar_config(1, n_q * hd, n_q, n_kv, hd, 512, 512, 0, code, PAGE, 16, case.get("batch", 1), 511, 1e4, 1e-6)
        st["ctx"] = T.tidar_create(cfg)
        if "pool" in st:
            st["kv4"] = T.tidar_kv4_cache(st["pool"].data_ptr(), st["table"].data_ptr() if "table" in st else None,
                                          st.get("pps", 0), st["n_pages"])
        if "k_pages" in st:
            st["kv"] = T.tidar_kv_cache(st["k_pages"].data_ptr(), st["v_pages"].data_ptr(), st["table"].data_ptr(),
                                        st["pps"], st["n_pages"])
        if "table" in st:
            n = T.tidar_attention_workspace_bytes(st["ctx"], case["batch"], case["nc"], case["nb"], case["bl"], st["hint"])
            st["ws"] = torch.empty(n, dtype=torch.uint8, device=DEV)
    return st


def _table_lengths(case):
    """Lengths and new rows of every sequence: decodes of one row, and every fourth a prompt's chunk of up to `new`."""
    B, P = case["batch"], case["prefix"]
    length = [max(0, P - i * P // B) for i in range(B)]
    new = [case["new"] if case["new"] == 1 else 1 + (7 * i) % case["new"] if i % 4 == 1 else 1 for i in range(B)]
    return length, new


def _table_pages(length, new):
    """Pages of every sequence (every third has one to spare, that a rejected draft left behind) and how many it misses."""
    held = [-(-p // PAGE) + (i % 3 == 2) for i, p in enumerate(length)]
    return held, [max(0, -(-(p + n) // PAGE) - h) for p, n, h in zip(length, new, held)]


def _prepare_table(case, g, st):
    length, new = _table_lengths(case)
    B = case["batch"]
    pps = max(-(-(p + n) // PAGE) for p, n in zip(length, new)) + 2
    held, need = _table_pages(length, new)
    n_free = max(1, sum(need) * 9 // 10) if case["short"] else sum(need) + 5
    n_pages = sum(held) + n_free + 4096                    # the rest belongs to nobody here
    ids = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    h = torch.tensor(held, device=DEV)
    at = (h.cumsum(0) - h)[:, None] + torch.arange(pps, device=DEV)
    table = torch.where(torch.arange(pps, device=DEV) < h[:, None], ids[at.clamp(max=n_pages - 1)], -1).to(torch.int32)
    i32 = {"dtype": torch.int32, "device": DEV}
    st.update(lens=torch.tensor(length, **i32), new=torch.tensor(new, **i32), free=ids[sum(held):sum(held) + n_free].contiguous(), table=table,
              n_pages=n_pages, held=torch.tensor(held, **i32), held_out=torch.empty(B, **i32), start=torch.empty(B + 1, **i32), slots=torch.empty(sum(new) + 3, **i32),
              granted=torch.empty(B, **i32), taken=torch.empty(1, **i32))
    if own:
        import paper_2511_08923_amd as T
        st["ctx"] = T.tidar_create(T.tidar_config(1, 128, 4, 4, 32, 512, 512, 0, T.TIDAR_F32, PAGE, 4, B, 511, 1e4, 1e-6))
    return st


# ---------------------------------------------------------------- one pass
def run(st):
    kind = st["case"]["kind"]
    if own:
        return _own(st)
    return {"table": _plain_table, "store": _plain_store}.get(kind, _plain_attention)(st)


def _own(st):
    import paper_2511_08923_amd as T
    c = st["case"]
    if c["kind"] == "table":
        T.tidar_table_extend(st["ctx"], c["batch"], st["lens"], st["new"], st["held"], st["free"], st["free"].numel(), st["table"],
                             st["n_pages"], st["start"], st["slots"], st["held_out"], st["granted"], st["taken"])
        return {k: st[k] for k in ("table", "start", "slots", "held_out", "granted", "taken")}
    if c["kind"] == "store":
        T.tidar_kv4_store(st["ctx"], st["kv4"], 0, c["rows"], st["slots"], st["k"], st["v"])
        T.tidar_kv4_load(st["ctx"], st["kv4"], 0, c["rows"], st["slots"], st["k_out"], st["v_out"])
        return {"k": st["k_out"], "v": st["v_out"]}
    rows = (c["nc"], c["nb"], c["bl"], c["cond0"], c["window"], c["sinks"])
    if c["kind"] == "kv4":
        T.tidar_kv4_attention(st["ctx"], st["kv4"], 0, c["batch"], st["lens"], st["q"], st["k_new"], st["v_new"], *rows,
                              st["out"], st["hint"], st["ws"])
        return {"out": st["out"]}
    T.tidar_window_attention(st["ctx"], st["kv"], 0, c["batch"], st["lens"], st["q"], st["k_new"], st["v_new"], *rows,
                             st["out"], st["hint"], st["ws"])
    return {"out": st["out"], "k_pages": st["k_pages"], "v_pages": st["v_pages"]}


def _plain_table(st):
    P, n, table, free = st["lens"].long(), st["new"].long(), st["table"], st["free"]
    B, pps = table.shape
    held = st["held"].long()
    need = ((P + n + PAGE - 1) // PAGE - held).clamp(min=0)
    off, end = need.cumsum(0) - need, n.cumsum(0)
    ok = (need == 0) | (off + need <= free.numel())                                 # nothing needed, nothing to wait for
    j = torch.arange(pps, device=DEV)
    take = ok[:, None] & (j >= held[:, None]) & (j < (held + need)[:, None])
    at = (off[:, None] + j - held[:, None]).clamp(0, free.numel() - 1)
    table.copy_(torch.where(take, free[at], table))
    r = torch.arange(st["slots"].numel(), device=DEV)
    b = torch.searchsorted(end, r, right=True).clamp(max=B - 1)
    pos = (P[b] + r - (end[b] - n[b])).clamp(0, pps * PAGE - 1)
    slots = torch.where(ok[b] & (r < end[-1]), table[b, pos // PAGE] * PAGE + pos % PAGE, -1).to(torch.int32)
    start = torch.cat((torch.zeros_like(end[:1]), end)).to(torch.int32)
    taken = torch.where(ok & (need > 0), off + need, 0).amax().view(1).to(torch.int32)
    now = torch.where(ok, held + need, held).to(torch.int32)
    return {"table": table, "start": start, "slots": slots, "held_out": now, "granted": ok.to(torch.int32), "taken": taken}


def _plain_store(st):
    nb = HEADS[st["case"]["heads"]][2] // 32
    slots = st["slots"].long()
    real = slots >= 0
    page, slot = torch.where(real, slots // PAGE, st["n_pages"]), torch.where(real, slots % PAGE, 0)    # padding: the spare page
    _put(st["pool"], nb, page, slot, st["k"].float(), st["v"].float())
    k, v = _get(st["pool"], nb, page, slot)
    keep = real[:, None, None]
    return {"k": torch.where(keep, k, 0).to(st["k"].dtype), "v": torch.where(keep, v, 0).to(st["v"].dtype)}


def _plain_attention(st):
    c = st["case"]
    n_q, n_kv, hd = HEADS[c["heads"]]
    B, nc, bl = c["batch"], c["nc"], c["bl"]
    nm, R, L, dev = c["nb"] * bl, c["nc"] + c["nb"] * bl, st["lens"].long()[:, None], DEV
    at = torch.arange(st["hint"] + nc, device=dev)
    page, slot = st["table"].long()[:, at // PAGE], (at % PAGE).expand(B, -1)
    if c["kind"] == "kv4":
        k, v = _get(st["pool"], hd // 32, page, slot)                               # [B][position][kv head][head_dim]
        k_mask, v_mask = st["k_new"].float(), st["v_new"].float()
    else:
        i = torch.arange(nc, device=dev)
        new_page, new_slot = st["table"].long().gather(1, (L + i) // PAGE), (L + i) % PAGE
        st["k_pages"][new_page, :, new_slot, :] = st["k_new"][:, :nc]
        st["v_pages"][new_page, :, :, new_slot] = st["v_new"][:, :nc]
        k, v = st["k_pages"][page, :, slot, :].float(), st["v_pages"][page, :, :, slot].float()
        k_mask, v_mask = st["k_new"][:, nc:].float(), st["v_new"][:, nc:].float()
    k, v = torch.cat((k, k_mask), 1).transpose(1, 2).contiguous(), torch.cat((v, v_mask), 1).transpose(1, 2).contiguous()
    r, m = torch.arange(R, device=dev), torch.arange(nm, device=dev)
    block = torch.where(r < nc, -1, (r - nc) // bl)                                 # the rows' blocks, what they see, where they are
    seen = torch.where(r < nc, r + 1, c["cond0"] + block)
    place = L + torch.where(r < nc, r, seen + (r - nc) % bl)                        # [B][R]
    key = torch.cat((at.expand(B, -1), L + c["cond0"] + m // bl + m % bl), 1)       # the keys' positions
    see = torch.cat((at < (L + seen)[:, :, None], (block[:, None] == m // bl).expand(B, -1, -1)), 2)
    if c["window"]:
        see = see & ((key[:, None, :] > place[:, :, None] - c["window"]) | (key[:, None, :] < c["sinks"]))
    q = st["q"].float().view(B, R, n_kv, n_q // n_kv, hd).permute(0, 2, 3, 1, 4).reshape(B, n_kv, -1, hd)
    s = (torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(hd)).view(B, n_kv, -1, R, key.shape[1])
    s = s.masked_fill(~see[:, None, None], -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    p = (p / p.sum(-1, keepdim=True)).view(B, n_kv, -1, key.shape[1])
    out = torch.matmul(p, v).view(B, n_kv, -1, R, hd).permute(0, 3, 1, 2, 4).reshape(B, R, n_q, hd).to(st["q"].dtype)
    return {"out": out} if c["kind"] == "kv4" else {"out": out, "k_pages": st["k_pages"], "v_pages": st["v_pages"]}


# ---------------------------------------------------------------- what a pass cannot do without
def _pairs(case):
    """(query, key) pairs that are seen and keys that any row sees, over all sequences."""
    nc, nb, bl, w, t = case["nc"], case["nb"], case["bl"], case["window"], case["sinks"]
    pairs = keys = 0
    for L in _lengths(case):
        rows = [(L + r, L + r + 1) for r in range(nc)]                              # position, cached keys in front of it
        rows += [(L + case["cond0"] + j + s, L + case["cond0"] + j) for j in range(nb) for s in range(bl)]
        low = L + nc
        for pos, n in rows:
            lo = max(0, min(n, pos - w + 1)) if w else 0
            pairs += n - lo + min(lo, t)
            low = min(low, lo)
        for s in range(bl if nb else 0):                                            # the block's own keys
            pairs += nb * (bl - max(0, s - w + 1) if w else bl)
        keys += L + nc - low + min(low, t) + nb * bl
    return pairs, keys


def work(case):
    if case["kind"] == "table":
        length, new = _table_lengths(case)
        taken = sum(_table_pages(length, new)[1])
        return {"bytes": 4 * (4 * len(new) + 2 * taken + 3 * len(new) + 1 + sum(new) + 4), "flops": 0}
    n_q, n_kv, hd = HEADS[case["heads"]]
    size = 2 if case["dtype"] == "bf16" else 4
    row4 = n_kv * (hd // 2 + hd // 32)
    if case["kind"] == "store":
        return {"bytes": case["rows"] * (4 + 2 * (2 * n_kv * hd * size + row4)), "flops": 0}
    pairs, keys = _pairs(case)
    mask = case["batch"] * case["nb"] * case["bl"]
    R = case["nc"] + case["nb"] * case["bl"]
    cached = 2 * (keys - mask) * (row4 if case["kind"] == "kv4" else n_kv * hd * size)
    io = 2 * case["batch"] * R * n_q * hd * size + 2 * mask * n_kv * hd * size
    if case["kind"] == "window":
        io += 2 * case["batch"] * case["nc"] * n_kv * hd * size                     # the new rows go into the cache
    return {"bytes": cached + io, "flops": 4 * hd * n_q * pairs}


# ---------------------------------------------------------------- the definition, in 64 bits
def exact(case, seed):
    if case["kind"] == "table":
        return None
    st = prepare(case, seed)
    nb = HEADS[case["heads"]][2] // 32
    if case["kind"] == "store":
        real = (st["slots"] >= 0)[:, None, None].double()
        return {"k": real * _nearest(st["k"].double()), "v": real * _nearest(st["v"].double())}
    outs = []
    for b, L in enumerate(_lengths(case)):
        outs.append(_exact_sequence(case, st, b, L, nb))
    out = torch.stack(outs)
    if case["kind"] == "kv4":
        return {"out": out}
    kp, vp = st["k_pages"].double(), st["v_pages"].double()
    for b, L in enumerate(_lengths(case)):
        for i in range(case["nc"]):
            page, slot = int(st["table"][b, (L + i) // PAGE]) if i == 0 or (L + i) % PAGE == 0 else page, (L + i) % PAGE
            kp[page, :, slot] = st["k_new"][b, i].double()
            vp[page, :, :, slot] = st["v_new"][b, i].double()
    return {"out": out, "k_pages": kp, "v_pages": vp}


def _nearest(x):
    """Every element of x [..., head_dim] (64 bits) as the nearest of its block's 15 levels; of two as near, the one whose
    index in 0, 1/2, 1, 3/2, 2, 3, 4, 6 is even."""
    y = x.reshape(*x.shape[:-1], -1, 32)
    top = y.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 7))
    e = torch.where(top > 7 * torch.exp2(e), e + 1, torch.where(top <= 7 * torch.exp2(e - 1), e - 1, e)).clamp(-125, 125)
    level = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    z, best, far = (y / torch.exp2(e)).abs(), torch.zeros_like(y), torch.full_like(y, math.inf)
    for i in (0, 2, 4, 6, 1, 3, 5, 7):                      # the even ones first: another has to be nearer
        d = (z - level[i]).abs()
        best, far = torch.where(d < far, level[i], best), torch.minimum(d, far)
    return (torch.sign(y) * best * torch.exp2(e)).reshape(x.shape)


def _exact_rows4(st, b, n, nb):
    """Cached K and V [n][kv head][head_dim] of sequence b in 64 bits, nibble by nibble from the bytes."""
    at = torch.arange(n, device=DEV)
    block = st["pool"][st["table"][b].long()[at // PAGE]].long()                    # [n][kv head][bytes]
    t = (at % PAGE)[:, None, None]
    d = torch.arange(32 * nb, device=DEV)[None, None, :]
    got = []
    for code_at, scale_at in (((d // 32) * 256 + t * 16 + (d % 32) // 2, 512 * nb + (d // 32) * 16 + t),
                              (256 * nb + (t // 4) * 64 * nb + (d // 8) * 16 + (t % 4) * 4 + (d % 8) // 2,
                               528 * nb + (d // 32) * 16 + t)):
        shape = (n, block.shape[1], 32 * nb)
        nibble = (block.gather(2, code_at.expand(shape)) >> (4 * (d % 2))) & 15
        exp, half = (nibble >> 1) & 3, (nibble & 1).double()
        mag = torch.where(exp == 0, half / 2, (1 + half / 2) * torch.exp2((exp - 1).double()))
        scale = torch.exp2((block.gather(2, scale_at.expand(shape)) - 127).double())
        got.append(torch.where(nibble > 7, -mag, mag) * scale)
    return got


def _exact_sequence(case, st, b, L, nb):
    n_q, n_kv, hd = HEADS[case["heads"]]
    nc, bl, w, t = case["nc"], case["bl"], case["window"] or 1 << 40, case["sinks"]
    if case["kind"] == "kv4":
        k, v = _exact_rows4(st, b, L + nc, nb)
    else:
        at = torch.arange(L, device=DEV)
        page = st["table"][b].long()[at // PAGE]
        k, v = st["k_pages"][page, :, at % PAGE, :].double(), st["v_pages"][page, :, :, at % PAGE].double()
    k, v = torch.cat((k, st["k_new"][b].double())), torch.cat((v, st["v_new"][b].double()))
    where = list(range(L + nc)) + [L + case["cond0"] + j + s for j in range(case["nb"]) for s in range(bl)]
    where = torch.tensor(where, device=DEV)
    n_cache = L + nc
    group = n_q // n_kv
    out = torch.empty(st["q"].shape[1], n_q, hd, dtype=torch.float64, device=DEV)
    rows = [(0, nc, -1)] + [(nc + j * bl, nc + (j + 1) * bl, j) for j in range(case["nb"])]
    for r0, r1, j in rows:                                  # the causal rows, then block by block
        if j < 0:
            pos = L + torch.arange(r0, r1, device=DEV)
            see = (where <= pos[:, None]) & (torch.arange(len(where), device=DEV) < n_cache)
        else:
            pos = L + case["cond0"] + j + torch.arange(bl, device=DEV)
            i = torch.arange(len(where), device=DEV)
            mine = (i >= n_cache + j * bl) & (i < n_cache + (j + 1) * bl)
            see = ((i < L + case["cond0"] + j) | mine).expand(bl, -1)
        see = see & ((pos[:, None] - where < w) | (where < t))
        for h in range(n_kv):
            q = st["q"][b, r0:r1, h * group:(h + 1) * group].double().transpose(0, 1)          # [group][rows][hd]
            s = torch.matmul(q, k[:, h].t().contiguous()) * hd ** -0.5
            s = torch.where(see, s, torch.full_like(s, -math.inf))
            out[r0:r1, h * group:(h + 1) * group] = torch.matmul(torch.softmax(s, -1), v[:, h].contiguous()).transpose(0, 1)
    return out
