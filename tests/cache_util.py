"""The operators around the paged cache from their definitions, in 64 bits and without the library: the 4-bit levels, the
page format, the mask with window and sinks, attention and page tables.  Plain loops and searches, for small sizes."""
import math

import torch

LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def quantise(x):
    """x [..., hd] float64 -> (signed codes [..., hd], scale bytes [..., nb]).  NaN blocks: byte 255, codes unspecified (0)."""
    hd = x.shape[-1]
    nb = (hd + 31) // 32
    pad = torch.zeros(*x.shape[:-1], nb * 32, dtype=torch.float64)
    pad[..., :hd] = x
    blk = pad.unflatten(-1, (nb, 32))
    amax = blk.abs().amax(-1)
    odd = ~torch.isfinite(blk).all(-1)
    e = torch.full_like(amax, 125.0)
    for i in range(124, -126, -1):                       # the smallest that still holds 1/7 of the largest magnitude
        e = torch.where(amax <= 7 * 2.0 ** i, torch.full_like(e, float(i)), e)
    mag = (blk / torch.exp2(e).unsqueeze(-1)).abs()
    dist = (mag.unsqueeze(-1) - torch.tensor(LEVELS, dtype=torch.float64)).abs()
    dist = torch.where(torch.isnan(dist), torch.zeros_like(dist), dist)
    order = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7])       # ties go to the even code: even codes first, argmin takes the first
    code = order[dist[..., order].argmin(-1)]
    code = torch.where(odd.unsqueeze(-1), torch.zeros_like(code), code + 8 * (torch.signbit(blk)).long())
    byte = torch.where(odd, torch.full_like(e, 255.0), e + 127).long()
    return code.flatten(-2), byte


def values(code, byte, hd):
    lv = torch.tensor(LEVELS + [-x for x in LEVELS], dtype=torch.float64)
    x = lv[code].unflatten(-1, (-1, 32)) * torch.exp2(byte.double() - 127).unsqueeze(-1)
    x = torch.where((byte == 255).unsqueeze(-1), torch.full_like(x, math.nan), x)
    return x.flatten(-2)[..., :hd]


def fake4(x):
    """The values that a cache in 4 bits holds for x, float64."""
    code, byte = quantise(x.double())
    return values(code, byte, x.shape[-1])


def put_rows(pool, hd, slots, k, v):
    """Rows k, v [n][n_kv][hd] into the byte pool [pages][n_kv][544 nb] at the slots, byte by byte."""
    nb = (hd + 31) // 32
    for x, is_k in ((k, True), (v, False)):
        code, byte = quantise(x.double())
        for i, s in enumerate(slots):
            if s < 0 or s >= pool.shape[0] * 16:
                continue
            page, t = s // 16, s % 16
            pair = (code[i, :, 0::2] + 16 * code[i, :, 1::2]).to(torch.uint8)           # [n_kv][16 nb]
            for j in range(16 * nb):                     # byte j: elements 2j, 2j + 1
                at = (j // 16) * 256 + t * 16 + j % 16 if is_k else 256 * nb + (t // 4) * 64 * nb + (j // 4) * 16 + (t % 4) * 4 + j % 4
                pool[page, :, at] = pair[:, j]
            for blk in range(nb):
                pool[page, :, (512 if is_k else 528) * nb + blk * 16 + t] = byte[i, :, blk].to(torch.uint8)


def mask(L, nc, nb, bl, cond0, window, sinks):
    """[R][L + nc + nb * bl] bool: the hybrid mask, from what it says about every single pair."""
    keys = [(p, -1) for p in range(L + nc)] + [(L + cond0 + j + s, j) for j in range(nb) for s in range(bl)]
    rows = [(L + r, -1, L + r + 1) for r in range(nc)]
    rows += [(L + cond0 + j + s, j, L + cond0 + j) for j in range(nb) for s in range(bl)]
    kp, kb = (torch.tensor([k[i] for k in keys]) for i in range(2))
    out = torch.zeros(len(rows), len(keys), dtype=torch.bool)
    for i, (pos, blk, below) in enumerate(rows):
        see = ((kb < 0) & (kp < below)) | ((kb == blk) & (blk >= 0))
        if window:
            see &= (kp > pos - window) | (kp < sinks)
        out[i] = see
    return out


def attention(q, k, v, see):
    """q [R][n_q][hd], k, v [K][n_kv][hd] float64, see [R][K].  Returns the output and sum_k w |v|, which bounds how far rounded
    weights can move it.  A masked key takes no part, whatever it holds."""
    R, n_q, hd = q.shape
    n_kv = k.shape[1]
    out, size = torch.empty_like(q), torch.empty_like(q)
    for h in range(n_q):
        g = h // (n_q // n_kv)
        kk, vv = k[:, g], v[:, g]
        s = torch.where(see, (q[:, h] @ torch.nan_to_num(kk, 0.0, 0.0, 0.0).T) / math.sqrt(hd), torch.tensor(-math.inf, dtype=torch.float64))
        bad_k = ~torch.isfinite(kk).all(-1)              # a visible key that is not a number
        w = torch.softmax(s, -1)
        o = w @ torch.nan_to_num(vv, 0.0, 0.0, 0.0)
        for i in torch.nonzero(~torch.isfinite(vv).all(-1)).flatten().tolist():
            odd = torch.where(torch.isfinite(vv[i]), torch.zeros_like(vv[i]), vv[i])
            o = torch.where(see[:, i:i + 1], o + odd, o)
        o[(see & bad_k).any(-1)] = math.nan
        out[:, h] = o
        size[:, h] = w @ torch.nan_to_num(vv, 0.0, 0.0, 0.0).abs()
    return out, size


def extend(prefix, new, has, free, table, n_pages, slot_cap):
    """Page tables and slot maps, one sequence after another.  Lists in; (table, row_start, slots, held_out, granted, n_taken) out."""
    table = [list(r) for r in table]
    cap, now = len(table[0]) * 16, list(has)
    start, slots, granted, taken, off = [0], [-1] * slot_cap, [], 0, 0
    for b, (P, n) in enumerate(zip(prefix, new)):
        rows = n if 0 <= n <= cap else 0
        row0 = start[-1]
        start.append(row0 + rows)
        if rows != n or P < 0 or P + n > cap or has[b] > len(table[0]) or -(-P // 16) > has[b]:
            granted.append(-1)
            continue
        held, need = has[b], max(0, -(-(P + n) // 16) - has[b])
        part = free[off:off + need]
        room = (need == 0 or off + need <= len(free)) and (rows == 0 or row0 + rows <= slot_cap)
        off += need
        if not room:
            granted.append(0)
            continue
        if need:
            taken = off
        old = table[b][P // 16:min(held, -(-(P + n) // 16))] if n > 0 else []
        if any(not 0 <= p < n_pages for p in part + old):
            granted.append(-1)
            continue
        granted.append(1)
        now[b] = held + need
        table[b][held:held + need] = part
        for i in range(n):
            slots[row0 + i] = table[b][(P + i) // 16] * 16 + (P + i) % 16
    return table, start, slots, now, granted, taken
