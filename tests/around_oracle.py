"""The calls around the reading of a retrieval from their definitions in 64 bits on the CPU, and how far a kernel's result may
be off.

Bounds.  u: the largest relative error of a rounding to the result's type, half of its last place (bfloat16 2^-8, float16
2^-11, float32 2^-24); ``least`` what is below its normal numbers.  Everything before that rounding is done in 32 bits: a sum of n terms is
off by at most n 2^-24 of the terms' sizes, whatever its order."""
import math

import torch

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}
E32 = 2.0 ** -24
MOST = {t: torch.finfo(t).max for t in UNIT}


def check(got, want, tol, what=""):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fine = want.isfinite()
    assert torch.equal(got[~fine].isnan(), want[~fine].isnan()) and torch.equal(got[~fine].nan_to_num(7.0), want[~fine].nan_to_num(7.0)), what
    far = (got - want).abs() - tol
    far = torch.where(fine, far, -1.0)
    far = torch.where(got.isnan() & fine, math.inf, far)
    assert far.numel() == 0 or far.max() <= 0, f"{what}: {int((far > 0).sum())} of {far.numel()} off, worst by {far.max():.3e} at {far.argmax().item()}"


# ---------------------------------------------------------------- rows of a table
def embed(table, ids, scale=1.0):
    ids = ids.cpu().long()
    good = (ids >= 0) & (ids < table.shape[0])
    want = torch.zeros(*ids.shape, table.shape[1], dtype=torch.float64)
    want[good] = table.detach().cpu()[ids[good]].double() * scale
    return want, (UNIT[table.dtype] + 2 * E32) * want.abs() + LEAST[table.dtype]


def embed_grad(dout, ids, num_entities, scale=1.0, out=None, dtype=None):
    """``out``: what stood there, of an accumulating call (then rows without an id come back as they were, exactly)."""
    dtype = dtype or dout.dtype
    ids, x = ids.cpu().reshape(-1).long(), dout.detach().cpu().double().reshape(ids.numel(), dout.shape[-1])
    good = (ids >= 0) & (ids < num_entities)
    sums, sizes, n = (torch.zeros(num_entities, w, dtype=torch.float64) for w in (x.shape[1], x.shape[1], 1))
    sums.index_add_(0, ids[good], x[good])
    sizes.index_add_(0, ids[good], x[good].abs())
    n.index_add_(0, ids[good], torch.ones(int(good.sum()), 1, dtype=torch.float64))
    want, tol = scale * sums, abs(scale) * sizes * (n + 2) * E32
    if out is not None:
        old = out.detach().cpu().double()
        want, tol = want + old, tol + E32 * (want.abs() + old.abs())
    tol = tol + UNIT[dtype] * (want.abs() + tol) + LEAST[dtype]
    return want, torch.where(n > 0, tol, 0.0)


# ---------------------------------------------------------------- answers
def policy(logits, target, advantage=None, old=None, ref=None, weight=None, clip=(0.2, 0.2), kl=0.0, scale=1.0, mask=None, mask_row=None,
           dloss=1.0):
    """(results, bounds): "logp" and "lse", and with an advantage "loss" and "dlogits".

    An exponential's argument (x - top) scale is off by 2 roundings, the exponential by two more; a sum's terms go by 64 threads at
    least, or V / 512 in turn (rows of up to 1,024 by 16 threads, 64 terms each in four sums: 22 in turn); so each of exp's relative errors enters lse by its share p."""
    (R, V), dtype = logits.shape, logits.dtype
    x = logits.detach().cpu().double() * scale
    hidden = torch.zeros(R, V, dtype=torch.bool)
    if mask is not None:
        bits = ((mask.cpu()[:, :, None] >> torch.arange(64)) & 1).reshape(mask.shape[0], -1)[:, :V].bool()
        at = torch.arange(R) if mask_row is None else mask_row.cpu().long()
        inside = (at >= 0) & (at < mask.shape[0])
        hidden = torch.ones(R, V, dtype=torch.bool)
        hidden[inside] = ~bits[at[inside]]
    x = torch.where(hidden, -math.inf, x)
    lse = torch.logsumexp(x, 1) if V else torch.full((R,), -math.inf, dtype=torch.float64)
    safe = torch.where(lse == -math.inf, 0.0, lse)[:, None]
    p = torch.where(x == -math.inf, 0.0, torch.exp(x - safe))
    top = x.amax(1, keepdim=True) if V else torch.zeros(R, 1, dtype=torch.float64)
    below = torch.where(p > 0, (x - top).abs(), 0.0)
    in_turn = 80 + V / 512
    lse_tol = E32 * (in_turn + 8 + 4 * (p * below).sum(1) + 4 * torch.where(top == -math.inf, 0.0, top.abs()).squeeze(1) + 4 * safe.abs().squeeze(1))
    t = target.cpu().long()
    pads = (t < 0) | (t >= V)
    said = x.gather(1, t.clamp(0, V - 1)[:, None]).squeeze(1) if V else torch.full((R,), -math.inf, dtype=torch.float64)
    logp = torch.where(pads, 0.0, torch.where(said == -math.inf, -math.inf, said - safe.squeeze(1)))
    logp_tol = lse_tol + 4 * E32 * torch.where(logp == -math.inf, 0.0, logp.abs())
    res, tol = {"logp": logp, "lse": lse}, {"logp": logp_tol, "lse": lse_tol}
    if advantage is None:
        return res, tol
    counts = ~pads & (logp != -math.inf)
    lp = torch.where(counts, logp, 0.0)
    A = advantage.cpu().double()
    w = torch.where(counts, torch.ones(R, dtype=torch.float64) if weight is None else weight.cpu().double(), 0.0)
    o = lp if old is None else old.cpu().double()
    ratio = torch.where(counts, torch.exp(lp - o), 1.0)
    stopped = torch.where(A >= 0, ratio > 1 + clip[1], ratio < 1 - clip[0])
    bound = torch.where(A >= 0, 1 + clip[1] + 0 * A, 1 - clip[0] + 0 * A)
    loss, slope = -torch.where(stopped, bound, ratio) * A, -torch.where(stopped, 0.0, ratio) * A
    d = torch.zeros(R, dtype=torch.float64) if ref is None or not kl else torch.where(counts, ref.cpu().double() - lp, 0.0)
    loss = loss + kl * (torch.expm1(d) - d)
    slope = slope - kl * torch.expm1(d)
    # of logp's error: by the slope's size; of the ratio, its exponential and the products: a few roundings
    apart = (lp - o).abs()
    steep = ratio * A.abs() + kl * torch.exp(d)
    near = logp_tol + 4 * E32 * (1 + apart + d.abs() + lp.abs() + (0.0 if old is None else o.abs()))
    slope_tol = w.abs() * (steep * near * 1.1 + 8 * E32 * (steep + (bound * A).abs() + kl))
    loss_tol = w.abs() * (steep * near * 1.1 + 8 * E32 * (loss.abs() + steep + (bound * A).abs() + kl * (1 + d.abs())))
    loss, slope, loss_tol, slope_tol = (torch.where(counts, x, 0.0) for x in (loss, slope, loss_tol, slope_tol))  # whatever stands beside rows that do not count
    res["loss"] = (w * loss).sum()
    tol["loss"] = loss_tol.sum() + E32 * (w * loss).abs().sum()
    g, g_tol = (w * slope * scale * dloss)[:, None], (slope_tol * scale * abs(dloss))[:, None]
    hot = torch.zeros(R, V, dtype=torch.float64)
    if V:
        hot[torch.arange(R), t.clamp(0, V - 1)] = 1.0
    hot[~counts] = 0.0
    share_tol = p * (lse_tol[:, None] + 4 * E32 * (2 + torch.where(p > 0, (x - safe).abs() + x.abs(), 0.0)))
    res["dlogits"] = torch.where(counts[:, None], g * (hot - p), 0.0)
    tol["dlogits"] = g_tol * (hot - p).abs() + 1.1 * g.abs() * (share_tol + 4 * E32 * (hot - p).abs())
    tol["dlogits"] = torch.where(counts[:, None], tol["dlogits"] + UNIT[dtype] * (res["dlogits"].abs() + tol["dlogits"]) + LEAST[dtype], 0.0)
    # what rounds to more than the type holds (float16: from 65,520 on, half a step above its largest) is infinite
    over = res["dlogits"].abs() - tol["dlogits"] > torch.finfo(dtype).max * (1 + torch.finfo(dtype).eps / 4)
    res["dlogits"] = torch.where(over, torch.sign(res["dlogits"]) * math.inf, res["dlogits"])
    return res, tol


# ---------------------------------------------------------------- the end of a step
def clip(grads, max_norm, scale=1.0, to=None):
    """(norm, its bound, [(gradient, bound)])."""
    norm = abs(scale) * math.sqrt(math.fsum(float((g.detach().cpu().double() ** 2).sum()) for g in grads))
    by = scale * (max_norm / norm if norm > max_norm else 1.0)
    got = []
    for i, g in enumerate(grads):
        dtype = g.dtype if to is None else to[i]
        want = g.detach().cpu().double() * by
        got.append((want, (UNIT[dtype] + 4 * E32) * want.abs() + LEAST[dtype]))
    return torch.tensor(norm, dtype=torch.float64), torch.tensor(2 * E32 * norm, dtype=torch.float64), got


# ---------------------------------------------------------------- tables in 4 bits
def groups_of(dim):
    return (dim + 31) // 32


def row_bytes(kv_heads, dim):
    return -(-40 * kv_heads * groups_of(dim) // 16) * 16


def pack(keys, values):
    """uint8 rows from the definition, element by element, and where a quotient is so near a half that 32 bits may round it either way."""
    n, K, D = keys.shape
    G = groups_of(D)
    rows, near = torch.zeros(n, row_bytes(K, D), dtype=torch.uint8), torch.zeros(n, 2, K, D, dtype=torch.bool)
    for which, x in enumerate((keys, values)):
        x = x.detach().cpu().float()
        for g in range(G):
            part = x[:, :, 32 * g:32 * g + 32]
            low, high = part.amin(2), part.amax(2)
            base, scale = low.to(torch.bfloat16), ((high - low) / torch.tensor(15.0)).to(torch.bfloat16)
            bad = ~(part.isfinite().all(2) & base.isfinite() & scale.isfinite())
            nan = torch.tensor(0x7fc0, dtype=torch.int16).view(torch.bfloat16)
            base, scale = (torch.where(bad, nan, t) for t in (base, scale))
            s = scale.double()[:, :, None]
            ratio = torch.where(s > 0, (part.double() - base.double()[:, :, None]) / torch.where(s > 0, s, 1.0), 0.0)
            near[:, which, :, 32 * g:32 * g + 32] = ((ratio - ratio.floor()) - 0.5).abs() < 2.0 ** -16
            code = torch.where(bad[:, :, None], 0.0, ratio.round().clamp(0, 15)).to(torch.uint8)
            for i in range(part.shape[2]):
                d = 32 * g + i
                word = (i // 8) * G + g if which == 0 else d // 8
                at = which * 16 * K * G + torch.arange(K) * 16 * G + 4 * word + (d % 8) // 2
                rows[:, at] |= code[:, :, i] << (4 * (d % 2))
            at = 32 * K * G + 8 * (torch.arange(K) * G + g) + 4 * which
            for j, t in enumerate((scale, base)):
                two = t.contiguous().view(torch.uint8).view(n, K, 2)
                rows[:, at + 2 * j], rows[:, at + 2 * j + 1] = two[:, :, 0], two[:, :, 1]
    return rows, near


def unpack(rows, K, D):
    """(values, scales, bases) in 64 bits, each [2, n, K, D]: of keys, of values."""
    rows = rows.cpu()
    n, G = rows.shape[0], groups_of(D)
    got = torch.zeros(3, 2, n, K, D, dtype=torch.float64)
    heads = torch.arange(K)
    for which in (0, 1):
        for d in range(D):
            g, i = d // 32, d % 32
            word = (i // 8) * G + g if which == 0 else d // 8
            code = (rows[:, which * 16 * K * G + heads * 16 * G + 4 * word + (d % 8) // 2] >> (4 * (d % 2))) & 15
            at = 32 * K * G + 8 * (heads * G + g) + 4 * which
            scale, base = (torch.stack([rows[:, at + 2 * j], rows[:, at + 2 * j + 1]], 2).contiguous().view(torch.bfloat16).squeeze(2).double() for j in (0, 1))
            got[0, which, :, :, d], got[1, which, :, :, d], got[2, which, :, :, d] = base + scale * code.double(), scale, base
    return got


def read_packed(q, packed, off, entity=None, *, kv_heads, scale=None, cap=0.0, bias=None, buckets=None, hop=None, q_pos=None):
    """(results, bounds).  A score is made of scale x (16 + code) x q and of sums of q, all in 32 bits: off by some 2^-20 of the terms'
    sizes (128 terms, in any order).  The weights p x scale are rounded to q's type before the second product, with codes from -7.5 to 7.5;
    that product's terms are 16 + code, and what takes the 16 away."""
    Q, T, H, D = q.shape
    K, G, unit, least = kv_heads, H // kv_heads, UNIT[q.dtype], LEAST[q.dtype]
    scale = D ** -0.5 if scale is None else scale
    x, s, b = unpack(packed, K, D)
    q64, off = q.detach().cpu().double(), off.cpu().tolist()
    E = packed.shape[0]
    entity = torch.arange(E) if entity is None else entity.cpu().long()
    hop = torch.zeros(len(entity), dtype=torch.long) if hop is None else hop.cpu().long()
    out, out_tol = torch.zeros_like(q64), torch.zeros_like(q64) + least
    lse, lse_tol = torch.full((Q, T, H), -math.inf, dtype=torch.float64), torch.zeros(Q, T, H, dtype=torch.float64)
    M = 0 if buckets is None else buckets.numel() // 2
    for i in range(Q):
        at = torch.arange(off[i], off[i + 1])
        at = at[(entity[at] >= 0) & (entity[at] < E)]
        rows = entity[at]
        if not len(at):
            continue
        pos = 0 if q_pos is None else int(q_pos[i])
        for h in range(H):
            kk, ks, kb = (t[0, rows, h // G] for t in (x, s, b))
            vv, vs, vb = (t[1, rows, h // G] for t in (x, s, b))
            z = scale * (q64[i, :, h] @ kk.T)
            z_tol = abs(scale) * 2.0 ** -20 * (q64[i, :, h].abs() @ (31 * ks.abs() + kb.abs()).T)
            y = cap * torch.tanh(z / cap) if cap else z
            if bias is not None:
                y = y + bias.detach().cpu().double()[h][buckets.cpu().long()[(hop[at] - pos).clamp(-M, M) + M]][None]
            lse[i, :, h] = torch.logsumexp(y, 1)
            p = torch.softmax(y, 1)
            off_by = z_tol.amax(1) + 2.0 ** -17 * (1 + y.abs().amax(1))
            lse_tol[i, :, h] = off_by + 2.0 ** -17 * lse[i, :, h].abs()
            out[i, :, h] = p @ vv
            terms = p @ (vs * ((vv - vb) / torch.where(vs == 0, 1.0, vs) - 7.5).abs())
            sizes = p @ (40 * vs.abs() + vb.abs())
            out_tol[i, :, h] = 1.5 * unit * (out[i, :, h].abs() + terms) + 2.0 ** -16 * sizes + 2 * off_by[:, None] * (p @ vv.abs()) + least
    return {"out": out, "lse": lse}, {"out": out_tol, "lse": lse_tol}
