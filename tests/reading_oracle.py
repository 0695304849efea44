"""The calls that read a retrieval into a language model, from their definitions in 64 bits on the CPU, one document, head
and row at a time, and how far a kernel's result may be off.

Bounds.  Let u be the largest relative error of a rounding to the 16-bit type, half of its last place:
2^-8 for bfloat16 (8 significant bits), 2^-11 for float16 (11).  A
kernel rounds the weights p (or the score gradients dz) to 16 bits before the second product and its result once more, and
keeps everything else in 32 bits.  So |out - exact| <= u |out| + u sum p |v|, and likewise for dv, dq and dk with the sums of
their own terms; besides, the backward takes delta = sum dout out from the rounded out, which shifts dy by at most
p u sum |dout| (|out| + sum p |v|).  Scores carry 32-bit errors: exp2, reciprocal and products of 128 terms, below 2^-16
relative to p for scores up to 2^6.  Every bound is taken 1.5 times plus 2^-16 of the terms, and what a 16-bit type cannot
hold (its smallest subnormal) on top."""
import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}
SLOP = 2.0 ** -16


def score(z, cap):
    return cap * torch.tanh(z / cap) if cap else z


def visible(rows, keys, causal, prefix):
    i, j = torch.arange(rows)[:, None], torch.arange(keys)[None, :]
    return (j < prefix) | (j <= i + keys - rows) if causal else torch.ones(rows, keys, dtype=torch.bool)


def attention(q, k, v, q_off, k_off, scale=None, cap=0.0, causal=False, prefix=None, bias=None, buckets=None, q_pos=None,
              k_pos=None, dout=None):
    """(results, bounds): dicts of 64-bit tensors; with ``dout`` also the gradients."""
    unit, least = UNIT[q.dtype], SMALLEST[q.dtype]
    q, k, v = (t.detach().cpu().double() for t in (q, k, v))
    scale = q.shape[2] ** -0.5 if scale is None else scale
    H, G = q.shape[1], q.shape[1] // k.shape[1]
    names = ["out", "lse"] + (["dq", "dk", "dv"] if dout is not None else [])
    like = {"out": q, "lse": q[..., 0], "dq": q, "dk": k, "dv": v}
    res = {n: torch.zeros_like(like[n]) for n in names}
    tol = {n: torch.zeros_like(like[n]) for n in names}
    if bias is not None:
        table = bias.detach().cpu().double()
        buckets = buckets.cpu().long()
        M = buckets.numel() // 2
        if dout is not None:
            res["dbias"], tol["dbias"] = torch.zeros_like(table), torch.zeros_like(table)
    if dout is not None:
        dout = dout.detach().cpu().double()
    q_off, k_off = q_off.tolist(), k_off.tolist()
    for d in range(len(q_off) - 1):
        a, b, c, e = q_off[d], q_off[d + 1], k_off[d], k_off[d + 1]
        R, K = b - a, e - c
        see = visible(R, K, causal, 0 if prefix is None else int(prefix[d]))
        if bias is not None:
            qp = torch.arange(R) + K - R if q_pos is None else q_pos[a:b].cpu().long()
            kp = torch.arange(K) if k_pos is None else k_pos[c:e].cpu().long()
            kind = buckets[(kp[None] - qp[:, None]).clamp(-M, M) + M]
        for h in range(H):
            kh, vh, qh = k[c:e, h // G], v[c:e, h // G], q[a:b, h]
            z = scale * (qh @ kh.T)
            t = torch.tanh(z / cap) if cap else torch.zeros_like(z)
            y = score(z, cap) + (table[h][kind] if bias is not None else 0.0)
            y = torch.where(see, y, torch.tensor(-math.inf, dtype=torch.float64))
            lse = torch.logsumexp(y, 1) if K else torch.full((R,), -math.inf, dtype=torch.float64)
            p = torch.where(see, torch.exp(y - torch.where(lse == -math.inf, 0.0, lse)[:, None]), 0.0)
            out, terms = p @ vh, p @ vh.abs()
            res["out"][a:b, h], res["lse"][a:b, h] = out, lse
            tol["out"][a:b, h] = 1.5 * unit * (out.abs() + terms) + SLOP * terms + least
            tol["lse"][a:b, h] = 2.0 ** -17 * (1 + lse.abs())
            if dout is None:
                continue
            do = dout[a:b, h]
            dp = do @ vh.T
            off = unit * (do.abs() * (out.abs() + terms)).sum(1, keepdim=True)  # of delta
            dy = p * (dp - (do * out).sum(1, keepdim=True))
            slope = scale * (1 - t * t)
            dz = dy * slope
            part = p * (do.abs() @ vh.abs().T + (do.abs() * out.abs()).sum(1, keepdim=True))  # terms of dy
            dy_tol = 1.5 * p * off + 4 * SLOP * part
            dz_tol = (dy_tol * slope.abs() + 1.5 * unit * dz.abs() + least)
            res["dq"][a:b, h] = dz @ kh
            tol["dq"][a:b, h] = dz_tol @ kh.abs() + 1.5 * unit * (dz @ kh).abs() + least
            res["dk"][c:e, h // G] += dz.T @ qh
            tol["dk"][c:e, h // G] += dz_tol.T @ qh.abs() + least
            res["dv"][c:e, h // G] += p.T @ do
            tol["dv"][c:e, h // G] += 1.5 * unit * (p.T @ do.abs()) + SLOP * (p.T @ do.abs()) + least + least * do.abs().sum(0)
            if bias is not None:
                for x in range(table.shape[1]):
                    res["dbias"][h, x] += dy[kind == x].sum()
                    tol["dbias"][h, x] += dy_tol[kind == x].sum()
    if dout is not None:
        for n in ("dk", "dv"):
            tol[n] += 1.5 * unit * res[n].abs()
        if bias is not None:
            tol["dbias"] += 1.5 * unit * res["dbias"].abs() + least
    return res, tol


def read(q, keys, values, off, entity=None, scale=None, cap=0.0, bias=None, buckets=None, hop=None, q_pos=None):
    """``read_entities`` as the attention of one document per query."""
    n, T, H, D = q.shape
    off = off.cpu()
    entity = torch.arange(keys.shape[0]) if entity is None else entity.cpu().long()
    hop = torch.zeros(len(entity), dtype=torch.long) if hop is None else hop.cpu().long()
    good = (entity >= 0) & (entity < keys.shape[0])
    lists = [torch.arange(int(off[i]), int(off[i + 1])) for i in range(n)]
    lists = [x[good[x]] for x in lists]
    at = torch.cat(lists) if lists else torch.zeros(0, dtype=torch.long)
    k_off = torch.tensor([0] + [len(x) for x in lists]).cumsum(0)
    qp = (torch.zeros(n, dtype=torch.long) if q_pos is None else q_pos.cpu().long()).repeat_interleave(T)
    res, tol = attention(q.reshape(n * T, H, D), keys.cpu()[entity[at]], values.cpu()[entity[at]], torch.arange(n + 1) * T, k_off,
                         scale, cap, False, None, bias, buckets, qp, hop[at])
    return ({"out": res["out"].view(n, T, H, D), "lse": res["lse"].view(n, T, H)},
            {"out": tol["out"].view(n, T, H, D), "lse": tol["lse"].view(n, T, H)})


def entity_mask(off, ids, num_ids):
    words = [[0] * ((num_ids + 63) // 64) for _ in range(len(off) - 1)]
    for q in range(len(off) - 1):
        for x in ids[int(off[q]):int(off[q + 1])].tolist():
            if 0 <= x < num_ids:
                words[q][x // 64] |= 1 << (x % 64)
    return [[w - (1 << 64) if w >> 63 else w for w in row] for row in words]


def logits(x, history=None, history_off=None, repetition=None, presence=None, frequency=None, bias_off=None, bias_id=None,
           bias_value=None, mask=None):
    x = x.detach().cpu().double().clone()
    for b in range(x.shape[0]):
        if history is not None:
            said = history[int(history_off[b]):int(history_off[b + 1])].tolist()
            for v in {w for w in said if 0 <= w < x.shape[1]}:
                if repetition is not None:
                    r = float(repetition[b])
                    x[b, v] = x[b, v] / r if x[b, v] > 0 else x[b, v] * r
                x[b, v] -= (0 if presence is None else float(presence[b])) + said.count(v) * (0 if frequency is None else float(frequency[b]))
        if bias_id is not None:
            s, e = int(bias_off[b]), int(bias_off[b + 1])
            for v, add in dict(zip(bias_id[s:e].tolist(), bias_value[s:e].tolist())).items():
                if 0 <= v < x.shape[1]:
                    x[b, v] += add
        if mask is not None:
            bits = torch.tensor([int(mask[b, v // 64]) >> (v % 64) & 1 for v in range(x.shape[1])], dtype=torch.bool)
            x[b][~bits] = -math.inf
    return x


def check(got, res, tol, what=""):
    """Every element of ``got`` within its bound; infinities equal."""
    got = got.detach().cpu().double()
    assert got.shape == res.shape, (what, got.shape, res.shape)
    fine = torch.isfinite(res)
    assert torch.equal(got[~fine], res[~fine]), what + ": infinities differ"
    off = (got - res)[fine].abs()
    bad = ~(off <= tol[fine])
    if bad.any():
        at = int((off / tol[fine].clamp(min=1e-300)).nan_to_num(nan=1e300).argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside; {float(got[fine][at])} for {float(res[fine][at])} +- {float(tol[fine][at])}")
