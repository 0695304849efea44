"""The measured calls of the operators around the reading of a retrieval: entity rows into a model and their gradient back
into the table, the loss of answers that were held to masks, the end of a training step, and tables of 4 bits.

``embed``   rows of a table by the ids of retrieved lists, scaled; ``embed_grad`` their gradient, summed by entity
``policy``  clipped policy loss with a KL term over answers sampled under masks, with its gradient
``clip``    the norm of all gradients, and the gradients scaled to it
``pack``    keys and values by entity into 4 bits, and back into the values that these stand for
``read``    single tokens attend to entity lists whose keys and values lie in such a table

A packed row holds, one behind the other: the keys' codes (per head 4 ng words of 32 bits, ng = ceil(dim / 32), word
c ng + g for the elements 32 g + 8 c .. + 7, four bits each from the lowest on), the values' codes (per head 4 ng words, word w for the
elements 8 w .. + 7), and per head and group of 32 elements the keys' scale and base and the values' scale and base (bfloat16
each); zeros up to a multiple of 16 bytes.  An element is base + scale x code.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
MAX_DISTANCE, BUCKETS = 128, 32
HEADS = [(8, 8, 64), (16, 4, 128), (32, 8, 128), (16, 8, 64), (12, 4, 96), (6, 2, 80), (5, 5, 40), (8, 1, 128)]
CLIP = 0.2


def _embed(name, op, lists, ids, table, dim, dtype, skew):
    """``ids``: of the longest list; ``skew``: the larger, the more often the same few entities are listed."""
    return {"name": name, "op": op, "lists": lists, "ids": ids, "table": table, "dim": dim, "dtype": dtype, "skew": skew}


def _policy(name, rows, vocab, masks, kl, dtype):
    return {"name": name, "op": "policy", "rows": rows, "vocab": vocab, "masks": masks, "kl": kl, "dtype": dtype}


def _clip(name, table, width, matrices, dtype, to):
    return {"name": name, "op": "clip", "table": table, "width": width, "matrices": matrices, "dtype": dtype, "to": to}


def _pack(name, entities, heads, dim, dtype):
    return {"name": name, "op": "pack", "entities": entities, "kv_heads": heads, "dim": dim, "dtype": dtype}


def _read(name, queries, tokens, entities, table, heads, dtype, cap=30.0, bias=True):
    return {"name": name, "op": "read", "docs": queries, "tokens": tokens, "entities": entities, "table": table,
            "heads": heads[0], "kv_heads": heads[1], "dim": heads[2], "dtype": dtype, "cap": cap, "bias": bias}


def listed():
    return [
        # the neighbourhood of one question becomes rows of a prompt: latency
        _embed("embed_one", "embed", 1, 300, 10_000, 512, "bf16", 1),
        # a full batch of questions to 3M entities
        _embed("embed_1024", "embed", 1024, 1500, 3_000_000, 512, "bf16", 2),
        # a training step on short questions with a few facts each
        _embed("embed_grad_short", "embed_grad", 16, 124, 10_000, 512, "fp32", 2),
        # an ordinary training batch to 407K concepts: hubs are in most lists, most concepts in none
        _embed("embed_grad_256", "embed_grad", 256, 4000, 407_000, 1024, "bf16", 4),
        # the next relations of 64 sampled paths (500 relations), each held to the whitelist of its query
        _policy("policy_relations", 64, 500, 64, 0.05, "fp32"),
        # the tokens of a batch of sampled answers over a vocabulary, the answers of a question under one mask
        _policy("policy_vocab", 2048, 150_001, 32, 0.05, "bf16"),
        # a small reader's gradients: a table of 10K entities and its matrices
        _clip("clip_small", 10_000, 64, 7, "fp32", "fp32"),
        # a table of 3M entities and forty matrices, kept for the optimizer in 32 bits
        _clip("clip_large", 3_000_000, 256, 40, "bf16", "fp32"),
        # the entities that one update has changed
        _pack("pack_update", 2000, 8, 128, "bf16"),
        # the whole table of a graph of 407K concepts
        _pack("pack_table", 407_000, 8, 128, "bf16"),
        # one generated token of one question reads its neighbourhood
        _read("packed_one", 1, 1, 900, 10_000, (32, 8, 128), "bf16"),
        # a full batch of 1,024 questions, four tokens each, to 3M entities
        _read("packed_1024", 1024, 4, 3000, 3_000_000, (16, 8, 64), "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "embed_grad", "policy", "policy", "clip", "pack", "read", "read", "read"])
    half = rng.choice(["bf16", "fp16"])
    if op in ("embed", "embed_grad"):
        dim, dtype = rng.choice([64, 80, 100, 128, 333, 512, 768, 1024, 2000, 4096]), rng.choice(["bf16", "fp16", "fp32"])
        most = 400_000_000 if op == "embed" else 200_000_000  # elements of the lists, and of a table
        lists, ids = _log_int(rng, 1, 1024), _log_int(rng, 1, 6000)
        while lists > 1 and lists * ids * dim > most:
            lists = (lists + 1) // 2
        c = _embed("", op, lists, min(ids, most // dim), _log_int(rng, 1000, min(3_000_000, most // dim)), dim, dtype, rng.choice([1, 2, 4, 8]))
    elif op == "policy":
        rows, vocab = _log_int(rng, 1, 4096), _log_int(rng, 100, 200_000)
        rows = max(1, min(rows, 2048 * 150_001 // vocab))
        c = _policy("", rows, vocab, rng.choice([0, 1, (rows + 7) // 8, rows]), rng.choice([0.0, 0.02, 0.1]), rng.choice(["bf16", "bf16", "fp16", "fp32"]))
    elif op == "clip":
        width = rng.choice([64, 100, 256, 333, 512])
        c = _clip("", _log_int(rng, 1000, 3_000_000 * 256 // width), width, rng.randint(0, 50), rng.choice(["bf16", "fp16", "fp32"]), "fp32")
        c["to"] = rng.choice([c["dtype"], "fp32"])
        if c["dtype"] == "fp32":
            c["table"] = (c["table"] + 1) // 2
    elif op == "pack":
        _, heads, dim = rng.choice(HEADS)
        c = _pack("", _log_int(rng, 1, 407_000), heads, dim, rng.choice(["bf16", "fp16", "fp32"]))
        if c["dtype"] == "fp32":
            c["entities"] = (c["entities"] + 1) // 2
    else:
        heads, cap, bias = rng.choice(HEADS), rng.choice([0.0, 20.0, 50.0]), rng.random() < 0.7
        queries, entities = _log_int(rng, 1, 1024), _log_int(rng, 1, 400_000)
        tokens = rng.choice([1, 1, 1, 2, 3, 4])
        table = max(entities, _log_int(rng, 10_000, 3_000_000 * 512 // (heads[1] * heads[2])))
        largest = 1024 * 3000 * 16 * 64 * 4
        while queries > 1 and queries * entities * heads[0] * heads[2] * tokens > largest:
            queries = (queries + 1) // 2
        entities = min(entities, max(1, largest // (queries * heads[0] * heads[2] * tokens)))
        c = _read("", queries, tokens, entities, table, heads, half, cap, bias)
    del c["name"]
    return c


# ------------------------------------------------------------------------- inputs
def _lengths(n, most, salt):
    """``n`` lengths up to ``most`` (the first), every eighth of them 0: fixed by the case."""
    rng = random.Random(n * 1_000_003 + most * 101 + salt)
    got = [0 if i % 8 == 7 else round(most * rng.random() ** 0.7) for i in range(n)]
    got[0] = most
    return got


def _offsets(lengths):
    off = [0]
    for n in lengths:
        off.append(off[-1] + n)
    return torch.tensor(off, dtype=torch.int64)


def _randn(gen, shape, dtype, scale=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype).mul_(scale)


def _rand(gen, n):
    return torch.rand(n, generator=gen, device="cuda")


def _shapes(case):
    """Gradients of a reader: its table, then projections, biases and norms."""
    w = case["width"]
    kinds = [(w, w), (w, 4 * w), (w,), (4 * w + 1, w), (), (w, w // 2), (0, w)]
    return [(case["table"], w)] + [kinds[i % len(kinds)] for i in range(case["matrices"])]


def _bucket_of_distance():
    """int32[2 * MAX_DISTANCE + 1]: half of the buckets for each sign, near distances alone, far ones by their logarithm."""
    half, got = BUCKETS // 2, []
    for d in range(-MAX_DISTANCE, MAX_DISTANCE + 1):
        n = abs(d)
        far = half // 2 + int(math.log(max(n, 1) / (half // 2)) / math.log(MAX_DISTANCE / (half // 2)) * (half - half // 2))
        got.append((half if d > 0 else 0) + (n if n < half // 2 else min(far, half - 1)))
    return torch.tensor(got, dtype=torch.int32)


def _groups(dim):
    return (dim + 31) // 32


def _row_bytes(kv_heads, dim):
    return (40 * kv_heads * _groups(dim) + 15) // 16 * 16


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    make = {"embed": _prepare_embed, "embed_grad": _prepare_embed, "policy": _prepare_policy, "clip": _prepare_clip,
            "pack": _prepare_pack, "read": _prepare_read}[case["op"]]
    return {"case": case} | make(case, gen)


def _prepare_embed(case, gen):
    n, E, dtype = sum(_lengths(case["lists"], case["ids"], 1)), case["table"], DTYPES[case["dtype"]]
    # hubs have low ids here, and are listed often; some places pad
    ids = (torch.rand(n, generator=gen, device="cuda", dtype=torch.float64) ** case["skew"] * E).to(torch.int32).clamp_(max=E - 1)
    ids[_rand(gen, n) < 0.02] = -1
    got = {"ids": ids, "scale": case["dim"] ** 0.5}
    if case["op"] == "embed":
        return got | {"table": _randn(gen, (E, case["dim"]), dtype, 0.05)}
    return got | {"dout": _randn(gen, (n, case["dim"]), dtype, 0.01)}


def _prepare_policy(case, gen):
    R, V, M, dtype = case["rows"], case["vocab"], case["masks"], DTYPES[case["dtype"]]
    logits = _randn(gen, (R, V), dtype, 3.0)
    words, mask, mask_row = (V + 63) // 64, None, None
    target = (_rand(gen, R) * V).long().clamp_(max=V - 1)
    if M:
        bits = [torch.randint(-2 ** 63, 2 ** 63 - 1, (M, words), generator=gen, device="cuda") for _ in range(2)]
        mask = bits[0] & bits[1]
        mask_row = torch.arange(R, device="cuda") * M // R
        # an answer's token is one that its mask allows: the first from a random place on, were there none, the place itself
        look = (target[:, None] + torch.arange(256, device="cuda")) % V
        open_ = (mask[mask_row[:, None], look // 64] >> (look % 64)) & 1
        target = look.gather(1, open_.argmax(1, keepdim=True)).squeeze(1)
        if M > 1:
            mask[1] = 0  # nothing is allowed
        mask_row = mask_row.to(torch.int32)
    target = target.to(torch.int32)
    target[_rand(gen, R) < 0.05] = -1  # padding of answers
    weight = (target >= 0).float() / R
    # the policies that sampled and that is kept near: a little off; ratios stand clear of the clip's borders
    near = _near_logp(logits, target, mask, mask_row)
    off = (torch.randint(-8, 9, (R,), generator=gen, device="cuda") * 0.05 + (_rand(gen, R) - 0.5) * 0.03)
    return {"logits": logits, "target": target, "advantage": torch.randn(R, generator=gen, device="cuda") + 0.3, "old": near - off,
            "ref": near + torch.randn(R, generator=gen, device="cuda") * 0.3, "weight": weight, "mask": mask, "mask_row": mask_row,
            "scale": 1 / 1.5}


def _near_logp(logits, target, mask, mask_row):
    """About what the tokens' log probabilities are (0 where a row has none)."""
    got = torch.zeros(logits.shape[0], device="cuda")
    for a in range(0, logits.shape[0], 512):
        x = logits[a:a + 512].float() / 1.5
        at = target[a:a + 512, None].long().clamp(min=0)
        if mask is not None:
            x = x.masked_fill_(~_allowed(mask, mask_row[a:a + 512], x.shape[1]), -math.inf)
        got[a:a + 512] = x.gather(1, at).squeeze(1) - x.logsumexp(1)
    return torch.where(got.isfinite(), got, 0.0)


def _prepare_clip(case, gen):
    grads = [_randn(gen, s, DTYPES[case["dtype"]], 1e-3) for s in _shapes(case)]
    return {"grads": grads, "out": [torch.empty_like(g, dtype=DTYPES[case["to"]]) for g in grads], "scale": 0.25,
            "max_norm": 0.25 * 1e-3 * 0.7 * math.sqrt(sum(g.numel() for g in grads))}


def _prepare_pack(case, gen):
    shape = (case["entities"], case["kv_heads"], case["dim"])
    k, v = (_randn(gen, shape, DTYPES[case["dtype"]]) for _ in range(2))
    k *= (torch.rand(case["kv_heads"], case["dim"], generator=gen, device="cuda") * 3).to(k.dtype)  # keys' channels differ
    return {"keys": k, "values": v}


def _prepare_read(case, gen):
    dtype, H, K, D, E = DTYPES[case["dtype"]], case["heads"], case["kv_heads"], case["dim"], case["table"]
    G, bytes_ = _groups(D), _row_bytes(K, D)
    lengths = _lengths(case["docs"], case["entities"], 2)
    off = _offsets(lengths)
    n = int(off[-1])
    packed = torch.randint(-2 ** 63, 2 ** 63 - 1, (E, bytes_ // 8), generator=gen, device="cuda").view(torch.uint8)
    # sixteen steps from 2 to 3 below 0 up: values around 0 with deviations of about 1.5
    scale = 0.3 + 0.1 * torch.rand(E, K * G * 2, generator=gen, device="cuda")
    base = -7.5 * scale + 0.2 * torch.randn(E, K * G * 2, generator=gen, device="cuda")
    packed[:, 32 * K * G:40 * K * G] = torch.stack([scale, base], 2).to(torch.bfloat16).view(E, -1).view(torch.uint8)
    packed[:, 40 * K * G:] = 0
    size = torch.tensor(lengths, device="cuda")
    doc = torch.repeat_interleave(torch.arange(len(lengths), device="cuda"), size, output_size=n)
    at = torch.arange(n, device="cuda") - off[:-1].cuda()[doc]
    first, behind = at * E // size[doc], (at + 1) * E // size[doc]  # lists ascend
    entity = (first + (torch.rand(n, generator=gen, device="cuda", dtype=torch.float64) * (behind - first)).long()).to(torch.int32)
    return {"q": _randn(gen, (case["docs"], case["tokens"], H, D), dtype, 1.0), "packed": packed, "off": off.cuda(), "entity": entity,
            "hop": torch.randint(0, 4, (n,), generator=gen, device="cuda").to(torch.uint8),
            "bias": _randn(gen, (H, BUCKETS), dtype) if case["bias"] else None,
            "buckets": _bucket_of_distance().cuda() if case["bias"] else None, "scale": D ** -0.5, "cap": case["cap"]}


# ------------------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    op = case["op"]
    if not own:
        return {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "policy": _plain_policy, "clip": _plain_clip,
                "pack": _plain_pack, "read": _plain_read}[op](state)
    import paper_2604_18913_amd as lkg
    if op == "embed":
        return lkg.embed_entities(state["table"], state["ids"], scale=state["scale"])
    if op == "embed_grad":
        return lkg.embed_entities_backward(state["dout"], state["ids"], case["table"], scale=state["scale"])
    if op == "policy":
        return lkg.policy_loss(state["logits"], state["target"], state["advantage"], old=state["old"], ref=state["ref"],
                               weight=state["weight"], clip=(CLIP, CLIP), kl=case["kl"], scale=state["scale"],
                               mask=state["mask"], mask_row=state["mask_row"], gradient=True)
    if op == "clip":
        norm = lkg.clip_gradients(state["grads"], state["max_norm"], scale=state["scale"], out=state["out"])
        return {"norm": norm, "grads": state["out"]}
    if op == "pack":
        packed = lkg.pack_entities(state["keys"], state["values"])
        return lkg.unpack_entities(packed, case["kv_heads"], case["dim"], dtype=state["keys"].dtype)
    return lkg.read_packed(state["q"], state["packed"], state["off"], state["entity"], kv_heads=case["kv_heads"], hop=state["hop"],
                           scale=state["scale"], cap=state["cap"], bias=state["bias"], buckets=state["buckets"])


def _plain_embed(state):
    ids = state["ids"].long()
    x = state["table"][ids.clamp(min=0)].float() * state["scale"]
    return (x * (ids >= 0)[:, None]).to(state["table"].dtype)


def _plain_embed_grad(state):
    ids, dout, E = state["ids"].long(), state["dout"], state["case"]["table"]
    sums = torch.zeros(E + 1, dout.shape[1], device=dout.device)
    sums.index_add_(0, torch.where(ids < 0, E, ids), dout.float())
    return (sums[:E] * state["scale"]).to(dout.dtype)


def _allowed(mask, mask_row, vocab):
    ids = torch.arange(vocab, device=mask.device)
    return ((mask[:, ids // 64] >> (ids % 64)) & 1).bool()[mask_row.long()]


def _plain_policy(state):
    case, target = state["case"], state["target"].long()
    x = state["logits"].float() * state["scale"]
    if state["mask"] is not None:
        x.masked_fill_(~_allowed(state["mask"], state["mask_row"], x.shape[1]), -math.inf)
    top = x.amax(1, keepdim=True).clamp_(min=-1e30)
    at = target.clamp(min=0)[:, None]
    said = x.gather(1, at).squeeze(1)
    p = x.sub_(top).exp_()
    total = p.sum(1)
    lse = top.squeeze(1) + total.log()
    logp = torch.where(said == -math.inf, -math.inf, said - lse)
    counted = (target >= 0) & (logp > -math.inf)
    lp, A = torch.where(counted, logp, 0.0), state["advantage"]
    ratio, apart = (lp - state["old"]).exp(), state["ref"] - lp
    inside = ratio * A
    border = ratio.clamp(1 - CLIP, 1 + CLIP) * A
    row = -torch.minimum(inside, border) + case["kl"] * (apart.exp() - apart - 1)
    slope = torch.where(inside <= border, -inside, 0.0) + case["kl"] * (1 - apart.exp())
    w = torch.where(counted, state["weight"], 0.0)
    slope = slope * w * state["scale"]
    p *= (-slope / total.clamp(min=1e-30))[:, None]
    p.scatter_add_(1, at, slope[:, None])
    return {"loss": (row * w).sum(), "logp": torch.where(target < 0, 0.0, logp), "lse": lse, "dlogits": p.to(state["logits"].dtype)}


def _plain_clip(state):
    grads, scale = state["grads"], state["scale"]
    norm = torch.stack([g.float().square().sum() for g in grads]).sum().sqrt() * scale
    by = scale * (state["max_norm"] / norm.clamp(min=1e-30)).clamp(max=1.0)
    return {"norm": norm, "grads": [(g.float() * by).to(o.dtype) for g, o in zip(grads, state["out"])]}


def _plain_rounded(x):
    """What 4 bits a group of 32 keep of ``x``, in its type."""
    E, K, D = x.shape
    G = _groups(D)
    y = x.float()
    inside = torch.arange(G * 32, device=x.device).view(G, 32) < D
    y = torch.nn.functional.pad(y, (0, G * 32 - D)).view(E, K, G, 32)
    low = torch.where(inside, y, math.inf).amin(3, keepdim=True)
    high = torch.where(inside, y, -math.inf).amax(3, keepdim=True)
    base = low.to(torch.bfloat16).float()
    scale = ((high - low) / torch.full_like(low, 15.0)).to(torch.bfloat16).float()
    code = torch.where(scale > 0, (y - base) / scale, 0.0).round_().clamp_(0, 15)
    return (base + scale * code).view(E, K, G * 32)[:, :, :D].to(x.dtype)


def _plain_pack(state):
    return _plain_rounded(state["keys"]), _plain_rounded(state["values"])


def _plain_unpacked(rows, K, D):
    """Keys and values [n, K, D] in 32 bits of packed rows."""
    n, G = rows.shape[0], _groups(D)
    codes = rows[:, :32 * K * G]
    codes = torch.stack([codes & 15, codes >> 4], 2).view(n, 2, K, 32 * G)
    keys = codes[:, 0].reshape(n, K, 4, G, 8).transpose(2, 3).reshape(n, K, G, 32)
    values = codes[:, 1].reshape(n, K, G, 32)
    p = rows[:, 32 * K * G:40 * K * G].contiguous().view(torch.bfloat16).view(n, K, G, 2, 2).float()
    return [(c * p[:, :, :, i, :1] + p[:, :, :, i, 1:]).view(n, K, 32 * G)[:, :, :D] for i, c in enumerate((keys, values))]


def _plain_read(state):
    """One entry of a list at a time: its scores, the largest and the sum of its list, its share of the values."""
    q, off, dtype, K = state["q"], state["off"], state["q"].dtype, state["case"]["kv_heads"]
    Q, T, H, D = q.shape
    n = state["entity"].numel()
    keys, values = _plain_unpacked(state["packed"][state["entity"].long()], K, D)
    owner = torch.repeat_interleave(torch.arange(Q, device=q.device), off[1:] - off[:-1], output_size=n)
    s = (q.float().view(Q, T, K, H // K, D)[owner] * keys[:, None, :, None, :]).sum(4).view(n, T * H)
    s *= state["scale"]
    if state["cap"]:
        s = (s / state["cap"]).tanh_().mul_(state["cap"])
    if state["bias"] is not None:
        bucket = state["buckets"][state["hop"].long().clamp(max=MAX_DISTANCE) + MAX_DISTANCE].long()
        s += state["bias"].float().t()[bucket].repeat(1, T)
    top = torch.full((Q, T * H), -math.inf, device=q.device)
    top.scatter_reduce_(0, owner[:, None].expand(n, T * H), s, "amax")
    p = (s - top[owner]).exp_()
    total = torch.zeros(Q, T * H, device=q.device).index_add_(0, owner, p)
    share = p.view(n, T, K, H // K, 1) * values[:, None, :, None, :]
    o = torch.zeros(Q, T, K, H // K, D, device=q.device).index_add_(0, owner, share).view(Q, T, H, D)
    o /= total.view(Q, T, H, 1).clamp(min=1e-30)
    return {"out": o.to(dtype), "lse": (top + total.log()).view(Q, T, H)}


# ------------------------------------------------------------------------- definition in 64 bits
def exact(case, seed):
    state = prepare(case, seed)
    return {"embed": _exact_embed, "embed_grad": _exact_embed_grad, "policy": _exact_policy, "clip": _exact_clip,
            "pack": _exact_pack, "read": _exact_read}[case["op"]](state)


def _exact_embed(state):
    ids = state["ids"]
    got = torch.zeros(ids.numel(), state["table"].shape[1], dtype=torch.float64, device="cuda")
    kept = (ids >= 0).nonzero().squeeze(1)
    got[kept] = state["table"].index_select(0, ids[kept].long()).double().mul_(state["scale"])
    return got


def _exact_embed_grad(state):
    """Sums of neighbours in the order of the ids: differences of running sums, a part of the columns at a time."""
    ids, dout, E = state["ids"].long(), state["dout"], state["case"]["table"]
    got = torch.zeros(E, dout.shape[1], dtype=torch.float64, device="cuda")
    by_id, order = torch.sort(ids, stable=True)
    order = order[int((ids < 0).sum()):]
    who, count = torch.unique_consecutive(by_id[by_id >= 0], return_counts=True)
    for c in range(0, dout.shape[1], 64):
        parts = dout[:, c:c + 64][order].double()
        got[who, c:c + 64] = torch.segment_reduce(parts, "sum", lengths=count, axis=0) * state["scale"]
    return got


def _exact_policy(state):
    case, R = state["case"], state["case"]["rows"]
    got = {"loss": torch.zeros((), dtype=torch.float64, device="cuda"),
           "logp": torch.zeros(R, dtype=torch.float64, device="cuda"), "lse": torch.zeros(R, dtype=torch.float64, device="cuda"),
           "dlogits": torch.zeros(R, case["vocab"], dtype=torch.float64, device="cuda")}
    place = torch.arange(64, device="cuda")
    target = state["target"].tolist()
    for a in range(0, R, 256):
        b = min(R, a + 256)
        x = state["logits"][a:b].double() * state["scale"]
        if state["mask"] is not None:
            bits = ((state["mask"][state["mask_row"][a:b].long()][:, :, None] >> place) & 1).reshape(b - a, -1)[:, :case["vocab"]]
            x = torch.where(bits == 1, x, -math.inf)
        lse = torch.logsumexp(x, 1)
        got["lse"][a:b] = lse
        t = torch.tensor(target[a:b], device="cuda")
        lp = x.gather(1, t.clamp(min=0)[:, None])[:, 0]
        gone = lp == -math.inf
        lp = torch.where(gone, -math.inf, lp - lse)
        got["logp"][a:b] = torch.where(t < 0, 0.0, lp)
        use = ~gone & (t >= 0)
        lp = torch.where(use, lp, state["old"][a:b].double())
        A, old, ref, w = (state[n][a:b].double() for n in ("advantage", "old", "ref", "weight"))
        w = torch.where(use, w, 0.0)
        rho = torch.exp(lp - old)
        stopped = torch.where(A >= 0, rho > 1 + CLIP, rho < 1 - CLIP)
        gain = torch.where(stopped, torch.where(A >= 0, 1 + CLIP, 1 - CLIP) * A, rho * A)
        got["loss"] += (w * (case["kl"] * (torch.expm1(ref - lp) - (ref - lp)) - gain)).sum()
        g = w * (torch.where(stopped, 0.0, -rho * A) - case["kl"] * torch.expm1(ref - lp)) * state["scale"]
        share = torch.where(x == -math.inf, 0.0, torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)[:, None]))
        d = -g[:, None] * share
        d[torch.arange(b - a, device="cuda"), t.clamp(min=0)] += g
        got["dlogits"][a:b] = d
    return got


def _exact_clip(state):
    total = math.fsum(float(torch.linalg.vector_norm(g, dtype=torch.float64)) ** 2 for g in state["grads"] if g.numel())
    norm = abs(state["scale"]) * math.sqrt(total)
    by = state["scale"] * (state["max_norm"] / norm if norm > state["max_norm"] else 1.0)
    return {"norm": torch.tensor(norm, dtype=torch.float64, device="cuda"), "grads": [g.double() * by for g in state["grads"]]}


def _exact_pack(state):
    def kept(x):
        got = torch.zeros(x.shape, dtype=torch.float64, device="cuda")
        for a in range(0, x.shape[2], 32):
            y = x[:, :, a:a + 32].double()
            low, high = y.min(2, keepdim=True).values, y.max(2, keepdim=True).values
            base, step = low.to(torch.bfloat16).double(), ((high - low) / 15).to(torch.bfloat16).double()
            code = torch.round((y - base) / torch.where(step > 0, step, 1.0)).clamp(0, 15)
            got[:, :, a:a + 32] = base + step * torch.where(step > 0, code, 0.0)
        return got
    return kept(state["keys"]), kept(state["values"])


def _exact_values(rows, K, D, which):
    """Keys (0) or values (1) of packed rows, element by element of the format."""
    G = _groups(D)
    d = torch.arange(D, device="cuda")
    word = (d % 32) // 8 * G + d // 32 if which == 0 else d // 8
    head = torch.arange(K, device="cuda")[:, None]
    byte = which * 16 * K * G + head * 16 * G + word * 4 + d % 8 // 2
    code = (rows[:, byte] >> ((d % 2) * 4).to(torch.uint8)) & 15
    at = 32 * K * G + 8 * (head * G + d // 32) + 4 * which
    held = [(rows[:, at + i].int() + (rows[:, at + i + 1].int() << 8)).to(torch.int16).view(torch.bfloat16).double() for i in (0, 2)]
    return code.double() * held[0] + held[1]


def _exact_read(state):
    q, off, K = state["q"].double(), state["off"].tolist(), state["case"]["kv_heads"]
    Q, T, H, D = q.shape
    G = H // K
    out, lse = torch.zeros_like(q), torch.full((Q, T, H), -math.inf, dtype=torch.float64, device="cuda")
    for i in range(Q):
        if off[i] == off[i + 1]:
            continue
        rows = state["packed"][state["entity"][off[i]:off[i + 1]].long()]
        k, v = (_exact_values(rows, K, D, which).transpose(0, 1) for which in (0, 1))
        z = q[i].view(T, K, G, D).permute(1, 0, 2, 3).reshape(K, T * G, D)
        z = torch.matmul(z, k.transpose(1, 2).contiguous()) * state["scale"]
        if state["cap"]:
            z = state["cap"] * torch.tanh(z / state["cap"])
        z = z.view(K, T, G, -1)
        if state["bias"] is not None:
            kind = state["buckets"].long()[state["hop"][off[i]:off[i + 1]].long() + MAX_DISTANCE]
            z = z + state["bias"].double()[:, kind].view(K, 1, G, -1)
        p = torch.softmax(z, 3)
        out[i] = torch.matmul(p.view(K, T * G, -1), v.contiguous()).view(K, T, G, D).transpose(0, 1).reshape(T, H, D)
        lse[i] = torch.logsumexp(z, 3).transpose(0, 1).reshape(T, H)
    return {"out": out, "lse": lse}


# ------------------------------------------------------------------------- work
def _distinct(n, E, skew):
    """Entities that n draws of ``_prepare_embed`` are expected to hit: id i has the share ((i + 1)^(1/skew) - i^(1/skew)) / E^(1/skew)."""
    edge = torch.arange(E + 1, dtype=torch.float64).div_(E).pow_(1 / skew)
    return float((1 - (1 - (edge[1:] - edge[:-1])).clamp_(min=0).pow_(n)).sum())


def work(case):
    """Each input read once and each output written once; of tables the different rows that are listed, as expected."""
    op, size = case["op"], SIZE.get(case["dtype"])
    if op in ("embed", "embed_grad"):
        n, E, D = sum(_lengths(case["lists"], case["ids"], 1)), case["table"], case["dim"]
        rows = _distinct(n, E, case["skew"]) if op == "embed" else E
        return {"bytes": int(4 * n + size * D * (n + rows)), "flops": 0 if op == "embed" else n * D}
    if op == "policy":
        R, V = case["rows"], case["vocab"]
        return {"bytes": 2 * size * R * V + 8 * case["masks"] * ((V + 63) // 64) + 32 * R, "flops": 6 * R * V}
    if op == "clip":
        n = sum(math.prod(s) for s in _shapes(case))
        return {"bytes": n * (size + SIZE[case["to"]]), "flops": 3 * n}
    if op == "pack":
        n, K, D = case["entities"], case["kv_heads"], case["dim"]
        return {"bytes": n * (4 * size * K * D + _row_bytes(K, D)), "flops": 8 * n * K * D}
    H, K, D, E = case["heads"], case["kv_heads"], case["dim"], case["table"]
    lengths = _lengths(case["docs"], case["entities"], 2)
    n, missed = sum(lengths), 1.0
    for m in lengths:
        missed *= 1 - min(m / E, 1)
    return {"bytes": int(_row_bytes(K, D) * E * (1 - missed) + 5 * n + case["docs"] * case["tokens"] * H * (4 * D + 4)),
            "flops": 4 * n * case["tokens"] * H * D}
