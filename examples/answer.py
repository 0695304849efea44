#!/usr/bin/env python3
"""From a retrieval to an answer: a question's k-hop neighbourhood is read by a small model: rows of an entity table, ragged attention
over them and the text, logits over the entities.  First it samples answers from the lists and is paid for near ones, then it learns the
true ones, all with gradients.  In serving one token reads the list from tables by entity, of 16 and of 4 bits, and the answer is held
to the list.

    python examples/answer.py            # needs an MI355X
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import kggen
import paper_2604_18913_amd as lkg

HEADS, KV_HEADS, DIM, TOKENS, HOPS, BUCKETS, FAR, CAP = 8, 2, 64, 6, 2, 12, 32, 30.0
TEXT_AT = HOPS + 1  # entities stand at their hop, the text behind them


def main(steps=40, questions=32, policy_steps=4):
    gen = torch.Generator().manual_seed(1)
    w = kggen.config1()
    graph = lkg.Graph(w.subj, w.rel, w.obj, w.num_entities, w.num_relations)
    res = graph.khop(w.seed_off[:questions + 1], w.seeds[:w.seed_off[questions]], HOPS)
    off, (entity, hop, _) = torch.from_numpy(res.offsets()).cuda(), res.fetch(want_pred=False)
    lengths = (off[1:] - off[:-1]).tolist()
    at = off.tolist()
    truth = torch.stack([entity[at[i] + (37 * i) % lengths[i]] for i in range(questions)]).long()  # an entity of the list

    def new(*shape, scale):
        return (torch.randn(*shape, generator=gen) * scale).cuda().requires_grad_()

    width = HEADS * DIM
    table, words = new(w.num_entities, width, scale=1.0), new(questions * TOKENS, width, scale=1.0)  # words: one set per question
    to_q, to_k, to_v, to_out = (new(width, n * DIM, scale=width ** -0.5) for n in (HEADS, KV_HEADS, KV_HEADS, HEADS))
    bias = new(HEADS, BUCKETS, scale=0.1)
    buckets = lkg.distance_buckets(BUCKETS, FAR)
    half = torch.bfloat16

    # documents: a question's entities, then its text; rows are the text's tokens, which see all entities and the text so far
    order, k_pos = [], []
    for i, n in enumerate(lengths):
        order += list(range(at[i], at[i + 1])) + [int(off[-1]) + i * TOKENS + j for j in range(TOKENS)]
        k_pos += hop[at[i]:at[i + 1]].tolist() + [TEXT_AT + j for j in range(TOKENS)]
    order, k_pos = torch.tensor(order).cuda(), torch.tensor(k_pos, dtype=torch.int32).cuda()
    q_pos = (TEXT_AT + torch.arange(TOKENS, dtype=torch.int32)).repeat(questions).cuda()
    ends = torch.arange(questions + 1)
    q_off, k_off = (ends * TOKENS).cuda(), off + ends.cuda() * TOKENS
    kw = dict(cap=CAP, causal=True, prefix=torch.tensor(lengths, dtype=torch.int32).cuda(), buckets=buckets, q_pos=q_pos, k_pos=k_pos)
    last = torch.arange(questions).cuda() * TOKENS + TOKENS - 1
    parameters = [table, words, to_q, to_k, to_v, to_out, bias]
    optimizer = torch.optim.Adam(parameters, lr=0.0003)
    mask = lkg.entity_mask(off, entity, w.num_entities)  # an answer is an entity of its question's list

    def attention():
        read = torch.cat([lkg.embed_entities(table, entity), words])[order]
        k, v = ((read @ m).view(-1, KV_HEADS, DIM).to(half) for m in (to_k, to_v))
        return lkg.attend((words @ to_q).view(-1, HEADS, DIM).to(half), k, v, q_off, k_off, bias=bias.to(half), **kw)[0][last]

    def answers():
        return attention().float().flatten(1) @ to_out @ table.t()

    def step(optimizer, loss):
        optimizer.zero_grad()
        loss.backward()
        norms.append(float(lkg.clip_gradients([p.grad for p in parameters], 10.0)))
        optimizer.step()

    losses, norms, rewards = [], [], []
    even = torch.full((questions,), 1.0 / questions, device="cuda")
    owner = torch.arange(questions, dtype=torch.int32, device="cuda").repeat_interleave(4)
    hops = torch.full((questions, w.num_entities), HOPS + 1, dtype=torch.uint8, device="cuda")
    hops[torch.arange(questions, device="cuda").repeat_interleave(off[1:] - off[:-1]), entity.long()] = hop
    held = dict(scale=0.05, mask=mask, mask_row=owner)
    for _ in range(policy_steps):  # four answers per question, two steps on each, kept near what gave them
        with torch.no_grad():
            logits = answers()
            tokens = torch.multinomial(lkg.constrain_logits(logits * held["scale"], mask=mask).softmax(1), 4, replacement=True).int()
            reward = (hops.gather(1, tokens.long()) < HOPS).float()
            advantage = (reward - reward.mean(1, keepdim=True)).flatten()
            sampled = lkg.token_logp(logits[owner.long()], tokens.flatten(), **held)["logp"]
        rewards.append(float(reward.mean()))
        for _ in range(2):
            step(optimizer, lkg.policy_loss(answers()[owner.long()], tokens.flatten(), advantage, old=sampled, ref=sampled, kl=0.05,
                                 weight=even.repeat_interleave(4) / 4, **held)["loss"])

    optimizer = torch.optim.Adam(parameters, lr=0.01)
    for _ in range(steps):  # the true answers: with an advantage of 1 the loss's gradient is that of -log p
        got = lkg.policy_loss(answers(), truth.int(), torch.ones_like(even), weight=even)
        losses.append(-float(got["logp"].mean()))
        step(optimizer, got["loss"])

    # serving: keys and values of all entities are made once; a question's last token reads its list from them, and its text by
    # attention; the two are joined by their sums
    with torch.no_grad():
        want = attention().float()
        keys, values = ((table @ m).view(-1, KV_HEADS, DIM).to(half) for m in (to_k, to_v))
        q = (words @ to_q).view(questions, TOKENS, HEADS, DIM).to(half)[:, -1:].contiguous()
        b, token = bias.to(half), torch.full((questions,), TEXT_AT + TOKENS - 1, dtype=torch.int32).cuda()
        kw = dict(hop=hop, q_pos=token, cap=CAP, bias=b, buckets=buckets)
        graph_part = lkg.read_entities(q, keys, values, off, entity, **kw)
        four_bits = lkg.read_packed(q, lkg.pack_entities(keys, values), off, entity, kv_heads=KV_HEADS, **kw)["out"].float()
        k, v = ((words @ m).view(-1, KV_HEADS, DIM).to(half) for m in (to_k, to_v))
        text, text_lse = lkg.attend(q[:, 0], k, v, ends.cuda(), q_off, cap=CAP, bias=b, buckets=buckets, q_pos=token, k_pos=q_pos)
        lse = torch.logaddexp(graph_part["lse"][:, 0], text_lse)
        joined = sum((x.float() * torch.exp(part - lse)[..., None] for x, part in ((graph_part["out"][:, 0], graph_part["lse"][:, 0]), (text, text_lse))))
        logits = lkg.constrain_logits(joined.flatten(1) @ to_out @ table.t(), mask=mask)
        answer = logits.argmax(1)
    return {"losses": losses, "norms": norms, "rewards": rewards,
            "packed_off_by": float((four_bits - graph_part["out"].float()).norm() / graph_part["out"].float().norm()),
            "right": int((answer == truth).sum()), "questions": questions, "off_by": float((joined - want).abs().max() / want.abs().max()),
            "in_list": all(int(answer[i]) in set(entity[at[i]:at[i + 1]].tolist()) for i in range(questions))}


if __name__ == "__main__":
    got = main()
    print("its own answers: %s of them near" % ", ".join("%.2f" % r for r in got["rewards"]))
    print("training: loss %.3f -> %.3f in %d steps" % (got["losses"][0], got["losses"][-1], len(got["losses"])))
    print("read from a table of 4 bits, the entities' part differs by %.2f of its size" % got["packed_off_by"])
    print("serving: %d of %d answers right, all of them from the lists: %s; read from the tables and joined, outputs differ from training's by %.1e"
          % (got["right"], got["questions"], got["in_list"], got["off_by"]))
