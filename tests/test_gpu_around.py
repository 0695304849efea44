"""The calls around the reading as they are used together: a retrieval's lists become rows, answers held to the lists are trained, the step
ends, and the trained table is read in 4 bits."""
import importlib.util
import os

import pytest
import torch

import around_oracle as oracle
import kggen
import paper_2604_18913_amd as lkg

pytestmark = pytest.mark.gpu
DIM, LIST = 40, 48


def _retrieval(questions=24):
    w = kggen.config1()
    g = lkg.Graph(w.subj, w.rel, w.obj, w.num_entities, w.num_relations)
    res = g.khop(w.seed_off[:questions + 1], w.seeds[:w.seed_off[questions]], 2)
    off, (entity, hop, _) = torch.from_numpy(res.offsets()).cuda(), res.fetch(want_pred=False)
    padded = torch.full((questions, LIST), -1, dtype=torch.int32, device="cuda")  # the lists' beginnings as rows of one length
    for i in range(questions):
        mine = entity[off[i]:off[i + 1]][:LIST]
        padded[i, :len(mine)] = mine
    return w.num_entities, off, entity, hop, padded


def _model(entities, seed=1):
    g = torch.Generator().manual_seed(seed)
    table, answers = (torch.randn(entities, DIM, generator=g) * s for s in (0.2, 0.2))
    return table, answers


def _terms(questions, logp, seed=2):
    g = torch.Generator().manual_seed(seed)
    near = lambda s: (logp + torch.randn(questions, generator=g).cuda() * s).contiguous()
    return dict(advantage=torch.randn(questions, generator=g).cuda(), old=near(0.02), ref=near(0.3), weight=torch.full((questions,), 1 / questions).cuda())


def _logits(table, answers, padded):
    rows = lkg.embed_entities(table, padded, scale=2.0)
    return rows, rows.mean(1), rows.mean(1) @ answers.t()


def test_a_training_step():
    entities, off, entity, _, padded = _retrieval()
    table, answers = (x.cuda().requires_grad_() for x in _model(entities))
    mask = lkg.entity_mask(off, entity, entities)
    target = padded[:, 3].contiguous()  # (-1 of shorter lists: those do not count)
    kw = dict(kl=0.1, scale=0.7, mask=mask)
    with torch.no_grad():
        terms = _terms(len(target), lkg.token_logp(_logits(table, answers, padded)[2], target, scale=0.7, mask=mask)["logp"])
    rows, pooled, logits = _logits(table, answers, padded)
    loss = lkg.policy_loss(logits, target, **terms, **kw)["loss"]
    loss.backward()

    # torch's backward is the calls one behind the other, bit by bit
    with torch.no_grad():
        rows, pooled, logits = _logits(table, answers, padded)
        got = lkg.policy_loss(logits, target, **terms, **kw)
        assert torch.equal(got["loss"], loss)
        dlogits = lkg.policy_loss_backward(torch.tensor(1.0, device="cuda"), logits, target, lse=got["lse"], **terms, **kw)
        dpooled = dlogits @ answers
        drows = (dpooled / LIST)[:, None].expand(-1, LIST, -1).contiguous()
        assert torch.equal(answers.grad, (pooled.t() @ dlogits).t())
        assert torch.equal(table.grad, lkg.embed_entities_backward(drows, padded, entities, scale=2.0))

    # .. and the formula's gradient in 64 bits.  Logits are sums of 40 products of sums of 48 terms, 90 roundings of 2^-24 of terms that sum up
    # to less than 4: off by 2^-15; so are the exponents (twice) and what is made of them, relative to slope x (share + 1).  The sums
    # behind have up to 24 x 48, 2,080 and 40 terms, whose roundings are 2^-24 of their terms' sizes each: 2^-12 of the sizes' sums in all
    # holds with a third to spare (4 x 2^-15 + 3,272 x 2^-24 = 0.0003; 2^-11.6).
    t64, a64 = (x.detach().cpu().double().requires_grad_() for x in (table, answers))
    good = (padded >= 0).cpu()
    p64 = (t64[padded.cpu().long().clamp(min=0)] * good[..., None] * 2.0).mean(1)
    l64 = p64 @ a64.t()
    assert float((p64.abs() @ a64.abs().t()).max()) < 4
    allowed = torch.zeros(len(target), entities, dtype=torch.bool)
    at = off.tolist()
    for i in range(len(target)):
        allowed[i, entity[at[i]:at[i + 1]].cpu().long()] = True
    lp = torch.log_softmax((0.7 * l64).masked_fill(~allowed, float("-inf")), 1).gather(1, target.cpu().long().clamp(min=0)[:, None])[:, 0]
    counts = (target >= 0).cpu()
    assert counts.any()
    lp = torch.where(counts, lp, 0.0)
    t = {n: x.cpu().double() for n, x in terms.items()}
    t["weight"] = torch.where(counts, t["weight"], 0.0)
    ratio = (lp - t["old"]).exp()
    each = -torch.minimum(ratio * t["advantage"], ratio.clamp(0.8, 1.2) * t["advantage"]) + 0.1 * ((t["ref"] - lp).exp() - (t["ref"] - lp) - 1)
    want = (t["weight"] * each).sum()
    assert bool(((ratio - 0.8).abs() > 1e-3).all() and ((ratio - 1.2).abs() > 1e-3).all())  # clear of the clip's borders
    want.backward()
    with torch.no_grad():
        share = torch.softmax((0.7 * l64).masked_fill(~allowed, float("-inf")), 1)
        steep = t["weight"] * 0.7 * (ratio * t["advantage"].abs() + 0.1 * ((t["ref"] - lp).exp() + 1))
        size = steep[:, None] * (share + torch.nn.functional.one_hot(target.cpu().long().clamp(min=0), entities))
        rows_size = (size @ a64.abs() / LIST)[:, None].expand(-1, LIST, -1)
        table_size = oracle.embed_grad(rows_size.contiguous(), padded, entities, 2.0, dtype=torch.float32)[0]
    oracle.check(table.grad, t64.grad, 1.5 * 2.0 ** -12 * table_size + 1e-30, "table")
    oracle.check(answers.grad, a64.grad, 1.5 * 2.0 ** -12 * (size.t() @ p64.detach().abs()) + 1e-30, "answers")
    assert abs(float(loss) - float(want)) <= 2.0 ** -12 * float((t["weight"] * (ratio * t["advantage"].abs() + 0.1 * ((t["ref"] - lp).exp() + 1 + (t["ref"] - lp).abs()))).sum())

    grads = [table.grad.clone(), answers.grad.clone()]
    norm, bound, ends = oracle.clip(grads, 0.01)
    oracle.check(lkg.clip_gradients(grads, 0.01), norm, bound, "norm")
    for g, (x, b) in zip(grads, ends):
        oracle.check(g, x, b, "gradient")


def test_gradients_against_differences():
    """Along a direction in both parameters: (f(h) - f(-h)) / 2h of the same calls' loss, f to 2^-20 of its terms (some 4 together), h = 2^-6: off
    by 2^-19 x 4 / 2^-5 = 2^-12, and by h^2 / 6 = 2^-14.6 of the third derivative, which the step sizes keep below 1."""
    entities, off, entity, _, padded = _retrieval()
    table, answers = (x.cuda().requires_grad_() for x in _model(entities, 3))
    mask = lkg.entity_mask(off, entity, entities)
    target = padded[:, 1].contiguous()
    with torch.no_grad():
        terms = _terms(len(target), lkg.token_logp(_logits(table, answers, padded)[2], target, mask=mask)["logp"], 4)

    def f(a, b):
        return lkg.policy_loss(_logits(a, b, padded)[2], target, clip=(10.0, 10.0), kl=0.1, mask=mask, **terms)["loss"]
    f(table, answers).backward()
    g = torch.Generator().manual_seed(5)
    da, db = ((torch.randn(x.shape, generator=g) * 0.2).cuda() for x in (table, answers))
    slope = float((table.grad.double() * da).sum() + (answers.grad.double() * db).sum())
    with torch.no_grad():
        h = 2.0 ** -6
        by = float(f(table + h * da, answers + h * db).double() - f(table - h * da, answers - h * db).double()) / (2 * h)
    assert abs(slope - by) < 2.0 ** -11, (slope, by)


def test_a_step_in_a_graph():
    """Forward, loss with its gradient, gradients and clipping captured together, replayed on new inputs with eager work in between."""
    entities, off, entity, _, padded = _retrieval()
    table, answers = (x.cuda() for x in _model(entities))
    mask = lkg.entity_mask(off, entity, entities)
    target = padded[:, 2].contiguous()
    terms = _terms(len(target), torch.full((len(target),), -3.0, device="cuda"))

    def step():
        _, pooled, logits = _logits(table, answers, padded)
        got = lkg.policy_loss(logits, target, kl=0.1, mask=mask, gradient=True, **terms)
        grads = [lkg.embed_entities_backward((got["dlogits"] @ answers / LIST)[:, None].expand(-1, LIST, -1).contiguous(), padded, entities, scale=2.0),
                 got["dlogits"].t() @ pooled]
        return got["loss"], lkg.clip_gradients(grads, 0.02), grads
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, norm, grads = step()
    for i in range(4):
        table.copy_(_model(entities, 10 + i)[0])
        padded.copy_(padded.flip(0))
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        assert torch.equal(loss, want[0]) and torch.equal(norm, want[1]) and all(torch.equal(a, b) for a, b in zip(grads, want[2])), i


def test_serving_from_a_packed_table():
    entities, off, entity, hop, _ = _retrieval()
    g = torch.Generator().manual_seed(6)
    table = torch.randn(entities, 64, generator=g).cuda()
    keys, values = ((table @ (torch.randn(64, 2 * 64, generator=g) / 8).cuda()).view(entities, 2, 64).bfloat16() for _ in range(2))
    q = torch.randn(len(off) - 1, 1, 8, 64, generator=g).bfloat16()
    bias, buckets = torch.randn(8, 6, generator=g).bfloat16(), lkg.distance_buckets(6, 3, device="cpu")
    packed = lkg.pack_entities(keys, values)
    kw = dict(kv_heads=2, cap=30.0)
    got = lkg.read_packed(q.cuda(), packed, off, entity, hop=hop, bias=bias.cuda(), buckets=buckets.cuda(), **kw)
    res, tol = oracle.read_packed(q, packed.cpu(), off.cpu(), entity.cpu(), hop=hop.cpu(), bias=bias, buckets=buckets, **kw)
    for name in ("out", "lse"):
        oracle.check(got[name], res[name], tol[name], name)
    # a few rows learn, and are packed again in their places: as the whole table packed again
    ids = torch.arange(0, entities, 7, device="cuda")
    keys[ids], values[ids] = keys[ids] * 1.5, values[ids] - 1.0
    packed[ids] = lkg.pack_entities(keys[ids], values[ids])
    assert torch.equal(packed, lkg.pack_entities(keys, values))
    # read as the 16-bit table of what the rows stand for
    k16, v16 = lkg.unpack_entities(packed, 2, 64, dtype=torch.bfloat16)
    wide = lkg.read_entities(q.cuda(), k16, v16, off, entity, hop=hop, bias=bias.cuda(), buckets=buckets.cuda(), cap=30.0)
    four = lkg.read_packed(q.cuda(), packed, off, entity, hop=hop, bias=bias.cuda(), buckets=buckets.cuda(), **kw)
    # keys and values rounded to bfloat16 once more: 2^-8 of scores of some 2 and of values of some 3, and both results' own roundings
    assert float((wide["out"].float() - four["out"].float()).abs().max()) < 2.0 ** -8 * (2 * 2 * 3 + 3 + 2 * 3)


def test_the_example_trains_and_serves_with_them():
    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "answer.py")
    spec = importlib.util.spec_from_file_location("answer", at)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    got = example.main(steps=3, questions=8, policy_steps=2)
    assert len(got["losses"]) == 3 and len(got["rewards"]) == 2 and got["in_list"]
    assert len(got["norms"]) == 3 + 2 * 2 and all(0 <= n < float("inf") for n in got["norms"])  # (a model that is always right has no gradient)
    assert got["norms"][0] > 0
    assert 0 < got["packed_off_by"] < 1  # 4 bits: a step is a fifteenth of a group's range
