"""The calls that read a retrieval into a language model against their 64-bit definitions (bounds: reading_oracle)."""
import math

import pytest
import torch

import paper_2604_18913_amd as lkg
import reading_oracle as oracle

pytestmark = pytest.mark.gpu
HALVES = [torch.bfloat16, torch.float16]


def _gpu(x):
    return x.cuda() if isinstance(x, torch.Tensor) else x


def _inputs(seed, dtype, rows, keys, heads, kv_heads, dim, bias=False, far=16, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: (torch.randn(*s, generator=g) * spread).to(dtype)
    q_off, k_off = (torch.tensor([0] + list(x)).cumsum(0) for x in (rows, keys))
    n, m = sum(rows), sum(keys)
    a = dict(q=r(n, heads, dim), k=r(m, kv_heads, dim), v=r(m, kv_heads, dim), q_off=q_off, k_off=k_off)
    if bias:
        a |= dict(bias=r(heads, 12), buckets=lkg.distance_buckets(12, far, device="cpu"))
    return a, r(n, heads, dim)


def _attend(a, dout):
    b = {k: _gpu(x) for k, x in a.items()}
    out, lse = lkg.attend(**b)
    d = _gpu(dout)
    dq, dk, dv, dbias = lkg.attend_backward(d, b.pop("q"), b.pop("k"), b.pop("v"), out, lse, b.pop("q_off"), b.pop("k_off"), **b)
    return dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv, dbias=dbias)


def _check(a, dout, what=""):
    got = _attend(a, dout)
    res, tol = oracle.attention(**a, dout=dout)
    for name in res:
        oracle.check(got[name], res[name], tol[name], f"{what} {name}")
    return got


LENGTHS = {
    "one": ([1], [1]), "row_of_keys": ([1], [300]), "tile": ([32], [64]), "tile_and_one": ([33], [65]), "block": ([128], [128]),
    "block_and_one": ([129], [129]), "ragged": ([5, 0, 40, 1, 131, 17], [70, 3, 0, 1, 131, 200]), "long": ([70], [1000]),
    "tall": ([500], [30]), "many": ([3] * 150, [7, 0, 2] * 50),
}


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lengths", list(LENGTHS))
def test_lengths(lengths, causal):
    rows, keys = LENGTHS[lengths]
    a, dout = _inputs(len(rows), torch.bfloat16, rows, keys, 4, 2, 64, bias=True)
    if causal:
        a["prefix"] = torch.tensor([(7 * i) % 50 for i in range(len(rows))], dtype=torch.int32)
    _check({**a, "causal": causal, "cap": 4.0}, dout, lengths)


@pytest.mark.parametrize("dtype", HALVES, ids=["bf16", "fp16"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("cap", [0.0, 3.0, 50.0])
@pytest.mark.parametrize("heads, kv_heads, dim", [(4, 4, 128), (6, 2, 80), (5, 1, 40), (2, 2, 8), (12, 4, 96)])
def test_heads_types_and_scores(heads, kv_heads, dim, cap, bias, dtype):
    a, dout = _inputs(7, dtype, [37, 2, 90], [50, 140, 90], heads, kv_heads, dim, bias=bias)
    _check({**a, "causal": True, "cap": cap, "prefix": torch.tensor([30, 0, 11], dtype=torch.int32)}, dout)


@pytest.mark.parametrize("scale", [-0.3, 0.0, 1.0])
def test_scales(scale):
    a, dout = _inputs(8, torch.bfloat16, [40], [80], 2, 1, 64)
    _check({**a, "scale": scale}, dout)
    _check({**a, "scale": scale, "cap": 2.0}, dout)


def test_many_heads_share_a_key_head():
    a, dout = _inputs(9, torch.bfloat16, [3, 9], [40, 5], 128, 1, 64, bias=True)
    _check({**a, "causal": True}, dout)


def test_positions_of_retrieved_entities_and_far_ones():
    a, dout = _inputs(10, torch.float16, [60, 20], [300, 20], 4, 2, 64, bias=True, far=3)
    g = torch.Generator().manual_seed(1)
    k_pos = -1 - torch.randint(0, 4, (320,), generator=g, dtype=torch.int32)
    q_pos = torch.arange(80, dtype=torch.int32)
    _check({**a, "q_pos": q_pos, "k_pos": k_pos}, dout)
    k_pos[::3], q_pos[::2] = 2 ** 31 - 1, -2 ** 31  # (the difference does not fit)
    _check({**a, "q_pos": q_pos, "k_pos": k_pos}, dout)


def test_large_scores_and_equal_ones():
    a, dout = _inputs(11, torch.bfloat16, [50], [200], 2, 2, 64, spread=6.0)
    res, _ = oracle.attention(**a)
    got = lkg.attend(**{k: _gpu(x) for k, x in a.items()})
    # one key has nearly all the weight: scores of a few hundred are known to 2^-16 of themselves
    assert torch.allclose(got[1].cpu().double(), res["lse"], rtol=2e-5)
    a["k"][:] = a["k"][:1]
    a["q"] /= 16
    _check(a, dout / 16)


def test_rows_that_see_nothing():
    a, dout = _inputs(12, torch.bfloat16, [40, 8], [10, 0], 2, 2, 64, bias=True)
    got = _check({**a, "causal": True}, dout)  # the first 30 rows of 40 stand before the first key
    assert (got["out"][:30] == 0).all() and (got["lse"][:30] == -math.inf).all() and (got["dq"][:30] == 0).all()
    assert (got["out"][40:] == 0).all() and (got["dq"][40:] == 0).all()
    empty = {**a, "k": a["k"][:0], "v": a["v"][:0], "k_off": torch.zeros(3, dtype=torch.int64)}
    got = _attend(empty, dout)
    assert all((got[n] == 0).all() for n in ("out", "dq", "dbias")) and (got["lse"] == -math.inf).all() and got["dk"].numel() == 0


def test_no_rows_and_no_documents():
    a, dout = _inputs(13, torch.bfloat16, [0, 0], [5, 0], 2, 2, 64, bias=True)
    got = _attend(a, dout)
    assert got["out"].numel() == 0 and (got["dk"] == 0).all() and (got["dv"] == 0).all() and (got["dbias"] == 0).all()
    a, dout = _inputs(13, torch.bfloat16, [], [], 2, 2, 64)
    a |= dict(q_off=torch.zeros(1, dtype=torch.int64), k_off=torch.zeros(1, dtype=torch.int64))
    assert _attend(a, dout)["out"].numel() == 0


def test_strided_inputs():
    a, dout = _inputs(14, torch.bfloat16, [30, 50], [60, 20], 4, 2, 64)
    want = _attend(a, dout)
    packed = torch.full((80, 8, 72), math.nan, dtype=torch.bfloat16)  # q, k and v of a row beside each other, gaps behind a head
    packed[:, :4, :64], packed[:, 4:6, :64], packed[:, 6:, :64] = a["q"], a["k"], a["v"]
    packed = packed.cuda()
    b = {**{k: _gpu(x) for k, x in a.items()}, "q": packed[:, :4, :64], "k": packed[:, 4:6, :64], "v": packed[:, 6:, :64]}
    out, lse = lkg.attend(**b)
    assert torch.equal(out, want["out"]) and torch.equal(lse, want["lse"])
    grads = lkg.attend_backward(_gpu(dout), b["q"], b["k"], b["v"], out, lse, b["q_off"], b["k_off"])
    assert all(torch.equal(x, want[n]) for x, n in zip(grads, ("dq", "dk", "dv")))


def test_documents_do_not_see_each_other():
    a, dout = _inputs(15, torch.bfloat16, [30, 20, 9], [60, 20, 70], 2, 1, 64, bias=True)
    want = _attend(a, dout)
    a["q"][30:50], a["k"][60:80], a["v"][60:80] = math.nan, math.inf, math.nan
    got = _attend(a, dout)
    for n in ("out", "lse", "dq"):
        assert torch.equal(got[n][:30], want[n][:30]) and torch.equal(got[n][50:], want[n][50:])
    for n in ("dk", "dv"):
        assert torch.equal(got[n][:60], want[n][:60]) and torch.equal(got[n][80:], want[n][80:])


def test_same_bits_every_time():
    a, dout = _inputs(16, torch.bfloat16, [300, 40], [700, 300], 8, 2, 128, bias=True)
    a |= dict(causal=True, cap=20.0)
    first = _attend(a, dout)
    for _ in range(3):
        again = _attend(a, dout)
        assert all(torch.equal(first[n], again[n]) for n in first)


def test_offsets_that_point_outside():
    a, dout = _inputs(17, torch.bfloat16, [30], [60], 2, 1, 64)
    want = _attend(a, dout)
    got = _attend({**a, "q_off": torch.tensor([-5, 1000]), "k_off": torch.tensor([-(1 << 40), 1 << 40])}, dout)
    assert torch.equal(got["out"], want["out"])


def test_attend_on_another_stream_and_in_a_graph():
    a, dout = _inputs(18, torch.bfloat16, [70, 20], [90, 33], 4, 2, 64, bias=True)
    want = _attend(a, dout)
    b, d = {k: _gpu(x) for k, x in a.items()}, _gpu(dout)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pos = (b["q"], b["k"], b["v"])
    kw = dict(bias=b["bias"], buckets=b["buckets"])
    with torch.cuda.stream(side):
        out, lse = lkg.attend(*pos, b["q_off"], b["k_off"], **kw)
        grads = lkg.attend_backward(d, *pos, out, lse, b["q_off"], b["k_off"], **kw)
    side.synchronize()
    assert torch.equal(out, want["out"]) and all(torch.equal(x, want[n]) for x, n in zip(grads, ("dq", "dk", "dv", "dbias")))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = lkg.attend(*pos, b["q_off"], b["k_off"], **kw)
        grads = lkg.attend_backward(d, *pos, out, lse, b["q_off"], b["k_off"], **kw)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want["out"]) and all(torch.equal(x, want[n]) for x, n in zip(grads, ("dq", "dk", "dv", "dbias")))
        torch.randn(1000, device="cuda").sum().item()


def test_attend_refusals():
    a, dout = _inputs(19, torch.bfloat16, [4], [6], 2, 1, 64, bias=True)
    b = {k: _gpu(x) for k, x in a.items()}
    for wrong in (dict(q=b["q"].float()), dict(k=b["k"].half()), dict(v=b["v"][:5]), dict(k=b["k"].transpose(0, 1)), dict(q_off=b["q_off"].int()),
                  dict(k_off=b["k_off"][:1]), dict(bias=b["bias"].float()), dict(buckets=None), dict(buckets=b["buckets"][1:]), dict(bias=None),
                  dict(prefix=torch.zeros(1, dtype=torch.int32, device="cuda")), dict(q_pos=torch.zeros(3, dtype=torch.int32, device="cuda")),
                  dict(k_off=a["k_off"]), dict(q=b["q"].transpose(1, 2))):
        with pytest.raises(ValueError):
            lkg.attend(**{**b, **wrong})
    with pytest.raises(lkg.LogosKGError, match="aligned"):
        lkg.attend(**{**b, "k": torch.zeros(6 * 68, dtype=torch.bfloat16, device="cuda").view(6, 1, 68)[:, :, :64]})
    with pytest.raises(lkg.LogosKGError, match="dim"):
        lkg.attend(**{**b, **{n: b[n][..., :60].contiguous() for n in "qkv"}})


# ------------------------------------------------------------------------- read_entities
def _lists(seed, lengths, entities, hops=4):
    g = torch.Generator().manual_seed(seed)
    off = torch.tensor([0] + list(lengths)).cumsum(0)
    n = int(off[-1])
    return off, torch.randint(0, max(entities, 1), (n,), generator=g, dtype=torch.int32), torch.randint(0, hops, (n,), generator=g, dtype=torch.uint8)


def _read(seed, dtype, lengths, tokens, heads, kv_heads, dim, entities=500, bias=True, **kw):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g).to(dtype)
    off, entity, hop = _lists(seed, lengths, entities)
    a = dict(q=r(len(lengths), tokens, heads, dim), keys=r(entities, kv_heads, dim), values=r(entities, kv_heads, dim), off=off, entity=entity, hop=hop)
    if bias:
        a |= dict(bias=r(heads, 6), buckets=lkg.distance_buckets(6, 3, device="cpu"))
    return {**a, **kw}


def _check_read(a, what=""):
    got = lkg.read_entities(**{k: _gpu(x) for k, x in a.items()})
    res, tol = oracle.read(**a)
    for n in ("out", "lse"):
        oracle.check(got[n], res[n], tol[n], f"{what} {n}")
    return got


@pytest.mark.parametrize("lengths", [[1], [0], [31], [32, 33], [128], [129], [0, 5, 0, 700, 1], [3000], [64] * 70, [20_000, 3, 0, 9000]],
                         ids=lambda x: "x".join(map(str, x[:5])))
def test_read_lengths(lengths):
    _check_read(_read(len(lengths), torch.bfloat16, lengths, 1, 8, 2, 64, cap=5.0))


@pytest.mark.parametrize("dtype", HALVES, ids=["bf16", "fp16"])
@pytest.mark.parametrize("cap, bias", [(0.0, False), (0.0, True), (4.0, False), (30.0, True)])
@pytest.mark.parametrize("tokens, heads, kv_heads, dim", [(1, 4, 4, 128), (2, 6, 2, 80), (3, 5, 1, 40), (1, 2, 2, 8), (9, 16, 2, 64)])
def test_read_heads_types_and_scores(tokens, heads, kv_heads, dim, cap, bias, dtype):
    _check_read(_read(3, dtype, [40, 0, 333, 150], tokens, heads, kv_heads, dim, bias=bias, cap=cap))


def test_read_padding_and_bad_ids():
    a = _read(4, torch.bfloat16, [100, 40, 300], 2, 4, 2, 64)
    a["entity"][::3] = -1
    a["entity"][1::7] = 500
    a["entity"][100:140] = 2 ** 31 - 1  # nothing left of the second list
    got = _check_read(a)
    assert (got["out"][1] == 0).all() and (got["lse"][1] == -math.inf).all()


def test_read_rows_in_place_and_positions():
    a = _read(5, torch.float16, [300, 200], 2, 4, 2, 64)
    a |= dict(entity=None, hop=torch.randint(0, 255, (500,), dtype=torch.uint8), q_pos=torch.tensor([3, -7], dtype=torch.int32))
    _check_read(a)
    _check_read({**a, "hop": None})


def test_read_strided_table():
    a = _read(6, torch.bfloat16, [70, 400], 1, 4, 2, 64)
    want = lkg.read_entities(**{k: _gpu(x) for k, x in a.items()})
    both = torch.full((500, 2, 2, 72), math.nan, dtype=torch.bfloat16)
    both[:, 0, :, :64], both[:, 1, :, :64] = a["keys"], a["values"]
    both = both.cuda()
    got = lkg.read_entities(**{**{k: _gpu(x) for k, x in a.items()}, "keys": both[:, 0, :, :64], "values": both[:, 1, :, :64]})
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])


def test_read_unlisted_rows_are_not_read():
    a = _read(7, torch.bfloat16, [200, 90], 1, 4, 2, 64)
    want = lkg.read_entities(**{k: _gpu(x) for k, x in a.items()})
    other = torch.ones(500, dtype=torch.bool)
    other[a["entity"].long()] = False
    a["keys"][other], a["values"][other] = math.inf, math.nan
    got = lkg.read_entities(**{k: _gpu(x) for k, x in a.items()})
    assert torch.equal(got["out"], want["out"])


def test_read_places_beyond_32_bits():
    # a table whose last rows lie past 2^31 elements and 2^32 bytes
    entities, dim = 2 ** 21 + 5000, 128
    keys = torch.zeros(entities, 8, dim, dtype=torch.bfloat16, device="cuda")
    values = torch.zeros(entities, 8, dim, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(8)
    last = torch.randn(64, 8, dim, generator=g).to(torch.bfloat16)
    keys[-64:], values[-64:] = last.cuda(), last.flip(0).cuda()
    q = torch.randn(1, 1, 8, dim, generator=g).to(torch.bfloat16)
    entity = torch.arange(entities - 64, entities, dtype=torch.int32)
    got = lkg.read_entities(q.cuda(), keys, values, torch.tensor([0, 64]).cuda(), entity.cuda())
    res, tol = oracle.read(q, last, last.flip(0), torch.tensor([0, 64]))
    oracle.check(got["out"], res["out"], tol["out"])


def test_read_in_a_graph():
    a = {k: _gpu(x) for k, x in _read(9, torch.bfloat16, [900, 0, 4000], 1, 8, 2, 128).items()}
    want = lkg.read_entities(**a)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = lkg.read_entities(**a)
    for _ in range(3):
        got["out"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
        torch.randn(1000, device="cuda").sum().item()


# ------------------------------------------------------------------------- masks, logits
@pytest.mark.parametrize("num_ids", [1, 63, 64, 65, 1000, 70_001])
@pytest.mark.parametrize("lengths", [[0], [1], [5, 0, 300], [2000], [64] * 40, [0] * 100 + [3] * 5])
def test_entity_mask(lengths, num_ids):
    off, ids, _ = _lists(num_ids, lengths, num_ids)
    ids[::11], ids[3::13] = -1, num_ids
    for order in (ids, torch.cat([x.sort().values for x in ids.split(lengths)])):
        got = lkg.entity_mask(off.cuda(), order.cuda(), num_ids)
        assert got.cpu().tolist() == oracle.entity_mask(off, order, num_ids)


def _logit_case(seed, dtype, rows, vocab, history, biases, mask=True):
    g = torch.Generator().manual_seed(seed)
    pick = lambda n, most: [0 if i % 3 == 2 else int(torch.randint(0, most + 1, (1,), generator=g)) for i in range(n)]
    h_off, b_off = (torch.tensor([0] + pick(rows, most)).cumsum(0) for most in (history, biases))
    a = dict(logits=(torch.randn(rows, vocab, generator=g) * 3).to(dtype), history_off=h_off,
             history=torch.randint(-2, vocab + 2, (int(h_off[-1]),), generator=g, dtype=torch.int32),
             repetition=torch.rand(rows, generator=g) + 0.75, presence=torch.rand(rows, generator=g), frequency=torch.rand(rows, generator=g),
             bias_off=b_off, bias_id=torch.randint(-1, vocab + 1, (int(b_off[-1]),), generator=g, dtype=torch.int32),
             bias_value=torch.randn(int(b_off[-1]), generator=g) * 5)
    if mask:
        a["mask"] = torch.randint(-2 ** 63, 2 ** 63 - 1, (rows, (vocab + 63) // 64), generator=g)
    return a


def _check_logits(a):
    got = lkg.constrain_logits(**{k: _gpu(x) for k, x in a.items()})
    res = oracle.logits(a["logits"], **{k: x for k, x in a.items() if k != "logits"})
    # five roundings in 32 bits of terms up to the count's penalty, one to the type
    unit = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[a["logits"].dtype]
    fine = torch.isfinite(res)
    oracle.check(got, res, unit * res.abs().where(fine, torch.tensor(0.0, dtype=torch.float64)) + 2.0 ** -16, "logits")


@pytest.mark.parametrize("dtype", [torch.float32, *HALVES], ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows, vocab, history, biases", [(1, 1, 3, 1), (3, 500, 8, 4), (2, 8192, 50, 9), (2, 8193, 400, 9), (4, 20_011, 3000, 300), (70, 65, 9, 2)])
def test_logits(rows, vocab, history, biases, dtype):
    _check_logits(_logit_case(vocab, dtype, rows, vocab, history, biases))
    _check_logits(_logit_case(vocab + 1, dtype, rows, vocab, history, biases, mask=False))


def test_logits_parts_alone():
    a = _logit_case(3, torch.float32, 5, 300, 20, 6)
    for keep in (("logits",), ("logits", "mask"), ("logits", "bias_off", "bias_id", "bias_value"), ("logits", "history", "history_off", "repetition"),
                 ("logits", "history", "history_off", "frequency"), ("logits", "history", "history_off", "presence", "mask")):
        _check_logits({k: a[k] for k in keep})


def test_logits_nothing_allowed_and_hidden_values():
    a = {k: _gpu(x) for k, x in _logit_case(4, torch.bfloat16, 3, 200, 9, 3).items()}
    a["mask"][:] = 0
    a["logits"][:, ::2] = math.nan
    a["logits"][:, 1::4] = math.inf
    assert (lkg.constrain_logits(**a) == -math.inf).all()


def test_logits_in_place_and_strided():
    a = {k: _gpu(x) for k, x in _logit_case(5, torch.float16, 6, 701, 30, 5).items()}
    want = lkg.constrain_logits(**a)
    wide = torch.full((6, 800), 7.0, dtype=torch.float16, device="cuda")
    wide[:, 50:751] = a["logits"]
    got = lkg.constrain_logits(**{**a, "logits": wide[:, 50:751]}, out=wide[:, 50:751])
    assert torch.equal(got, want) and (wide[:, :50] == 7).all() and (wide[:, 751:] == 7).all()


def test_logits_and_mask_refusals():
    a = {k: _gpu(x) for k, x in _logit_case(6, torch.float32, 3, 100, 9, 3).items()}
    for wrong in (dict(logits=a["logits"].double()), dict(logits=a["logits"].t()), dict(history_off=None), dict(history=None), dict(bias_value=None),
                  dict(mask=a["mask"][:, :1].contiguous()), dict(repetition=a["repetition"].half()), dict(history=a["history"].long()),
                  dict(out=torch.empty(3, 101, device="cuda")), dict(bias_off=a["bias_off"][1:])):
        with pytest.raises(ValueError):
            lkg.constrain_logits(**{**a, **wrong})
    with pytest.raises(ValueError):
        lkg.entity_mask(a["history_off"], a["history"].long(), 10)


# ------------------------------------------------------------------------- from a retrieval to an answer
def test_from_a_retrieval_to_an_answer():
    import kggen
    w = kggen.config1()
    g = lkg.Graph(w.subj, w.rel, w.obj, w.num_entities, w.num_relations)
    res = g.khop(w.seed_off, w.seeds, 2)
    off, (entity, hop, _) = torch.from_numpy(res.offsets()).cuda(), res.fetch(want_pred=False)
    Q = off.numel() - 1
    gen = torch.Generator().manual_seed(1)
    keys, values = (torch.randn(w.num_entities, 2, 64, generator=gen).to(torch.bfloat16) for _ in range(2))
    q = torch.randn(Q, 1, 8, 64, generator=gen).to(torch.bfloat16)
    bias, buckets = torch.randn(8, 6, generator=gen).to(torch.bfloat16), lkg.distance_buckets(6, 3, device="cpu")
    got = lkg.read_entities(q.cuda(), keys.cuda(), values.cuda(), off, entity, hop=hop, bias=bias.cuda(), buckets=buckets.cuda(), cap=30.0)
    want, tol = oracle.read(q, keys, values, off.cpu(), entity.cpu(), cap=30.0, bias=bias, buckets=buckets, hop=hop.cpu())
    oracle.check(got["out"], want["out"], tol["out"])
    mask = lkg.entity_mask(off, entity, w.num_entities)
    logits = torch.randn(Q, w.num_entities, device="cuda")
    answer = lkg.constrain_logits(logits, mask=mask).argmax(1)
    for i in range(Q):
        mine = entity[off[i]:off[i + 1]].long()
        assert answer[i] == mine[logits[i][mine].argmax()]
