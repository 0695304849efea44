"""The calls that read a retrieval at the ends of their ranges (bounds: reading_oracle, as in test_gpu_reading)."""
import math

import numpy as np
import pytest
import torch

import paper_2604_18913_amd as lkg
import reading_oracle as oracle
from test_gpu_reading import HALVES, LENGTHS, _attend, _check, _check_logits, _check_read, _gpu, _inputs, _logit_case, _read

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------- attention
@pytest.mark.parametrize("dtype", HALVES, ids=["bf16", "fp16"])
@pytest.mark.parametrize("heads, dim, buckets, far", [(2, 128, 64, 1024), (35, 128, 64, 63), (2, 96, 33, 1024), (64, 64, 64, 34), (4, 128, 1, 5)])
def test_most_biases(heads, dim, buckets, far, dtype):
    # heads of one key head: the tables and sums of the gradients at the limits of LDS, and one bucket alone
    a, dout = _inputs(1, dtype, [70, 3], [140, 60], heads, 1, dim)
    g = torch.Generator().manual_seed(2)
    a |= dict(bias=torch.randn(heads, buckets, generator=g).to(dtype), buckets=torch.randint(0, buckets, (2 * far + 1,), generator=g, dtype=torch.int32))
    a["k_pos"] = torch.randint(-far - 3, far + 4, (200,), generator=g, dtype=torch.int32)
    _check({**a, "cap": 9.0}, dout)


@pytest.mark.parametrize("heads, far", [(4, 560), (36, 62), (3, 1024)])  # 4 x 1121 = 4484 places, 36 x 125 = 4500
def test_biases_beyond_the_limit_are_refused(heads, far):
    a, dout = _inputs(2, torch.bfloat16, [5], [9], heads, 1, 128)
    a |= dict(bias=torch.zeros(heads, 4, dtype=torch.bfloat16), buckets=torch.zeros(2 * far + 1, dtype=torch.int32))
    b = {k: _gpu(x) for k, x in a.items()}
    with pytest.raises(lkg.LogosKGError, match="BIAS_PLACES"):
        lkg.attend(**b)
    with pytest.raises(lkg.LogosKGError, match="BIAS_PLACES"):
        lkg.read_entities(b["q"][None, :1], b["k"], b["v"], torch.tensor([0, 9]).cuda(), bias=b["bias"], buckets=b["buckets"])


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
def test_tiles_of_several_blocks(dim, bias):
    # rows and keys beyond one block each way, all of whose tiles but the last are whole
    a, dout = _inputs(3, torch.bfloat16, [400, 190], [700, 129], 4, 2, dim, bias=bias)
    _check({**a, "causal": True, "prefix": torch.tensor([150, 0], dtype=torch.int32), "cap": 6.0}, dout)
    _check(a, dout)


def test_single_rows_and_axes_with_any_stride():
    a, dout = _inputs(4, torch.bfloat16, [1], [1], 1, 1, 64)
    odd = lambda x: x.cuda().as_strided(x.shape, (77, 33, 1))  # (an axis of one has no stride to speak of)
    out, lse = lkg.attend(odd(a["q"]), odd(a["k"]), odd(a["v"]), _gpu(a["q_off"]), _gpu(a["k_off"]))
    assert torch.equal(out.cpu(), a["v"])
    r = _read(4, torch.bfloat16, [50], 1, 1, 1, 64, bias=False)
    want = _check_read(r)
    b = {k: _gpu(x) for k, x in r.items()}
    got = lkg.read_entities(**{**b, "keys": b["keys"].as_strided((500, 1, 64), (64, 5, 1))})
    assert torch.equal(got["out"], want["out"])


def test_a_given_stream():
    a, dout = _inputs(5, torch.bfloat16, [300] * 8, [900] * 8, 8, 2, 128, bias=True)
    b, d = {k: _gpu(x) for k, x in a.items()}, _gpu(dout)
    pos = [b.pop(n) for n in ("q", "k", "v", "q_off", "k_off")]
    out, lse = lkg.attend(*pos, **b)
    want = (out, lse, *lkg.attend_backward(d, *pos[:3], out, lse, *pos[3:], **b))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):  # memory that goes round between the calls is that stream's own
        out, lse = lkg.attend(*pos, **b, stream=side)
        got = (out, lse, *lkg.attend_backward(d, *pos[:3], out, lse, *pos[3:], **b, stream=side))
        torch.full((1 << 22,), math.nan, device="cuda")
        side.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    r = {k: _gpu(x) for k, x in _read(5, torch.bfloat16, [9000, 40], 1, 8, 2, 64).items()}
    want = lkg.read_entities(**r)
    got = lkg.read_entities(**r, stream=side)
    mask = lkg.entity_mask(r["off"], r["entity"], 500, stream=side)
    logits = torch.zeros(2, 500, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    held = lkg.constrain_logits(logits, mask=mask, stream=side)
    side.synchronize()
    assert torch.equal(got["out"], want["out"])
    assert (held == 0).sum(1).tolist() == [len(set(x.tolist())) for x in r["entity"].cpu().split([9000, 40])]


def test_gradients_against_differences():
    # the loss sum(out * dout) along a direction of every input; out is rounded once (2^-11), so steps are wide
    a, dout = _inputs(6, torch.float16, [40, 21], [90, 33], 4, 2, 64, bias=True)
    a |= dict(causal=True, cap=4.0, prefix=torch.tensor([20, 5], dtype=torch.int32))
    b, d = {k: _gpu(x) for k, x in a.items()}, _gpu(dout)
    def loss(**other):
        return float((lkg.attend(**{**b, **other})[0].double() * d.double()).sum())
    out, lse = lkg.attend(**b)
    rest = {k: x for k, x in b.items() if k not in ("q", "k", "v", "q_off", "k_off")}
    grads = dict(zip(("q", "k", "v", "bias"), lkg.attend_backward(d, b["q"], b["k"], b["v"], out, lse, b["q_off"], b["k_off"], **rest)))
    for n, grad in grads.items():
        step = grad.float() / grad.float().norm() * 0.5  # along the gradient the difference is largest
        up, down = (b[n].float() + step).half(), (b[n].float() - step).half()
        want = loss(**{n: up}) - loss(**{n: down})
        got = float((grad.double() * (up.double() - down.double())).sum())
        # third order terms of a step of 1/2 along one direction, and the roundings of out: a fiftieth
        assert abs(got - want) <= 0.02 * abs(want), (n, got, want)


# ------------------------------------------------------------------------- masks
def _mask_words(off, ids, num_ids):
    bits = np.zeros((len(off) - 1, (num_ids + 63) // 64), dtype=np.uint64)
    for i in range(len(off) - 1):
        x = ids[off[i]:off[i + 1]]
        x = x[(x >= 0) & (x < num_ids)].astype(np.uint64)
        np.bitwise_or.at(bits[i], (x >> np.uint64(6)).astype(np.int64), np.uint64(1) << (x & np.uint64(63)))
    return bits.view(np.int64)


@pytest.mark.parametrize("ascending", [False, True])
@pytest.mark.parametrize("lengths, num_ids", [([70_000], 100_001), ([200_000, 3, 0, 90_000], 64_064), ([140_001, 0], 65), ([900, 0, 40], 110_000_000)])
def test_masks_of_long_lists_and_of_many_ids(lengths, num_ids, ascending):
    rng = np.random.default_rng(len(lengths))
    off = np.concatenate([[0], np.cumsum(lengths)])
    ids = rng.integers(-5, num_ids + 5, off[-1]).astype(np.int32)
    ids[::1001] = -2 ** 31
    if ascending:
        for i in range(len(lengths)):
            ids[off[i]:off[i + 1]].sort()
    out = torch.full((len(lengths), (num_ids + 63) // 64), -1, dtype=torch.int64, device="cuda")
    got = lkg.entity_mask(torch.from_numpy(off).cuda(), torch.from_numpy(ids).cuda(), num_ids, out=out)
    assert np.array_equal(got.cpu().numpy(), _mask_words(off, ids, num_ids))


# ------------------------------------------------------------------------- logits
@pytest.mark.parametrize("dtype", [torch.float32, *HALVES], ids=["fp32", "bf16", "fp16"])
def test_logits_after_a_history_beyond_16_bits(dtype):
    a = _logit_case(1, dtype, 3, 9001, 30, 5)
    g = torch.Generator().manual_seed(1)
    said = torch.tensor([0, 1, 2, 4095, 4096, 4097, 8000, 9000])
    long = said[torch.randint(0, 8, (70_000,), generator=g)].int()
    few, one = a["history"][:20], torch.full((66_000,), 4097, dtype=torch.int32)
    a |= dict(history=torch.cat([long, few, one]), history_off=torch.tensor([0, 70_000, 70_020, 136_020]), frequency=torch.full((3,), 2.0 ** -10))
    _check_logits(a)


@pytest.mark.parametrize("vocab", [300, 20_000])
def test_logits_with_more_biases_than_a_block_lists(vocab):
    a = _logit_case(2, torch.float32, 2, vocab, 10, 3)
    g = torch.Generator().manual_seed(2)
    a |= dict(bias_off=torch.tensor([0, 3000, 3700]), bias_id=torch.randint(-3, min(vocab, 900) + 3, (3700,), generator=g, dtype=torch.int32),
              bias_value=torch.randn(3700, generator=g))
    _check_logits(a)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_logits_and_out_at_different_places(shift, dtype):
    a = {k: _gpu(x) for k, x in _logit_case(3, dtype, 4, 5001, 300, 40).items()}
    want = lkg.constrain_logits(**a)
    room = torch.full((4 * 5001 + 8,), 3.0, dtype=dtype, device="cuda")
    got = lkg.constrain_logits(**a, out=room[shift:shift + 4 * 5001].view(4, 5001))
    assert torch.equal(got, want) and (room[:shift] == 3).all() and (room[shift + 4 * 5001:] == 3).all()


def test_logits_of_offsets_that_point_outside():
    a = {k: _gpu(x) for k, x in _logit_case(4, torch.float32, 2, 400, 20, 5).items()}
    n, m = a["history"].numel(), a["bias_id"].numel()
    want = lkg.constrain_logits(**{**a, "history_off": torch.tensor([0, n, n]).cuda(), "bias_off": torch.tensor([0, 0, m]).cuda()})
    got = lkg.constrain_logits(**{**a, "history_off": torch.tensor([-9, 1 << 40, n]).cuda(), "bias_off": torch.tensor([-(1 << 50), 0, 1 << 33]).cuda()})
    assert torch.equal(got, want)


# ------------------------------------------------------------------------- attention on either side of the rule for few rows
@pytest.mark.parametrize("dtype", HALVES, ids=["bf16", "fp16"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("heads, kv_heads, dim", [(32, 8, 128), (8, 8, 64), (24, 3, 96)])
def test_few_rows_and_many(heads, kv_heads, dim, bias, dtype):
    # 1,100 rows fill more blocks than the rule for few rows allows, their first 37 do not; both see the same keys, and rows
    # between 32 and 64 keys of both masks' ends
    a, _ = _inputs(21, dtype, [1100], [1130], heads, kv_heads, dim, bias=bias)
    if heads == 8:
        a["q"], a["q_off"] = a["q"].repeat(8, 1, 1)[:4500], torch.tensor([0, 4500])
        a["k"], a["v"], a["k_off"] = a["k"].repeat(5, 1, 1)[:4530], a["v"].repeat(5, 1, 1)[:4530], torch.tensor([0, 4530])
    n, m = a["q"].shape[0], a["k"].shape[0]
    kw = dict(causal=True, cap=5.0, prefix=torch.tensor([45], dtype=torch.int32).cuda(), **({"bias": a["bias"].cuda(), "buckets": a["buckets"].cuda()} if bias else {}))
    q, k, v = (a[x].cuda() for x in "qkv")
    many, many_lse = lkg.attend(q, k, v, a["q_off"].cuda(), a["k_off"].cuda(), **kw)
    few, few_lse = lkg.attend(q[:37], k[:67], v[:67], torch.tensor([0, 37]).cuda(), torch.tensor([0, 67]).cuda(), **kw)
    # the same rows of the same keys: each within the oracle's bound of the same value
    small = {**a, "q": a["q"][:37], "k": a["k"][:67], "v": a["v"][:67], "q_off": torch.tensor([0, 37]), "k_off": torch.tensor([0, 67]),
             "causal": True, "cap": 5.0, "prefix": torch.tensor([45], dtype=torch.int32)}
    assert m - n == 30
    res, tol = oracle.attention(**small)
    for got, lse in ((few, few_lse), (many[:37], many_lse[:37])):
        oracle.check(got, res["out"], tol["out"], "out")
        oracle.check(lse, res["lse"], tol["lse"], "lse")


@pytest.mark.parametrize("lengths", [([1], [1]), ([31, 1, 0, 33], [31, 33, 5, 0]), ([40], [2000]), ([3] * 9, [1, 0, 129, 128, 127, 32, 33, 5, 400])])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dim", [40, 128])
def test_few_rows(dim, causal, lengths):
    a, dout = _inputs(22, torch.float16, *lengths, 4, 1, dim, bias=True, far=30)
    if causal:
        a["prefix"] = torch.tensor([(5 * i + 1) % 40 for i in range(len(lengths[0]))], dtype=torch.int32)
    _check({**a, "causal": causal}, dout)


# heads so many that a document of one row is over the rule's limit: the form for many rows at lengths where it can go wrong
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lengths", [n for n in LENGTHS if n != "many"])
def test_lengths_under_many_heads(lengths, causal):
    rows, keys = LENGTHS[lengths]
    a, dout = _inputs(len(rows), torch.bfloat16, rows, keys, 264, 264, 16, bias=True)
    if causal:
        a["prefix"] = torch.tensor([(7 * i) % 50 for i in range(len(rows))], dtype=torch.int32)
    _check({**a, "causal": causal, "cap": 4.0}, dout, lengths)


@pytest.mark.parametrize("dtype", HALVES, ids=["bf16", "fp16"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("cap", [0.0, 3.0, 50.0])
@pytest.mark.parametrize("heads, kv_heads, dim", [(132, 132, 128), (264, 132, 96), (260, 260, 64), (520, 260, 40)])
def test_many_heads_types_and_scores(heads, kv_heads, dim, cap, bias, dtype):
    a, dout = _inputs(7, dtype, [37, 2, 90], [50, 140, 90], heads, kv_heads, dim, bias=bias)
    got = lkg.attend(**{k: _gpu(x) for k, x in {**a, "causal": True, "cap": cap, "prefix": torch.tensor([30, 0, 11], dtype=torch.int32)}.items()})
    res, tol = oracle.attention(**a, causal=True, cap=cap, prefix=torch.tensor([30, 0, 11], dtype=torch.int32))
    for x, n in zip(got, ("out", "lse")):
        oracle.check(x, res[n], tol[n], n)


def test_many_heads_rows_that_see_nothing_far_positions_and_other_documents():
    a, dout = _inputs(12, torch.bfloat16, [40, 8, 30], [10, 0, 70], 260, 260, 16, bias=True)
    got = _check({**a, "causal": True}, dout)
    assert (got["out"][:30] == 0).all() and (got["lse"][:30] == -math.inf).all() and (got["out"][40:48] == 0).all()
    g = torch.Generator().manual_seed(1)
    k_pos, q_pos = -1 - torch.randint(0, 4, (80,), generator=g, dtype=torch.int32), torch.arange(78, dtype=torch.int32)
    k_pos[::3], q_pos[::2] = 2 ** 31 - 1, -2 ** 31
    want = _check({**a, "q_pos": q_pos, "k_pos": k_pos}, dout)
    a["q"][:40], a["k"][:10], a["v"][:10] = math.nan, math.inf, math.nan
    got = _attend({**a, "q_pos": q_pos, "k_pos": k_pos}, dout)
    assert all(torch.equal(got[n][40:], want[n][40:]) for n in ("out", "lse", "dq"))


def test_many_heads_large_scores():
    a, dout = _inputs(11, torch.bfloat16, [50], [200], 260, 260, 64, spread=6.0)
    res, _ = oracle.attention(**a)
    got = lkg.attend(**{k: _gpu(x) for k, x in a.items()})
    assert torch.allclose(got[1].cpu().double(), res["lse"], rtol=2e-5)  # (as with few heads)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("docs", [7, 8, 40])
def test_documents_of_very_different_lengths(docs, causal):
    # blocks enough to be put in order from eight documents on; some documents have no rows, some no keys
    rows = [(97 * i) % 260 if i % 5 else 0 for i in range(docs)]
    keys = [(61 * i * i) % 390 if i % 7 else 0 for i in range(docs)]
    a, dout = _inputs(23, torch.bfloat16, rows, keys, 64, 32, 16, bias=True)
    if causal:
        a["prefix"] = torch.tensor([(13 * i) % 90 for i in range(docs)], dtype=torch.int32)
    got = _check({**a, "causal": causal}, dout)
    again = _attend({**a, "causal": causal}, dout)
    assert all(torch.equal(got[n], again[n]) for n in got)


# ------------------------------------------------------------------------- biases that hide
def _hiding(dtype, low, kv_heads, heads, cap):
    """Keys at distance 5 and beyond read a bucket whose bias is `low`; the case without them, and which they are."""
    a, dout = _inputs(24, dtype, [70], [300], heads, kv_heads, 64)
    g = torch.Generator().manual_seed(3)
    hidden = torch.rand(300, generator=g) < 0.4
    hidden[64:130] = True  # (a whole tile of them)
    near = torch.randint(0, 3, (300,), generator=g, dtype=torch.int32)
    buckets = torch.tensor([0, 0, 0, 0, 0, 0, 1, 0, 2, 2, 3], dtype=torch.int32)  # distances -5 .. 5
    bias = torch.randn(heads, 4, generator=g).to(dtype)
    bias[:, 3] = low
    a |= dict(bias=bias, buckets=buckets, cap=cap, q_pos=torch.zeros(70, dtype=torch.int32), k_pos=torch.where(hidden, 9 + near, near))
    seen = {**a, "k": a["k"][~hidden], "v": a["v"][~hidden], "k_pos": a["k_pos"][~hidden], "k_off": torch.tensor([0, int((~hidden).sum())])}
    return a, seen, hidden, dout


@pytest.mark.parametrize("heads, kv_heads", [(4, 2), (260, 260)])
@pytest.mark.parametrize("cap", [0.0, 6.0])
@pytest.mark.parametrize("dtype, low", [(torch.bfloat16, -math.inf), (torch.bfloat16, torch.finfo(torch.bfloat16).min), (torch.float16, -math.inf), (torch.float16, -65504.0)])
def test_biases_that_hide_keys(dtype, low, cap, heads, kv_heads):
    a, seen, hidden, dout = _hiding(dtype, low, kv_heads, heads, cap)
    got = _attend(a, dout)
    res, tol = oracle.attention(**{**seen, "bias": seen["bias"].clone().clamp(min=-9.0)}, dout=dout)  # (no key is left that reads it)
    for n in ("out", "lse", "dq"):
        oracle.check(got[n], res[n], tol[n], n)
    for n in ("dk", "dv"):
        oracle.check(got[n].cpu()[~hidden], res[n], tol[n], n)
        assert (got[n].cpu()[hidden] == 0).all()
    oracle.check(got["dbias"].cpu()[:, :3], res["dbias"][:, :3], tol["dbias"][:, :3], "dbias")
    assert (got["dbias"][:, 3] == 0).all()


@pytest.mark.parametrize("heads, kv_heads", [(4, 2), (260, 260)])
@pytest.mark.parametrize("cap", [0.0, 6.0])
def test_biases_that_hide_everything(cap, heads, kv_heads):
    a, seen, hidden, dout = _hiding(torch.bfloat16, -math.inf, kv_heads, heads, cap)
    a["bias"][:] = -math.inf
    got = _attend(a, dout)
    assert all((got[n] == 0).all() for n in ("out", "dq", "dk", "dv", "dbias")) and (got["lse"] == -math.inf).all()


@pytest.mark.parametrize("length", [40, 3000])
@pytest.mark.parametrize("cap", [0.0, 6.0])
def test_read_biases_that_hide(cap, length):
    a = _read(25, torch.bfloat16, [length, 90], 2, 4, 2, 64, cap=cap)
    a["buckets"] = torch.tensor([0, 0, 0, 0, 1, 2, 3], dtype=torch.int32)  # hops 0 .. 3
    a["bias"][:, 3] = -math.inf
    a["hop"][length:] = 3  # nothing left of the second list
    got = lkg.read_entities(**{k: _gpu(x) for k, x in a.items()})
    keep = a["hop"] != 3
    seen = {**a, "entity": a["entity"][keep], "hop": a["hop"][keep], "off": torch.tensor([0, int(keep.sum()), int(keep.sum())]), "bias": a["bias"].clone().clamp(min=-9.0)}
    res, tol = oracle.read(**seen)
    for n in ("out", "lse"):
        oracle.check(got[n], res[n], tol[n], n)
    assert (got["out"][1] == 0).all() and (got["lse"][1] == -math.inf).all()


@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("dim, heads, kv_heads", [(64, 4, 2), (96, 12, 4)])
def test_gradients_of_rows_with_few_keys(dim, heads, kv_heads, cap):
    # dy = p (dP - delta) cancels where keys are few: with one it is 0.  delta from the rounded output would be off by 2^-9 of
    # sums of `dim` products (some 1e-2); in 32 bits by 2^-22 of p, that is 1e-5 of the same
    a, dout = _inputs(26, torch.bfloat16, [50, 130, 7], [1, 1, 1], heads, kv_heads, dim, bias=True)
    got = _attend({**a, "cap": cap}, dout)
    assert got["dq"].abs().max() < 2e-4
    # two and three keys: the roundings of dz and of the result, 0.0017 of the norm each
    a, dout = _inputs(27, torch.bfloat16, [50, 130, 64], [2, 3, 2], heads, kv_heads, dim, bias=True)
    got = _check({**a, "cap": cap}, dout)
    want = oracle.attention(**a, cap=cap, dout=dout)[0]["dq"]
    assert (got["dq"].cpu().double() - want).norm() < 0.0035 * want.norm()
