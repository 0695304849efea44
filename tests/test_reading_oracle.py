"""Pins of the 64-bit definitions that the reading calls are tested against, and what those calls refuse before they
touch a GPU (no GPU needed)."""
import ctypes
import math
import os

import pytest
import torch

import paper_2604_18913_amd as lkg
import reading_oracle as oracle
from paper_2604_18913_amd import reading


def _case(seed, rows, keys, heads=2, kv_heads=1, dim=8, buckets=6, far=4):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16)
    q_off, k_off = (torch.tensor([0] + x).cumsum(0) for x in (rows, keys))
    q, k, v = r(sum(rows), heads, dim), r(sum(keys), kv_heads, dim), r(sum(keys), kv_heads, dim)
    return q, k, v, q_off, k_off, r(heads, buckets), lkg.distance_buckets(buckets, far, device="cpu"), r(sum(rows), heads, dim)


def test_attention_by_hand():
    # two keys, products 1 and 3, scale 1, bias +2 on the first: weights e^3 : e^3
    q = torch.tensor([[[1.0] + [0.0] * 7]], dtype=torch.bfloat16)
    k = torch.zeros(2, 1, 8, dtype=torch.bfloat16)
    k[0, 0, 0], k[1, 0, 0] = 1.0, 3.0
    v = torch.zeros(2, 1, 8, dtype=torch.bfloat16)
    v[0, 0, 1], v[1, 0, 1] = 4.0, 8.0
    off = torch.tensor([0, 1]), torch.tensor([0, 2])
    bias, buckets = torch.tensor([[0.0, 2.0]], dtype=torch.bfloat16), torch.tensor([1, 0, 0], dtype=torch.int32)
    res, _ = oracle.attention(q, k, v, *off, scale=1.0, bias=bias, buckets=buckets)  # the row stands at 1: distances -1, 0
    assert res["out"][0, 0, 1] == pytest.approx(6.0) and res["lse"][0, 0] == pytest.approx(3 + math.log(2))
    res, _ = oracle.attention(q, k, v, *off, scale=1.0, cap=2.0)
    w = [math.exp(2 * math.tanh(z / 2)) for z in (1, 3)]
    assert res["out"][0, 0, 1] == pytest.approx((4 * w[0] + 8 * w[1]) / sum(w))


def test_masks_by_hand():
    assert oracle.visible(2, 4, True, 0).tolist() == [[True, True, True, False], [True] * 4]
    assert oracle.visible(3, 3, True, 2).tolist() == [[True, True, False], [True, True, False], [True, True, True]]
    assert oracle.visible(3, 2, True, 0).tolist() == [[False, False], [True, False], [True, True]]
    assert oracle.visible(2, 0, True, 5).shape == (2, 0)


@pytest.mark.parametrize("cap", [0.0, 1.5])
@pytest.mark.parametrize("causal", [False, True])
def test_gradients_are_differences(cap, causal):
    q, k, v, q_off, k_off, bias, buckets, dout = _case(3, [3, 0, 4], [5, 2, 2])
    kw = dict(cap=cap, causal=causal, prefix=torch.tensor([2, 0, 1]) if causal else None, buckets=buckets)

    def value(q, k, v, bias):
        res, _ = oracle.attention(q, k, v, q_off, k_off, bias=bias, **kw)
        return float((res["out"] * dout.double()).sum())

    res, _ = oracle.attention(q, k, v, q_off, k_off, bias=bias, dout=dout, **kw)
    inputs = {"q": q, "k": k, "v": v, "bias": bias}
    g = torch.Generator().manual_seed(1)
    oracle.UNIT[torch.float64], oracle.SMALLEST[torch.float64] = 0.0, 0.0
    try:
        wide = {n: t.double() for n, t in inputs.items()}
        for name in inputs:
            way = torch.randn(wide[name].shape, generator=g, dtype=torch.float64)
            step = 1e-6
            up, down = ({**wide, name: wide[name] + s * step * way} for s in (1, -1))
            slope = (value(**up) - value(**down)) / (2 * step)
            assert slope == pytest.approx(float((res["d" + name] * way).sum()), rel=1e-6, abs=1e-7)
    finally:
        del oracle.UNIT[torch.float64], oracle.SMALLEST[torch.float64]


def test_read_is_attention_over_the_listed_rows():
    g = torch.Generator().manual_seed(5)
    q = torch.randn(2, 3, 2, 8, generator=g).to(torch.float16)
    keys, values = (torch.randn(9, 1, 8, generator=g).to(torch.float16) for _ in range(2))
    res, _ = oracle.read(q, keys, values, torch.tensor([0, 0, 4]), torch.tensor([8, -1, 2, 9]), scale=1.0)
    assert (res["out"][0] == 0).all() and (res["lse"][0] == -math.inf).all()
    z = q[1, 2, 1].double() @ keys[[8, 2], 0].double().T
    assert torch.allclose(res["out"][1, 2, 1], torch.softmax(z, 0) @ values[[8, 2], 0].double())


def test_mask_and_logits_by_hand():
    assert oracle.entity_mask(torch.tensor([0, 3, 3]), torch.tensor([0, 65, 200]), 100) == [[1, 2], [0, 0]]
    x = torch.tensor([[2.0, -2.0, 1.0, 0.5]])
    got = oracle.logits(x, history=torch.tensor([0, 1, 0, -1, 9]), history_off=torch.tensor([0, 5]), repetition=torch.tensor([2.0]),
                        presence=torch.tensor([0.25]), frequency=torch.tensor([0.5]), bias_off=torch.tensor([0, 3]),
                        bias_id=torch.tensor([3, 2, 3]), bias_value=torch.tensor([9.0, 1.0, 2.0]), mask=torch.tensor([[0b1111]]))
    assert got.tolist() == [[2 / 2 - 0.25 - 1.0, -4 - 0.25 - 0.5, 2.0, 2.5]]
    assert oracle.logits(x, mask=torch.tensor([[0b0010]])).tolist() == [[-math.inf, -2.0, -math.inf, -math.inf]]


def test_distance_buckets():
    b = lkg.distance_buckets(8, 16, device="cpu").tolist()
    assert len(b) == 33 and b[16] == 0 and b[15] == 1 and b[17] == 5  # near ones alone, the sign its half
    assert b[0] == b[1] == 3 and b[32] == 7 and sorted(set(b)) == [0, 1, 2, 3, 5, 6, 7]
    one = lkg.distance_buckets(8, 16, both_sides=False, device="cpu").tolist()
    assert one[16:] == [0] * 17 and one[12:17] == [4, 3, 2, 1, 0] and one[0] == 7
    for bad in ((1, 4), (32, 3)):
        with pytest.raises(ValueError):
            lkg.distance_buckets(*bad, device="cpu")


def test_cpu_tensors_are_refused():
    q, k, v, q_off, k_off, bias, buckets, dout = _case(1, [2], [3])
    with pytest.raises(ValueError, match="on the GPU"):
        lkg.read_entities(q[None], k, v, k_off, k_off[:0].int())
    with pytest.raises(ValueError, match="on the GPU"):
        lkg.entity_mask(k_off, k_off[:0].int(), 10)
    with pytest.raises(ValueError, match="on the GPU"):
        lkg.constrain_logits(torch.zeros(1, 4))
    with pytest.raises(ValueError, match="on the GPU"):
        reading._attention(q, k, v, q_off, k_off, None, 0.0, False, None, None, None, None, None, q, q, None)


def test_struct_sizes_match_the_header():
    assert [ctypes.sizeof(s) for s in (reading._Score, reading._Attention, reading._AttentionGrad, reading._EntityRead,
                                       reading._Logits)] == [32, 216, 64, 208, 144]


# what the C entry points refuse, before anything is launched
def _status(call, *structs):
    if not os.path.exists(lkg.library_path()):
        from paper_2604_18913_amd import build_ext
        build_ext.build(verbose=False)
    lib = reading._load()
    rc = getattr(lib, call)(*[ctypes.addressof(s) if s is not None else None for s in structs])
    return rc, lib.logoskg_last_error().decode()


def _attention(**kw):
    base = dict(struct_size=216, dtype=1, num_docs=1, heads=2, kv_heads=1, dim=64, num_rows=4, num_keys=4, q_off=64, k_off=64, q=64,
                k=64, v=64, q_row=128, q_head=64, k_row=64, k_head=64, v_row=64, v_head=64, out=64, lse=64)
    score = kw.pop("score", reading._Score(1.0, 0.0, None, None, 0, 0))
    return reading._Attention(**{**base, **kw}, score=score)


@pytest.mark.parametrize("wrong, says", [
    (dict(struct_size=8), "struct_size"), (dict(dtype=0), "type"), (dict(dtype=9), "type"), (dict(heads=3, kv_heads=2), "multiple"),
    (dict(kv_heads=0), "multiple"), (dict(heads=256), "128 heads"), (dict(dim=12), "dim"), (dict(dim=136), "dim"), (dict(dim=0), "dim"),
    (dict(num_rows=-1), "count"), (dict(num_keys=1 << 31), "count"), (dict(num_docs=0), "without a document"),
    (dict(q_off=None), "offsets"), (dict(q=None), "NULL"), (dict(lse=None), "NULL"), (dict(v=None), "NULL"),
    (dict(q=72), "aligned"), (dict(k_row=65), "multiple of 8"), (dict(out=68), "aligned"),
    (dict(score=reading._Score(1.0, -1.0, None, None, 0, 0)), "cap"), (dict(score=reading._Score(math.nan, 0.0, None, None, 0, 0)), "scale"),
    (dict(score=reading._Score(1.0, 0.0, 64, None, 4, 4)), "buckets"), (dict(score=reading._Score(1.0, 0.0, 64, 64, 65, 4)), "num_buckets"),
    (dict(score=reading._Score(1.0, 0.0, 64, 64, 4, 1025)), "max_distance"),
    (dict(heads=128, score=reading._Score(1.0, 0.0, 64, 64, 4, 100)), "BIAS_PLACES"),
])
def test_attention_refusals(wrong, says):
    rc, text = _status("logoskg_attend", _attention(**wrong))
    assert rc == 1 and says in text and text.startswith("logoskg_attend")
    assert reading._load().logoskg_attend_backward_bytes(ctypes.addressof(_attention(**wrong))) == -1


def test_backward_refusals():
    grad = dict(struct_size=64, dout=64, dq=64, dk=64, dv=64, workspace=64, workspace_bytes=1 << 20)
    for wrong, rc, says in [(dict(struct_size=0), 1, "struct_size"), (dict(dout=None), 1, "dout"), (dict(dk=None), 1, "dk"), (dict(dq=72), 1, "aligned"),
                            (dict(workspace_bytes=8), 4, "workspace"), (dict(workspace=None), 4, "workspace")]:
        got, text = _status("logoskg_attend_backward", _attention(), reading._AttentionGrad(**{**grad, **wrong}))
        assert got == rc and says in text, (wrong, text)
    biased = _attention(score=reading._Score(1.0, 0.0, 64, 64, 4, 4))
    got, text = _status("logoskg_attend_backward", biased, reading._AttentionGrad(**grad))
    assert got == 1 and "dbias" in text


@pytest.mark.parametrize("wrong, rc, says", [
    (dict(struct_size=1), 1, "struct_size"), (dict(tokens=0), 1, "count"), (dict(num_entries=-1), 1, "count"), (dict(off=None), 1, "NULL"),
    (dict(keys=None), 1, "NULL"), (dict(value_head=4), 1, "multiple of 8"), (dict(entity=None, num_entities=3), 1, "fewer rows"),
    (dict(num_entities=1 << 31), 1, "num_entities"), (dict(dtype=0), 1, "type"), (dict(num_entries=100_000, num_queries=3), 4, "workspace"),
])
def test_read_refusals(wrong, rc, says):
    base = dict(struct_size=208, dtype=2, num_queries=1, tokens=1, heads=4, kv_heads=4, dim=64, num_entries=9, num_entities=9, off=64,
                entity=64, q=64, keys=64, values=64, key_row=256, key_head=64, value_row=256, value_head=64, out=64, lse=64)
    got, text = _status("logoskg_read_entities", reading._EntityRead(**{**base, **wrong}, score=reading._Score(1.0, 0.0, None, None, 0, 0)))
    assert got == rc and says in text


def test_mask_and_logits_refusals():
    lib = reading._load()
    for args in [(0, None, 64, 5, 1, 9, 64, None), (0, 64, 64, -1, 1, 9, 64, None), (0, 64, 64, 5, 1, 1 << 32, 64, None), (0, 64, 64, 5, 1, 9, 72, None),
                 (0, 64, 64, 5, 1, 9, None, None)]:
        assert lib.logoskg_entity_mask(*args) == 1
    base = dict(struct_size=144, dtype=0, num_rows=2, vocab=10, row=10, logits=64, out=64)
    for wrong in (dict(struct_size=0), dict(dtype=3), dict(row=9), dict(logits=None), dict(num_rows=-1), dict(vocab=1 << 31),
                  dict(history_off=64, num_history=4), dict(bias_off=64, num_bias=2, bias_id=64)):
        rc, text = _status("logoskg_constrain_logits", reading._Logits(**{**base, **wrong}))
        assert rc == 1 and text.startswith("logoskg_constrain_logits")
