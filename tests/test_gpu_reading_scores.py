"""Scores that the attention's kernels take apart: biases that hide the first tiles of a row, caps of any size, rows whose few
keys leave little of their gradient (bounds: reading_oracle)."""
import math

import pytest
import torch

import paper_2604_18913_amd as lkg
import reading_oracle as oracle
from test_gpu_reading import HALVES, _attend, _check, _check_read, _gpu, _inputs, _read

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------- biases that hide the first tiles of a row
@pytest.mark.parametrize("heads, kv_heads", [(4, 2), (260, 260)])  # (few rows, many)
@pytest.mark.parametrize("dtype, cap, size", [(torch.float16, 0.0, 3.0), (torch.float16, 50.0, 3.0), (torch.bfloat16, 0.0, 40.0), (torch.bfloat16, 50.0, 3.0)])
@pytest.mark.parametrize("low", [-math.inf, -1e10])  # (-1e10 hides by its size alone: beside it, 32 bits hold scores to 512)
def test_first_tiles_hidden_by_their_bias(low, dtype, cap, size, heads, kv_heads):
    # four whole tiles that read a hiding bucket, under scores of which 16 bits could not hold the exponential, then keys that
    # are seen; the second document has hidden keys only
    if dtype is torch.float16 and low > -math.inf:
        low = -65504.0
    a, dout = _inputs(41, dtype, [70, 40], [300, 200], heads, kv_heads, 64, spread=1.5)
    g = torch.Generator().manual_seed(41)
    k_pos = torch.randint(0, 3, (500,), generator=g, dtype=torch.int32)
    k_pos[:256], k_pos[300:] = 9, 9
    a["k"][:256] *= size
    a["k"][300:] *= size
    bias = torch.randn(heads, 4, generator=g).to(dtype)
    bias[:, 3] = low
    a |= dict(bias=bias, buckets=torch.tensor([0, 0, 0, 0, 0, 0, 1, 0, 2, 2, 3], dtype=torch.int32), cap=cap,
              q_pos=torch.zeros(110, dtype=torch.int32), k_pos=k_pos)
    if low > -math.inf:  # (keys that all read a finite bias share their row's weight: no such document here)
        a |= dict(q=a["q"][:70], q_off=torch.tensor([0, 70]), k=a["k"][:300], v=a["v"][:300], k_off=torch.tensor([0, 300]), q_pos=a["q_pos"][:70], k_pos=k_pos[:300])
        _check(a, dout[:70])
    else:
        got = _check(a, dout)
        assert all((got[n][70:] == 0).all() for n in ("out", "dq")) and (got["lse"][70:] == -math.inf).all()
        assert all((got[n][300:] == 0).all() and (got[n][:256] == 0).all() for n in ("dk", "dv")) and (got["dbias"][:, 3] == 0).all()


@pytest.mark.parametrize("heads, kv_heads", [(4, 2), (132, 132)])
@pytest.mark.parametrize("dtype, cap", [(torch.float16, 0.0), (torch.float16, 50.0), (torch.bfloat16, 20.0)])
def test_a_window_made_by_a_hiding_bucket(dtype, cap, heads, kv_heads):
    # causal text whose keys 60 or more places back are hidden: the last rows' first tiles hold nothing else
    a, dout = _inputs(42, dtype, [420], [420], heads, kv_heads, 64, spread=2.0)
    buckets = torch.zeros(2 * 60 + 1, dtype=torch.int32)
    buckets[0], buckets[1:30] = 2, 1
    bias = torch.zeros(heads, 3, dtype=dtype)
    bias[:, 1], bias[:, 2] = 0.5, -math.inf
    _check({**a, "causal": True, "cap": cap, "bias": bias, "buckets": buckets}, dout)


def _low(dtype, low, heads, kv_heads):
    a, dout = _inputs(46, dtype, [70], [200], heads, kv_heads, 64, spread=1.5)
    return {**a, "bias": torch.full((heads, 4), low, dtype=dtype), "buckets": torch.tensor([0, 1, 2, 3, 0], dtype=torch.int32)}, dout


@pytest.mark.parametrize("heads, kv_heads", [(4, 2), (260, 260)])
@pytest.mark.parametrize("low", [-7.2e4, -1e6, -1e9, -1e14, -6e14, -1e30, -math.inf])
def test_rows_that_see_low_biases_alone(low, heads, kv_heads):
    a, dout = _low(torch.bfloat16, low, heads, kv_heads)
    got = _attend(a, dout)
    assert all((got[n] == 0).all() for n in ("out", "dq", "dk", "dv", "dbias")) and (got["lse"] == -math.inf).all()
    r = _read(46, torch.bfloat16, [300, 40], 1, heads, kv_heads, 64)
    r["bias"][:] = low
    got = lkg.read_entities(**{k: _gpu(x) for k, x in r.items()})
    assert (got["out"] == 0).all() and (got["lse"] == -math.inf).all()


@pytest.mark.parametrize("heads, kv_heads", [(4, 2), (260, 260)])
@pytest.mark.parametrize("dtype, low", [(torch.float16, -65504.0), (torch.bfloat16, -65536.0)])
def test_rows_that_see_the_least_biases_alone(dtype, low, heads, kv_heads):
    # float16's lowest value is a number yet: beside 94,500 (in units of log 2) 32 bits hold scores to 2^-8, weights to 0.003, and
    # lse to as much; with the roundings to 16 bits below a hundredth of the norm
    a, dout = _low(dtype, low, heads, kv_heads)
    got, (want, _) = _attend(a, dout), oracle.attention(**a, dout=dout)
    for n in want:
        assert (got[n].cpu().double() - want[n]).norm() < 0.01 * want[n].norm(), n


# ------------------------------------------------------------------------- caps of any size
CAPS = [1e-30, 1e-9, 1e3, 1e4, 1e6, 1e8, 1e30]


@pytest.mark.parametrize("heads, kv_heads, dim", [(4, 2, 64), (4, 2, 128), (264, 264, 16)])
@pytest.mark.parametrize("cap", CAPS)
def test_attention_under_any_cap(cap, heads, kv_heads, dim):
    # causal, so that most tiles have hidden keys; a row and a key of zeros, whose products are 0
    a, dout = _inputs(43, torch.float16, [90, 30], [90, 140], heads, kv_heads, dim, bias=True)
    a["q"][7], a["k"][11] = 0, 0
    _check({**a, "causal": True, "cap": cap}, dout)
    _check({**a, "causal": False, "cap": cap}, dout)


@pytest.mark.parametrize("cap", [0.25, 0.5])
@pytest.mark.parametrize("dtype", HALVES, ids=["bf16", "fp16"])
@pytest.mark.parametrize("heads, kv_heads, dim, rows, keys", [(260, 260, 72, [5], [80]), (132, 132, 16, [1, 85, 3], [13, 473, 104]), (12, 3, 80, [33, 12, 50], [22, 67, 200]), (6, 3, 128, [196], [9])])
def test_gradients_of_scores_near_their_cap(heads, kv_heads, dim, rows, keys, dtype, cap):
    # slopes from 1 down to 1e-8 of the scale, of either sign of the score, each known to the roundings of its own size
    a, dout = _inputs(47, dtype, rows, keys, heads, kv_heads, dim, bias=True)
    _check({**a, "cap": cap}, dout)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("cap", CAPS)
def test_read_under_any_cap(cap, dim):
    a = _read(44, torch.float16, [40, 0, 700], 2, 4, 2, dim, cap=cap)
    a["q"][0, 0] = 0
    _check_read(a)


# ------------------------------------------------------------------------- rows with few keys among others
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("rows, prefix", [(100, 0), (300, 0), (200, 2)])
@pytest.mark.parametrize("heads, kv_heads, dim", [(4, 4, 64), (2, 2, 128), (4, 2, 64)])
def test_gradients_of_the_first_rows_of_causal_text(heads, kv_heads, dim, rows, prefix, cap):
    # row 0 sees one key: its dq is 0, and delta in 32 bits leaves 1e-5 of sums of `dim` products; the next rows see a few: the
    # roundings of dz and of the result, 0.0017 of the norm each
    a, dout = _inputs(45, torch.bfloat16, [rows], [rows], heads, kv_heads, dim, bias=True)
    a |= dict(causal=True, cap=cap, prefix=torch.tensor([prefix], dtype=torch.int32))
    got = _check(a, dout)
    want = oracle.attention(**a, dout=dout)[0]["dq"]
    if prefix == 0:
        assert got["dq"][0].abs().max() < 2e-4
    few = slice(1, 6)
    assert (got["dq"][few].cpu().double() - want[few]).norm() < 0.0035 * want[few].norm()
