"""The calls that read a retrieval on a part of a batch: offsets that begin behind the first entry and end before the last, as
a slice of a batch's offsets with its whole arrays gives them (bounds: reading_oracle)."""
import math

import pytest
import torch

import paper_2604_18913_amd as lkg
import reading_oracle as oracle
from test_gpu_reading import HALVES, _attend, _check_logits, _gpu, _inputs, _lists, _logit_case, _read

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------- read_entities
@pytest.mark.parametrize("dtype", HALVES, ids=["bf16", "fp16"])
@pytest.mark.parametrize("off, entries", [([200, 250, 300], 300), ([128, 128, 200], 210), ([127, 130], 130), ([1000, 1128, 1128, 3000], 3500),
                                          ([5000, 5000], 5000), ([300, 700, 39_000], 40_000), ([20_000, 20_000, 20_256, 40_000], 40_000)])
def test_read_of_lists_that_begin_behind_the_first_entry(off, entries, dtype):
    # (40,000 entries under eight key heads are cut into blocks of 256, the others into blocks of 128)
    a = _read(31, dtype, [entries], 1, 8, 8, 64, cap=5.0)
    g = torch.Generator().manual_seed(31)
    a |= dict(q=torch.randn(len(off) - 1, 1, 8, 64, generator=g).to(dtype), off=torch.tensor(off))
    res, tol = oracle.read(**a)
    for _ in range(3):
        got = lkg.read_entities(**{k: _gpu(x) for k, x in a.items()})
        for n in ("out", "lse"):
            oracle.check(got[n], res[n], tol[n], n)


@pytest.mark.parametrize("first, last", [(0, 3), (2, 5), (5, 9), (8, 9)])
def test_read_of_a_slice_of_a_batch(first, last):
    a = _read(32, torch.bfloat16, [900, 0, 40, 300, 1, 0, 700, 129, 64], 2, 4, 2, 64)
    part = {**a, "q": a["q"][first:last].contiguous(), "off": a["off"][first:last + 1].contiguous()}
    got = lkg.read_entities(**{k: _gpu(x) for k, x in part.items()})
    res, tol = oracle.read(**a)
    for n in ("out", "lse"):
        oracle.check(got[n], res[n][first:last], tol[n][first:last], n)


# ------------------------------------------------------------------------- masks and logits
@pytest.mark.parametrize("num_ids", [500, 70_001, 110_000_000])  # (the last by atomics)
def test_masks_of_lists_that_begin_behind_the_first_entry(num_ids):
    off, ids, _ = _lists(33, [2000], num_ids)
    off = torch.tensor([300, 400, 400, 1500])
    got = lkg.entity_mask(off.cuda(), ids.cuda(), num_ids).cpu()
    for i in range(3):
        mine = ids[off[i]:off[i + 1]].unique()
        words = torch.nonzero(got[i]).flatten()
        bits = [(int(w) * 64 + b) for w in words for b in range(64) if int(got[i, w]) >> b & 1]
        assert bits == mine.tolist()


def test_logits_of_lists_that_begin_behind_the_first_entry():
    a = _logit_case(34, torch.float32, 4, 5000, 300, 40)
    n, m = a["history"].numel(), a["bias_id"].numel()
    assert n > 60 and m > 20
    _check_logits({**a, "history_off": torch.tensor([30, 33, 33, n - 20, n - 4]), "bias_off": torch.tensor([5, 5, 9, m - 6, m - 1])})


# ------------------------------------------------------------------------- attention
PARTS = [([130, 170, 170, 400], 450, [70, 200, 260, 500], 640), ([1, 2], 3, [1, 2], 3), ([300, 300, 428], 428, [128, 257, 257], 300),
         ([0, 129], 131, [0, 128], 129), ([127, 128, 256], 1000, [128, 129, 257], 1100)]


def _part(seed, dtype, q_off, rows, k_off, keys, heads, kv_heads, dim):
    a, dout = _inputs(seed, dtype, [rows], [keys], heads, kv_heads, dim, bias=True)
    a |= dict(q_off=torch.tensor(q_off), k_off=torch.tensor(k_off), causal=True, cap=4.0,
              prefix=torch.tensor([(7 * i + 3) % 50 for i in range(len(q_off) - 1)], dtype=torch.int32))
    return a, dout


@pytest.mark.parametrize("part", PARTS, ids=lambda x: "-".join(map(str, x[0])))
@pytest.mark.parametrize("heads, kv_heads, dim", [(4, 2, 64), (12, 4, 96), (264, 264, 16)])  # (few rows, many)
def test_attention_of_documents_that_begin_behind_the_first_row(heads, kv_heads, dim, part):
    q_off, rows, k_off, keys = part
    a, dout = _part(35, torch.bfloat16, q_off, rows, k_off, keys, heads, kv_heads, dim)
    got = _attend(a, dout)
    res, tol = oracle.attention(**a, dout=dout)
    for n in ("out", "lse", "dq"):
        oracle.check(got[n][q_off[0]:q_off[-1]], res[n][q_off[0]:q_off[-1]], tol[n][q_off[0]:q_off[-1]], n)
    for n in ("dk", "dv"):
        oracle.check(got[n][k_off[0]:k_off[-1]], res[n][k_off[0]:k_off[-1]], tol[n][k_off[0]:k_off[-1]], n)
    oracle.check(got["dbias"], res["dbias"], tol["dbias"], "dbias")


def _stale():
    """Leaves NaN in the memory that the next tensors take."""
    junk = [torch.full((1 << n,), math.nan, device="cuda") for n in range(8, 24) for _ in range(3)]
    torch.cuda.synchronize()
    del junk


def _check_spare(got, q_off, k_off):
    for n, (a, b) in {"out": (q_off[0], q_off[-1]), "dq": (q_off[0], q_off[-1]), "dk": (k_off[0], k_off[-1]), "dv": (k_off[0], k_off[-1])}.items():
        assert (got[n][:a] == 0).all() and (got[n][b:] == 0).all(), n
    assert (got["lse"][:q_off[0]] == -math.inf).all() and (got["lse"][q_off[-1]:] == -math.inf).all()


@pytest.mark.parametrize("part", PARTS + [([0, 0], 200, [0, 0], 300), ([700, 700], 700, [900, 900], 900), ([500, 500, 500], 900, [0, 300, 300], 300)],
                         ids=lambda x: "-".join(map(str, x[0])))
@pytest.mark.parametrize("heads, kv_heads, dim", [(4, 2, 64), (6, 2, 80), (264, 264, 16), (35, 1, 24)])
def test_rows_and_keys_that_no_document_holds(heads, kv_heads, dim, part):
    a, dout = _part(36, torch.bfloat16, *part, heads, kv_heads, dim)
    _stale()
    _check_spare(_attend(a, dout), part[0], part[2])


@pytest.mark.parametrize("heads, kv_heads", [(8, 2), (64, 32)])  # (the second batch's blocks are put in order)
def test_a_batch_in_longer_buffers_under_a_graph(heads, kv_heads):
    # buffers for 900 rows and 1,500 keys, offsets that change from replay to replay
    a, dout = _inputs(37, torch.bfloat16, [100] * 9, [150] * 10, heads, kv_heads, 32, bias=True)
    a["q_off"], a["k_off"] = (torch.cat([torch.zeros(1, dtype=torch.int64), x.sort().values]) for x in (a["q_off"][1:10], a["k_off"][1:10]))
    b, d = {k: _gpu(x) for k, x in a.items()}, _gpu(dout)
    pos = [b.pop(n) for n in ("q", "k", "v", "q_off", "k_off")]

    def call():
        out, lse = lkg.attend(*pos, causal=True, **b)
        return dict(zip(("out", "lse", "dq", "dk", "dv", "dbias"), (out, lse, *lkg.attend_backward(d, *pos[:3], out, lse, *pos[3:], causal=True, **b))))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for docs in (9, 4, 1, 6):
        q_off, k_off = a["q_off"].clamp(max=100 * docs - 13), a["k_off"].clamp(max=150 * docs - 20)
        pos[3].copy_(q_off)
        pos[4].copy_(k_off)
        for x in got.values():
            x.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        want = call()
        assert all(torch.equal(got[n], want[n]) for n in got)
        _check_spare(got, q_off.tolist(), k_off.tolist())
