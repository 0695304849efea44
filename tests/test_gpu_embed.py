"""embed_entities and its gradient against their 64-bit definitions (bounds: around_oracle)."""
import pytest
import torch

import around_oracle as oracle
import paper_2604_18913_amd as lkg

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
TYPE_NAMES = ["fp32", "bf16", "fp16"]


def _table(seed, entities, dim, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(entities, dim, generator=g) * scale).to(dtype)


def _ids(seed, n, entities, skew=1):
    g = torch.Generator().manual_seed(seed)
    return (torch.rand(n, generator=g, dtype=torch.float64) ** skew * entities).int().clamp(max=max(entities - 1, 0))


def _forward(table, ids, scale=1.0, cuda=None):
    oracle.check(lkg.embed_entities(table.cuda() if cuda is None else cuda, ids.cuda(), scale=scale), *oracle.embed(table, ids, scale), "embed")


def _backward(dout, ids, entities, scale=1.0, out=None, accumulate=False, dtype=None):
    kw = {} if out is None else {"out": out.cuda(), "accumulate": accumulate}
    if out is None and dtype is not None:
        kw["out"] = torch.full((entities, dout.shape[-1]), 7.0, dtype=dtype, device="cuda")  # what stood there does not matter
    got = lkg.embed_entities_backward(dout.cuda(), ids.cuda(), entities, scale=scale, **kw)
    oracle.check(got, *oracle.embed_grad(dout, ids, entities, scale, out if accumulate else None, got.dtype), "gradient")
    again = lkg.embed_entities_backward(dout.cuda(), ids.cuda(), entities, scale=scale, **({} if out is None else {"out": out.cuda(), "accumulate": accumulate}))
    assert again.dtype is not got.dtype or torch.equal(again, got)  # the same bits
    return got


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_NAMES)
@pytest.mark.parametrize("dim", [1, 3, 8, 15, 64, 100, 333, 512, 4104])
def test_rows_of_all_sizes(dim, dtype):
    table, ids = _table(dim, 37, dim, dtype), _ids(1, 41, 37)
    ids[5], ids[6], ids[7], ids[40] = -1, 37, 2 ** 31 - 1, -2 ** 31
    _forward(table, ids, 22.6)
    _backward(_table(2, 41, dim, dtype), ids, 37, 0.3)


@pytest.mark.parametrize("shape", [(0,), (1,), (), (3, 0), (2, 5, 7)])
def test_shapes_of_ids(shape):
    table = _table(3, 10, 24, torch.bfloat16)
    n = 1
    for s in shape:
        n *= s
    ids = _ids(4, n, 10).reshape(shape)
    _forward(table, ids)
    _backward(_table(5, n, 24, torch.bfloat16).reshape(*shape, 24), ids, 10)


def test_empty_tables():
    ids = _ids(6, 9, 5)
    assert (lkg.embed_entities(torch.zeros(0, 16, device="cuda"), ids.cuda()) == 0).all()
    assert lkg.embed_entities(torch.zeros(5, 0, device="cuda"), ids.cuda()).shape == (9, 0)
    assert lkg.embed_entities_backward(torch.ones(9, 16, device="cuda"), ids.cuda(), 0).shape == (0, 16)
    assert lkg.embed_entities_backward(torch.ones(9, 0, device="cuda"), ids.cuda(), 5).shape == (5, 0)


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_NAMES)
def test_strides(dtype):
    wide, ids = _table(7, 20, 77, dtype), _ids(8, 30, 20)
    for a, b in [(0, 64), (1, 65), (3, 40), (76, 77)]:
        _forward(wide[:, a:b], ids, cuda=wide.cuda()[:, a:b])
    _forward(wide[:1].expand(20, -1), ids, cuda=wide.cuda()[:1].expand(20, -1))  # one row for all
    _forward(wide[::3, :50], ids, cuda=wide.cuda()[::3, :50])
    # a gradient inside a wider one: what lies beside it stays
    dout, out = _table(9, 30, 40, dtype), wide.cuda()
    lkg.embed_entities_backward(dout.cuda(), ids.cuda(), 20, out=out[:, 5:45])
    oracle.check(out[:, 5:45], *oracle.embed_grad(dout, ids, 20))
    assert torch.equal(out[:, :5].cpu(), wide[:, :5]) and torch.equal(out[:, 45:].cpu(), wide[:, 45:])


# around the ends of chunks and tiles, and of the list that one block sorts
@pytest.mark.parametrize("n", [1, 7, 8, 9, 63, 64, 65, 1023, 1025, 4095, 4096, 4097, 8192, 12_289, 65_535, 65_536, 70_001])
@pytest.mark.parametrize("entities", [1, 2, 255, 256, 5000])
def test_lengths(n, entities):
    _backward(_table(10, n, 12, torch.float32), _ids(n, n, entities), entities)


@pytest.mark.parametrize("skew", [1, 3, 9])
@pytest.mark.parametrize("n, dim, dtype", [(3000, 72, torch.bfloat16), (30_000, 20, torch.float16), (100_000, 8, torch.float32)])
def test_hubs(n, dim, dtype, skew):
    ids = _ids(11, n, 3000, skew)
    ids[::17] = -1
    _backward(_table(12, n, dim, dtype, 0.1), ids, 3000, 8.0)


@pytest.mark.parametrize("n", [100, 5000, 70_000])
def test_one_entity_all_and_none(n):
    dout = _table(13, n, 40, torch.bfloat16, 0.01)
    _backward(dout, torch.full((n,), 3, dtype=torch.int32), 9)
    _backward(dout, torch.full((n,), -5, dtype=torch.int32), 9)
    _backward(dout, torch.arange(n, dtype=torch.int32).flip(0), n)
    _backward(dout, (torch.arange(n) % 2 * 8).int(), 9)


@pytest.mark.parametrize("entities", [(1 << 11) - 1, 1 << 11, (1 << 16) + 1, (1 << 22) - 1, 1 << 22])
@pytest.mark.parametrize("n", [2000, 20_000])
def test_bits_of_ids(n, entities):
    ids = _ids(14, n, entities)
    ids[0], ids[1], ids[2], ids[3] = 0, entities - 1, entities, entities - 1
    _backward(_table(15, n, 2, torch.float32), ids, entities)


@pytest.mark.parametrize("n", [50, 6000])
def test_ids_of_thirty_bits(n):
    entities = 1 << 30
    out = torch.ones(entities, 1, dtype=torch.bfloat16, device="cuda")
    ids = _ids(16, n, entities)
    ids[1], ids[2] = entities - 1, ids[3]
    dout = _table(17, n, 1, torch.bfloat16)
    lkg.embed_entities_backward(dout.cuda(), ids.cuda(), entities, out=out, accumulate=True)
    who, back = torch.unique(ids, return_inverse=True)
    oracle.check(out[who.long().cuda()], *oracle.embed_grad(dout, back.int(), len(who), out=torch.ones(len(who), 1)  , dtype=torch.bfloat16))
    out[who.long().cuda()] = 1.0
    assert bool((out == 1).all())


@pytest.mark.parametrize("dtype", TYPES[1:], ids=TYPE_NAMES[1:])
@pytest.mark.parametrize("n", [300, 9000])
def test_wide_gradients_and_accumulation(n, dtype):
    dout, ids = _table(18, n, 48, dtype), _ids(19, n, 400, 2)
    _backward(dout, ids, 400, 2.0, dtype=torch.float32)
    for to in (dtype, torch.float32):
        _backward(dout, ids, 400, 0.5, out=_table(20, 400, 48, to), accumulate=True)


# (lanes at the end of such rows begin before their own columns)
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_NAMES)
@pytest.mark.parametrize("dim", [1, 3, 5, 9, 13, 67, 333])
@pytest.mark.parametrize("n", [40, 13_000])
def test_accumulation_into_rows_of_odd_sizes(n, dim, dtype):
    dout, ids = _table(21, n, dim, dtype, 0.1), _ids(22, n, 300, 3)
    for to in {dtype, torch.float32}:
        _backward(dout, ids, 300, 0.5, out=_table(23, 300, dim, to), accumulate=True)


@pytest.mark.parametrize("run", [7, 8, 9, 63, 64, 65, 66, 127, 1000, 4000])
@pytest.mark.parametrize("before", [0, 1, 7, 8, 90])
@pytest.mark.parametrize("dim, dtype", [(3, torch.float32), (40, torch.bfloat16), (333, torch.float16)])
def test_runs_of_one_entity(before, run, dim, dtype):
    ids = torch.cat([torch.arange(before), torch.full((run,), 100), torch.tensor([101, 103])]).int()[torch.randperm(before + run + 2, generator=torch.Generator().manual_seed(28))]
    dout = _table(29, len(ids), dim, dtype, 0.1)
    _backward(dout, ids, 110)
    _backward(dout, ids, 110, 2.0, out=_table(30, 110, dim, dtype), accumulate=True)


@pytest.mark.parametrize("n", [12_288, 131_072, 262_143, 262_145])
@pytest.mark.parametrize("entities, skew", [(3000, 4), (300_000, 1)])
def test_long_lists(n, entities, skew):
    _backward(_table(24, n, 4, torch.float32), _ids(25, n, entities, skew), entities)


@pytest.mark.parametrize("dim, dtype", [(2048, torch.bfloat16), (1021, torch.float32)])
def test_large_tables_whose_rows_are_mostly_named(dim, dtype):
    """Cleared between the sums: gaps of no, few and many rows, and those at both ends.  Whole numbers: sums are exact."""
    n, entities = 62_000, 64_000
    g = torch.Generator().manual_seed(26)
    ids = torch.cat([torch.arange(3, 30_000), torch.arange(30_000, 56_000, 2), torch.full((100,), 57_000), torch.tensor([63_998])])
    ids = torch.cat([ids, ids[torch.randint(0, len(ids), (n - len(ids),), generator=g)]])[torch.randperm(n, generator=g)].int().cuda()
    dout = torch.randint(-1, 2, (n, dim), generator=g).to(dtype).cuda()
    want = torch.zeros(entities, dim, device="cuda").index_add_(0, ids.long(), dout.float())
    assert want.abs().max() <= 256
    for _ in range(2):
        got = lkg.embed_entities_backward(dout, ids, entities, out=torch.full((entities, dim), 5.0, dtype=dtype, device="cuda"))
        assert torch.equal(got.float(), want)


def test_tables_beyond_32_bits():
    entities, dim = 600_000, 4096  # 2.4e9 elements
    table = torch.zeros(entities, dim, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([entities - 1, 524_289, 0, entities - 2], dtype=torch.int32)
    table[ids.long().cuda()] = torch.arange(1.0, 5.0, device="cuda", dtype=torch.bfloat16)[:, None]
    assert lkg.embed_entities(table, ids.cuda())[:, ::999].float().cpu().tolist() == [[float(i)] * 5 for i in range(1, 5)]
    got = lkg.embed_entities_backward(torch.ones(4, dim, dtype=torch.bfloat16, device="cuda"), ids.cuda(), entities, out=table)
    assert got.data_ptr() == table.data_ptr() and bool((table[ids.long().cuda()] == 1).all()) and float(table.sum(dtype=torch.float32)) == 4 * dim


def test_infinities_and_nan_stay_in_their_rows():
    dout, ids = _table(21, 500, 16, torch.bfloat16), _ids(22, 500, 20)
    dout[7, 3], dout[8, 4] = float("inf"), float("nan")
    got = lkg.embed_entities_backward(dout.cuda(), ids.cuda(), 20).cpu()
    bad = ~got.isfinite()
    assert bad.sum() == 2 and bad[ids[7].long(), 3] and bad[ids[8].long(), 4]
    table = _table(23, 4, 8, torch.float16)
    table[2] = float("nan")
    assert torch.equal(lkg.embed_entities(table.cuda(), torch.tensor([0, -1, 2], dtype=torch.int32).cuda()).isnan().any(1).cpu(), torch.tensor([False, False, True]))


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_NAMES)
def test_torch_s_backward(dtype):
    table, ids = _table(24, 50, 40, dtype).cuda().requires_grad_(), _ids(25, 6 * 20, 50).reshape(6, 20)
    out = lkg.embed_entities(table, ids.cuda(), scale=3.0)
    dout = _table(26, 120, 40, dtype).reshape(6, 20, 40)
    out.backward(dout.cuda())
    oracle.check(out, *oracle.embed(table, ids, 3.0))
    oracle.check(table.grad, *oracle.embed_grad(dout, ids, 50, 3.0))
    table.grad = None
    # a gradient that is one value for all, and a table that is read twice
    two = lkg.embed_entities(table, ids.cuda()).float().sum() + lkg.embed_entities(table, ids.cuda()).float().sum()
    two.backward()
    want, tol = oracle.embed_grad(torch.ones(120, 40), ids, 50)
    oracle.check(table.grad, 2 * want, 2 * tol + 2 * oracle.UNIT[dtype] * 2 * want.abs())
    with torch.no_grad():
        assert not lkg.embed_entities(table, ids.cuda()).requires_grad


def test_streams_and_graphs():
    n, entities = 9000, 700
    table, ids, dout = _table(27, entities, 64, torch.bfloat16).cuda(), _ids(28, n, entities, 2).cuda(), _table(29, n, 64, torch.bfloat16).cuda()
    want, grad = lkg.embed_entities(table, ids, scale=2.0), lkg.embed_entities_backward(dout, ids, entities)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other, other_grad = lkg.embed_entities(table, ids, scale=2.0, stream=side), lkg.embed_entities_backward(dout, ids, entities, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(other, want) and torch.equal(other_grad, grad)
    few = ids[:500].contiguous()
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, b = lkg.embed_entities(table, ids, scale=2.0), lkg.embed_entities_backward(dout, ids, entities)
    with torch.cuda.graph(second, pool=graph.pool()):
        c = lkg.embed_entities_backward(dout[:500], few, entities)
    for seed in range(4):
        ids.copy_(_ids(30 + seed, n, entities, 2))
        few.copy_(ids[:500])
        dout.copy_(_table(40 + seed, n, 64, torch.bfloat16))
        graph.replay()
        got = a.clone(), b.clone()
        second.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], lkg.embed_entities(table, ids, scale=2.0)) and torch.equal(got[1], lkg.embed_entities_backward(dout, ids, entities))
        assert torch.equal(c, lkg.embed_entities_backward(dout[:500], few, entities))


def test_what_the_binding_refuses():
    table, ids = torch.zeros(4, 8, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    for bad, says in [(lambda: lkg.embed_entities(table, ids.long()), "int32"), (lambda: lkg.embed_entities(table.t(), ids), "last axis"), (lambda: lkg.embed_entities(table.double(), ids), "not supported"),
                      (lambda: lkg.embed_entities(table[0], ids), "entities, dim"), (lambda: lkg.embed_entities(table, ids[::2]), "contiguous"),
                      (lambda: lkg.embed_entities_backward(table, ids, 4), "shape"), (lambda: lkg.embed_entities_backward(table[:3], ids, 4, accumulate=True), "needs out"),
                      (lambda: lkg.embed_entities_backward(table[:3], ids, 5, out=table), "shape"), (lambda: lkg.embed_entities_backward(table[:3], ids, 4, out=table.half()), "float32"),
                      (lambda: lkg.embed_entities_backward(table[:1].expand(3, 8), ids, 4), "contiguous"), (lambda: lkg.embed_entities_backward(table[:3], ids, 4, out=table), "shares memory")]:
        with pytest.raises(ValueError, match=says):
            bad()
    with pytest.raises(lkg.LogosKGError, match="overlap"):
        lkg.embed_entities_backward(table[:3].clone(), ids, 4, out=table[:1].expand(4, 8))


def test_more_ids_than_a_launch_takes(memory_given_back):
    n = (1 << 34) + 3000  # four rows of one element a thread: 2^32 threads and some
    table = torch.tensor([[1.0], [2.0], [3.0]], dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    ids[-2500:] = 2
    ids[-1], ids[0] = 5, 1
    got = lkg.embed_entities(table, ids)
    assert got.shape == (n, 1) and got[0] == 2 and got[-1] == 0
    assert bool((got[1:-2500] == 1).all()) and bool((got[-2500:-1] == 3).all())


def test_tangents_are_not_lost():
    table, ids = torch.ones(5, 8, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    with torch.autograd.forward_ad.dual_level():
        assert lkg.embed_entities(table, ids).shape == (3, 8)
        with pytest.raises(NotImplementedError, match="jvp"):
            lkg.embed_entities(torch.autograd.forward_ad.make_dual(table, torch.ones_like(table)), ids)
