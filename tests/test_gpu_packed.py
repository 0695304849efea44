"""Tables in 4 bits and attention to them against their 64-bit definitions (bounds: around_oracle)."""
import math

import pytest
import torch

import around_oracle as oracle
import paper_2604_18913_amd as lkg

pytestmark = pytest.mark.gpu
HALVES = [torch.bfloat16, torch.float16]


def _kv(seed, n, heads, dim, dtype=torch.bfloat16, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return tuple((torch.randn(n, heads, dim, generator=g) * size).to(dtype) for _ in range(2))


def _gpu(a):
    return {k: x.cuda() if isinstance(x, torch.Tensor) else x for k, x in a.items()}


# ---------------------------------------------------------------- rows
def _check_rows(got, keys, values):
    want, near = oracle.pack(keys, values)
    n, K, D = keys.shape
    got = got.cpu()
    if not torch.equal(got, want):
        a, b = oracle.unpack(got, K, D), oracle.unpack(want, K, D)
        assert torch.equal(got[:, 32 * K * oracle.groups_of(D):], want[:, 32 * K * oracle.groups_of(D):]), "scales and bases, and what lies behind them"
        off = a[0] != b[0]
        assert not (off & ~near.transpose(0, 1)).any() and ((a[0] - b[0]).abs() <= 1.01 * b[1].abs()).all()


@pytest.mark.parametrize("dtype", [torch.float32, *HALVES], ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("heads, dim", [(1, 8), (1, 16), (2, 32), (3, 40), (5, 72), (4, 96), (8, 128), (7, 104), (1, 128)])
def test_rows(heads, dim, dtype):
    k, v = _kv(dim, 9, heads, dim, dtype, 3.0)
    got = lkg.pack_entities(k.cuda(), v.cuda())
    _check_rows(got, k, v)
    for to in (torch.float32, *HALVES):
        back = lkg.unpack_entities(got, heads, dim, dtype=to)
        want = oracle.unpack(got, heads, dim)[0]
        for x, y in zip(back, want):
            oracle.check(x, y, (oracle.UNIT[to] + oracle.E32) * y.abs() + oracle.LEAST[to])


@pytest.mark.parametrize("n", [0, 1, 63, 64, 65, 5000])
def test_numbers_of_rows(n):
    k, v = _kv(1, n, 2, 64)
    _check_rows(lkg.pack_entities(k.cuda(), v.cuda()), k, v)


def test_strides_and_rows_of_a_larger_table():
    k, v = _kv(2, 12, 6, 48)
    both = torch.cat([k, v], 2).cuda()
    got = lkg.pack_entities(both[:, :, :48], both[:, :, 48:])
    _check_rows(got, k, v)
    assert torch.equal(lkg.pack_entities(both[:, 1::2, :48], both[:, 1::2, 48:]), lkg.pack_entities(k[:, 1::2].cuda(), v[:, 1::2].cuda()))
    odd = torch.zeros(12, 6, 51, dtype=torch.bfloat16, device="cuda")
    odd[:, :, 3:] = k.cuda()
    assert torch.equal(lkg.pack_entities(odd[:, :, 3:], v.cuda()), got)
    assert torch.equal(lkg.pack_entities(k.cuda()[:1].expand(12, 6, 48), v.cuda()), lkg.pack_entities(k[:1].expand(12, 6, 48).contiguous().cuda(), v.cuda()))
    table = torch.full((20, got.shape[1] + 16), 77, dtype=torch.uint8, device="cuda")
    lkg.pack_entities(k.cuda(), v.cuda(), out=table[4:16, :got.shape[1]])
    assert torch.equal(table[4:16, :-16], got) and (table[:4] == 77).all() and (table[16:] == 77).all() and (table[:, -16:] == 77).all()
    table[torch.tensor([19, 0]).cuda(), :-16] = lkg.pack_entities(k[:2].cuda(), v[:2].cuda())
    assert torch.equal(table[19, :-16], got[0])


def test_odd_groups():
    """Constant groups, tiny and huge ranges, zeros, infinities and NaN."""
    k, v = _kv(3, 10, 1, 64, torch.float32)
    k[0], k[1], k[2, :, 5], k[3, :, 40], k[4] = 1.5, 0.0, math.inf, math.nan, 1e-38
    v[0, :, 3], v[1, :, :32], v[2] = 1e38, -3e38, torch.linspace(-3e38, 3e38, 64)
    v[3], v[4], v[5, :, :] = torch.linspace(1e-40, 3e-40, 64), 65504.0, -0.0
    got = lkg.pack_entities(k.cuda(), v.cuda())
    _check_rows(got, k, v)
    back = lkg.unpack_entities(got, 1, 64, dtype=torch.float32)
    assert (back[0][0] == 1.5).all() and (back[0][1] == 0).all()
    assert back[0][2, 0, :32].isnan().all() and back[0][2, 0, 32:].isfinite().all() and back[0][3, 0, 32:].isnan().all()
    assert (back[1][5] == 0).all()


# ---------------------------------------------------------------- attention
def _case(seed, lengths, heads, kv_heads, dim, dtype=torch.bfloat16, tokens=1, entities=300, bias=False, far=6, size=1.0, **kw):
    g = torch.Generator().manual_seed(seed)
    rows, _ = oracle.pack(*_kv(seed + 1, entities, kv_heads, dim, dtype, size))
    n = sum(lengths)
    a = dict(q=torch.randn(len(lengths), tokens, heads, dim, generator=g).to(dtype), packed=rows, off=torch.tensor([0] + list(lengths)).cumsum(0),
             entity=torch.randint(0, max(entities, 1), (n,), generator=g).int(), kv_heads=kv_heads)
    if bias:
        a |= dict(bias=torch.randn(heads, 8, generator=g).to(dtype), buckets=lkg.distance_buckets(8, far, device="cpu"), hop=torch.randint(0, 4, (n,), generator=g).to(torch.uint8))
    return a | kw


def _check(a, what=""):
    got = lkg.read_packed(**_gpu(a))
    res, tol = oracle.read_packed(**a)
    for name in res:
        oracle.check(got[name], res[name], tol[name], f"{what} {name}")
    return got


@pytest.mark.parametrize("dtype", HALVES, ids=["bf16", "fp16"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("cap", [0.0, 3.0])
@pytest.mark.parametrize("heads, kv_heads, dim", [(4, 4, 128), (6, 2, 80), (5, 5, 40), (2, 2, 8), (12, 4, 96), (8, 1, 128), (16, 8, 64), (9, 9, 32), (11, 11, 24), (32, 8, 128)])
def test_heads_types_and_scores(heads, kv_heads, dim, cap, bias, dtype):
    _check(_case(7, [37, 2, 0, 90], heads, kv_heads, dim, dtype, bias=bias, cap=cap, entities=60))


@pytest.mark.parametrize("lengths", [[1], [0], [63], [64], [65], [127, 1, 128, 129], [0, 0, 700, 0], [3] * 40, [1, 0] * 9, [5000]], ids=str)
@pytest.mark.parametrize("kv_heads", [1, 8])
def test_lengths(lengths, kv_heads):
    got = _check(_case(8, lengths, 8, kv_heads, 64, bias=True, cap=5.0))
    for i, n in enumerate(lengths):
        if n == 0:
            assert (got["out"][i] == 0).all() and (got["lse"][i] == -math.inf).all()


# lists that a block has alone, and that several share
@pytest.mark.parametrize("dtype", HALVES, ids=["bf16", "fp16"])
@pytest.mark.parametrize("heads, kv_heads, dim", [(4, 4, 128), (6, 2, 80), (5, 5, 40), (2, 2, 8), (12, 4, 96), (8, 1, 128), (16, 8, 64), (9, 9, 32)])
@pytest.mark.parametrize("lengths, tokens", [([1100], 1), ([1030, 0, 2100, 3], 3), ([600], 5)], ids=str)
def test_lists_of_several_blocks(lengths, tokens, heads, kv_heads, dim, dtype):
    _check(_case(26, lengths, heads, kv_heads, dim, dtype, bias=True, cap=5.0, tokens=tokens))


@pytest.mark.parametrize("lengths", [[512], [513], [1023], [1024], [1025], [4095, 1] + [0] * 9, [4096, 1] + [0] * 9, [0, 4096] + [0] * 8, [64] * 64, [64] * 63 + [65]], ids=lambda x: f"{len(x)}_{sum(x)}")
@pytest.mark.parametrize("heads, kv_heads, dim", [(8, 1, 128), (4, 2, 64)])
def test_where_lists_begin_to_share_blocks(lengths, heads, kv_heads, dim):
    _check(_case(27, lengths, heads, kv_heads, dim))


@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 5, 9, 33, 70])
@pytest.mark.parametrize("heads, kv_heads", [(8, 1), (4, 4), (20, 4)])
def test_tokens(tokens, heads, kv_heads):
    _check(_case(9, [30, 100], heads, kv_heads, 48, tokens=tokens, bias=True, q_pos=torch.tensor([2, -3], dtype=torch.int32)))


@pytest.mark.parametrize("scale", [-0.3, 0.0, 1.0])
def test_scales(scale):
    _check(_case(10, [80], 4, 2, 64, scale=scale))


@pytest.mark.parametrize("size", [1e-6, 1e-3, 300.0])
@pytest.mark.parametrize("dtype", HALVES, ids=["bf16", "fp16"])
def test_small_and_large_values(size, dtype):
    """Weights are p times a scale: in float16 they would leave its range."""
    a = _case(11, [200, 70], 4, 2, 64, dtype)
    g = torch.Generator().manual_seed(1)
    keys = torch.randn(300, 2, 64, generator=g)
    a["packed"], _ = oracle.pack(keys, torch.randn(300, 2, 64, generator=g) * size)
    got, (res, tol) = lkg.read_packed(**_gpu(a)), oracle.read_packed(**a)
    least = oracle.LEAST[dtype]
    assert ((got["out"].cpu().double() - res["out"]).abs() <= tol["out"]).all()
    assert float((got["out"].cpu().double() - res["out"]).norm()) <= 2 * oracle.UNIT[dtype] * float(res["out"].norm()) + least * res["out"].numel() ** 0.5
    # scales of a list that grow a thousandfold and more from tile to tile
    k, v = torch.randn(300, 2, 64, generator=g), torch.randn(300, 2, 64, generator=g) * torch.logspace(-7, 3, 300)[:, None, None]
    a["packed"], _ = oracle.pack(k, v)
    a["entity"] = torch.arange(270).int() + 30
    _check(a)


def test_ids_outside_the_table_and_no_ids():
    a = _case(12, [50, 40], 4, 2, 64, entities=100)
    a["entity"][::3] = torch.tensor([-1, 100, 2 ** 31 - 1, -2 ** 31] * 8, dtype=torch.int32)[:30]
    _check(a)
    a["entity"][:50] = -1  # a whole list
    got = _check(a)
    assert (got["out"][0] == 0).all() and (got["lse"][0] == -math.inf).all()
    b = _case(13, [30, 70], 4, 2, 64, entities=100)
    del b["entity"]
    _check(b)
    empty = _case(14, [0, 0], 4, 2, 64, entities=0)
    assert (_check(empty)["out"] == 0).all()


def test_offsets_of_a_part_of_a_batch():
    a = _case(15, [300, 200, 100], 4, 2, 64)
    a["off"] = torch.tensor([130, 290, 290, 555])
    got = _check(a)
    b = _gpu(a)
    b["off"] = torch.tensor([-7, 290, 290, 9999]).cuda()
    wild = lkg.read_packed(**b)  # taken into the list
    assert wild["out"].isfinite().all() and torch.equal(wild["out"][1], got["out"][1])
    b["off"] = torch.tensor([290, 130, 600, 20]).cuda()  # no offsets at all (they ascend): nothing outside the arrays is read or written
    lkg.read_packed(**b)
    assert all(torch.equal(x, got[n]) for n, x in lkg.read_packed(**_gpu(a)).items())


def test_biases_that_hide():
    a = _case(16, [150, 90], 4, 2, 64, bias=True, cap=8.0)
    kind = a["buckets"][a["hop"].long() + 6]
    a["bias"][:, kind[:64].unique()[0]] = -math.inf
    a["bias"][2, :] = torch.finfo(torch.bfloat16).min
    got = lkg.read_packed(**_gpu(a))
    b = {**a, "bias": torch.where(a["bias"] < -7e4, torch.tensor(-1e300, dtype=torch.float64), a["bias"].double())}
    res, tol = oracle.read_packed(**b)
    for h in (0, 1, 3):
        assert ((got["out"][:, :, h].cpu().double() - res["out"][:, :, h]).abs() <= tol["out"][:, :, h].clamp(max=0.05)).all()
    assert (got["out"][:, :, 2] == 0).all() and (got["lse"][:, :, 2] == -math.inf).all()


def test_nan_stays_in_its_lists():
    a = _case(17, [70, 70, 70], 4, 2, 64)
    k, v = _kv(3, 300, 2, 64)
    k[5, 1, 3], v[6, 0, 3] = math.nan, math.inf
    a["packed"], _ = oracle.pack(k, v)
    a["entity"][a["entity"] == 5], a["entity"][a["entity"] == 6] = 7, 8
    a["entity"][10], a["entity"][80] = 5, 6
    got = lkg.read_packed(**_gpu(a))
    bad = got["out"].isnan().any(3).any(1).cpu()
    assert bad.tolist() == [[False, False, True, True], [True, True, False, False], [False] * 4]
    assert got["out"][1, :, :2, 32:].isfinite().all()


def test_rows_of_a_wider_table_and_far_ones():
    a = _case(18, [120], 4, 2, 64)
    wide = torch.full((300, a["packed"].shape[1] + 48), 255, dtype=torch.uint8, device="cuda")
    wide[:, 16:16 + a["packed"].shape[1]] = a["packed"].cuda()
    b = _gpu(a)
    want = lkg.read_packed(**b)
    got = lkg.read_packed(**{**b, "packed": wide[:, 16:16 + a["packed"].shape[1]]})
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
    big = torch.zeros(4_000_000, 1280, dtype=torch.uint8, device="cuda")  # 5.1 GB, 8 heads of 128
    k, v = _kv(19, 50, 8, 128)
    big[-50:] = lkg.pack_entities(k.cuda(), v.cuda())
    c = _gpu(_case(20, [50], 8, 8, 128, entities=50))
    near = lkg.read_packed(**{**c, "packed": big[-50:], "entity": torch.arange(50).int().cuda()})
    far = lkg.read_packed(**{**c, "packed": big, "entity": torch.arange(4_000_000 - 50, 4_000_000).int().cuda()})
    assert torch.equal(near["out"], far["out"]) and float(far["out"].abs().max()) > 0


def test_the_same_bits_streams_and_graphs():
    a = _gpu(_case(21, [400, 30, 700], 8, 4, 96, bias=True, cap=4.0))
    want = lkg.read_packed(**a)
    again = lkg.read_packed(**a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = lkg.read_packed(**a, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(x[n], want[n]) for x in (again, other) for n in want)
    k, v = (x.cuda() for x in _kv(22, 300, 4, 96))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lkg.pack_entities(k, v, out=a["packed"])
        got = lkg.read_packed(**a)
        back = lkg.unpack_entities(a["packed"], 4, 96, dtype=torch.bfloat16)
    for seed in range(4):
        for x, y in zip((k, v), _kv(30 + seed, 300, 4, 96)):
            x.copy_(y)
        a["q"].copy_(_case(40 + seed, [400, 30, 700], 8, 4, 96)["q"])
        graph.replay()
        torch.cuda.synchronize()
        want = lkg.read_packed(**{**a, "packed": lkg.pack_entities(k, v)})
        assert all(torch.equal(got[n], want[n]) for n in want)
        assert all(torch.equal(x, y) for x, y in zip(back, lkg.unpack_entities(a["packed"], 4, 96, dtype=torch.bfloat16)))


@pytest.mark.parametrize("far", [1024, 200])
def test_biases_of_many_distances(far):
    a = _case(23, [90, 40], 4 if far == 1024 else 20, 2 if far == 1024 else 2, 64, bias=True, far=far, q_pos=torch.tensor([-900, 2 ** 31 - 1], dtype=torch.int32))
    _check(a)


def test_what_the_binding_refuses():
    a = _gpu(_case(24, [9], 4, 2, 64))
    k, v = (x.cuda() for x in _kv(25, 9, 2, 64))
    for bad, says in [(lambda: lkg.read_packed(**{**a, "kv_heads": 4}), "uint8"), (lambda: lkg.read_packed(**{**a, "kv_heads": 0}), "kv_heads"), (lambda: lkg.read_packed(**{**a, "packed": a["packed"].int()}), "uint8"),
                      (lambda: lkg.read_packed(**{**a, "q": a["q"].float()[0]}), "q must be"), (lambda: lkg.read_packed(**{**a, "entity": a["entity"].long()}), "int32"),
                      (lambda: lkg.pack_entities(k, v[:5]), "one shape"), (lambda: lkg.pack_entities(k, v.half()), "bfloat16"), (lambda: lkg.pack_entities(k, v, out=a["packed"][:5]), "rows"),
                      (lambda: lkg.pack_entities(k[:, :, :12], v[:, :, :12]), "multiple of 8"), (lambda: lkg.unpack_entities(a["packed"], 2, 128, dtype=torch.float32), "uint8"),
                      (lambda: lkg.unpack_entities(a["packed"], 2, 64, dtype=torch.float64), "not supported"),
                      (lambda: lkg.pack_entities(k, v, out=v.view(torch.uint8).view(9, 256)[:, :160]), "shares memory")]:
        with pytest.raises(ValueError, match=says):
            bad()
    with pytest.raises(lkg.LogosKGError, match="type"):
        lkg.read_packed(**{**a, "q": a["q"].float()})
    with pytest.raises(lkg.LogosKGError, match="multiple"):
        lkg.read_packed(**{**a, "q": a["q"][:, :, :3].contiguous()})


@pytest.mark.parametrize("packed", [False, True], ids=["16 bits", "4 bits"])
def test_more_lists_than_a_launch_takes(packed, memory_given_back):
    """2^26 lists and some of one entry, the last one of 5,000, in four heads: 2^32 threads and more of the reading and of the join."""
    lists, entities = (1 << 26) + 40, 6001
    values = (torch.arange(entities, device="cuda") % 50).to(torch.bfloat16)[:, None, None].expand(-1, 4, 8).contiguous()
    keys = torch.zeros_like(values)
    off = torch.arange(lists + 1, device="cuda")
    off[-1] = lists - 1 + 5000
    entity = (torch.arange(lists - 1 + 5000, device="cuda") % entities).int()
    q = torch.ones(lists, 1, 4, 8, dtype=torch.bfloat16, device="cuda")
    got = lkg.read_packed(q, lkg.pack_entities(keys, values), off, entity, kv_heads=4) if packed else lkg.read_entities(q, keys, values, off, entity)
    out, lse = got["out"], got["lse"]
    want = (entity[:lists - 1] % 50).to(torch.bfloat16)
    for h in range(4):
        for c in (0, 7):
            assert bool((out[:-1, 0, h, c] == want).all())
    assert bool((lse[:-1] == 0).all())
    assert float((out[-1].float() - float((entity[-5000:] % 50).double().mean())).abs().max()) < 25 * 2 ** -7 and float((lse[-1] - math.log(5000)).abs().max()) < 1e-4


@pytest.mark.parametrize("dtype", [torch.float32, *HALVES], ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("offset, spread", [(0.0, 1.0), (1000.0, 1.0), (-1000.0, 1.0), (1000.0, 1e-3), (257.0, 30.0), (-3.0, 0.1), (5e4, 100.0)])
def test_groups_that_stand_far_from_nothing(offset, spread, dtype):
    """With lo and R a group's smallest element and range, u = 2^-8: its base is off by u |lo|, its step s by u of itself, so the
    last code's place by u (|lo| + R).  An element between the first and the last code is off by s / 2, one outside by what
    those places are; the value, a product and sum in 32 bits and a rounding to float32, by 2^-23 of its size."""
    g = torch.Generator().manual_seed(50)
    k, v = ((offset + torch.rand(200, 3, 64, generator=g) * spread).to(dtype) for _ in range(2))
    rows = lkg.pack_entities(k.cuda(), v.cuda())
    _check_rows(rows, k, v)
    for x, y in zip((k, v), lkg.unpack_entities(rows, 3, 64, dtype=torch.float32)):
        x, y = (t.cpu().double().view(200, 3, 2, 32) for t in (x, y))
        lo, hi = x.amin(3, keepdim=True), x.amax(3, keepdim=True)
        step = (hi - lo) / 15 * (1 + 2 ** -8)
        bound = torch.maximum(step / 2, 2.0 ** -8 * (lo.abs() + hi - lo)) * (1 + 2 ** -20) + 2.0 ** -23 * (x.abs() + y.abs())
        assert bool(((x - y).abs() <= bound).all())
