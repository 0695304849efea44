"""token_logp, policy_loss and its gradient against their 64-bit definitions (bounds: around_oracle)."""
import math

import pytest
import torch

import around_oracle as oracle
import paper_2604_18913_amd as lkg

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
TYPE_NAMES = ["fp32", "bf16", "fp16"]


def _case(seed, rows, vocab, dtype=torch.float32, masks=None, spread=3.0, kl=0.07, scale=0.8, **kw):
    """Ratios stand clear of the clip's borders; a third of the ids of a mask are open, its rows' targets nearly always."""
    g = torch.Generator().manual_seed(seed)
    logits = (torch.randn(rows, vocab, generator=g) * spread).to(dtype)
    target = torch.randint(0, max(vocab, 1), (rows,), generator=g).int()
    a = dict(logits=logits, target=target, advantage=torch.randn(rows, generator=g), kl=kl, scale=scale, weight=torch.rand(rows, generator=g) / max(rows, 1)) | kw
    if masks is not None:
        open_ = torch.rand(masks, (vocab + 63) // 64 * 64, generator=g) < 0.34
        a["mask_row"] = torch.randint(0, masks, (rows,), generator=g).int()
        for r in range(0, rows, 2):
            open_[int(a["mask_row"][r]), int(target[r])] = True
        a["mask"] = (open_.view(masks, -1, 64).long() << torch.arange(64)).sum(2)
    lp = oracle.policy(logits, target, scale=scale, mask=a.get("mask"), mask_row=a.get("mask_row"))[0]["logp"]
    lp = torch.where(lp.isfinite(), lp, 0.0).float()
    off = torch.randint(-8, 9, (rows,), generator=g) * 0.05 + (torch.rand(rows, generator=g) - 0.5) * 0.02
    return a | dict(old=lp - off, ref=lp + torch.randn(rows, generator=g) * 0.3)


def _gpu(a):
    return {k: x.cuda() if isinstance(x, torch.Tensor) else x for k, x in a.items()}


def _check(a, cuda=None, what=""):
    b = _gpu(a) if cuda is None else cuda
    res, tol = oracle.policy(**a)
    got = lkg.policy_loss(**b, gradient=True)
    few = {k: b[k] for k in ("logits", "target", "scale", "mask", "mask_row") if k in b}
    alone = lkg.policy_loss(**b)
    logp = lkg.token_logp(**few)
    rest = {k: x for k, x in b.items() if k not in ("logits", "target", "advantage")}
    dlogits = lkg.policy_loss_backward(torch.tensor(1.0, device="cuda"), b["logits"], b["target"], b["advantage"], got["lse"], **rest)
    for name in res:
        oracle.check(got[name], res[name], tol[name], f"{what} {name}")
        if name != "dlogits":
            assert torch.equal(alone[name].nan_to_num(5.0), got[name].nan_to_num(5.0)), name
    for name in ("logp", "lse"):
        assert torch.equal(logp[name].nan_to_num(5.0), got[name].nan_to_num(5.0)), name
    # the backward makes logp of the rounded lse: one more rounding of that, by which slopes and shares move
    more = 4 * oracle.E32 * (1 + torch.where(res["lse"].isfinite(), res["lse"], 0.0).abs())[:, None] * (res["dlogits"].abs() + _steep(a))
    oracle.check(dlogits, res["dlogits"], tol["dlogits"] + more, f"{what} backward")
    return got


def _steep(a):
    """How much a row's dlogits move with its logp, at most."""
    lp = oracle.policy(**{k: a[k] for k in ("logits", "target", "scale", "mask", "mask_row") if k in a})[0]["logp"]
    lp = torch.where(lp.isfinite(), lp, 0.0)
    old, ref = (lp if a.get(k) is None else a[k].double() for k in ("old", "ref"))
    w = 1.0 if a.get("weight") is None else a["weight"].double().abs()
    return (w * a["scale"] * (torch.exp(lp - old).clamp(max=1e4) * a["advantage"].abs() + a["kl"] * torch.exp((ref - lp).clamp(max=20)))).nan_to_num(0.0)[:, None]  # (NaN: of a row that does not count)


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_NAMES)
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 63, 64, 65, 500, 4095, 4096, 4097, 10_001])
def test_sizes_and_types(vocab, dtype):
    _check(_case(vocab, 5, vocab, dtype), what="open")
    _check(_case(vocab, 9, vocab, dtype, masks=4), what="masked")


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_NAMES)
def test_a_large_vocabulary(dtype):
    _check(_case(1, 12, 150_001, dtype, masks=3))


@pytest.mark.parametrize("rows", [0, 1, 3, 300])
def test_rows(rows):
    got = _check(_case(2, rows, 40, masks=2))
    assert rows or float(got["loss"]) == 0.0


def test_no_vocabulary():
    a = _gpu(dict(logits=torch.zeros(3, 0), target=torch.tensor([0, -1, 5], dtype=torch.int32), advantage=torch.ones(3)))
    got = lkg.policy_loss(**a, gradient=True)
    assert got["loss"] == 0 and (got["logp"] == 0).all() and (got["lse"] == -math.inf).all() and got["dlogits"].shape == (3, 0)


@pytest.mark.parametrize("change", [dict(old=None), dict(weight=None), dict(kl=0.0, ref=None), dict(clip=(0.0, 0.0)), dict(clip=(0.1, 0.3)), dict(clip=(5.0, 1e30)), dict(scale=3.0),
                                    dict(scale=1e-3)])
def test_options(change):
    a = _case(3, 40, 300, masks=5, scale=change.get("scale", 0.8))
    _check(a | change)


def test_strided_logits_and_gradients_in_place():
    a = _case(4, 6, 200, torch.bfloat16, masks=2)
    for lead, width in [(0, 256), (1, 203), (3, 300), (8, 208)]:
        wide = torch.full((6, width + lead), float("nan"), dtype=torch.bfloat16)
        wide[:, lead:lead + 200] = a["logits"]
        _check(a, _gpu(a) | {"logits": wide.cuda()[:, lead:lead + 200]})


def test_rows_that_do_not_count():
    a = _case(5, 8, 100, masks=3)
    a["mask"][1] = 0
    a["mask_row"] = torch.tensor([0, 1, 2, -1, 3, 0, 2, 2 ** 31 - 1], dtype=torch.int32)
    a["target"][[2, 5]] = torch.tensor([-1, 100], dtype=torch.int32)
    a["advantage"][2], a["old"][5], a["weight"][3], a["ref"][1] = math.nan, math.inf, math.nan, -math.inf  # of rows that do not count
    got = _check(a)
    assert got["logp"][[1, 3, 4, 7]].tolist() == [-math.inf] * 4 and got["logp"][[2, 5]].tolist() == [0, 0]
    assert (got["lse"][[1, 3, 4, 7]] == -math.inf).all() and (got["dlogits"][[1, 2, 3, 4, 5, 7]] == 0).all()


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_NAMES)
def test_infinities_nan_and_lowest_values(dtype):
    low = torch.finfo(dtype).min
    a = _case(6, 6, 90, dtype, masks=2)
    a["mask_row"][:] = 0
    a["target"][:] = 10
    hidden = [v for v in range(90) if not a["mask"][0, v // 64] >> (v % 64) & 1 and v != 10]
    a["mask"][0, 0] |= 1 << 10
    a["logits"][:, hidden[:3]] = torch.tensor([math.nan, math.inf, -math.inf], dtype=dtype)  # hidden places do not matter
    open_ = [v for v in range(90) if v not in hidden and v != 10]
    a["logits"][0, open_[:4]] = -math.inf
    a["logits"][1, open_] = low
    a["logits"][2, 10] = -math.inf       # an answer that cannot be
    a["old"] = oracle.policy(a["logits"], a["target"], scale=a["scale"], mask=a["mask"], mask_row=a["mask_row"])[0]["logp"].clamp(min=-50).float()
    a["ref"] = a["old"] - 0.1
    _check(a)
    # a whole row at the type's lowest value is a row of equal ones
    a["logits"][3] = low
    got = lkg.token_logp(a["logits"].cuda(), a["target"].cuda(), scale=1.0)
    assert abs(float(got["logp"][3]) + math.log(90)) < 1e-5
    a["logits"][4, open_[0]] = math.nan  # one in sight spoils its row, and the loss
    b = _gpu(a)
    got = lkg.policy_loss(**b, gradient=True)
    assert got["loss"].isnan() and got["lse"].isnan().tolist() == [False] * 4 + [True, False]
    assert got["dlogits"][5].isfinite().all() and got["dlogits"][4].isnan().any()
    b["weight"][4] = 0.0  # .. unless it weighs nothing
    got = lkg.policy_loss(**b, gradient=True)
    assert got["loss"].isfinite() and (got["dlogits"][4] == 0).all()


def test_far_policies():
    a = _case(7, 8, 30)
    a["old"] = torch.tensor([-200.0, 200.0, -200.0, 200.0, -math.inf, -math.inf, 0.0, 0.0])
    a["advantage"] = torch.tensor([1.0, 1.0, -1.0, -1.0, 1.0, 0.0, 0.0, 0.0])
    a["kl"], a["ref"] = 0.0, None
    got = lkg.policy_loss(**_gpu(a), gradient=True)
    w = a["weight"].double()
    # far above: held at 1.2 where that is better, without bound (an infinite loss) where it is worse; far below the other way round
    each = torch.stack([lkg.policy_loss(**_gpu({k: x[i:i + 1] if isinstance(x, torch.Tensor) else x for k, x in a.items()}))["loss"] for i in range(8)]).cpu().double()
    assert torch.allclose(each[[0, 3, 4]], torch.stack([-1.2 * w[0], 0.8 * w[3], -1.2 * w[4]]), rtol=1e-6)
    assert each[1] == 0 and each[2] == math.inf and (each[5:] == 0).all()
    assert (got["dlogits"][[0, 1, 3, 4, 5, 6, 7]] == 0).all()


@pytest.mark.parametrize("vocab", [50, 5000])
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_NAMES)
def test_torch_s_backward(dtype, vocab):
    a = _case(8, 30, vocab, dtype, masks=3)
    b = _gpu(a)
    b["logits"].requires_grad_()
    got = lkg.policy_loss(**b)
    (got["loss"] * 3.0).backward()
    res, tol = oracle.policy(**a, dloss=3.0)
    more = 3 * 4 * oracle.E32 * (1 + res["lse"].abs().nan_to_num(0.0, posinf=0.0))[:, None] * (res["dlogits"].abs() + _steep(a))
    oracle.check(b["logits"].grad, res["dlogits"], tol["dlogits"] + more)
    assert not got["logp"].requires_grad and not got["lse"].requires_grad
    direct = lkg.policy_loss(**b, gradient=True)
    assert not direct["dlogits"].requires_grad and not direct["loss"].requires_grad
    with torch.no_grad():
        assert not lkg.policy_loss(**b)["loss"].requires_grad


def test_gradient_is_that_of_differences():
    a = _case(9, 4, 12, masks=2)
    a["weight"] = None
    got = lkg.policy_loss(**_gpu(a), gradient=True)["dlogits"].cpu().double()
    step = 2.0 ** -5
    for r in range(4):
        for v in range(12):
            two = []
            for sign in (1, -1):
                x = a["logits"].clone()
                x[r, v] += sign * step
                two.append(float(lkg.policy_loss(**_gpu({**a, "logits": x}))["loss"]))
            # third derivatives of the row's loss, at most some 4 (r A + kl e^d) scale^3, times step^2 / 6; 32-bit losses over 2 steps
            bound = 4 * float(_steep({**a, "weight": None})[r]) * step ** 2 + 8 * oracle.E32 * 10 / step
            crossed = any(abs(float(torch.exp(lkg.token_logp(**_gpu({k: a[k] for k in ("logits", "target", "scale", "mask", "mask_row")}))["logp"].cpu()[r] - a["old"][r])) - b) < 0.06 for b in (0.8, 1.2))
            assert crossed or abs((two[0] - two[1]) / (2 * step) - got[r, v]) <= bound, (r, v)


def test_streams_and_graphs():
    a = _gpu(_case(10, 64, 6000, torch.bfloat16, masks=4))
    want = lkg.policy_loss(**a, gradient=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = lkg.policy_loss(**a, gradient=True, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(got[k], want[k]) for k in want)
    rest = {k: x for k, x in a.items() if k not in ("logits", "target", "advantage")}
    dloss = torch.tensor(2.0, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = lkg.policy_loss(**a, gradient=True)
        back = lkg.policy_loss_backward(dloss, a["logits"], a["target"], a["advantage"], got["lse"], **rest)
    for seed in range(4):
        new = _case(20 + seed, 64, 6000, torch.bfloat16, masks=4)
        for k in ("logits", "target", "advantage", "old", "ref", "weight", "mask", "mask_row"):
            a[k].copy_(new[k])
        graph.replay()
        torch.cuda.synchronize()
        want = lkg.policy_loss(**a, gradient=True)
        assert all(torch.equal(got[k], want[k]) for k in want)
        assert torch.equal(back, lkg.policy_loss_backward(dloss, a["logits"], a["target"], a["advantage"], want["lse"], **rest))


def test_logits_beyond_32_bits():
    rows, vocab = 70_000, 32_768  # 2.3e9 elements
    logits = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    target = (torch.arange(rows, device="cuda") % vocab).int()
    got = lkg.policy_loss(logits, target, torch.ones(rows, device="cuda"), gradient=True)
    assert torch.allclose(got["logp"], torch.full((rows,), -math.log(vocab), device="cuda")) and abs(float(got["loss"]) + rows) < 1
    last = got["dlogits"][-1].double()
    assert abs(float(last[(rows - 1) % vocab]) + 1) < 0.01 and abs(float(last[5]) * vocab - 1) < 0.01


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_NAMES)
@pytest.mark.parametrize("rows, vocab", [(6, 300), (100, 300), (6, 5000), (6, 60_000)])
def test_nan_and_infinity_among_allowed_logits(rows, vocab, dtype):
    a = _case(13, rows, vocab, dtype)
    a["logits"][0, 7], a["logits"][1, vocab - 1], a["logits"][2, 3] = math.nan, math.inf, math.inf
    a["target"][:4] = torch.tensor([5, 6, 3, -1], dtype=torch.int32)
    a["logits"][3, 0] = math.nan  # of a row that pads
    a = a | dict(old=None, ref=torch.zeros(rows), kl=0.1)
    got = lkg.policy_loss(**_gpu(a), gradient=True)
    assert got["lse"][:4].isnan().all() and got["logp"][:3].isnan().all() and got["logp"][3] == 0 and got["loss"].isnan()
    assert got["dlogits"][:3].isnan().all() and (got["dlogits"][3] == 0).all()
    rest = {k: x[4:] if isinstance(x, torch.Tensor) else x for k, x in a.items()}
    res, tol = oracle.policy(**rest)
    for name in ("logp", "lse", "dlogits"):
        oracle.check(got[name][4:], res[name], tol[name], name)


def test_what_the_binding_refuses():
    a = _gpu(_case(11, 4, 70, masks=2))
    for change, says in [(dict(target=a["target"].long()), "int32"), (dict(target=a["target"][:3]), "shape"), (dict(advantage=a["advantage"].double()), "float32"), (dict(mask=a["mask"][:, :1]), "mask"),
                         (dict(mask_row=None), "shape"), (dict(mask_row=a["mask_row"].long()), "int32"), (dict(mask=None), "mask_row without"), (dict(ref=None), "kl without ref"),
                         (dict(logits=a["logits"].t()), "contiguous rows"), (dict(logits=a["logits"].double()), "not supported"), (dict(weight=a["weight"][:2]), "shape"),
                         (dict(mask=a["mask"][:0]), "without rows")]:
        with pytest.raises(ValueError, match=says):
            lkg.policy_loss(**{**a, **change})
    with pytest.raises(ValueError, match="dloss"):
        lkg.policy_loss_backward(torch.ones(1, device="cuda"), a["logits"], a["target"], a["advantage"], a["weight"])
    with pytest.raises(lkg.LogosKGError, match="scale"):
        lkg.policy_loss(**{**a, "scale": 0.0})


# A vocabulary for every kernel: by 16, 64, 256 (twice) and 1,024 lanes a row (under masks in two sweeps, else whole rows of two sizes, and two sweeps)
KERNELS = [300, 1501, 6001, 20_001, 60_001, 120_001, 200_001]


def _raw(call, a, dlogits, lse=None, dloss=None, logits=None):
    """The C call on a gradient that the caller has; (loss, logp, lse) of a forward."""
    from paper_2604_18913_amd import training
    from paper_2604_18913_amd.binding import _check as check, _load, _stream_handle
    x = a["logits"] if logits is None else logits
    head, device, rows = training._answers(x, a["target"], a.get("mask"), a.get("mask_row"))
    terms = training._terms(a["advantage"], a.get("old"), a.get("ref"), a.get("weight"), a.get("clip", (0.2, 0.2)), a.get("kl", 0.0), a.get("scale", 1.0), rows, device)
    loss, logp = torch.empty((), device="cuda"), torch.empty(rows, device="cuda")
    lse = torch.empty(rows, device="cuda") if lse is None else lse
    check(getattr(_load(), call)(training._policy_of(*head, *terms, logp.data_ptr(), lse.data_ptr(), loss.data_ptr(), dlogits.data_ptr(), 0 if dloss is None else dloss.data_ptr(),
                                                     _stream_handle(None, device))))
    return loss, logp, lse


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_NAMES)
@pytest.mark.parametrize("masks", [None, 2], ids=["open", "masked"])
@pytest.mark.parametrize("vocab", KERNELS)
def test_rows_that_do_not_count_under_a_loss_that_is_not_finite(vocab, masks, dtype):
    rows, pad = 9, 512
    a = _case(30, rows, vocab, dtype, masks=masks)
    idle = torch.tensor([True, True, False, True, True, False, True, masks is not None, True])
    a["target"][[0, 1, 3, 4, 8]] = torch.tensor([-1, -100, vocab, 2 ** 31 - 1, -3], dtype=torch.int32)
    a["weight"][6] = 0.0
    if masks:
        a["mask_row"] = torch.tensor([0, 1, 0, 1, 0, 0, 1, -1, 0], dtype=torch.int32)
        for r in (2, 5):
            a["mask"][0, int(a["target"][r]) // 64] |= -2 ** 63 if int(a["target"][r]) % 64 == 63 else 1 << int(a["target"][r]) % 64
        hidden = ~((a["mask"][0][:, None] >> torch.arange(64)) & 1).reshape(-1)[:vocab].bool()
    b = _gpu(a)
    lse = lkg.token_logp(**{k: b[k] for k in ("logits", "target", "scale", "mask", "mask_row") if k in b})["lse"]
    for dloss in (math.inf, -math.inf, math.nan):
        flat = torch.full((pad + rows * vocab + pad,), 7.0, dtype=dtype, device="cuda")
        got = flat[pad:pad + rows * vocab].view(rows, vocab)
        _raw("logoskg_policy_loss_backward", b, got, lse, torch.tensor(dloss, device="cuda"))
        assert (flat[:pad] == 7).all() and (flat[-pad:] == 7).all()
        assert (got[idle] == 0).all() and not got[~idle].isfinite().all(1).any()
        if masks:
            assert (got[[2, 5]][:, hidden] == 0).all()


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_NAMES)
@pytest.mark.parametrize("rows, vocab", [(100, 300)] + [(6, v) for v in KERNELS])
def test_hidden_ids_get_no_gradient_whatever_their_row_holds(rows, vocab, dtype):
    a = _case(31, rows, vocab, dtype, masks=2)
    a["mask_row"][:] = 0
    a["target"][:] = 70
    a["mask"][0, 0] |= 1 << 9
    a["mask"][0, 1] |= 1 << 70 - 64
    hidden = ~((a["mask"][0][:, None] >> torch.arange(64)) & 1).reshape(-1)[:vocab].bool()
    a["logits"][0, 9], a["logits"][1, 9], a["logits"][2, 70] = math.nan, math.inf, math.nan
    a["logits"][3, hidden.nonzero()[:2, 0]] = torch.tensor([math.nan, math.inf], dtype=dtype)
    a["old"][4], a["advantage"][4] = -1000.0, -1.0  # a ratio above 32 bits
    b = _gpu(a)
    got = lkg.policy_loss(**b, gradient=True)
    rest = {k: x for k, x in b.items() if k not in ("logits", "target", "advantage")}
    back = lkg.policy_loss_backward(torch.tensor(1.0, device="cuda"), b["logits"], b["target"], b["advantage"], got["lse"], **rest)
    for d in (got["dlogits"], back):
        assert (d[:, hidden] == 0).all()
        assert d[0, ~hidden].isnan().all() and d[1, ~hidden].isnan().all() and d[2, ~hidden].isnan().all() and d[4, 70] == math.inf and d[5].isfinite().all()


@pytest.mark.parametrize("rows, vocab, masked", [((1 << 28) + 40, 6, False), ((1 << 28) + 40, 6, True), ((1 << 24) + 40, 2064, False)])
def test_more_rows_than_a_launch_takes(rows, vocab, masked, memory_given_back):
    """Rows of 16 lanes (2^28 and more), and of 256 (2^24 and more): 2^32 threads and more."""
    logits = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    target = (torch.arange(rows, device="cuda") % 6).int()
    kw = dict(mask=torch.tensor([[63]], device="cuda"), mask_row=torch.zeros(rows, dtype=torch.int32, device="cuda")) if masked else {}
    logits[-1, 0] = 2.0
    target[-1] = 0
    logp = lkg.token_logp(logits, target, **kw)["logp"]
    share = math.exp(2) / (math.exp(2) + vocab - 1)
    assert abs(float(logp[:-1].min()) + math.log(vocab)) < 1e-5 and abs(float(logp[:-1].max()) + math.log(vocab)) < 1e-5 and abs(float(logp[-1]) - math.log(share)) < 1e-5
    if vocab < 10:  # (the gradient too)
        got = lkg.policy_loss(logits, target, torch.ones(rows, device="cuda"), gradient=True, **kw)
        assert torch.equal(got["logp"], logp) and abs(float(got["loss"]) / -rows - 1) < 1e-6
        one = got["dlogits"].abs().amax(1)  # of the target: 1 - its share
        assert float((one[:-1].float() - 5 / 6).abs().max()) < 0.01 and abs(float(one[-1]) - (1 - share)) < 0.01


@pytest.mark.parametrize("dtype, size", [(torch.float32, 1e4), (torch.float32, -1e5), (torch.float16, 3000.0), (torch.bfloat16, -400.0), (torch.float32, 65.0)])
@pytest.mark.parametrize("masks", [None, 3], ids=["open", "masked"])
@pytest.mark.parametrize("rows, vocab", [(100, 300)] + [(6, v) for v in KERNELS])
def test_rows_far_from_nothing(rows, vocab, masks, dtype, size):
    """Rows whose logits stand far from 0 keep the bits of those near it, in one pass and from lse.

    With b what an id is below its row's largest, in units of the exponent: its term is off by 2^-24 (4 b + 2), the sum by those and by up to
    250 additions and scalings in turn (1,024 threads with 195 terms each, 256 with 128, in steps of 16), its logarithm by four of its own last places, and
    logp by the four more of what it is."""
    a = _case(32, rows, vocab, dtype, scale=0.5)
    a["logits"] = (a["logits"].float() * 1.5 + size / 0.5).to(dtype)
    few = dict(scale=0.5)
    if masks:
        a |= {k: x for k, x in _case(32, rows, vocab, dtype, masks=masks).items() if k in ("mask", "mask_row")}
        few |= {k: a[k] for k in ("mask", "mask_row")}
    lp = oracle.policy(a["logits"], a["target"], **few)[0]["logp"]
    lp = torch.where(lp.isfinite(), lp, 0.0)
    g = torch.Generator().manual_seed(33)
    a["old"] = (lp - torch.randint(-8, 9, (rows,), generator=g) * 0.05 + 0.011).float()
    a["ref"] = (lp + torch.randn(rows, generator=g) * 0.3).float()
    res, _ = oracle.policy(**a)
    x = a["logits"].double() * 0.5
    if masks:
        bits = ((a["mask"][:, :, None] >> torch.arange(64)) & 1).reshape(masks, -1)[:, :vocab].bool()
        x = torch.where(bits[a["mask_row"].long()], x, -math.inf)
    top = x.amax(1, keepdim=True)
    b = torch.where(x == -math.inf, 0.0, top - x)
    p, logsum = torch.softmax(x, 1), torch.logsumexp(x - top, 1, keepdim=True)
    rest = oracle.E32 * (250 + 4 * (p * b).sum(1, keepdim=True) + 4 * logsum)
    said = b.gather(1, a["target"].long()[:, None])
    counts = res["logp"].isfinite()[:, None]
    lp, old, ref, A, w = (t.double()[:, None] for t in (lp, a["old"], a["ref"], a["advantage"], a["weight"]))
    lp_tol = rest + oracle.E32 * (4 * said + 4 * lp.abs())
    near = lp_tol + 4 * oracle.E32 * (1 + lp.abs() + old.abs() + ref.abs())
    steep = torch.exp(lp - old) * A.abs() + a["kl"] * torch.exp(ref - lp)
    slope_tol = 0.5 * w * steep * (1.1 * near + 8 * oracle.E32)
    hot = torch.zeros_like(p).scatter_(1, a["target"].long()[:, None], 1.0)
    slope = 0.5 * w * steep  # at most
    tol = slope_tol * (hot - p).abs() + 1.1 * slope * (p * (rest + 4 * oracle.E32 * (b + 1)) + hot * lp_tol * torch.exp(lp) + 4 * oracle.E32 * (hot - p).abs())
    tol = torch.where(counts, tol + oracle.UNIT[dtype] * (res["dlogits"].abs() + tol) + oracle.LEAST[dtype], 0.0)
    c = _gpu(a)
    got = lkg.policy_loss(**c, gradient=True)
    oracle.check(got["dlogits"], res["dlogits"], tol, "one pass")
    oracle.check(got["logp"], res["logp"], torch.where(counts, lp_tol, 0.0).squeeze(1), "logp")
    rest = {k: t for k, t in c.items() if k not in ("logits", "target", "advantage")}
    oracle.check(lkg.policy_loss_backward(torch.tensor(1.0, device="cuda"), c["logits"], c["target"], c["advantage"], got["lse"], **rest), res["dlogits"], tol, "backward")


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_NAMES)
@pytest.mark.parametrize("masks", [None, 3], ids=["open", "masked"])
@pytest.mark.parametrize("rows, vocab", [(9, 7), (100, 299), (100, 304)] + [(9, v) for v in KERNELS])
def test_gradients_in_place_of_the_logits(rows, vocab, masks, dtype):
    a = _case(34, rows, vocab, dtype, masks=masks)
    a["target"][[2, 5]] = torch.tensor([-1, vocab], dtype=torch.int32)
    a["logits"][3] += 200  # (its sum is made again by the backward)
    b = _gpu(a)
    want = lkg.policy_loss(**b, gradient=True)
    x = b["logits"].clone()
    loss, logp, lse = _raw("logoskg_policy_loss", b, x, logits=x)
    assert torch.equal(x, want["dlogits"]) and torch.equal(loss, want["loss"]) and torch.equal(logp, want["logp"]) and torch.equal(lse, want["lse"])
    rest = {k: t for k, t in b.items() if k not in ("logits", "target", "advantage")}
    dloss = torch.tensor(-1.5, device="cuda")
    back = lkg.policy_loss_backward(dloss, b["logits"], b["target"], b["advantage"], lse, **rest)
    x = b["logits"].clone()
    _raw("logoskg_policy_loss_backward", b, x, lse, dloss, logits=x)
    assert torch.equal(x, back)
    one = {k: t[3:4].clone() if k not in ("mask", "kl", "scale") else t for k, t in b.items()}  # of one row, whose stride does not matter
    x = one["logits"].clone()
    _raw("logoskg_policy_loss", one, x, logits=x)
    assert torch.equal(x, lkg.policy_loss(**one, gradient=True)["dlogits"])


def test_tangents_are_not_lost():
    a = _gpu(_case(35, 4, 30))
    with torch.autograd.forward_ad.dual_level():
        a["logits"] = torch.autograd.forward_ad.make_dual(a["logits"], torch.ones_like(a["logits"]))
        with pytest.raises(NotImplementedError, match="jvp"):
            lkg.policy_loss(**a)


def test_the_largest_scale():
    a = _gpu(dict(logits=torch.tensor([[1.0, 0.5, -2.0], [0.25, 0.25, 0.0]]), target=torch.tensor([0, 1], dtype=torch.int32), advantage=torch.ones(2), scale=2e38))
    got = lkg.policy_loss(**a, gradient=True)
    assert got["logp"][0] == 0 and abs(float(got["logp"][1]) + math.log(2)) < 1e-6
    assert got["dlogits"][0].tolist() == [0, 0, 0] and torch.allclose(got["dlogits"][1], torch.tensor([1e38, -1e38, 0.0], device="cuda"))
