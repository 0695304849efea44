"""The definitions in around_oracle against plain torch on the CPU and against differences, and what the calls around the
reading refuse before they touch a GPU (no GPU needed)."""
import ctypes
import math

import pytest
import torch

import around_oracle as oracle
import paper_2604_18913_amd as lkg
from paper_2604_18913_amd import packed, reading, training
from test_reading_oracle import _status


def test_embedding_is_torch_s():
    g = torch.Generator().manual_seed(1)
    table = torch.randn(9, 5, generator=g, dtype=torch.float64).float().requires_grad_()
    ids, dout = torch.tensor([[3, 8, 3], [0, 3, 8]], dtype=torch.int32), torch.randn(2, 3, 5, generator=g)
    got = torch.nn.functional.embedding(ids.long(), table) * 1.5
    oracle.check(got, *oracle.embed(table, ids, 1.5))
    got.backward(dout)
    oracle.check(table.grad, *oracle.embed_grad(dout, ids, 9, 1.5))
    padded = torch.tensor([3, -1, 9, 2 ** 31 - 1, -2 ** 31, 0], dtype=torch.int32)
    want, _ = oracle.embed(table, padded)
    assert (want[1:5] == 0).all() and (want[0] != 0).any()
    old = torch.randn(9, 5, generator=g)
    want, tol = oracle.embed_grad(dout, ids, 9, 2.0, out=old)
    assert torch.equal(want[1], old[1].double()) and (tol[1] == 0).all() and (tol[3] > 0).all()


def _case(seed=2, rows=6, vocab=11, **kw):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    return dict(logits=r(rows, vocab).float(), target=torch.randint(0, vocab, (rows,), generator=g).int(), advantage=r(rows), old=-2 + r(rows) * 0.3,
                ref=-2 + r(rows) * 0.3, weight=r(rows).abs(), kl=0.1, scale=0.7, **kw)


@pytest.mark.parametrize("masked", [False, True])
def test_policy_gradient_is_that_of_differences_and_of_torch(masked):
    a = _case()
    if masked:
        a |= dict(mask=torch.tensor([[0b10111101111], [0b11111111111], [0]]), mask_row=torch.tensor([0, 1, 0, 2, 7, 1], dtype=torch.int32))
    res, _ = oracle.policy(**a)
    step, base = 2.0 ** -10, a["logits"].double()
    for r, v in [(0, 0), (0, 4), (1, 3), (2, int(a["target"][2])), (5, 10)]:
        up, down = base.clone(), base.clone()
        up[r, v] += step
        down[r, v] -= step
        two = [oracle.policy(**{**a, "logits": x.to(torch.float32)})[0]["loss"] for x in (up, down)]
        assert abs((two[0] - two[1]) / (2 * step) - res["dlogits"][r, v]) < 1e-3
    x = base.clone().requires_grad_()
    bits = None
    y = x * a["scale"]
    if masked:
        bits = ((a["mask"][a["mask_row"].long().clamp(max=2)][:, None, 0:1].squeeze(1) >> torch.arange(11)) & 1).bool()
        bits[4] = False
        y = torch.where(bits, y, -math.inf)
    lp = torch.log_softmax(y, 1).gather(1, a["target"].long()[:, None]).squeeze(1)
    counts = lp.isfinite()
    lp = torch.where(counts, lp, 0.0)
    ratio = torch.exp(lp - a["old"])
    row = -torch.minimum(ratio * a["advantage"], ratio.clamp(0.8, 1.2) * a["advantage"])
    d = a["ref"] - lp
    loss = (torch.where(counts, a["weight"], 0.0) * (row + a["kl"] * (torch.exp(d) - d - 1))).sum()
    loss.backward()
    assert torch.allclose(loss.detach(), res["loss"], rtol=1e-9)
    assert torch.allclose(x.grad.nan_to_num(0.0), res["dlogits"], atol=1e-12)


def test_policy_rows_that_do_not_count():
    a = _case(rows=4, vocab=8)
    a["target"] = torch.tensor([-1, 8, 3, 3], dtype=torch.int32)
    a["logits"][2, 3] = -math.inf
    a["mask"] = torch.tensor([[255], [255], [255], [255 - 8]])
    res, tol = oracle.policy(**a)
    assert res["logp"].tolist() == [0.0, 0.0, -math.inf, -math.inf] and res["loss"] == 0 and (res["dlogits"] == 0).all() and (tol["dlogits"] == 0).all()


def test_clip_is_torch_s():
    g = torch.Generator().manual_seed(3)
    grads = [torch.randn(s, generator=g) for s in [(3, 4), (7,), (), (0, 2)]]
    params = [torch.zeros_like(x).requires_grad_() for x in grads]
    for most in (0.5, 100.0):
        for p, x in zip(params, grads):
            p.grad = x.clone()
        norm = torch.nn.utils.clip_grad_norm_(params, most)
        want, tol, each = oracle.clip(grads, most)
        assert abs(norm - want) < 1e-5 * want
        for p, (x, t) in zip(params, each):
            assert torch.allclose(p.grad.double(), x, rtol=1e-5)


@pytest.mark.parametrize("kv_heads, dim", [(1, 8), (2, 32), (3, 40), (5, 96), (2, 128)])
def test_packed_rows_come_back(kv_heads, dim):
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn(6, kv_heads, dim, generator=g).to(torch.bfloat16) for _ in range(2))
    rows, _ = oracle.pack(k, v)
    x, s, b = oracle.unpack(rows, kv_heads, dim)
    assert rows.shape[1] % 16 == 0 and rows.shape[1] == packed.packed_row_bytes(kv_heads, dim) == lkg.packed_row_bytes(kv_heads, dim)
    for i, y in enumerate((k, v)):  # half a step, and what base and scale lose in bfloat16: 2^-8 of them, a range being 15 steps
        assert ((x[i] - y.double()).abs() <= s[i] * 0.5 + b[i].abs() * 2.0 ** -8 + s[i] * 15 * 2.0 ** -8).all()
    flat = torch.full((1, kv_heads, dim), 1.5).to(torch.bfloat16)
    assert torch.equal(oracle.unpack(oracle.pack(flat, flat)[0], kv_heads, dim)[0], flat.double().expand(2, -1, -1, -1))


def test_read_packed_is_the_reading_of_what_rows_stand_for():
    import reading_oracle
    g = torch.Generator().manual_seed(5)
    k, v, q = torch.randn(40, 2, 40, generator=g), torch.randn(40, 2, 40, generator=g), torch.randn(3, 2, 4, 40, generator=g).to(torch.bfloat16)
    rows, _ = oracle.pack(k, v)
    off, entity = torch.tensor([0, 7, 7, 30]), torch.randint(-1, 41, (30,), generator=g).int()
    x = oracle.unpack(rows, 2, 40)[0]
    kw = dict(cap=3.0, bias=torch.randn(4, 8, generator=g), buckets=lkg.distance_buckets(8, 6, device="cpu"), hop=torch.randint(0, 4, (30,), generator=g).to(torch.uint8))
    got, _ = oracle.read_packed(q, rows, off, entity, kv_heads=2, **kw)
    want, _ = reading_oracle.read(q, x[0], x[1], off, entity, **kw)
    for name in want:
        assert torch.allclose(got[name], want[name], atol=1e-12), name


# ---------------------------------------------------------------- refusals
def test_struct_sizes_match_the_header():
    assert [ctypes.sizeof(s) for s in (training._Embedding, training._EmbeddingGrad, training._Policy, training._Gradient, packed._Pack)] == [80, 104, 168, 32, 104]


def test_cpu_tensors_are_refused():
    ids, x = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 8)
    for call in (lambda: lkg.embed_entities(x, ids), lambda: lkg.embed_entities_backward(x, ids, 4), lambda: lkg.token_logp(x, ids),
                 lambda: lkg.policy_loss(x, ids, x[:, 0]), lambda: lkg.policy_loss_backward(x[0, 0], x, ids, x[:, 0], x[:, 0]), lambda: lkg.clip_gradients([x], 1.0),
                 lambda: lkg.pack_entities(x[None], x[None]), lambda: lkg.unpack_entities(x.byte(), 1, 8, dtype=torch.float32),
                 lambda: lkg.read_packed(x[None, None], x.byte(), ids.long(), kv_heads=2)):
        with pytest.raises(ValueError, match="on the GPU"):
            call()


@pytest.mark.parametrize("wrong, says", [
    (dict(struct_size=1), "struct_size"), (dict(dtype=3), "type"), (dict(scale=math.nan), "scale"), (dict(scale=math.inf), "scale"),
    (dict(num_ids=-1), "count"), (dict(dim=-1), "count"), (dict(row=-8), "count"), (dict(ids=None), "NULL"), (dict(out=None), "NULL"), (dict(table=None), "NULL"),
    (dict(table=65), "aligned")])
def test_embedding_refusals(wrong, says):
    base = dict(struct_size=80, dtype=1, scale=1.0, num_ids=3, num_entities=4, dim=8, row=8, ids=64, table=64, out=64)
    rc, text = _status("logoskg_embed_entities", training._Embedding(**{**base, **wrong}))
    assert rc == 1 and says in text and text.startswith("logoskg_embed_entities")


@pytest.mark.parametrize("wrong, rc, says", [
    (dict(struct_size=1), 1, "struct_size"), (dict(dtype=-1), 1, "type"), (dict(table_dtype=2), 1, "dtable"), (dict(scale=math.nan), 1, "scale"),
    (dict(num_ids=1 << 31), 1, "count"), (dict(num_entities=(1 << 31) - 1), 1, "count"), (dict(row=7), 1, "overlap"), (dict(ids=None), 1, "NULL"),
    (dict(dout=None), 1, "NULL"), (dict(dtable=None), 1, "NULL"), (dict(workspace=72), 1, "aligned"), (dict(workspace_bytes=8), 4, "workspace"),
    (dict(workspace=None), 4, "workspace"), (dict(dout=65), 1, "aligned"), (dict(dtable=65), 1, "aligned")])
def test_embedding_gradient_refusals(wrong, rc, says):
    base = dict(struct_size=104, dtype=1, table_dtype=1, scale=1.0, num_ids=3, num_entities=4, dim=8, row=8, ids=64, dout=64, dtable=64, workspace=64, workspace_bytes=1 << 20)
    e = training._EmbeddingGrad(**{**base, **wrong})
    got, text = _status("logoskg_embed_entities_backward", e)
    assert got == rc and says in text, text
    nbytes = reading._load().logoskg_embed_entities_backward_bytes(ctypes.addressof(e))
    assert (nbytes == -1) == (rc == 1)


_POLICY = dict(struct_size=168, dtype=0, num_rows=2, vocab=10, row=10, logits=64, target=64, scale=1.0, kl=0.1, clip_low=0.2, clip_high=0.2, advantage=64, ref=64,
               logp=64, lse=64, loss=64, dlogits=64)


@pytest.mark.parametrize("wrong, rc, says", [
    (dict(struct_size=0), 1, "struct_size"), (dict(dtype=9), 1, "type"), (dict(vocab=1 << 30, row=1 << 30), 1, "count"), (dict(num_rows=-1), 1, "count"), (dict(vocab=1 << 31), 1, "count"), (dict(num_masks=-1), 1, "count"),
    (dict(row=9), 1, "overlap"), (dict(logits=None), 1, "NULL"), (dict(target=None), 1, "NULL"), (dict(lse=None), 1, "NULL"), (dict(mask=64, num_masks=1), 1, "fewer masks"),
    (dict(scale=0.0), 1, "scale"), (dict(scale=-1.0), 1, "scale"), (dict(scale=math.inf), 1, "scale"), (dict(scale=math.nan), 1, "scale"), (dict(logits=66), 1, "aligned"),
    (dict(kl=-0.1), 1, "kl"), (dict(kl=math.nan), 1, "kl"), (dict(clip_low=-1.0), 1, "clip"), (dict(clip_high=math.nan), 1, "clip"), (dict(advantage=None), 1, "advantage"),
    (dict(ref=None), 1, "ref"), (dict(loss=None), 1, "loss"), (dict(logp=None), 1, "logp"), (dict(row=12, dlogits=64), 1, "in place")])
def test_policy_refusals(wrong, rc, says):
    got, text = _status("logoskg_policy_loss", training._Policy(**{**_POLICY, **wrong}))
    assert got == rc and says in text and text.startswith("logoskg_policy_loss"), text


def test_further_policy_refusals():
    for wrong, says in [(dict(dlogits=None), "dlogits"), (dict(lse=None), "NULL"), (dict(scale=0.0), "scale")]:
        rc, text = _status("logoskg_policy_loss_backward", training._Policy(**{**_POLICY, **wrong}))
        assert rc == 1 and says in text
    rc, text = _status("logoskg_token_logp", training._Policy(**{**_POLICY, "logp": None}))
    assert rc == 1 and "logp" in text
    x = torch.zeros(2, 3)
    with pytest.raises(ValueError, match="mask_row without"):
        training._answers(_Fake(x), torch.zeros(2, dtype=torch.int32), None, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="kl without ref"):
        training._terms(x[:, 0], None, None, None, (0.2, 0.2), 0.1, 1.0, 2, 0)


@pytest.mark.parametrize("call", ["logoskg_token_logp", "logoskg_policy_loss", "logoskg_policy_loss_backward"])
def test_policy_rows_whose_numbers_leave_32_bits_are_refused(call):
    for rows in (2 ** 31 - 1, 2 ** 31 - 2 ** 16):
        rc, text = _status(call, training._Policy(**{**_POLICY, "num_rows": rows, "vocab": 1, "row": 1}))
        assert rc == 1 and "count" in text, text


class _Fake:
    """A tensor that says it is on the GPU."""

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 0


def _gradients(*entries):
    return b"".join(training._gradient_of(*e) for e in entries)


@pytest.mark.parametrize("entries, kw, rc, says", [
    ([(64, 64, -1, 0, 0)], {}, 1, "count"), ([(64, 64, 4, 3, 0)], {}, 1, "type"), ([(0, 64, 4, 0, 0)], {}, 1, "NULL"), ([(64, 0, 4, 0, 0)], {}, 1, "NULL"),
    ([(66, 66, 4, 0, 0)], {}, 1, "aligned"), ([(64, 64, 4, 0, 0)], dict(max_norm=-1.0), 1, "max_norm"), ([(64, 64, 4, 0, 0)], dict(max_norm=math.nan), 1, "max_norm"),
    ([(64, 64, 4, 0, 0)], dict(scale=math.inf), 1, "scale"), ([(64, 64, 4, 0, 0)], dict(norm=None), 1, "norm"), ([(64, 64, 4, 0, 0)], dict(nbytes=8), 4, "workspace"),
    # the same tensor twice, one inside another, one that is written and read as another, itself in another type
    ([(64, 64, 4, 0, 0), (64, 64, 4, 0, 0)], {}, 1, "share"), ([(64, 64, 4, 0, 0), (72, 72, 1, 0, 0)], {}, 1, "share"),
    ([(64, 640, 4, 0, 0), (640, 1280, 4, 0, 0)], {}, 1, "share"), ([(64, 64, 4, 1, 0)], {}, 1, "share"), ([(64, 68, 4, 0, 0)], {}, 1, "share"),
])
def test_clip_refusals(entries, kw, rc, says):
    lib, data = reading._load(), _gradients(*entries)
    got = lib.logoskg_clip_gradients(0, data, len(entries), kw.get("max_norm", 1.0), kw.get("scale", 1.0), kw.get("norm", 4096), 8192, kw.get("nbytes", 1 << 20), None)
    text = lib.logoskg_last_error().decode()
    assert got == rc and says in text, text


def test_clip_gradients_that_are_read_twice_are_fine():
    # (two gradients of one tensor, each to its own place, share what is read alone: refused for another reason here, the workspace)
    lib = reading._load()
    data = _gradients((64, 6400, 4, 0, 0), (64, 12800, 4, 0, 0), (64, 64, 0, 0, 0))
    assert lib.logoskg_clip_gradients(0, data, 3, 1.0, 1.0, 4096, 8192, 0, None) == 4
    with pytest.raises(ValueError, match="no gradients"):
        lkg.clip_gradients([None], 1.0)
    with pytest.raises(ValueError, match="outputs"):
        lkg.clip_gradients([None], 1.0, out=[])


@pytest.mark.parametrize("wrong, says", [
    (dict(struct_size=1), "struct_size"), (dict(dtype=3), "type"), (dict(dim=12), "dim"), (dict(dim=136), "dim"), (dict(dim=0), "dim"), (dict(kv_heads=0), "dim"),
    (dict(num_rows=-1), "count"), (dict(keys=None), "NULL"), (dict(packed=None), "NULL"), (dict(key_row=-1), "negative"), (dict(packed=72), "aligned"),
    (dict(packed_row=72), "aligned"), (dict(packed_row=64), "overlap"), (dict(keys=65), "aligned to"), (dict(values=65), "aligned to")])
def test_pack_refusals(wrong, says):
    base = dict(struct_size=104, dtype=1, kv_heads=2, dim=64, num_rows=3, keys=64, values=64, key_row=128, key_head=64, value_row=128, value_head=64, packed=64, packed_row=160)
    for call in ("logoskg_pack_entities", "logoskg_unpack_entities"):
        rc, text = _status(call, packed._Pack(**{**base, **wrong}))
        assert rc == 1 and says in text and text.startswith(call), text
    for heads, dim in ((0, 64), (1, 0), (1, 12), (1, 136), (-3, 64)):
        assert reading._load().logoskg_packed_row_bytes(heads, dim) == 0
    with pytest.raises(ValueError, match="multiple of 8"):
        lkg.packed_row_bytes(2, 12)


@pytest.mark.parametrize("wrong, rc, says", [
    (dict(struct_size=1), 1, "struct_size"), (dict(dtype=0), 1, "type"), (dict(dim=12), 1, "dim"), (dict(tokens=0), 1, "count"), (dict(num_entries=-1), 1, "count"), (dict(off=None), 1, "NULL"),
    (dict(keys=None), 1, "NULL"), (dict(values=64), 1, "packed"), (dict(key_head=8), 1, "packed"), (dict(entity=None, num_entities=3), 1, "fewer rows"), (dict(key_row=312), 1, "stride"),
    (dict(key_row=160), 1, "stride"), (dict(q=72), 1, "aligned"), (dict(num_entities=1 << 31), 1, "num_entities"), (dict(num_entries=100_000, num_queries=3), 4, "workspace"),
    (dict(score=reading._Score(1.0, -1.0, None, None, 0, 0)), 1, "cap")])
def test_read_packed_refusals(wrong, rc, says):
    base = dict(struct_size=208, dtype=2, num_queries=1, tokens=1, heads=4, kv_heads=4, dim=64, num_entries=9, num_entities=9, off=64, entity=64, q=64, keys=64,
                key_row=320, out=64, lse=64, score=reading._Score(1.0, 0.0, None, None, 0, 0))
    e = reading._EntityRead(**{**base, **wrong})
    got, text = _status("logoskg_read_packed", e)
    assert got == rc and says in text, text
    assert (reading._load().logoskg_read_packed_bytes(ctypes.addressof(e)) == -1) == (rc == 1)


@pytest.mark.parametrize("name", ["advantage", "old", "ref", "weight"])
def test_gradients_that_the_policy_loss_does_not_have_are_refused(name):
    x = torch.zeros(2, 8)
    kw = dict(advantage=torch.zeros(2), old=torch.zeros(2), ref=torch.zeros(2), weight=torch.zeros(2))
    kw[name].requires_grad_()
    call = lambda **more: lkg.policy_loss(x, torch.zeros(2, dtype=torch.int32), kl=0.1, **kw, **more)
    with pytest.raises(ValueError, match=f"{name} requires a gradient"):
        call()
    for more in (torch.no_grad, torch.inference_mode):  # (nothing is asked for: refused for another reason)
        with more(), pytest.raises(ValueError, match="on the GPU"):
            call()
    with pytest.raises(ValueError, match="on the GPU"):
        call(gradient=True)
    kw[name] = torch.zeros(2)
    with torch.autograd.forward_ad.dual_level():
        kw[name] = torch.autograd.forward_ad.make_dual(kw[name], torch.ones(2))
        with pytest.raises(ValueError, match=f"{name} requires a gradient"):
            call()


@pytest.mark.parametrize("call", ["logoskg_token_logp", "logoskg_policy_loss", "logoskg_policy_loss_backward"])
def test_policy_scales_that_leave_32_bits_as_exponents_are_refused(call):
    rc, text = _status(call, training._Policy(**{**_POLICY, "scale": 3e38}))
    assert rc == 1 and "scale is above" in text, text
