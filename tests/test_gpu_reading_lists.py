"""Logits under lists of biases that fill whole pieces of a row (the definition: reading_oracle)."""
import pytest
import torch

import paper_2604_18913_amd as lkg
from test_gpu_reading import HALVES, _check_logits, _gpu, _logit_case

pytestmark = pytest.mark.gpu


def _dense(seed, dtype, vocab, lengths, history):
    """Ids of the whole row in any order, some twice, some none."""
    a = _logit_case(seed, dtype, len(lengths), vocab, history, 3)
    g = torch.Generator().manual_seed(seed)
    n = sum(lengths)
    return {**a, "bias_off": torch.tensor([0] + lengths).cumsum(0), "bias_id": torch.randint(-2, vocab + 2, (n,), generator=g, dtype=torch.int32),
            "bias_value": torch.randn(n, generator=g) * 5}


@pytest.mark.parametrize("dtype", [torch.float32, *HALVES], ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("vocab, lengths", [(1000, [4000, 513, 511, 0]), (9001, [30_000, 9001, 100]), (4096, [5000, 600])])
def test_logits_with_biases_on_all_ids(vocab, lengths, dtype):
    _check_logits(_dense(51, dtype, vocab, lengths, 700))
    a = _dense(52, dtype, vocab, lengths, 0)
    _check_logits({k: x for k, x in a.items() if k not in ("history", "history_off", "repetition", "presence", "frequency", "mask")})


def test_logits_with_biases_on_all_ids_after_a_history_beyond_16_bits():
    a = _dense(53, torch.float32, 9001, [20_000, 3000, 20_000], 5)
    g = torch.Generator().manual_seed(53)
    said = torch.tensor([0, 1, 2, 1023, 1024, 2047, 2048, 4095, 4096, 4097, 8000, 9000])
    long = said[torch.randint(0, 12, (70_000,), generator=g)].int()
    a |= dict(history=torch.cat([long, a["history"][:3], long[:66_000]]), frequency=torch.full((3,), 2.0 ** -10))
    a["history_off"] = torch.tensor([0, 70_000, a["history"].numel() - 66_000, a["history"].numel()])
    _check_logits(a)


def test_logits_with_biases_on_all_ids_in_place_and_out_of_line():
    a = {k: _gpu(x) for k, x in _dense(54, torch.bfloat16, 5001, [7000, 3000], 50).items()}
    want = lkg.constrain_logits(**a)
    room = torch.full((2 * 5001 + 8,), 3.0, dtype=torch.bfloat16, device="cuda")
    assert torch.equal(lkg.constrain_logits(**a, out=room[3:3 + 2 * 5001].view(2, 5001)), want)
    assert torch.equal(lkg.constrain_logits(**a, out=a["logits"]), want)


def test_a_bias_on_every_id_takes_no_search_per_id():
    # 1 ms where a list is gone through once per 1,024 ids; a search through it for every id took 320
    rows, vocab = 16, 150_001
    ids = torch.cat([torch.randperm(vocab, device="cuda", dtype=torch.int32) for _ in range(rows)])
    a = dict(logits=torch.zeros(rows, vocab, device="cuda"), bias_off=torch.arange(rows + 1, device="cuda") * vocab, bias_id=ids,
             bias_value=torch.arange(rows * vocab, device="cuda").float())
    got = lkg.constrain_logits(**a)
    assert torch.equal(got, torch.zeros_like(got).scatter_(1, ids.view(rows, vocab).long(), a["bias_value"].view(rows, vocab)))
    first, last = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    first.record()
    lkg.constrain_logits(**a)
    last.record()
    last.synchronize()
    assert first.elapsed_time(last) < 40
