"""Attention over a paged cache with more sequences than a workgroup has threads, and a bf16 model with adapters that writes on over one."""
import numpy as np
import pytest
import torch

import paper_2401_15207_amd as H
from hift_inputs import make_batch
from oracle import hift_oracle as O
from tests.hift_pair import make_pair, rel_l2
from tests.test_gpu_extend import calls_of, oracle_logits, write_on
from tests.test_gpu_paged import Made
from tests.test_gpu_step_fp32 import SMALL2

pytestmark = pytest.mark.gpu


def lengths(n, most, turn=7):
    return [i * turn % most for i in range(n)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("window", [0, 100])
def test_a_token_each_of_more_sequences_than_threads(dtype, window):
    """Runs over more than 256 entries: each thread of the search sums several, some of them empty."""
    tokens = [(c, 0 if i % 11 == 3 else 1) for i, c in enumerate(lengths(299, 90))]
    tokens.insert(140, (1300, 1))
    tokens.append((900, 1))
    m = Made(tokens, 2, 1, 64, 16, dtype, seed=5, more_rows=1)
    out, lse = m.attend(window=window)
    m.check(out, lse, window=window)
    again, lse2 = m.attend(window=window)
    assert torch.equal(again, out) and torch.equal(lse2, lse)


def test_several_blocks_of_rows_of_many_sequences():
    """fp32, two blocks of 32 rows a sequence: over 256 entries as well."""
    tokens = [(c, 1 + i % 8) for i, c in enumerate(lengths(139, 60))]
    tokens.insert(70, (1500, 8))
    m = Made(tokens, 8, 1, 32, 16, "fp32", seed=6)
    out, lse = m.attend()
    m.check(out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_chunks_of_more_sequences_than_threads(dtype):
    """The kernel of many rows takes them in the order that they have; sequences of few rows and of none among them."""
    tokens = [(c, (0, 1, 20, 36, 70)[i % 5]) for i, c in enumerate(lengths(280, 50))]
    m = Made(tokens, 4, 2, 16, 16, dtype, seed=7, more_rows=1)
    out, lse = m.attend()
    m.check(out, lse)


def test_adapters_answer_in_bf16():
    wl = SMALL2
    orc, _, theta = make_pair(wl, seed=8, jitter=0.02, dtype=1)
    gpu = H.HiftModel(dict(orc.cfg), wl["opt"], 1, wl["batch"], wl["seq"], init_params=theta, lora_rank=8, lora_alpha=8.0)
    lora = np.random.default_rng(1).normal(0, 0.05, gpu.lora_param_count()).astype(np.float32)
    gpu.lora_write(lora)
    tok, _ = make_batch(wl, 8, 1)
    merged = O.lora_merge(orc.cfg, O.bf16_round(orc.theta), O.bf16_round(lora.astype(np.float64)), 8, 8.0)
    want = oracle_logits(orc, merged, tok)
    got = write_on(gpu, tok, calls_of(*tok.shape)).numpy()
    # about 23 roundings to bf16 one after the other and three in each of the two layers more (low-rank product, its part of q or v, their sum), 2^-8 / sqrt(3) each in the
    # mean square, adding up like independent ones: 0.0122; twice that
    assert rel_l2(got, want) <= 0.0243
