"""A model writes on over a paged cache: logits of prompts in chunks and of single tokens against the oracle's logits of the whole texts."""
import os
import sys

import numpy as np
import pytest
import torch

import paper_2401_15207_amd as H
from hift_inputs import WORKLOADS, make_batch
from oracle import hift_oracle as O
from tests.hift_pair import make_pair, rel_l2, to_dev
from tests.test_gpu_step_fp32 import SMALL1, SMALL2, TIED0

pytestmark = pytest.mark.gpu
# heads 128 wide and sides that the packed-operand kernels take: rotation's block order, folded normalisation
WIDE = dict(WORKLOADS["C4"], n_layers=2, d_model=512, n_heads=4, d_ffn=1024, vocab=1000, max_seq=96, seq=96, batch=3)
MODELS = {"C1": WORKLOADS["C1"], "rope": SMALL2, "C1_tied": TIED0, "wide": WIDE}


def oracle_logits(orc, theta, tok):
    seen = {}

    def look(logits, rows):
        seen["x"] = logits
        return 0.0, np.zeros_like(logits)

    O.loss_and_grad(orc.cfg, theta, tok, np.full_like(tok, -1), objective=look)
    return seen["x"].reshape(*tok.shape, -1)


def cache_for(gpu, sequences, most, page=16, seed=0):
    c = gpu.cfg
    n = -(-most // page)
    shape = (c["n_layers"], sequences * n + 1, c["n_heads"], page, c["d_model"] // c["n_heads"])
    k, v = (torch.full(shape, float("nan"), device="cuda", dtype=torch.bfloat16 if c["dtype"] else torch.float32) for _ in range(2))
    pages = torch.randperm(sequences * n, generator=torch.Generator().manual_seed(seed)).to(torch.int32).view(sequences, n).cuda()
    return H.PagedCache(k, v, pages, torch.zeros(sequences, dtype=torch.int32, device="cuda"))


def write_on(gpu, tok, news, pick_last=False):
    """Feeds the texts tok [sequences, S] by `news` ([per call] tokens of each sequence); logits [sequences, S, V] (unfed or unpicked: nan)."""
    n, s = tok.shape
    cache = cache_for(gpu, n, s)
    out = torch.full((n, s, gpu.cfg["vocab"]), float("nan"))
    at = [0] * n
    for new in news:
        rows = torch.from_numpy(np.concatenate([tok[i, at[i]:at[i] + new[i]] for i in range(n)]).astype(np.int32)).cuda()
        starts = torch.tensor(np.cumsum([0] + list(new)), dtype=torch.int32, device="cuda")
        pick = (starts[1:] - 1).to(torch.int32) if pick_last else None
        got = gpu.extend(rows, starts, cache, max(new), max(a + b for a, b in zip(at, new)), pick=pick).float().cpu()
        row = 0
        for i in range(n):
            if pick_last:
                out[i, at[i] + new[i] - 1] = got[i]
            else:
                out[i, at[i]:at[i] + new[i]] = got[row:row + new[i]]
            row += new[i]
            at[i] += new[i]
        cache.lengths += torch.tensor(new, dtype=torch.int32, device="cuda")
    return out


def calls_of(n, s):
    """A ragged prompt, a chunk, then tokens one by one, one sequence pausing."""
    at = [s // 2 - i for i in range(n)]
    news = [list(at), [3 + i for i in range(n)]]
    at = [a + b for a, b in zip(at, news[1])]
    while max(s - a for a in at) > 0:
        new = [1 if a < s else 0 for a in at]
        if len(news) == 3:
            new[0] = 0
        news.append(new)
        at = [a + b for a, b in zip(at, new)]
    return news


@pytest.mark.parametrize("name", sorted(MODELS))
@pytest.mark.parametrize("unfused", [0, 7])
def test_fp32_against_the_oracle(name, unfused):
    wl = MODELS[name]
    orc, gpu, _ = make_pair(wl, seed=6, jitter=0.02, dtype=0, unfused=unfused)
    tok, _ = make_batch(wl, 6, 1)
    want = oracle_logits(orc, orc.theta, tok)
    got = write_on(gpu, tok, calls_of(*tok.shape)).numpy()
    # as the step's own parity tests: 1e-5 of the largest logit
    assert np.abs(got - want).max() <= 1e-5 * (np.abs(want).max() + 1)
    last = write_on(gpu, tok, calls_of(*tok.shape)[:1], pick_last=True).numpy()
    ends = calls_of(*tok.shape)[0]
    for i, e in enumerate(ends):
        assert np.abs(last[i, e - 1] - want[i, e - 1]).max() <= 1e-5 * (np.abs(want).max() + 1)


@pytest.mark.parametrize("name", ["rope", "wide", "C1"])
@pytest.mark.parametrize("how", [dict(), dict(unfused=7), dict(no_packed_copies=1), dict(master_on_host=1, state_on_host=1)])
def test_bf16_against_the_oracle(name, how):
    wl = MODELS[name]
    orc, gpu, _ = make_pair(wl, seed=7, jitter=0.02, dtype=1, **how)
    if (wl["d_model"] // wl["n_heads"]) % 8:
        pytest.skip("heads of no whole 16-byte pieces")
    tok, _ = make_batch(wl, 7, 1)
    want = oracle_logits(orc, orc.theta_half if hasattr(orc, "theta_half") else O.bf16_round(orc.theta), tok)
    got = write_on(gpu, tok, calls_of(*tok.shape)).numpy()
    # about 23 roundings to bf16 one after the other, 2^-8 / sqrt(3) each in the mean square, adding up like independent ones: 0.011; twice that
    assert rel_l2(got, want) <= 0.022


def test_adapters_answer():
    wl = MODELS["C1"]
    orc, _, theta = make_pair(wl, seed=8, jitter=0.02)
    gpu = H.HiftModel(dict(orc.cfg), wl["opt"], 1, wl["batch"], wl["seq"], init_params=theta, lora_rank=4, lora_alpha=8.0)
    lora = np.random.default_rng(1).normal(0, 0.05, gpu.lora_param_count()).astype(np.float32)
    gpu.lora_write(lora)
    tok, _ = make_batch(wl, 8, 1)
    want = oracle_logits(orc, O.lora_merge(orc.cfg, orc.theta, lora.astype(np.float64), 4, 8.0), tok)
    got = write_on(gpu, tok, calls_of(*tok.shape)).numpy()
    assert np.abs(got - want).max() <= 1e-5 * (np.abs(want).max() + 1)


def test_a_trained_model_answers_with_its_new_weights():
    """Prompts before and after a step, scores dropped by an extension, and training undisturbed by it."""
    wl = MODELS["rope"]
    orc, gpu, _ = make_pair(wl, seed=9, jitter=0.02, dtype=0)
    tok, lab = make_batch(wl, 9, 1)
    dtok, dlab = to_dev(tok, lab)
    for t in range(1, orc.k + 1):
        gid = orc.schedule_group_at(t)
        write_on(gpu, tok, [[tok.shape[1]] * tok.shape[0]])
        assert abs(gpu.step(dtok, dlab, gid) - orc.step(tok, lab, gid)) <= 1e-5 * 10
    want = oracle_logits(orc, orc.theta, tok)
    got = write_on(gpu, tok, calls_of(*tok.shape)).numpy()
    assert np.abs(got - want).max() <= 1e-4 * (np.abs(want).max() + 1)      # after updates the weights differ by the steps' own rounding
    gid = orc.schedule_group_at(1)
    gpu.score(dtok, dlab, gid)
    write_on(gpu, tok, [[1] * tok.shape[0]])
    with pytest.raises(H.HiftError):
        gpu.step_scored(dtok, dlab, gid, None, None)


def test_rows_of_no_sequence_and_refusals():
    wl = MODELS["C1"]
    orc, gpu, _ = make_pair(wl, seed=6, jitter=0.02)
    tok, _ = make_batch(wl, 6, 1)
    want = oracle_logits(orc, orc.theta, tok)
    cache = cache_for(gpu, 2, 32)
    rows = torch.from_numpy(np.concatenate([tok[0, :9], tok[1, :4], [0, 255, 7]]).astype(np.int32)).cuda()
    starts = torch.tensor([0, 9, 13], dtype=torch.int32, device="cuda")
    got = gpu.extend(rows, starts, cache, 9, 9).cpu().numpy()
    assert np.abs(got[:9] - want[0, :9]).max() <= 1e-5 * (np.abs(want).max() + 1)
    assert np.abs(got[9:13] - want[1, :4]).max() <= 1e-5 * (np.abs(want).max() + 1)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert gpu.extend(none, torch.zeros(3, dtype=torch.int32, device="cuda"), cache, 0, 0).shape == (0, 256)
    with pytest.raises(H.HiftError):
        gpu.extend(rows, starts, cache, 9, 33)          # beyond the position table
    with pytest.raises(H.HiftError):
        gpu.extend(rows.repeat(5), starts, cache, 9, 9)  # more rows than the model holds
    with pytest.raises(ValueError):
        gpu.extend(rows.long(), starts, cache, 9, 9)
    with pytest.raises(ValueError):
        gpu.extend(rows, starts[:2], cache, 9, 9)
    wrong = H.PagedCache(*(t.bfloat16() for t in cache.all), cache.pages, cache.lengths)
    with pytest.raises(H.HiftError):
        gpu.extend(rows, starts, wrong, 9, 9)
    with pytest.raises(ValueError):
        gpu.extend(rows, starts, H.PagedCache(cache.k, cache.v, cache.pages, cache.lengths), 9, 9)   # one layer
    _, enc, _ = make_pair(SMALL1, seed=1)
    hd = SMALL1["d_model"] // SMALL1["n_heads"]
    k = torch.zeros(SMALL1["n_layers"], 4, SMALL1["n_heads"], 16, hd, device="cuda")
    with pytest.raises(H.HiftError):
        enc.extend(rows, starts, H.PagedCache(k, k.clone(), cache.pages, cache.lengths), 9, 9)


def test_the_example_learns_from_its_own_answers():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import learn_from_own_answers as E
    rewards = E.run(workload="C1", batch=4, sweeps=1, prompt=6, answer=8, say=lambda *a, **k: None)
    assert len(rewards) == 4 and all(np.isfinite(r) and 0.0 <= r <= 1.0 for r in rewards)
