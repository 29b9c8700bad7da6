"""What hift_extend says of rows that belong to no sequence, of chunks without logits, and of how often it rounds."""
import numpy as np
import pytest
import torch

import paper_2401_15207_amd as H
from hift_inputs import WORKLOADS, make_batch
from oracle import hift_oracle as O
from tests.hift_pair import make_pair, rel_l2
from tests.test_gpu_extend import cache_for, oracle_logits, write_on
from tests.test_gpu_step_fp32 import SMALL2

pytestmark = pytest.mark.gpu
# as many rows as the packed-operand kernels want, so that weights have no other copy: the projection's kernel turns q and k by itself
PACKED = dict(WORKLOADS["C4"], n_layers=2, d_model=512, n_heads=4, d_ffn=1024, vocab=1000, max_seq=96, seq=96, batch=134)


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("name", ["C1", "rope"])
@pytest.mark.parametrize("dtype", [0, 1])
def test_logits_of_rows_of_no_sequence_are_zero(name, dtype):
    """Before, between and behind the sequences' rows, and beyond max_new; whatever ran before, picked or not."""
    wl = dict(C1=WORKLOADS["C1"], rope=SMALL2)[name]
    _, gpu, _ = make_pair(wl, seed=6, jitter=0.02, dtype=dtype)
    tok, _ = make_batch(wl, 6, 1)
    write_on(gpu, tok, [[tok.shape[1]] * tok.shape[0]])      # leaves activations of another batch in every row
    rows = torch.from_numpy(np.concatenate([[3, 9], tok[0, :9], tok[1, :4], [0, 7, 1]]).astype(np.int32)).cuda()
    starts = ints(2, 11, 15)
    alone = gpu.extend(rows[2:15].contiguous(), ints(0, 9, 13), cache_for(gpu, 2, 32), 9, 9)
    got = gpu.extend(rows, starts, cache_for(gpu, 2, 32), 9, 9)
    assert (got[:2] == 0).all() and (got[15:] == 0).all()
    # other tiles of rows in the contractions: sums of the same numbers in another order
    assert rel_l2(got[2:15].float().cpu().numpy(), alone.float().cpu().numpy()) <= (0.022 if dtype else 1e-5)
    few = gpu.extend(rows, starts, cache_for(gpu, 2, 32), 3, 9)
    stray = torch.ones(18, dtype=torch.bool, device="cuda")
    stray[[2, 3, 4, 11, 12, 13]] = False
    assert (few[stray] == 0).all() and (few[~stray] != 0).any(1).all()
    assert torch.equal(few[~stray], gpu.extend(rows, starts, cache_for(gpu, 2, 32), 3, 9)[~stray])
    picked = gpu.extend(rows, starts, cache_for(gpu, 2, 32), 9, 9, pick=ints(17, 2, 0, 14, 2, -5, 99))
    assert (picked[[0, 2, 5, 6]] == 0).all() and torch.equal(picked[1], picked[4])
    assert rel_l2(picked[[1, 3]].float().cpu().numpy(), got[[2, 14]].float().cpu().numpy()) <= (0.022 if dtype else 1e-5)
    assert (gpu.extend(rows, starts, cache_for(gpu, 2, 32), 0, 9) == 0).all()


@pytest.mark.parametrize("name", ["C1", "rope"])
def test_rows_without_any_sequence(name):
    wl = dict(C1=WORKLOADS["C1"], rope=SMALL2)[name]
    _, gpu, _ = make_pair(wl, seed=6, jitter=0.02)
    whole = cache_for(gpu, 2, 32)
    none = H.PagedCache(*whole.all, torch.empty(0, 2, dtype=torch.int32, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"))
    assert (gpu.extend(ints(5, 6, 7), ints(0), none, 3, 9) == 0).all()


@pytest.mark.parametrize("name", ["C1", "rope"])
def test_a_chunk_without_logits(name):
    """All chunks of a prompt but the last: nobody wants their logits."""
    wl = dict(C1=WORKLOADS["C1"], rope=SMALL2)[name]
    orc, gpu, _ = make_pair(wl, seed=6, jitter=0.02)
    tok, _ = make_batch(wl, 6, 1)
    want = oracle_logits(orc, orc.theta, tok)
    cache = cache_for(gpu, 1, 32)
    a, b = (torch.from_numpy(tok[0, i:j].astype(np.int32)).cuda() for i, j in ((0, 9), (9, 14)))
    assert gpu.extend(a, ints(0, 9), cache, 9, 9, pick=ints()).shape == (0, wl["vocab"])
    cache.lengths += 9
    got = gpu.extend(b, ints(0, 5), cache, 5, 14).cpu().numpy()
    assert np.abs(got - want[0, 9:14]).max() <= 1e-5 * (np.abs(want).max() + 1)


def test_keys_are_rounded_once():
    """bf16, where the projection's kernel rotates: a cached key is off by one rounding of the rotated sum, as in the model's own forward pass."""
    _, gpu, theta = make_pair(PACKED, seed=7, dtype=1)
    c = gpu.cfg
    d, heads, hd = c["d_model"], c["n_heads"], 128
    tok, _ = make_batch(PACKED, 7, 1)
    tok = tok[:3]
    spec = {n: (o, s) for n, s, _k, _u, o in H.tensor_list(c)[0]}
    take = lambda n: theta[spec[n][0]:spec[n][0] + int(np.prod(spec[n][1]))].reshape(spec[n][1]).astype(np.float64)
    gain = [n for n in spec if n.endswith(".g1")][0]
    assert (take(gain) == 1.0).all()
    x = take("tok_emb")[tok[:, :40]]
    rstd = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + c["norm_eps"])
    w = take(gain[:-2] + "wqkv")[d:2 * d]
    raw, size = (x * rstd) @ w.T, np.abs(x * rstd) @ np.abs(w.T)
    raw, size = raw.reshape(3, 40, heads, hd), size.reshape(3, 40, heads, hd)
    angle = np.arange(40)[:, None] * c["rope_base"] ** (-np.arange(0, hd, 2) / hd)
    cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]
    a, b, sa, sb = raw[..., :64], raw[..., 64:], size[..., :64], size[..., 64:]
    want = np.concatenate([a * cos - b * sin, b * cos + a * sin], -1)
    # sums of d products and of d squares in 32 bits, a few operations more; then one rounding
    slack = np.concatenate([sa * abs(cos) + sb * abs(sin), sb * abs(cos) + sa * abs(sin)], -1) * (2 * d + 16) * 2.0 ** -24
    cache = cache_for(gpu, 3, 96)
    at = [0, 0, 0]
    for news in ([30, 2, 11], [10, 1, 0], [0, 37, 29]):
        rows = np.concatenate([tok[i, at[i]:at[i] + news[i]] for i in range(3)]).astype(np.int32)
        gpu.extend(torch.from_numpy(rows).cuda(), ints(*np.cumsum([0] + news)), cache, max(news), 96)
        cache.lengths += ints(*news)
        at = [p + n for p, n in zip(at, news)]
    assert at == [40, 40, 40]
    k = cache.all[0][0]      # layer 0
    got = np.stack([k[cache.pages[s].long()].transpose(1, 2).reshape(-1, heads, hd)[:40].double().cpu().numpy() for s in range(3)])
    far = np.abs(got - want) / (2.0 ** -8 * np.abs(want) + 1.01 * slack)
    assert far.max() <= 1.0, f"off by up to {far.max():.2f} of one rounding"


@pytest.mark.parametrize("how", [dict(), dict(master_on_host=1, state_on_host=1), dict(unfused=1)])
def test_packed_weights_against_the_oracle(how):
    """With packed copies alone; with row-major ones beside them, which few rows take and the rotation is the cache's; and with the rotation apart."""
    orc, gpu, _ = make_pair(PACKED, seed=7, jitter=0.02, dtype=1, **how)
    tok, _ = make_batch(PACKED, 7, 1)
    tok = tok[:3]
    want = oracle_logits(orc, O.bf16_round(orc.theta), tok)
    got = write_on(gpu, tok, [[50, 49, 48], [3, 4, 5], [1, 1, 1], [0, 1, 1], [42, 41, 41]]).numpy()
    # about 23 roundings to bf16 one after the other, 2^-8 / sqrt(3) each in the mean square, adding up like independent ones: 0.011; twice that
    assert rel_l2(got, want) <= 0.022
