"""What hift_extend says of rows that belong to no sequence."""
import numpy as np
import pytest
import torch

import paper_2401_15207_amd as H
from hift_inputs import WORKLOADS, make_batch
from tests.hift_pair import make_pair, rel_l2
from tests.test_gpu_extend import cache_for, write_on
from tests.test_gpu_step_fp32 import SMALL2

pytestmark = pytest.mark.gpu


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
