"""A decoder that learns from scored answers, one group of layers a step, with orthogonalised updates.

Every step scores a batch (log probability of each answer token, entropy of each position, the model's own first choices), turns the scores and
a reward into derivatives on the device, and takes a HiFT step on them with the Muon optimizer: policy gradient with an entropy bonus, where the
tokens that the rule below calls good are rewarded against the batch's mean.  Needs an MI355X; tokens and weights are synthetic.

    python examples/learn_from_scores.py [--workload C1] [--batch 16] [--sweeps 30] [--dtype bf16]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np  # noqa: E402


def reward_of(tokens, vocab):
    """The rule to learn: an even token is followed by one of the lower half of the vocabulary, an odd one by one of the upper half."""
    import torch
    after = torch.roll(tokens, -1, 1)
    return torch.where((after < vocab // 2) == (tokens % 2 == 0), 1.0, 0.0)


def run(workload="C1", batch=16, sweeps=30, dtype="fp32", lr=5e-3, entropy_bonus=0.01, say=print):
    """Mean probability that the model's first choice follows the rule: before and after training."""
    import torch

    import paper_2401_15207_amd as H
    from hift_inputs import WORKLOADS, init_params, model_config, next_token_labels, uniform_tokens
    wl = WORKLOADS[workload]
    cfg = model_config(wl, dtype=1 if dtype == "bf16" else 0)
    opt = dict(kind="muon", lr=lr, momentum=0.9, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0)
    spec = [(name, shape, kind) for name, shape, kind, _unit, _offset in H.tensor_list(cfg)[0]]
    model = H.HiftModel(cfg, opt, wl["m"], batch, wl["seq"], init_params=init_params(0, spec, bf16_exact=dtype == "bf16"), state_on_host=1)
    groups = model.set_group_schedule("bottom2up", wl["m"])

    def data(step):
        tokens = uniform_tokens(1, step, batch, wl["seq"], cfg["vocab"])
        targets = next_token_labels(tokens)
        return torch.from_numpy(tokens).cuda(), torch.from_numpy(np.ascontiguousarray(targets)).cuda()

    def share():
        tokens, targets = data(10 ** 6)
        first = model.score(tokens, targets, top=1)["top_ids"][..., 0]
        return ((first < cfg["vocab"] // 2) == (tokens % 2 == 0)).float().mean().item()

    before = share()
    for step in range(1, sweeps * groups + 1):
        group = model.schedule_group_at(step)
        tokens, targets = data(step)
        scores = model.score(tokens, targets, group)
        has = (targets >= 0).float()
        count = has.sum()
        reward = reward_of(tokens, cfg["vocab"])
        advantage = (reward - (reward * has).sum() / count) * has
        # objective to descend: -(advantage logp + bonus entropy) per position with a target
        model.step_scored(tokens, targets, group, (-advantage / count).contiguous(), (-entropy_bonus * has / count).contiguous())
        if step % (5 * groups) == 0:
            say(f"sweep {step // groups}: mean log probability {(scores['logp'].sum() / count).item():.3f}, mean entropy "
                f"{(scores['entropy'] * has).sum().item() / count.item():.3f}, first choice follows the rule in {100 * share():.1f} %", flush=True)
    after = share()
    model.close()
    return before, after


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workload", default="C1")
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--sweeps", type=int, default=30)
    ap.add_argument("--dtype", choices=("fp32", "bf16"), default="fp32")
    ap.add_argument("--lr", type=float, default=5e-3)
    a = ap.parse_args()
    before, after = run(a.workload, a.batch, a.sweeps, a.dtype, a.lr)
    print(f"first choice follows the rule: {100 * before:.1f} % before, {100 * after:.1f} % after")
