"""A decoder that writes answers and learns from them: policy gradient from its own samples, one group of layers a step.

Every step the model continues prompts token by token over a paged cache (HiftModel.extend): the logits of each next token pass through the penalties for repeated
tokens and a mask of allowed ones (kernel_adjust_logits), the most probable alternatives and their log probabilities come from kernel_token_logprob, and one of
them is drawn.  The answers are then scored in one pass over the whole texts, at the temperature they were drawn at, and the HiFT step is taken on the derivatives
that their reward gives.  The gradient is that of the model's own distribution at this temperature: that answers were drawn with a penalty for repeated tokens, from
allowed ones alone and among the most probable, it leaves out.  Needs an MI355X; prompts and weights are synthetic.

    python examples/learn_from_own_answers.py [--workload C1] [--batch 16] [--sweeps 10] [--dtype fp32]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

TOP, PAGE, TEMPERATURE = 16, 16, 0.9


def answers(H, model, prompts, answer, allowed, temperature=TEMPERATURE, repetition=1.1):
    """Continues prompts [batch, length] (int32) by `answer` tokens each: the texts [batch, length + answer]."""
    import torch
    batch, length = prompts.shape
    c, dev = model.cfg, prompts.device
    vocab, total = c["vocab"], length + answer
    per = -(-total // PAGE)
    shape = (c["n_layers"], batch * per, c["n_heads"], PAGE, c["d_model"] // c["n_heads"])
    k, v = (torch.empty(shape, device=dev, dtype=torch.bfloat16 if c["dtype"] else torch.float32) for _ in range(2))
    cache = H.PagedCache(k, v, torch.arange(batch * per, device=dev, dtype=torch.int32).view(batch, per), torch.zeros(batch, device=dev, dtype=torch.int32))
    texts = torch.zeros(batch, total, device=dev, dtype=torch.int32)
    texts[:, :length] = prompts
    begin = torch.arange(batch, device=dev) * total
    top_logp, top_ids = torch.empty(batch, TOP, device=dev), torch.empty(batch, TOP, device=dev, dtype=torch.int32)
    new, tokens = length, prompts.reshape(-1)
    for at in range(length, total):
        starts = torch.arange(batch + 1, device=dev, dtype=torch.int32) * new
        logits = model.extend(tokens, starts, cache, new, at, pick=starts[1:] - 1)
        cache.lengths += new
        H.kernel_adjust_logits(logits, vocab, logits, texts.view(-1), begin, begin + at, repetition=repetition, allowed=allowed)
        H.kernel_token_logprob(logits, vocab, None, 1.0 / temperature, None, None, None, top_logp, top_ids)
        tokens = top_ids.gather(1, torch.multinomial(top_logp.exp(), 1)).view(-1).contiguous()
        texts[:, at] = tokens
        new = 1
    return texts


def reward_of(texts, length, vocab):
    """The rule to learn: an even token is followed by one of the lower half of the vocabulary, an odd one by one of the upper half.  One value an answer token."""
    before, token = texts[:, length - 1:-1], texts[:, length:]
    return ((token < vocab // 2) == (before % 2 == 0)).float()


def run(workload="C1", batch=16, sweeps=10, prompt=8, answer=16, dtype="fp32", lr=3e-3, say=print):
    """Mean reward of the answers of every step."""
    import torch

    import paper_2401_15207_amd as H
    from hift_inputs import WORKLOADS, init_params, model_config, uniform_tokens
    wl = WORKLOADS[workload]
    cfg = model_config(wl, dtype=1 if dtype == "bf16" else 0)
    total, vocab = prompt + answer, cfg["vocab"]
    opt = dict(kind="muon", lr=lr, momentum=0.9, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0)
    spec = [(name, shape, kind) for name, shape, kind, _unit, _offset in H.tensor_list(cfg)[0]]
    model = H.HiftModel(cfg, opt, wl["m"], batch, total, init_params=init_params(0, spec, bf16_exact=dtype == "bf16"), state_on_host=1)
    groups = model.set_group_schedule("bottom2up", wl["m"])
    torch.manual_seed(0)
    allowed = torch.full((1, -(-vocab // 32)), -1, device="cuda", dtype=torch.int32)
    allowed[0, 0] = -2      # token 0 is never an answer
    rewards = []
    for step in range(1, sweeps * groups + 1):
        group = model.schedule_group_at(step)
        prompts = torch.from_numpy(uniform_tokens(1, step, batch, prompt, vocab)).cuda()
        texts = answers(H, model, prompts, answer, allowed)
        reward = reward_of(texts, prompt, vocab)
        targets = torch.full_like(texts, -1)
        targets[:, prompt - 1:-1] = texts[:, prompt:]
        model.score(texts, targets, group, temperature=TEMPERATURE)
        d_logp = torch.zeros(batch, total, device="cuda")
        d_logp[:, prompt - 1:-1] = -(reward - reward.mean()) / reward.numel()
        model.step_scored(texts, targets, group, d_logp, None)
        rewards.append(reward.mean().item())
        if step % groups == 0:
            say(f"sweep {step // groups}: mean reward {rewards[-1]:.3f}", flush=True)
    model.close()
    return rewards


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workload", default="C1")
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--sweeps", type=int, default=10)
    ap.add_argument("--dtype", choices=("fp32", "bf16"), default="fp32")
    a = ap.parse_args()
    r = run(a.workload, a.batch, a.sweeps, dtype=a.dtype)
    print(f"mean reward {r[0]:.3f} at first, {r[-1]:.3f} in the end")
