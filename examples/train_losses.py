"""A small language model through the stages of its training, every loss and
its gradient from paper_2507_08784_amd.losses, every hidden weight's gradient
compressed by GreedyLore in the DistributedDataParallel communication hook:

  pretrain    cross entropy: the mean of the tokens' log-probabilities
  distill     a narrower student on the model's top logits and the hard labels
  preference  pairs of answers, against the pretrained model as the reference
  policy      answers sampled from the model, rewarded, the clipped loss with
              the KL term to the reference

    python examples/train_losses.py [--steps 60]

One process, one GPU, synthetic tokens (a random Markov chain).  As in the
paper, embedding and output layer are not compressed.  Prints each stage's
first and last loss.
"""
from __future__ import annotations

import argparse
import copy
import os
import socket
import sys

import torch
import torch.distributed as dist
from torch import nn
from torch.nn.parallel import DistributedDataParallel as DDP

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2507_08784_amd import losses  # noqa: E402
from paper_2507_08784_amd.ddp import GreedyLoreHook  # noqa: E402

VOCAB, STEPS_SEQ, BATCH = 503, 33, 32


class TinyLM(nn.Module):
    """Two hidden layers over the current, the previous and the mean past embedding."""

    def __init__(self, width):
        super().__init__()
        self.embed = nn.Embedding(VOCAB, width)
        self.first = nn.Linear(3 * width, 2 * width)
        self.second = nn.Linear(2 * width, width)
        self.head = nn.Linear(width, VOCAB, bias=False)

    def forward(self, ids):
        e = self.embed(ids)
        before = torch.cat([torch.zeros_like(e[:, :1]), e[:, :-1]], 1)
        mean = e.cumsum(1) / torch.arange(1, ids.shape[1] + 1, device=ids.device)[:, None]
        h = torch.relu(self.first(torch.cat([e, before, mean], -1)))
        return self.head(torch.relu(self.second(h)))

    def hidden(self):
        return [self.first.weight, self.second.weight]


class Chain:
    """Tokens of a random Markov chain: every token has eight likely successors."""

    def __init__(self, gen):
        self.gen = gen
        self.next = torch.randint(0, VOCAB, (VOCAB, 8), generator=gen, device="cuda")

    def batch(self, n, steps=STEPS_SEQ):
        ids = [torch.randint(0, VOCAB, (n,), generator=self.gen, device="cuda")]
        for _ in range(steps - 1):
            k = torch.randint(0, 8, (n,), generator=self.gen, device="cuda")
            ids.append(self.next[ids[-1], k])
        return torch.stack(ids, 1)


def train(name, model, steps, rank, lr, loss_of):
    """`steps` optimizer steps on loss_of(ddp model, step); the hidden weights
    are updated by the hook during backward."""
    hook = GreedyLoreHook(model.hidden(), rank=rank, tau=10, opt="adam", lr=lr)
    ddp = DDP(model, device_ids=[0])
    hook.register(ddp)
    taken = {p.data_ptr() for p in hook.compressed_parameters()}
    opt = torch.optim.AdamW([p for p in model.parameters() if p.data_ptr() not in taken], lr=lr)
    seen = []
    for t in range(steps):
        opt.zero_grad(set_to_none=True)
        loss = loss_of(ddp, t)
        loss.backward()
        opt.step()
        seen.append(loss.detach())
    hook.check_status()
    seen = torch.stack(seen).cpu()
    tenth = max(1, steps // 10)
    first, last = float(seen[:tenth].mean()), float(seen[-tenth:].mean())
    print(f"{name:10s} {steps:4d} steps  loss {first:.4f} -> {last:.4f}", flush=True)
    return first, last


def sample(model, ids, steps, gen):
    """`steps` tokens more, drawn from the model."""
    with torch.no_grad():
        for _ in range(steps):
            p = torch.softmax(model(ids)[:, -1], -1)
            ids = torch.cat([ids, torch.multinomial(p, 1, generator=gen)], 1)
    return ids


def main(steps=60):
    torch.manual_seed(0)
    gen = torch.Generator(device="cuda").manual_seed(1)
    chain = Chain(gen)
    out = {}

    # ---- pretraining: position t predicts token t + 1, the views are taken as they are
    model = TinyLM(96).cuda()

    def pretrain(ddp, t):
        ids = chain.batch(BATCH)
        return -losses.token_logprobs(ddp(ids)[:, :-1], ids[:, 1:]).logps.mean()

    out["pretrain"] = train("pretrain", model, 2 * steps, 8, 3e-3, pretrain)

    # ---- distillation: what would be stored of the teacher is its top 16 logits and their log-sum-exp
    student, tau = TinyLM(48).cuda(), 2.0

    def distill(ddp, t):
        ids = chain.batch(BATCH)
        with torch.no_grad():
            z = model(ids)[:, :-1]
            top = z.topk(16, -1)
            lse = torch.logsumexp(z / tau, -1)
        return losses.distill_loss(ddp(ids)[:, :-1], top.indices, top.values, temperature=tau, teacher_lse=lse,
                                   targets=ids[:, 1:], hard_weight=0.3).loss

    out["distill"] = train("distill", student, 2 * steps, 8, 3e-3, distill)

    # ---- preference: of two answers to a prompt, the one that keeps to even tokens
    ref = copy.deepcopy(model).eval()
    prompt, answer = 9, 24

    def preference(ddp, t):
        start = chain.batch(BATCH // 2, prompt)
        two = [sample(ref, start, answer, gen) for _ in range(2)]
        even = [(x[:, prompt:] % 2 == 0).sum(1) for x in two]
        swap = (even[1] > even[0])[:, None]
        ids = torch.cat([torch.where(swap, two[1], two[0]), torch.where(swap, two[0], two[1])])
        targets = ids[:, 1:].clone()
        targets[:, :prompt - 1] = -100                 # the prompt is not trained on
        with torch.no_grad():
            base = losses.token_logprobs(ref(ids)[:, :-1], targets).logps.sum(1)
        return losses.preference_loss(ddp(ids)[:, :-1], targets, base, beta=0.1).loss

    tuned = copy.deepcopy(model)
    out["preference"] = train("preference", tuned, 2 * steps, 8, 3e-4, preference)

    # ---- policy: the same wish as a reward; the answers of a step serve four updates
    actor, kept = copy.deepcopy(model), {}

    def policy(ddp, t):
        if t % 4 == 0:
            ids = sample(actor, chain.batch(BATCH, prompt), answer, gen)
            targets = ids[:, 1:].clone()
            targets[:, :prompt - 1] = -100
            reward = (ids[:, prompt:] % 2 == 0).float().mean(1)
            adv = (reward - reward.mean()) / (reward.std() + 1e-6)
            with torch.no_grad():
                old = losses.token_logprobs(actor(ids)[:, :-1], targets).logps
                base = losses.token_logprobs(ref(ids)[:, :-1], targets).logps
            kept.update(ids=ids, targets=targets, old=old, base=base, adv=adv[:, None].expand(old.shape),
                        reward=kept.get("reward", []) + [float(reward.mean())])
        return losses.policy_loss(ddp(kept["ids"])[:, :-1], kept["targets"], kept["old"], kept["adv"],
                                  ref_logps=kept["base"], kl_coef=0.01, reduction="sequence").loss

    out["policy"] = train("policy", actor, 2 * steps, 8, 1e-3, policy)
    out["reward"] = kept["reward"][0], sum(kept["reward"][-3:]) / len(kept["reward"][-3:])
    print(f"policy reward (share of even tokens) {out['reward'][0]:.3f} -> {out['reward'][1]:.3f}", flush=True)
    return out


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    a = ap.parse_args()
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        port = s.getsockname()[1]
    dist.init_process_group("nccl", init_method=f"tcp://127.0.0.1:{port}", rank=0, world_size=1)
    try:
        main(a.steps)
    finally:
        dist.destroy_process_group()
