"""A training loop around the scorer: sampled sequences are rewarded by their BLEU and a small policy
learns from that, with every loss of `paper_2510_05485_amd.losses`.

Prompts are class numbers, and each class has a reference sequence.  The policy is a table of
embeddings and a linear layer, so that the loop fits a page; a language model takes their place
without a change to the calls.

  distil   the policy follows a teacher's best logits (a teacher that is right most of the time)
  prefer   of two samples of a prompt the one with the higher BLEU is preferred
  reward   eight samples of a prompt compete: advantages are their BLEU against the group's mean

Run:  python -m paper_2510_05485_amd.example.train_step
"""
from __future__ import annotations

import torch

import paper_2510_05485_amd as tb

V, T, CLASSES, SAMPLES = 96, 16, 24, 8
DEVICE = "cuda:0"


class Policy(torch.nn.Module):
    def __init__(self, width: int = 64):
        super().__init__()
        self.prompt = torch.nn.Embedding(CLASSES, width)
        self.place = torch.nn.Embedding(T, width)
        self.head = torch.nn.Linear(width, V)

    def forward(self, prompts):
        """Logits [B, T, V] of the answers' positions."""
        x = torch.tanh(self.prompt(prompts).unsqueeze(1) * self.place.weight)
        return self.head(x)


def sample(logits, generator):
    p = torch.softmax(logits, -1).flatten(0, 1)
    return torch.multinomial(p, 1, generator=generator).view(logits.shape[:-1])


def run(steps: int = 60, seed: int = 0, say=print):
    """Mean BLEU of samples before training and behind each of the three parts."""
    torch.manual_seed(seed)
    gen = torch.Generator(device=DEVICE).manual_seed(seed + 1)
    policy = Policy().to(DEVICE)
    optimizer = torch.optim.Adam(policy.parameters(), lr=0.02)
    references = torch.randint(0, V, (CLASSES, T), generator=gen, device=DEVICE)
    lengths = torch.randint(T // 2, T + 1, (CLASSES,), generator=gen, device=DEVICE, dtype=torch.int32)
    scorers = {}

    def bleu(prompts, tokens):
        B = prompts.shape[0]
        if B not in scorers:
            scorers[B] = tb.BleuScorer(B, 1, T, T, vocab_size=V, smoothing="add-k", smooth_param=1.0, device=DEVICE)
        n = lengths[prompts]
        return scorers[B](tokens, n, references[prompts].unsqueeze(1), n.unsqueeze(1)).clone()

    every = torch.arange(CLASSES, device=DEVICE)
    means = []

    def report(name):
        with torch.no_grad():
            prompts = every.repeat(SAMPLES)
            means.append(float(bleu(prompts, sample(policy(prompts), gen)).mean()))
        say(f"{name}: mean BLEU {means[-1]:.3f}")

    def update(logits, grad):
        optimizer.zero_grad()
        logits.backward(grad)            # from the logits on into the model
        optimizer.step()

    report("untrained")

    # a teacher whose best logits hold the right token, at a wrong place in the order now and then
    ids = torch.rand(CLASSES, T, V, generator=gen, device=DEVICE).topk(8).indices
    ids[..., 0] = references
    best = torch.sort(torch.randn(CLASSES, T, 8, generator=gen, device=DEVICE), descending=True).values
    best[..., 0] += torch.where(torch.rand(CLASSES, T, generator=gen, device=DEVICE) < 0.7, 2.0, -1.0)
    for _ in range(steps):
        logits = policy(every)
        r = tb.distillation_loss_grad(logits.detach(), ids, best, lengths=lengths)
        update(logits, r.grad)
    report("distilled")

    frozen = Policy().to(DEVICE)
    frozen.load_state_dict(policy.state_dict())
    for _ in range(steps):
        with torch.no_grad():
            one, other = sample(policy(every), gen), sample(policy(every), gen)
            better = (bleu(every, one) >= bleu(every, other)).unsqueeze(-1)
            tokens = torch.cat([torch.where(better, one, other), torch.where(better, other, one)])
            prompts = every.repeat(2)
            ref_lp = tb.token_logprobs(frozen(prompts), tokens, lengths=lengths.repeat(2))
        logits = policy(prompts)
        r = tb.preference_loss_grad(logits.detach(), tokens, ref_lp, lengths=lengths.repeat(2), beta=0.5)
        update(logits, r.grad)
    report("preferences")

    frozen.load_state_dict(policy.state_dict())
    prompts, n = every.repeat_interleave(SAMPLES), lengths.repeat_interleave(SAMPLES)
    for _ in range(steps):
        with torch.no_grad():
            tokens = sample(policy(prompts), gen)
            reward = bleu(prompts, tokens).view(CLASSES, SAMPLES)
            advantages = ((reward - reward.mean(1, keepdim=True)) / (reward.std(1, keepdim=True) + 1e-4)).view(-1)
            old_lp = tb.token_logprobs(policy(prompts), tokens, lengths=n)
            ref_lp = tb.token_logprobs(frozen(prompts), tokens, lengths=n)
        for _ in range(2):               # two updates on each batch of samples: ratios leave 1
            logits = policy(prompts)
            r = tb.policy_loss_grad(logits.detach(), tokens, old_lp, advantages.contiguous(), ref_logprobs=ref_lp,
                                    lengths=n, kl_coef=0.02, entropy_coef=0.001)
            update(logits, r.grad)
    report("rewards")
    say("last policy loss %.4f, KL to the start %.3f, clipped %.3f, entropy %.3f" % tuple(r.terms.tolist()))
    return means


if __name__ == "__main__":
    run()
