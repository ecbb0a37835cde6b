"""Fine-tuning a small gated-MLP language model with this library's operators.

    python examples/finetune.py [--steps N]

Both objectives of a usual fine-tuning run, each a whole training step:

  1. preferences: pairs of answers, the preferred one following a hidden rule, scored against a frozen
     copy of the model (meq.token_logprobs) and learnt with meq.preference_loss;
  2. policy: answers sampled from the model, rewarded where they follow the rule, several updates per
     batch with meq.policy_loss (clipped ratios, a KL term against the frozen copy).

A step: the loss and the gradient of the logits in their place (bf16), torch's backward pass from
there, then MeqMuon for the hidden matrices and AdamW with 8-bit moments, its gradients clipped to a
norm, for the embedding, the head and the norm weight.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_35701_gb300 import meq  # noqa: E402


class Model:
    """Next-token model of one token: embedding, a gated MLP block, head. fp32 parameters, bf16 logits."""

    def __init__(self, vocab, dim, ffn, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=g, device="cuda") * cols ** -0.5).requires_grad_()

        self.hidden = [weight(ffn, dim), weight(ffn, dim), weight(dim, ffn)]   # gate, up, down
        self.rest = [weight(vocab, dim), weight(vocab, dim), torch.ones(1, dim, device="cuda", requires_grad=True)]

    def logits(self, tokens):
        (gate, up, down), (embed, head, norm) = self.hidden, self.rest
        x = embed[tokens]
        h = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * norm
        x = x + (torch.nn.functional.silu(h @ gate.T) * (h @ up.T)) @ down.T
        return (x @ head.T).bfloat16()


class Trainer:
    def __init__(self, model):
        self.model = model
        self.muon = meq.MeqMuon([tuple(p.shape) for p in model.hidden])
        self.adamw = meq.AdamW([tuple(p.shape) for p in model.rest], state_bits=8, beta2=0.95,
                               decay=[1.0 if p.shape[0] > 1 else 0.0 for p in model.rest])
        self.norm = torch.empty(2, device="cuda")

    def step(self, logits, grad, lr):
        """One update from the gradient of the logits; the optimizers' kernels follow on the same stream.
        lr is MeqMuon's: its updates have the same size whatever the gradient's, so it falls between the phases."""
        params = self.model.hidden + self.model.rest
        for p in params:
            p.grad = None
        logits.backward(grad)
        with torch.no_grad():
            self.muon.step([p.detach() for p in self.model.hidden], [p.grad for p in self.model.hidden], lr=lr, momentum=0.9,
                           weight_decay=0.01)
            grads = [p.grad for p in self.model.rest]
            self.adamw.grad_norm(grads, max_norm=1.0, out=self.norm)
            self.adamw.step([p.detach() for p in self.model.rest], grads, lr=0.5 * lr, weight_decay=0.01, grad_scale=self.norm[1:])

    def sync(self):
        self.muon.sync()
        self.adamw.sync()


def reference_logprobs(model, prompts, answers):
    with torch.no_grad():
        return meq.token_logprobs(model.logits(prompts), answers).logp


def preference_phase(model, frozen, trainer, vocab, steps, g, pairs=32, length=16):
    losses = []
    starts = torch.arange(0, (2 * pairs + 1) * length, length, device="cuda")
    for _ in range(steps):
        prompts = torch.randint(0, vocab, (2 * pairs, length), generator=g, device="cuda")
        answers = torch.randint(0, vocab, (2 * pairs, length), generator=g, device="cuda")
        answers[0::2] = (3 * prompts[0::2] + 1) % vocab   # the preferred ones follow the rule
        prompts, answers = prompts.view(-1), answers.view(-1)
        ref = reference_logprobs(frozen, prompts, answers)
        logits = model.logits(prompts)
        z = logits.detach()
        r = meq.preference_loss(z, answers, starts, ref, beta=0.1, grad=z)   # the gradient in the logits' place
        trainer.step(logits, r.grad, lr=5e-3)
        losses.append(r.loss)
    return torch.stack(losses)


def policy_phase(model, frozen, trainer, vocab, steps, g, batch=1024, updates=2):
    rewards = []
    for _ in range(steps):
        prompts = torch.randint(0, vocab, (batch,), generator=g, device="cuda")
        with torch.no_grad():
            z = model.logits(prompts)
            noise = -torch.log(-torch.log(torch.rand(z.shape, generator=g, device="cuda").clamp(1e-9, 1 - 1e-7)))
            answers = (z.float() + noise).argmax(-1)   # a sample of the softmax
            old = meq.token_logprobs(z, answers).logp
        ref = reference_logprobs(frozen, prompts, answers)
        reward = (answers == (3 * prompts + 1) % vocab).float()
        advantage = (reward - reward.mean()) / (reward.std() + 1e-3)
        weights = torch.full((batch,), 1.0 / batch, device="cuda")
        for _ in range(updates):
            logits = model.logits(prompts)
            z = logits.detach()
            r = meq.policy_loss(z, answers, old, advantage, weights, ref_logp=ref, clip_low=0.2, clip_high=0.28, kl_coef=0.001, grad=z)
            trainer.step(logits, r.grad, lr=1e-3)
        rewards.append(reward.mean())
    return torch.stack(rewards)


def main(steps=60, vocab=509, dim=128, ffn=344, seed=0):
    """The preference loss of each of steps // 6 steps, then the mean reward of each of `steps` batches."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    model, frozen = Model(vocab, dim, ffn, seed), Model(vocab, dim, ffn, seed)
    trainer = Trainer(model)
    losses = preference_phase(model, frozen, trainer, vocab, max(2, steps // 6), g).tolist()
    rewards = policy_phase(model, frozen, trainer, vocab, steps, g).tolist()
    trainer.sync()
    return losses, rewards


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    losses, rewards = main(ap.parse_args().steps)
    print(f"preference loss {losses[0]:.4f} -> {losses[-1]:.4f}; reward {rewards[0]:.3f} -> {rewards[-1]:.3f}")
