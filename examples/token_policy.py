"""A population of token policies trained with the library's token losses.

    python examples/token_policy.py [--vocab 4000 --steps 30 --seed 0]

Each policy answers a prompt with a few tokens of a vocabulary; its network is a small
one in PyTorch (any network that gives a row of logits for every position would do). The
library takes the logits from there:

  * the rollout records each token's log-probability, one row per live answer and step
    (``token_logprob``); a frozen reference policy's log-probabilities come from the same call;
  * two members are trained by the clipped policy loss (``learn_token_ppo``), whose
    gradient is written over the logits and carried back by the network; the parameters
    move by ``adam_step``;
  * the first member is trained further on pairs of its answers, the better one of two
    to the same prompt being the chosen one (``learn_token_pref``);
  * a new policy learns from the better member's largest logits (``learn_token_distill``).

An answer ends after a random number of tokens; the rows after its end carry token -1
and are left out by every call. A token earns 1 where it agrees with the prompt modulo 8,
so a policy that knows nothing earns 1/8 a token.
"""
import argparse
import pathlib
import sys

import torch

sys.path.insert(0, str(pathlib.Path(__file__).resolve().parents[1]))
from paper_2106_07551_gb300 import Context  # noqa: E402

PROMPTS, LENGTH, HIDDEN, CLASSES = 16, 6, 64, 8


class Policy:
    """logits = relu(E[prompt] + F[previous token's class] + G[position]) W + b, its fp32
    parameters in one flat tensor that ``adam_step`` moves."""

    def __init__(self, vocab, seed):
        gen = torch.Generator().manual_seed(seed)
        self.vocab = vocab
        self.shapes = [(PROMPTS, HIDDEN), (CLASSES, HIDDEN), (LENGTH, HIDDEN), (HIDDEN, vocab), (vocab,)]
        scale = [1.0, 1.0, 1.0, 0.3 * HIDDEN ** -0.5, 0.0]
        self.flat = torch.cat([(torch.randn(s, generator=gen) * f).flatten() for s, f in zip(self.shapes, scale)]).cuda()
        self.flat.requires_grad_(True)
        self.m, self.v, self.step = torch.zeros_like(self.flat), torch.zeros_like(self.flat), 0

    def copy(self):
        other = Policy(self.vocab, 0)
        other.flat.data.copy_(self.flat.data)
        return other

    def logits(self, prompt, previous, position):
        """[rows][vocab] in bf16, as the losses and the sampling read them."""
        at, parts = 0, []
        for s in self.shapes:
            n = torch.Size(s).numel()
            parts.append(self.flat[at:at + n].view(s))
            at += n
        e, f, g, w, b = parts
        h = torch.relu(e[prompt] + f[previous % CLASSES] + g[position])
        return (h @ w + b).bfloat16()

    def update(self, ctx, lr):
        self.step += 1
        ctx.adam_step(self.flat.data, self.flat.grad, self.m, self.v, self.step, lr)
        self.flat.grad = None


class Answers:
    """Sampled answers, one row per (answer, position), answers in a row."""

    def __init__(self, ctx, policy, prompts, gen):
        n, dev = prompts.numel(), prompts.device
        length = torch.randint(2, LENGTH + 1, (n,), generator=gen, device=dev)
        tokens = torch.full((n, LENGTH), -1, dtype=torch.int32, device=dev)
        logp = torch.zeros((n, LENGTH), device=dev)
        previous = torch.zeros(n, dtype=torch.long, device=dev)
        with torch.no_grad():
            for t in range(LENGTH):
                z = policy.logits(prompts, previous, torch.full_like(previous, t))
                chosen = torch.multinomial(torch.softmax(z.float(), -1), 1, generator=gen).view(-1)
                live = t < length
                token = torch.where(live, chosen, -1).int()
                step = torch.empty(n, device=dev)
                ctx.token_logprob(z, token, step)                  # one row per answer; those that ended are left out
                tokens[:, t], logp[:, t] = token, step
                previous = chosen
        self.length, self.tokens, self.logp = length, tokens.view(-1), logp.view(-1)
        self.prompt = prompts.repeat_interleave(LENGTH)
        self.position = torch.arange(LENGTH, device=dev).repeat(n)
        self.previous = torch.cat([torch.zeros((n, 1), dtype=torch.long, device=dev), tokens[:, :-1].clamp(min=0).long()], 1).view(-1)
        self.live = self.tokens >= 0
        self.reward = ((self.tokens % CLASSES == self.prompt % CLASSES) & self.live).float()

    def inputs(self):
        return self.prompt, self.previous, self.position

    def mean_reward(self):
        return float(self.reward.sum() / self.live.sum())


def reference_logp(ctx, policy, answers):
    out = torch.empty_like(answers.logp)
    with torch.no_grad():
        ctx.token_logprob(policy.logits(*answers.inputs()), answers.tokens, out)
    return out


def train_ppo(ctx, policy, reference, steps, answers_per_step, gen, lr=0.02):
    """Clipped policy loss with a KL term to the reference, two passes an iteration."""
    stats = torch.empty(5, device="cuda")
    rewards = []
    for _ in range(steps):
        prompts = torch.randint(PROMPTS, (answers_per_step,), generator=gen, device="cuda")
        a = Answers(ctx, policy, prompts, gen)
        rewards.append(a.mean_reward())
        advantage = a.reward - a.mean_reward()
        ref = reference_logp(ctx, reference, a)
        weight = torch.full_like(advantage, 1.0 / float(a.live.sum()))
        for _ in range(2):
            z = policy.logits(*a.inputs())
            g = z.detach().clone()                                 # autograd keeps z; the loss writes over the copy
            ctx.learn_token_ppo(g, a.tokens, a.logp, advantage, g, stats, weight=weight, ref_logp=ref, kl_coef=0.01,
                                entropy_coef=0.001)
            z.backward(g)
            policy.update(ctx, lr)
    ctx.sync()                                                     # errors on the device surface here
    return rewards, stats.tolist()


def train_pref(ctx, policy, steps, pairs, gen, lr=0.005):
    """Pairs of the policy's answers to one prompt, the better one (by reward a token)
    chosen; the policy at the start is the reference."""
    prompts = torch.randint(PROMPTS, (pairs,), generator=gen, device="cuda").repeat_interleave(2)
    a = Answers(ctx, policy, prompts, gen)
    score = a.reward.view(-1, LENGTH).sum(1) / a.length
    score = score.view(pairs, 2)
    better = (score[:, 1] > score[:, 0]).long()
    order = torch.stack([2 * torch.arange(pairs, device="cuda") + better, 2 * torch.arange(pairs, device="cuda") + 1 - better], 1)
    rows = (order.view(-1, 1) * LENGTH + torch.arange(LENGTH, device="cuda")).view(-1)
    rows = rows[a.live[rows]]                                      # answers of their own lengths, one after another
    offsets = torch.zeros(2 * pairs + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = a.length[order.view(-1)].cumsum(0)
    inputs = [x[rows] for x in a.inputs()]
    tokens, ref = a.tokens[rows].contiguous(), reference_logp(ctx, policy, a)[rows].contiguous()
    stats, losses = torch.empty(5, device="cuda"), []
    for _ in range(steps):
        z = policy.logits(*inputs)
        g = torch.empty_like(z)
        ctx.learn_token_pref(z.detach(), tokens, offsets, g, stats, ref_logp=ref, beta=0.5)
        z.backward(g)
        policy.update(ctx, lr)
        losses.append(stats[1].item())
    ctx.sync()
    return losses, stats.tolist()


def distill(ctx, teacher, student, steps, rows, gen, top=32, lr=0.02):
    """The student learns the teacher's `top` largest logits at random positions."""
    stats, losses = torch.empty(3, device="cuda"), []
    for _ in range(steps):
        inputs = [torch.randint(k, (rows,), generator=gen, device="cuda") for k in (PROMPTS, CLASSES, LENGTH)]
        with torch.no_grad():
            values, ids = teacher.logits(*inputs).topk(top, 1)
        z = student.logits(*inputs)
        g = torch.empty_like(z)
        ctx.learn_token_distill(z.detach(), ids.int(), values, g, stats)
        z.backward(g)
        student.update(ctx, lr)
        losses.append(stats[1].item())
    ctx.sync()
    return losses


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--vocab", type=int, default=4000)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--answers", type=int, default=512)
    ap.add_argument("--seed", type=int, default=0)
    args = ap.parse_args(argv)
    gen = torch.Generator(device="cuda").manual_seed(args.seed)
    base = Policy(args.vocab, args.seed)
    report = {"members": []}
    with Context(0) as ctx:
        members = []
        for k in range(2):
            member = base.copy()
            rewards, stats = train_ppo(ctx, member, base, args.steps, args.answers, gen, lr=(0.02, 0.01)[k])
            members.append(member)
            report["members"].append({"reward_first": rewards[0], "reward_last": rewards[-1], "stats": stats})
            print(f"member {k}: reward a token {rewards[0]:.3f} -> {rewards[-1]:.3f}, "
                  f"KL to the start {stats[3]:.3f}, entropy {stats[4]:.3f}")
        losses, stats = train_pref(ctx, members[0], args.steps, args.answers, gen)
        report["pref"] = {"losses": losses, "stats": stats}
        print(f"pairs of member 0: loss {losses[0]:.4f} -> {losses[-1]:.4f}, in order {stats[2]:.3f}")
        best = max(range(2), key=lambda k: report["members"][k]["reward_last"])
        student = Policy(args.vocab, args.seed + 1)
        losses = distill(ctx, members[best], student, 2 * args.steps, 2 * args.answers, gen)
        prompts = torch.randint(PROMPTS, (args.answers,), generator=gen, device="cuda")
        report["distill"] = {"losses": losses, "reward": Answers(ctx, student, prompts, gen).mean_reward()}
        ctx.sync()
        print(f"a new policy from member {best}: loss {losses[0]:.3f} -> {losses[-1]:.3f}, "
              f"reward a token {report['distill']['reward']:.3f}")
    return report


if __name__ == "__main__":
    main()
