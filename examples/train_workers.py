"""K workers train one small captioning policy with GMC on one GPU, using the
operators of a worker's pass: an encoder of channels-last images (group norm
with its activation, dropout joined to the residual stream) and a token head,
first on pairs of captions (preference loss), then on its own rollouts (clipped
policy loss with a KL term to the model the pairs left; the rollouts' log-probabilities
and entropies are the tokens' scores).

Each worker has images of its own few classes (non-IID) and masks of its own; the
gradients of all K workers go into gmc_iteration, which compresses them and updates
the shared parameters.  With --orthogonal the server takes the sum of the messages
through a momentum of its own and orthogonalises the weight matrices' part of it; with
--bonus the policy loss has an entropy bonus of that weight.

    python examples/train_workers.py [--orthogonal] [--bonus 0.01]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1905_12948_amd as gmc  # noqa: E402

K, CLASSES, PER_WORKER, T, V = 4, 12, 16, 8, 101   # workers, classes, images a worker, tokens, vocabulary
SIDE, INPUT, WIDTH, GROUPS, P_DROP, SEED = 6, 24, 64, 8, 0.1, 11
SHAPES = {"stem": (INPUT, WIDTH), "gamma": (WIDTH,), "beta": (WIDTH,), "mix": (WIDTH, WIDTH), "token": (V + 1, WIDTH),
          "place": (T, WIDTH), "head": (WIDTH, V)}


class GroupNorm(torch.autograd.Function):
    """gmc.group_norm and its backward call as one node of torch's graph."""

    @staticmethod
    def forward(ctx, x, gamma, beta):
        y, mean, rstd = gmc.group_norm(x, GROUPS, gamma, beta, act="silu")
        ctx.save_for_backward(x, mean, rstd, gamma, beta)
        return y

    @staticmethod
    def backward(ctx, dy):
        return gmc.group_norm_backward(dy.contiguous(), *ctx.saved_tensors, act="silu")


class Dropout(torch.autograd.Function):
    """residual + dropout(x), the mask drawn again in the backward pass."""

    @staticmethod
    def forward(ctx, x, residual, t, worker):
        ctx.where = dict(seed=SEED, t=t, worker=worker, site=0)
        return gmc.dropout(x, P_DROP, residual=residual, **ctx.where)

    @staticmethod
    def backward(ctx, dy):
        dy = dy.contiguous()
        return gmc.dropout_backward(dy, P_DROP, **ctx.where), dy, None, None


def parameters(w):
    """The named tensors of the flat vector w, as leaves of a graph."""
    out, at = {}, 0
    for name, shape in SHAPES.items():
        n = math.prod(shape)
        out[name] = w[at:at + n].view(shape).detach().requires_grad_()
        at += n
    return out


def logits_of(p, images, tokens, t=None, worker=0):
    """Logits [N, T, V] of each token after those before it; dropout only with a step t."""
    x = GroupNorm.apply((images @ p["stem"]).contiguous(), p["gamma"], p["beta"])
    mixed = (x @ p["mix"]).contiguous()
    x = x + mixed if t is None else Dropout.apply(mixed, x, t, worker)
    before = torch.cat([torch.full_like(tokens[:, :1], V), tokens[:, :-1]], 1)
    h = x.mean((1, 2))[:, None, :] + p["token"][before] + p["place"]
    return torch.nn.functional.silu(h) @ p["head"]


class Task:
    """Images with a class's pattern, and each class's caption."""

    def __init__(self, device):
        self.g = torch.Generator(device=device).manual_seed(SEED)
        self.pattern = torch.randn(CLASSES, SIDE, SIDE, INPUT, device=device, generator=self.g)
        self.caption = torch.randint(0, V, (CLASSES, T), device=device, generator=self.g)
        self.device = device

    def batch(self, worker):
        mine = torch.arange(worker, CLASSES, K, device=self.device)   # the worker's own classes
        cls = mine[torch.randint(0, len(mine), (PER_WORKER,), device=self.device, generator=self.g)]
        noise = torch.randn(PER_WORKER, SIDE, SIDE, INPUT, device=self.device, generator=self.g)
        return self.pattern[cls] + 0.3 * noise, self.caption[cls]


def gradient_row(p):
    return torch.cat([v.grad.reshape(-1) for v in p.values()])


class Server:
    """The server's side: gmc_iteration, or the messages' sum through orthogonal_step."""

    def __init__(self, w, orthogonal):
        self.w, self.w_prev, self.err = w, w.clone(), torch.zeros(K, len(w), device=w.device)
        # the server's momentum is the only one where it orthogonalises
        self.gmc = gmc.Gmc(len(w), K, "topk", ratio=0.05, beta=0.0 if orthogonal else 0.5, eta=1.0 if orthogonal else 0.5)
        self.message = self.gmc.alloc_messages(w.device)
        self.plan = None
        if orthogonal:
            table, at = [], 0
            for name, shape in SHAPES.items():
                if name in ("stem", "mix", "head"):
                    table.append((at, *shape))
                at += math.prod(shape)
            self.plan = gmc.Matrices(len(w), table, device=w.device)
            self.update, self.momentum = torch.empty_like(w), torch.zeros_like(w)

    def step(self, grads):
        if self.plan is None:
            self.gmc.iteration(self.w, self.w_prev, grads, self.err, *self.message)
        else:
            self.gmc.step(self.w, self.w_prev, grads, self.err, *self.message)
            self.gmc.aggregate(*self.message, self.update)
            gmc.orthogonal_step(self.plan, self.w, self.update, self.momentum, 0.02, mu=0.9, w_out=self.w_prev)
        self.w, self.w_prev = self.w_prev, self.w

    def close(self):
        self.gmc.close()
        if self.plan is not None:
            self.plan.close()


def policy_gradient(logits, tokens, old, advantage, ref, scores, bonus):
    """The logits' gradient of the clipped policy loss with a KL term, less bonus times the mean
    entropy; scores: gmc.token_scores of the same logits and tokens, for the bonus."""
    grad = gmc.policy_loss(logits, tokens, old, advantage, ref_logp=ref, kl_coef=0.01)[2]
    if bonus:
        share = torch.full(tokens.shape, -bonus / tokens.numel(), device=logits.device)
        grad += gmc.token_scores_backward(logits, scores[4], tokens, entropy=scores[1], dentropy=share)
    return grad


def train(pair_steps=40, policy_steps=40, device="cuda:0", log=print, orthogonal=False, bonus=0.0):
    """(first and last preference loss, first and last mean reward of the rollouts)."""
    task = Task(device)
    w = torch.cat([(torch.ones(s, device=device) if name == "gamma" else
                    torch.zeros(s, device=device) if name == "beta" else
                    torch.randn(s, device=device, generator=task.g) / math.sqrt(s[0])).reshape(-1)
                   for name, s in SHAPES.items()])
    server = Server(w, orthogonal)

    # 1. pairs: the class's caption is preferred to a random one
    frozen = parameters(server.w.clone())
    losses = []
    for t in range(pair_steps):
        rows, total = [], 0.0
        for k in range(K):
            images, chosen = task.batch(k)
            rejected = torch.randint(0, V, chosen.shape, device=device, generator=task.g)
            tokens, images = torch.cat([chosen, rejected]), torch.cat([images, images])
            with torch.no_grad():
                ref = gmc.preference_loss(logits_of(frozen, images, tokens).contiguous(), tokens, grad=False)[3]
            p = parameters(server.w)
            logits = logits_of(p, images, tokens, t, k)
            loss, _, _, _, grad = gmc.preference_loss(logits.detach(), tokens, ref, beta=0.5)
            logits.backward(grad)
            rows.append(gradient_row(p))
            total += loss.item() / K
        losses.append(total)
        server.step(torch.stack(rows))
    log("preference loss %.4f -> %.4f over %d iterations" % (losses[0], losses[-1], pair_steps))

    # 2. rollouts: reward for every token of the caption
    frozen = parameters(server.w.clone())
    rewards, entropies = [], []
    for t in range(policy_steps):
        rows, total, spread = [], 0.0, 0.0
        for k in range(K):
            images, caption = task.batch(k)
            p = parameters(server.w)
            with torch.no_grad():
                tokens = torch.zeros_like(caption)
                for j in range(T):
                    at = torch.softmax(logits_of(p, images, tokens)[:, j], -1)
                    tokens[:, j] = torch.multinomial(at, 1, generator=task.g)[:, 0]
                hit = (tokens == caption).float()
                advantage = (hit - hit.mean()) / (hit.std() + 0.05)
                # the rollouts' and the frozen model's log-probabilities
                old = gmc.token_scores(logits_of(p, images, tokens), tokens)[0]
                ref = gmc.token_scores(logits_of(frozen, images, tokens), tokens)[0]
            logits = logits_of(p, images, tokens, pair_steps + t, k)
            seen = logits.detach()
            scores = gmc.token_scores(seen, tokens)
            spread += scores[1].mean().item() / K
            logits.backward(policy_gradient(seen, tokens, old, advantage, ref, scores, bonus))
            rows.append(gradient_row(p))
            total += hit.mean().item() / K
        rewards.append(total)
        entropies.append(spread)
        server.step(torch.stack(rows))
    log("caption tokens right %.3f -> %.3f, entropy %.3f -> %.3f over %d iterations"
        % (rewards[0], rewards[-1], entropies[0], entropies[-1], policy_steps))
    server.close()
    return losses[0], losses[-1], rewards[0], rewards[-1]


def options(argv):
    """train's arguments from the command line's."""
    p = argparse.ArgumentParser(description="K workers train a small captioning policy.")
    p.add_argument("--orthogonal", action="store_true", help="the server orthogonalises the weight matrices' part of its step")
    p.add_argument("--bonus", type=float, default=0.0, help="weight of the entropy bonus in the policy loss (default: none)")
    return vars(p.parse_args(argv))


if __name__ == "__main__":
    train(**options(sys.argv[1:]))
