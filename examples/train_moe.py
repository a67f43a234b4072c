"""A one-layer mixture-of-experts language model trained with the operators of this package and SkewAdam.

    python examples/train_moe.py [--steps 60] [--device cuda:0] [--keep8]

Everything the optimizer's three tiers hold is trained by the package's own gradients: the token embedding (backbone,
`embed` / `embed_grad`), the router (float32, `route` / `route_backward`) and the stacked experts (`expert_matmul`,
`expert_matmul_grad`, `expert_combine`) and the head with its loss (`head_loss` / `head_loss_backward`: no logits are held). With
`keep8` the experts' activation is silu, and what the backward pass needs of it and of the tokens' rows is kept in 8 bits
(`expert_act`, `keep8`). The data is synthetic: sequences of a
random first-order Markov chain, so that the next token can be learned from the present one. Balance is kept by
the routing bias: 0.001 up for experts with fewer tokens than the average, down for those with more.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_19058_amd as P  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


class Model:
    """Weights, and their gradients in the buffers that the optimizer reads."""

    def __init__(self, vocab=512, d=128, f=256, experts=8, k=2, seed=0, device="cuda:0", keep8=False):
        g = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, std, dtype=BF16):
            return torch.empty(shape, device=device).normal_(0, std, generator=g).to(dtype)

        self.vocab, self.k, self.experts, self.keep8 = vocab, k, experts, keep8
        self.w = {"embed": normal(vocab, d, std=1.0), "router": normal(d, experts, std=d**-0.5, dtype=F32),
                  "up": normal(experts, d, f, std=d**-0.5), "down": normal(experts, f, d, std=f**-0.5),
                  "head": normal(d, vocab, std=d**-0.5)}
        self.g = {n: torch.zeros_like(w) for n, w in self.w.items()}
        self.bias = torch.zeros(experts, device=device)
        tier = {"embed": P.BACKBONE, "head": P.BACKBONE, "router": P.ROUTER, "up": P.EXPERT, "down": P.EXPERT}
        self.opt = P.SkewAdam([(tier[n], w, self.g[n], i, P.STATE_FP32 if w.dtype == F32 else 0)
                               for i, (n, w) in enumerate(self.w.items())])

    def forward(self, tokens, targets):
        """Losses of the next tokens, and what the backward pass needs."""
        w, s = self.w, {"tokens": tokens, "targets": targets}
        x = s["x"] = P.embed(tokens, w["embed"])
        s["logits"] = x.float() @ w["router"]
        s["weights"], s["chosen"] = P.route(s["logits"], self.k, score="sigmoid", bias=self.bias)
        plan = s["plan"] = P.expert_rows(s["chosen"], self.experts)
        h = P.expert_matmul(x, w["up"], plan, gather=True)
        if self.keep8:
            a, s["kept"] = P.expert_act(h, kind="silu", keep=True)
            s["x8"] = P.keep8(x)
        else:
            s["h"] = h
            a = s["a"] = P.expert_act(h, kind="relu")
        s["y"] = P.expert_matmul(a, w["down"], plan, dtype=F32)
        s["out"] = x + P.expert_combine(s["y"], plan, s["weights"], dtype=BF16)
        loss, s["lse"] = P.head_loss(s["out"], w["head"], targets)
        return loss, s

    def backward(self, s, dloss):
        """Gradients of every weight from those of the losses (tokens)."""
        w, g, plan = self.w, self.g, s["plan"]
        dout, _ = P.head_loss_backward(s["out"], w["head"], s["targets"], s["lse"], dloss, out=g["head"])
        dy, dweights = P.expert_combine_backward(dout, s["y"], plan, s["weights"])
        da = P.expert_matmul(dout, w["down"], plan, gather=True, transpose=True, scale=s["weights"])
        if self.keep8:
            a, dh, _ = P.expert_act_backward(da, s["kept"], kind="silu")
        else:
            a, dh = s["a"], da * (s["h"] > 0)
        P.expert_matmul_grad(a, dy, plan, out=g["down"])
        P.expert_matmul_grad(s["x8"] if self.keep8 else s["x"], dh, plan, gather=True, out=g["up"])
        dx = P.expert_combine(P.expert_matmul(dh, w["up"], plan, transpose=True, dtype=F32), plan)
        dlogits = P.route_backward(s["logits"], s["chosen"], dweights, score="sigmoid")
        g["router"].copy_(s["x"].float().T @ dlogits)
        dx += dout.float() + dlogits @ w["router"].T
        P.embed_grad(s["tokens"], dx.to(BF16), self.vocab, out=g["embed"])

    def balance(self, plan, step=1e-3):
        count = plan.offsets.diff().float()
        self.bias += step * torch.sign(count.mean() - count)


def batch(chain, n, g):
    """n pairs (token, next token) of the chain whose row t holds the probabilities of what follows t."""
    t = torch.randint(0, chain.shape[0], (n,), generator=g, device=chain.device)
    return t, torch.multinomial(chain[t], 1, generator=g).squeeze(1)


def train(steps=60, tokens=2048, device="cuda:0", log=print, keep8=False):
    """(first, last) mean loss of 10 steps, in nats a token."""
    model = Model(device=device, keep8=keep8)
    g = torch.Generator(device=device).manual_seed(1)
    chain = torch.softmax(4 * torch.randn(model.vocab, model.vocab, generator=g, device=device), -1)
    dloss = torch.full((tokens,), 1.0 / tokens, device=device)
    losses = []
    for step in range(1, steps + 1):
        x, target = batch(chain, tokens, g)
        loss, s = model.forward(x, target)
        losses.append(loss.mean())
        model.backward(s, dloss)
        model.balance(s["plan"])
        model.opt.step(step, lr=0.02, max_grad_norm=1.0)
        if step % 10 == 0:
            log(f"step {step}: loss {float(losses[-1]):.3f}, tokens an expert {s['plan'].offsets.diff().tolist()}")
    first, last = torch.stack(losses[:10]).mean(), torch.stack(losses[-10:]).mean()
    model.opt.close()
    return float(first), float(last)


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--device", default="cuda:0")
    ap.add_argument("--keep8", action="store_true")
    a = ap.parse_args()
    print("mean loss of the first and the last 10 steps: %.3f, %.3f" % train(a.steps, device=a.device, keep8=a.keep8))
