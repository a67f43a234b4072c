"""A one-layer mixture-of-experts language model trained with the operators of this package and SkewAdam.

    python examples/train_moe.py [--steps 60] [--device cuda:0]

Everything the optimizer's three tiers hold is trained by the package's own gradients: the token embedding (backbone,
`embed` / `embed_grad`), the router (float32, `route` / `route_backward`) and the stacked experts (`expert_matmul`,
`expert_matmul_grad`, `expert_combine`); the head is a plain matrix product. The data is synthetic: sequences of a
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

    def __init__(self, vocab=512, d=128, f=256, experts=8, k=2, seed=0, device="cuda:0"):
        g = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, std, dtype=BF16):
            return torch.empty(shape, device=device).normal_(0, std, generator=g).to(dtype)

        self.vocab, self.k, self.experts = vocab, k, experts
        self.w = {"embed": normal(vocab, d, std=1.0), "router": normal(d, experts, std=d**-0.5, dtype=F32),
                  "up": normal(experts, d, f, std=d**-0.5), "down": normal(experts, f, d, std=f**-0.5),
                  "head": normal(d, vocab, std=d**-0.5)}
        self.g = {n: torch.zeros_like(w) for n, w in self.w.items()}
        self.bias = torch.zeros(experts, device=device)
        tier = {"embed": P.BACKBONE, "head": P.BACKBONE, "router": P.ROUTER, "up": P.EXPERT, "down": P.EXPERT}
        self.opt = P.SkewAdam([(tier[n], w, self.g[n], i, P.STATE_FP32 if w.dtype == F32 else 0)
                               for i, (n, w) in enumerate(self.w.items())])

    def forward(self, tokens):
        """Logits of the next tokens, and what the backward pass needs."""
        w, s = self.w, {"tokens": tokens}
        x = s["x"] = P.embed(tokens, w["embed"])
        s["logits"] = x.float() @ w["router"]
        s["weights"], s["chosen"] = P.route(s["logits"], self.k, score="sigmoid", bias=self.bias)
        plan = s["plan"] = P.expert_rows(s["chosen"], self.experts)
        h = s["h"] = P.expert_matmul(x, w["up"], plan, gather=True)
        s["a"] = torch.relu(h)
        s["y"] = P.expert_matmul(s["a"], w["down"], plan, dtype=F32)
        s["out"] = x + P.expert_combine(s["y"], plan, s["weights"], dtype=BF16)
        return (s["out"] @ w["head"]).float(), s

    def backward(self, s, dscores):
        """Gradients of every weight from that of the scores (tokens, vocab)."""
        w, g, plan, d16 = self.w, self.g, s["plan"], dscores.to(BF16)
        g["head"].copy_(s["out"].T @ d16)
        dout = d16 @ w["head"].T
        dy, dweights = P.expert_combine_backward(dout, s["y"], plan, s["weights"])
        da = P.expert_matmul(dout, w["down"], plan, gather=True, transpose=True, scale=s["weights"])
        P.expert_matmul_grad(s["a"], dy, plan, out=g["down"])
        dh = da * (s["h"] > 0)
        P.expert_matmul_grad(s["x"], dh, plan, gather=True, out=g["up"])
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


def train(steps=60, tokens=2048, device="cuda:0", log=print):
    """(first, last) mean loss of 10 steps, in nats a token."""
    model = Model(device=device)
    g = torch.Generator(device=device).manual_seed(1)
    chain = torch.softmax(4 * torch.randn(model.vocab, model.vocab, generator=g, device=device), -1)
    losses = []
    for step in range(1, steps + 1):
        x, target = batch(chain, tokens, g)
        scores, s = model.forward(x)
        p = torch.softmax(scores, -1)
        losses.append(-p[torch.arange(tokens, device=device), target].log().mean())
        p[torch.arange(tokens, device=device), target] -= 1.0
        model.backward(s, p / tokens)
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
    a = ap.parse_args()
    print("mean loss of the first and the last 10 steps: %.3f, %.3f" % train(a.steps, device=a.device))
