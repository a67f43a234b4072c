"""The head's loss and its gradients from their definitions, in float64 (on the device of the inputs), with what the operators may be off by.

Error bounds, from the arithmetic (u = 2^-24, half an ulp of float32; A_tv = scale sum |x||w|):
  logit     float32 sums of d products, in any order and perhaps truncated: (2 d + 8) u A
  lse       the largest error of a logit of the row, and u times: 4 |z| of the powers' arguments, 2 of their values, 128 + V / 4096
            of the sums (32 in a lane, the tree, the runs, one after another)
  loss      the two together
  G         exp(z - lse) is off by e = error of z and lse, relatively; the factors by 4 u; float16 by 2^-11 of the value (half
            a step; two bf16 numbers, for few tokens or small heads, by 2^-16) and, below its smallest normal number, by 2^-39 of the largest factor (2^-25 where that is 2^14 or more)
  operands  x and w in float16 are exact but for 2^-39 of their columns' largest
  sums      float32 sums of K products: (2 K + 16) u, and the results' rounding
"""
import torch

U32 = 2.0**-24
UBF = 2.0**-8
F16, F16_LOW = 2.0**-11, 2.0**-39   # half a step; half a step below the normal numbers, of a largest value kept as 2^14 or more


class Ref:
    def __init__(self, x, w, targets, tied=False, scale=1.0):
        self.x, self.scale = x.double(), scale
        w = w.double()
        self.w = w if tied else w.T.contiguous()   # (V, d)
        self.tied = tied
        self.V, self.d = self.w.shape
        self.there = (targets >= 0) & (targets < self.V)
        self.x = torch.where(self.there[:, None], self.x, 0.0)
        self.y = torch.where(self.there, targets, 0).long()
        self.z = scale * (self.x @ self.w.T.contiguous())
        self.A = scale * (self.x.abs() @ self.w.abs().T.contiguous())
        self.lse_all = torch.logsumexp(self.z, 1)
        self.lse = torch.where(self.there, self.lse_all, 0.0)
        zy = self.z.gather(1, self.y[:, None]).squeeze(1)
        self.loss = torch.where(self.there, self.lse_all - zy, 0.0)
        self.ez = (2 * self.d + 8) * U32 * self.A
        big = self.z.abs().amax(1)
        self.e_lse = self.ez.amax(1) + (4 * big + 130 + self.V / 4096 + 4 * self.lse.abs()) * U32
        self.e_loss = self.e_lse + self.ez.gather(1, self.y[:, None]).squeeze(1) + 4 * U32 * (zy.abs() + self.loss.abs())

    def backward(self, dloss, dlse=None, out16=True):
        """(dx, its bound, dw, its bound)"""
        s = self.scale
        one = torch.where(self.there, s * dloss.double(), 0.0)
        both = one + (0.0 if dlse is None else torch.where(self.there, s * dlse.double(), 0.0))
        T = one.numel()
        n = torch.arange(T, device=one.device)
        p = torch.exp(self.z - self.lse_all[:, None])
        G = both[:, None] * p
        rest = -one * (-torch.expm1(self.z[n, self.y] - self.lse_all)) + (both - one) * p[n, self.y]
        G[n, self.y] = rest
        e = self.ez + self.e_lse[:, None] + (4 * self.z.abs() + 16) * U32
        eG = (both.abs() + one.abs())[:, None] * p * e.expm1().clamp(max=1e3)
        factor = torch.maximum(both.abs(), one.abs())
        eG += (F16 + 8 * U32) * G.abs() + 2 * F16_LOW * factor[:, None]
        eG = torch.where(self.there[:, None], eG, 0.0)
        ew, ex = F16_LOW * self.w.abs().amax(0), F16_LOW * self.x.abs().amax(0) if T else torch.zeros_like(self.w[0])
        Ga = G.abs() + eG
        dx, dw = G @ self.w, G.T.contiguous() @ self.x
        bx = eG @ self.w.abs() + Ga.sum(1, keepdim=True) * ew + (2 * self.V + 16) * U32 * (Ga @ self.w.abs())
        # what is left out of x_t is relative to its column's largest times the largest factor, where the token's own is its share of G
        share = torch.where(factor > 0, factor.max() / factor, 0.0) if T else factor
        bw = eG.T.contiguous() @ self.x.abs() + (Ga * share[:, None]).sum(0)[:, None] * ex + (2 * T + 16) * U32 * (Ga.T.contiguous() @ self.x.abs())
        bx = bx * 1.01 + (UBF if out16 else U32) * dx.abs() * 1.01 + 1e-37
        bw = bw * 1.01 + UBF * dw.abs() * 1.01 + 1e-37
        return dx, bx, (dw if self.tied else dw.T), (bw if self.tied else bw.T)
