"""Gradients of the latent ODE's encoder against automatic differentiation of a plain encoder in 64 bits."""
import numpy as np
import pytest

from test_gpu_sequence_passes import _mask

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


class _Plain:
    """The encoder's forward pass in torch, fp64.  Roundings are those of the encoder, and are passed through by the gradient: bf16
    where it stores bf16, 8 bits (the library's quantiser, which is tested on its own) where it multiplies."""

    def __init__(self, enc, rb):
        self.enc, self.rb, self.leaves = enc, rb, {}
        self.w = {lin: self._leaf(lin, lin.wq.dequantize()) for lin in enc.linears()}
        self.v = {k: self._leaf(k, t) for k, t in enc.vectors.items()}

    def _leaf(self, key, t):
        self.leaves[key] = t.detach().double().requires_grad_()
        return self.leaves[key]

    @staticmethod
    def low(v):
        return v + (v.detach().bfloat16().double() - v.detach())

    def product(self, lin, x, low=True):
        q = self.rb.rampde_fp8_quantize(x.detach().bfloat16()).dequantize().double()
        out = (x + (q - x.detach())) @ self.w[lin].t()
        return self.low(out) if low else out

    @staticmethod
    def norm(v, w):
        return v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-6) * w

    def recurrence(self, u, z, lengths):
        B, T, D = u.shape
        r = torch.sigmoid(z).repeat_interleave(D // z.shape[2], 2)
        h, out = torch.zeros(B, D, dtype=torch.float64, device=u.device), []
        for t in range(T):
            live = (t < lengths)[:, None]
            h = torch.where(live, h + r[:, t] * (u[:, t] - h), h)
            out.append(torch.where(live, h, 0.0))
        return torch.stack(out, 1), h

    def forward(self, obs, lengths, seed):
        enc, w, (B, T, n) = self.enc, self.enc.width, obs.shape
        keep = lambda i: torch.from_numpy(_mask(B * T * w, enc.p, seed, i << 40)).view(B * T, w).to(obs.device) if enc.p else 1.0  # noqa: E731
        y = self.product(enc.embed, obs.reshape(B * T, n).bfloat16().double(), low=False)
        x = self.low(self.norm(y, self.v["w_pre0"]))
        for i, (into, out) in enumerate(zip(enc.into, enc.out)):
            u, z, gate = self.product(into, x).split([w, enc.gates, w], 1)
            h, _ = self.recurrence(u.reshape(B, T, w), z.reshape(B, T, enc.gates), lengths)
            b = self.product(out, self.low(h.reshape(B * T, w)))
            y = y + enc.alpha * self.v[f"scale{i + 1}"] * torch.sigmoid(gate) * keep(i + 1) * self.norm(b, self.v[f"w_post{i + 1}"])
            x = self.low(self.norm(y, self.v[f"w_pre{i + 1}"]))
        x = self.low(x * keep(len(enc.into) + 1))
        u, z = self.product(enc.head, x).split([w, enc.gates], 1)
        return self.recurrence(u.reshape(B, T, w), z.reshape(B, T, enc.gates), lengths)[1]


@pytest.mark.parametrize("share,p", [(1, 0.0), (16, 0.1)])
def test_encoder_gradients_are_those_of_a_plain_encoder(share, p):
    """The backward pass quantises cotangents and activations to 8 bits (3 places of mantissa: 2^-3 / sqrt(12) of a value between 1 and 2,
    2.4 % of it on average).  A weight's gradient takes two of these roundings, and the cotangent that comes to the first layer has been
    through five products, one each: sqrt(7) 2.4 %, 6.4 % norm-wise, bounded by two and a half times that.  The roundings do not know of
    the gradient, so along it they cancel: its length is right to 3 %, in which a wrong factor on a path among several shows."""
    from paper_2510_23498_amd import binding as rb
    from paper_2510_23498_amd import latent
    enc = latent.Encoder(n_obs=12, width=64, blocks=2, share=share, p=p, seed=7)
    g = torch.Generator(device="cuda").manual_seed(8)
    for t in enc.vectors.values():
        t.add_(0.2 * torch.randn(t.shape, generator=g, device="cuda"))
    obs, _, lengths = latent.records(B=48, T=60, n_obs=12, width=64, seed=9)
    dy0 = torch.randn(48, 64, generator=g, device="cuda")
    y0 = enc.forward(obs, lengths, seed=11)
    enc.backward(dy0)
    plain = _Plain(enc, rb)
    want = plain.forward(obs.double(), lengths, 11)
    # (the same roundings but for those on the edge, which sums of other orders tip)
    assert (y0.double() - want).norm() <= 2e-2 * want.norm()
    (want * dy0.double()).sum().backward()
    got = {**{lin: lin.grad for lin in enc.linears()}, **enc.grads}
    names = {**{lin: f"linear {i}" for i, lin in enumerate(enc.linears())}, **{k: k for k in enc.grads}}
    seen = 0
    for key, leaf in plain.leaves.items():
        if leaf.grad is None:   # (a vector that the encoder does not use)
            assert not got[key].any()
            continue
        seen += 1
        a, b = got[key].double(), leaf.grad
        off, along = ((a - b).norm() / b.norm()).item(), ((a * b).sum() / (b * b).sum()).item()
        print(f"{names[key]}: {off:.4f} off, {along:.4f} along")
        assert off <= 0.16 and abs(along - 1) <= 0.03, (names[key], off, along)
    assert seen == len(enc.linears()) + 1 + 3 * len(enc.into)
