"""A latent ODE: a gated recurrent encoder reads a sequence of observations and gives the initial state of a neural ODE.

    python -m paper_2510_23498_amd.latent [steps]

trains one on synthetic records of different lengths.  The encoder is mixed precision throughout, as the time stepper is: the residual
stream and all states in fp32, activations in bf16, matrix products in 8 bits with power-of-two scales, dropout masks
regenerated in the backward pass.  Every block is an Euler step of it:
    [u, z, gate] = W_in x;   h = recurrence(u, z);   y <- y + alpha scale s(gate) dropout(N(W_out h) w_post);   x = N(y) w_pre
and a last recurrence without a block around it ends in the state y0 of the ODE.  Weights are fp32 tensors, quantised once per step.
"""
from __future__ import annotations

import sys
from typing import Dict, List, Optional

import numpy as np
import torch

from . import binding as rb

LOW = torch.bfloat16


class Linear:
    """y = x W^T in 8 bits; keeps what its backward pass needs"""

    def __init__(self, n_out: int, n_in: int, generator, device):
        self.w = torch.randn(n_out, n_in, generator=generator, device=device) * n_in ** -0.5
        self.grad = torch.zeros_like(self.w)
        self.wq, self.wt = rb.Fp8.empty(n_out, n_in, self.w.device), rb.Fp8.empty(n_in, n_out, self.w.device)
        self.quantise()

    def quantise(self):
        rb.rampde_fp8_quantize(self.w, "blocks", out=self.wq, out_t=self.wt)

    def forward(self, x: torch.Tensor, dtype=LOW) -> torch.Tensor:
        self.x = x
        return rb.rampde_fp8_matmul(rb.rampde_fp8_quantize(x), self.wq, dtype=dtype)

    def backward(self, dy: torch.Tensor, want_dx: bool = True) -> Optional[torch.Tensor]:
        rb.rampde_fp8_matmul(rb.rampde_fp8_quantize(dy, "cols"), rb.rampde_fp8_quantize(self.x, "cols"), out=self.grad, accumulate=True)
        return rb.rampde_fp8_matmul(rb.rampde_fp8_quantize(dy), self.wt, dtype=LOW) if want_dx else None


class Encoder:
    """Observations [B, T, n_obs] -> state [B, width] (fp32), `blocks` residual blocks, one gate per `share` channels"""

    def __init__(self, n_obs: int, width: int, blocks: int, share: int = 1, p: float = 0.1, seed: int = 0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.width, self.gates, self.p = width, width // share, p
        self.embed = Linear(width, n_obs, g, device)
        self.into = [Linear(2 * width + self.gates, width, g, device) for _ in range(blocks)]
        self.out = [Linear(width, width, g, device) for _ in range(blocks)]
        self.head = Linear(width + self.gates, width, g, device)
        self.vectors = {f"{k}{i}": torch.ones(width, device=device) for i in range(blocks + 1) for k in ("w_pre", "w_post", "scale")}
        self.grads = {k: torch.zeros_like(v) for k, v in self.vectors.items()}
        self.alpha = 1.0 / max(1, blocks)  # the Euler step

    def linears(self) -> List[Linear]:
        return [self.embed, *self.into, *self.out, self.head]

    def _join(self, i: int, seed: int, p: float) -> rb.Join:
        return rb.Join(alpha=self.alpha, p=p, seed=seed, offset=i << 40)

    def _split(self, u: torch.Tensor, B: int):
        """Views [B, T, ..] of a block's projection: inputs, gates of the recurrence, and the gate of the residual"""
        u, w = u.view(B, -1, u.shape[1]), self.width
        return u[:, :, :w], u[:, :, w:w + self.gates], u[:, :, w + self.gates:]

    def forward(self, obs: torch.Tensor, lengths: Optional[torch.Tensor] = None, seed: int = 0, train: bool = True,
                states: Optional[Dict[int, torch.Tensor]] = None) -> torch.Tensor:
        """`states` ({} at first) carries the recurrences of a program that passes its observations bit by bit"""
        B, T, n = obs.shape
        p, w = (self.p if train else 0.0), self.width
        st = {} if states is None else states
        y = self.embed.forward(obs.reshape(B * T, n).to(LOW), dtype=torch.float32)
        _, x, rstd = rb.rampde_join_fwd(self._join(0, seed, 0.0), y, w_pre=self.vectors["w_pre0"], low=LOW, save_rstd=train)
        self.saved = [(y, rstd)]
        for i, (into, out) in enumerate(zip(self.into, self.out)):
            u, z, gate = self._split(into.forward(x), B)
            h0 = st.get(i)
            h, st[i], before = rb.rampde_recurrence_fwd(u, z, h0=h0, lengths=lengths, save_states=train)
            b = out.forward(h.view(B * T, w))
            gate = gate.reshape(B * T, w)  # (a view)
            v = {k: self.vectors[f"{k}{i + 1}"] for k in ("w_post", "scale", "w_pre")}
            y, x, rstd = rb.rampde_join_fwd(self._join(i + 1, seed, p), y, b, gate=gate, save_rstd=train, **v)
            self.saved.append((y, rstd, u, z, gate, b, before))
        x = rb.rampde_dropout(x, p, seed, offset=(len(self.into) + 1) << 40) if p else x
        u, z, _ = self._split(self.head.forward(x), B)
        _, st["head"], before = rb.rampde_recurrence_fwd(u, z, h0=st.get("head"), lengths=lengths, save_states=train, want_h=False)
        self.tail = (u, z, before, lengths, seed, p)
        return st["head"]

    def backward(self, dy0: torch.Tensor) -> None:
        """Adds the gradients of the weights (Linear.grad, self.grads), given that of the state"""
        w = self.width
        u, z, before, lengths, seed, p = self.tail
        B, T, _ = u.shape
        du = torch.empty(B * T, w + self.gates, dtype=LOW, device=dy0.device)
        parts = self._split(du, B)
        rb.rampde_recurrence_bwd(u, z, before, None, dhT=dy0, lengths=lengths, dx=parts[0], dz=parts[1])
        dx = self.head.backward(du)
        if p:
            rb.rampde_dropout(dx, p, seed, offset=(len(self.into) + 1) << 40, out=dx)
        dy = None
        for i in reversed(range(len(self.into))):
            y, rstd, u, z, gate, b, before = self.saved[i + 1]
            v = {k: self.vectors[f"{k}{i + 1}"] for k in ("w_post", "scale", "w_pre")}
            dv = {f"d{k}": self.grads[f"{k}{i + 1}"] for k in v}
            du = torch.empty(B * T, 2 * w + self.gates, dtype=LOW, device=dy0.device)
            parts = self._split(du, B)
            g = rb.rampde_join_bwd(self._join(i + 1, seed, p), y, b, rstd, dy, dx, gate=gate, dgate=parts[2].reshape(B * T, w),
                                   **v, **dv)
            dh = self.out[i].backward(g.db).view(B, T, w)
            rb.rampde_recurrence_bwd(u, z, before, dh, lengths=lengths, dx=parts[0], dz=parts[1])
            dx, dy = self.into[i].backward(du), g.dy
        y, rstd = self.saved[0]
        g = rb.rampde_join_bwd(self._join(0, seed, 0.0), y, None, rstd, dy, dx, w_pre=self.vectors["w_pre0"], dw_pre=self.grads["w_pre0"])
        self.embed.backward(g.dy, want_dx=False)

    def update(self, rate: float) -> None:
        """A step of gradient descent on the fp32 weights; clears the gradients"""
        for lin in self.linears():
            lin.w.sub_(lin.grad, alpha=rate)
            lin.grad.zero_()
            lin.quantise()
        for k, v in self.vectors.items():
            v.sub_(self.grads[k], alpha=rate)
            self.grads[k].zero_()


class LatentODE:
    """Encoder -> y0 -> dense velocity network from t = 0 to 1 (rampde_odeint_fwd), squared distance of its end from a target"""

    def __init__(self, n_obs: int, width: int = 64, hidden: int = 128, blocks: int = 2, share: int = 1, p: float = 0.1, N: int = 8,
                 seed: int = 0, device="cuda"):
        self.encoder = Encoder(n_obs, width, blocks, share, p, seed, device)
        self.velocity = rb.Velocity.mlp((width, hidden, width))
        self.tableau = rb.Tableau([[0, 0], [1, 0]], [0.5, 0.5], [0, 1])
        self.policy = rb.Policy(low="bf16")
        self.grid = np.linspace(0.0, 1.0, N + 1)
        g = torch.Generator(device=device).manual_seed(seed + 1)
        self.theta = torch.randn(rb.rampde_num_params(self.velocity), generator=g, device=device) * 0.05

    def loss_and_gradients(self, obs, target, lengths=None, seed: int = 0) -> torch.Tensor:
        y0 = self.encoder.forward(obs, lengths, seed)
        yN, ckpt = rb.rampde_odeint_fwd(self.velocity, self.theta, y0, self.grid, self.tableau, self.policy)
        off = (yN - target) / target.numel()
        dy0, self.dtheta, _ = rb.rampde_odeint_bwd(self.velocity, self.theta, self.grid, self.tableau, self.policy, ckpt, off,
                                                   want_info=False)
        self.encoder.backward(dy0)
        return 0.5 * ((yN - target) ** 2).mean()

    def step(self, obs, target, lengths=None, seed: int = 0, rate: float = 1.0) -> torch.Tensor:
        loss = self.loss_and_gradients(obs, target, lengths, seed)
        self.theta.sub_(self.dtheta, alpha=rate)
        self.encoder.update(rate)
        return loss


def records(B: int, T: int, n_obs: int, width: int, seed: int = 0, device="cuda"):
    """Noisy damped oscillations observed for different numbers of steps, and a smooth function of their frequency and phase to predict"""
    g = torch.Generator(device=device).manual_seed(seed)
    f, ph = (torch.rand(B, 1, n_obs, generator=g, device=device) for _ in range(2))
    t = torch.arange(T, device=device, dtype=torch.float32)[None, :, None]
    obs = torch.exp(-t / T) * torch.sin(0.3 * f * t + 6.28 * ph) + 0.05 * torch.randn(B, T, n_obs, generator=g, device=device)
    lengths = torch.randint(max(1, T // 2), T + 1, (B,), generator=g, device=device, dtype=torch.int32)
    mix = torch.randn(n_obs, width, generator=g, device=device) / n_obs ** 0.5
    return obs, torch.tanh((f[:, 0] - 0.5 + torch.cos(6.28 * ph[:, 0])) @ mix), lengths


def main(steps: int = 100) -> None:
    model = LatentODE(n_obs=12)
    obs, target, lengths = records(B=64, T=200, n_obs=12, width=64)
    for i in range(steps):
        loss = model.step(obs, target, lengths, seed=i)
        if i % 20 == 0 or i + 1 == steps:
            print(f"step {i:4d}  loss {loss.item():.5f}", flush=True)


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 100)
