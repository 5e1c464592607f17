"""Seeded synthetic micro-gradient workloads.

This module only draws inputs; it contains none of the method's arithmetic (no
dot product, norm, distance or filtering).  The same tensors are handed to the
CUDA library and, as numpy views of the same bits, to the CPU oracle used by the
tests.

Model for every workload: one shared direction ``s`` and one private direction
``n_i`` per micro-gradient, all iid N(0, sigma_d^2) per element, mixed as

    g_i = sign(rho_i) * sqrt(|rho_i|) * s + sqrt(1 - |rho_i|) * n_i

so that the expected cosine between g_i and g_j is sign * sqrt(|rho_i rho_j|).
A negative rho flips the sign of the shared part.  This stands in for the
ResNet18 / ViT micro-gradients of the paper's experiments (Section 4), whose
datasets and weights are not available: late in training their pairwise cosine
distances sit near 1 and reach 1.1-1.6 (Figure 1), which the rho ranges below
reproduce.

The five named configurations:

  1  K=4  D=1,000,000     fp32  rho=(0.9, 0.5, 0.0, -0.3)  tau=0.97   seed 0
  2  K=4  D=11,227,812    fp32  ResNet18 (100 classes) tensor layout, per-tensor
                                sigma ~ lognormal(log 1e-3, 1), rho ~ U(-0.2, 0.6),
                                tau in {0.95, 0.97, 1.0}
  3  K=32 D=11,227,812    bf16  pairwise matrix, rho ~ U(-0.5, 0.9)
  4  K=8  D=124,439,808   fp32  rho ~ N(0.02, 0.05^2), tau=0.97
  5  K=8  D=1,000,000,000 bf16  rho ~ 50% U(0.3, 0.8) / 50% U(-0.3, 0.1), tau=0.97

Beside the mixtures, ``LanguageModel`` makes real micro-gradients: one microbatch after another through a small language
model whose memory-bound layers, 8-bit checkpoints and weight gradients are the library's own (``gaf_embedding`` and
its neighbours), each weight's gradient written straight into its slice of a flat buffer.

Configuration n uses seed n-1.  rho values are drawn first, from a CPU generator,
so they do not depend on the device; the vectors are drawn on the requested
device (CPU and GPU streams differ, which is fine: both consumers see the same
bits of one draw).
"""
from __future__ import annotations

import math
from dataclasses import dataclass, field
from typing import List, Optional, Sequence

import numpy as np
import torch

RESNET18_100_NUMEL = 11_227_812
GPT2_SMALL_NUMEL = 124_439_808


def resnet18_tensor_sizes(num_classes: int = 100) -> List[int]:
    """Element counts of ResNet18's parameter tensors in network order.

    Convolutions carry no bias; every batch-norm contributes a weight and a
    bias vector; the 128/256/512-channel stages open with a block that has a
    1x1 shortcut convolution plus batch-norm.
    """
    sizes: List[int] = [64 * 3 * 7 * 7, 64, 64]
    in_ch = 64
    for out_ch in (64, 128, 256, 512):
        for block in range(2):
            cin = in_ch if block == 0 else out_ch
            sizes += [out_ch * cin * 9, out_ch, out_ch]
            sizes += [out_ch * out_ch * 9, out_ch, out_ch]
            if block == 0 and cin != out_ch:
                sizes += [out_ch * cin, out_ch, out_ch]
        in_ch = out_ch
    sizes += [num_classes * 512, num_classes]
    return sizes


@dataclass
class Workload:
    name: str
    K: int
    D: int
    dtype: str                    # "f32" or "bf16"
    taus: List[float]
    rho: List[float]
    seed: int
    grads: List[torch.Tensor] = field(default_factory=list)
    order: Optional[List[int]] = None

    @property
    def elem_bytes(self) -> int:
        return 4 if self.dtype == "f32" else 2


def as_numpy_bits(t: torch.Tensor) -> np.ndarray:
    """Host numpy view of a gradient: float32 as is, bfloat16 as uint16 bit patterns."""
    t = t.detach().cpu().contiguous()
    if t.dtype == torch.bfloat16:
        return t.view(torch.int16).numpy().view(np.uint16)
    return t.numpy()


def _draw(K: int, D: int, dtype: str, rho: Sequence[float], seed: int,
          device: str, sigma, chunk: int = 1 << 24, stacked: bool = False) -> List[torch.Tensor]:
    """Draw K micro-gradients of D elements.  ``sigma`` is a float or a
    per-element float32 tensor on ``device``.  ``stacked``: the gradients are the
    rows of one matrix whose row stride is D rounded up to 128 elements (what an
    all-gather of padded flat gradients leaves); the values are the same either way."""
    tdtype = torch.float32 if dtype == "f32" else torch.bfloat16
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    if stacked:
        matrix = torch.zeros(K, (D + 127) // 128 * 128, dtype=tdtype, device=device)
        grads = [matrix[i, :D] for i in range(K)]
    else:
        grads = [torch.empty(D, dtype=tdtype, device=device) for _ in range(K)]
    alpha = [math.copysign(math.sqrt(abs(r)), r) for r in rho]
    beta = [math.sqrt(1.0 - abs(r)) for r in rho]
    for lo in range(0, D, chunk):
        hi = min(D, lo + chunk)
        sig = sigma[lo:hi] if torch.is_tensor(sigma) else float(sigma)
        s = torch.randn(hi - lo, generator=gen, device=device, dtype=torch.float32) * sig
        for i in range(K):
            n = torch.randn(hi - lo, generator=gen, device=device, dtype=torch.float32) * sig
            grads[i][lo:hi] = (alpha[i] * s + beta[i] * n).to(tdtype)
    return grads


def _clip_rho(r: Sequence[float]) -> List[float]:
    return [float(min(0.999, max(-0.999, x))) for x in r]


def mixture(K: int, D: int, dtype: str, rho: Sequence[float], seed: int,
            device: str = "cpu", sigma=1e-3, taus: Sequence[float] = (0.97,),
            name: str = "custom", stacked: bool = False) -> Workload:
    """A workload with explicit rho values (used by the tests for small and
    ragged shapes)."""
    rho = _clip_rho(rho)
    assert len(rho) == K
    w = Workload(name, K, D, dtype, [float(t) for t in taus], rho, seed)
    w.grads = _draw(K, D, dtype, rho, seed, device, sigma, stacked=stacked)
    return w


def config(n: int, device: str = "cpu", D: Optional[int] = None,
           K: Optional[int] = None, seed: Optional[int] = None, stacked: bool = False) -> Workload:
    """Named configuration ``n`` (1..5).  ``D``/``K`` override the size for
    scaled-down copies of the same recipe (the tensor layout of configuration 2
    is kept only at its native D); ``seed`` draws another instance of it."""
    seed = n - 1 if seed is None else seed
    rgen = np.random.RandomState(seed)
    if n == 1:
        K_, D_, dtype, taus = 4, 1_000_000, "f32", [0.97]
        rho = [0.9, 0.5, 0.0, -0.3]
        if K is not None and K != K_:
            rho = (rho * ((K + 3) // 4))[:K]
    elif n == 2:
        K_, D_, dtype, taus = 4, RESNET18_100_NUMEL, "f32", [0.95, 0.97, 1.0]
        rho = rgen.uniform(-0.2, 0.6, size=K or K_).tolist()
    elif n == 3:
        K_, D_, dtype, taus = 32, RESNET18_100_NUMEL, "bf16", []
        rho = rgen.uniform(-0.5, 0.9, size=K or K_).tolist()
    elif n == 4:
        K_, D_, dtype, taus = 8, GPT2_SMALL_NUMEL, "f32", [0.97]
        rho = rgen.normal(0.02, 0.05, size=K or K_).tolist()
    elif n == 5:
        K_, D_, dtype, taus = 8, 1_000_000_000, "bf16", [0.97]
        kk = K or K_
        pick = rgen.uniform(size=kk) < 0.5
        hi = rgen.uniform(0.3, 0.8, size=kk)
        lo = rgen.uniform(-0.3, 0.1, size=kk)
        rho = np.where(pick, hi, lo).tolist()
    else:
        raise ValueError("configurations are numbered 1..5")
    K_ = K or K_
    native = D is None or D == D_
    D_ = D or D_
    rho = _clip_rho(rho)

    sigma = 1e-3
    if n == 2 and native:
        sizes = resnet18_tensor_sizes(100)
        assert sum(sizes) == RESNET18_100_NUMEL
        per_tensor = np.exp(rgen.normal(math.log(1e-3), 1.0, size=len(sizes))).astype(np.float32)
        sigma = torch.repeat_interleave(torch.from_numpy(per_tensor),
                                        torch.tensor(sizes)).to(device)
    w = Workload(f"config{n}", K_, D_, dtype, taus, rho, seed)
    w.grads = _draw(K_, D_, dtype, rho, seed, device, sigma, stacked=stacked)
    return w


class LanguageModel:
    """Token embedding (scaled by sqrt(d)), RMS norm, a linear layer, RMS norm after the residual's addition, and the table once
    more as the output layer, under a cross-entropy loss: the smallest language model in which every layer operator of the library has its
    place.  The matrix products of the forward pass, the products that carry a gradient back through a linear layer, and the loss are
    plain torch.

    ``sizes``: name and shape of each weight; weight i starts at ``offsets[i]`` of a flat gradient (multiples of 8 elements, so
    that the offsets serve ``gaf_filter_accumulate_bucketed`` too); D: the flat gradient's length.
    """

    def __init__(self, V: int, d: int, seed: int = 0, dtype: torch.dtype = torch.bfloat16, device: str = "cuda"):
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)

        def draw(*shape, size, mean=0.0):
            return (mean + size * torch.randn(*shape, generator=gen, device=device)).to(dtype)
        self.V, self.d, self.dtype, self.device = V, d, dtype, device
        self.table = draw(V, d, size=0.3)
        self.w1, self.w2 = draw(d, size=0.1, mean=1.0), draw(d, size=0.1, mean=1.0)
        self.lin = draw(d, d, size=d ** -0.5)
        self.sizes = [("table", (V, d)), ("w1", (d,)), ("lin", (d, d)), ("w2", (d,))]
        self.offsets = [0]
        for _, shape in self.sizes:
            self.offsets.append(self.offsets[-1] + (math.prod(shape) + 7) // 8 * 8)
        self.D = self.offsets[-1]

    def views(self, flat: torch.Tensor) -> dict:
        """The weights' slices of a flat gradient, by name."""
        return {name: flat[at:at + math.prod(shape)].view(shape) for (name, shape), at in zip(self.sizes, self.offsets)}

    def new_workspace(self, T: int) -> torch.Tensor:
        from . import binding
        code = binding.GAF_F32 if self.dtype == torch.float32 else binding.GAF_BF16
        return binding.new_layer_workspace(T, max(self.V, self.d), code, V=self.V, device=self.device)

    def tokens(self, T: int, seed: int) -> torch.Tensor:
        """T tokens after Zipf's law, the last few padding (-1)."""
        gen = torch.Generator(device=self.device)
        gen.manual_seed(seed)
        u = torch.rand(T, generator=gen, device=self.device, dtype=torch.float64)
        t = (torch.exp(u * math.log(self.V + 1)).to(torch.int64) - 1).clamp(0, self.V - 1)
        t[T - T // 30:] = -1
        return t

    def micro_gradient(self, tokens: torch.Tensor, targets: torch.Tensor, flat: torch.Tensor, workspace: torch.Tensor) -> dict:
        """Forward and backward pass of one microbatch: the gradient into ``flat`` (float32 or bfloat16, all slices written).  The backward
        pass reads of the forward one the 8-bit checkpoints, the roots and the logits' gradient.  Returns the activations and their gradients by
        name, for tests (which keeps them all alive: a training step would let each go after its last use)."""
        from . import binding as gaf
        g, T, scale = self.views(flat), tokens.numel(), math.sqrt(self.d)
        y1c, h1c, y2c, h2c = (gaf.new_checkpoint(T, self.d, self.device) for _ in range(4))
        e = gaf.gaf_embedding(self.table, tokens, scale=scale)
        y1, _, r1 = gaf.gaf_rms_norm(e, self.w1, y_checkpoint=y1c, coded_y=True, h_checkpoint=h1c)
        z = (y1.float() @ self.lin.float().t()).to(self.dtype)
        y2, h2, r2 = gaf.gaf_rms_norm(z, self.w2, residual=e, y_checkpoint=y2c, coded_y=True, h_checkpoint=h2c)
        dlogits = torch.softmax(y2.float() @ self.table.float().t(), dim=1)
        dlogits[torch.arange(T, device=self.device), targets] -= 1.0
        dlogits = (dlogits.masked_fill((tokens < 0)[:, None], 0.0) / T).to(self.dtype)
        gaf.gaf_linear_weight_grad(dlogits, y2c, g["table"], workspace)
        dy2 = (dlogits.float() @ self.table.float()).to(self.dtype)
        dh2, _ = gaf.gaf_rms_norm_grad(dy2, h2c, self.w2, r2, g["w2"], workspace)
        gaf.gaf_linear_weight_grad(dh2, y1c, g["lin"], workspace)
        dy1 = (dh2.float() @ self.lin.float()).to(self.dtype)
        de, _ = gaf.gaf_rms_norm_grad(dy1, h1c, self.w1, r1, g["w1"], workspace, residual_grad=dh2)
        gaf.gaf_embedding_grad(de, tokens, g["table"], workspace, scale=scale, base=g["table"])
        return dict(tokens=tokens, e=e, y1=y1, h2=h2, y2=y2, r1=r1, r2=r2, dlogits=dlogits, dy2=dy2, dh2=dh2, dy1=dy1, de=de,
                    y1c=y1c, y2c=y2c, h1c=h1c, h2c=h2c)


def language_model(K: int, V: int, d: int, T: int, seed: int = 0, dtype: str = "f32", taus: Sequence[float] = (0.97,)) -> Workload:
    """K micro-gradients of a ``LanguageModel`` on microbatches of T tokens, made on the GPU by the library's layers."""
    from . import binding
    model = LanguageModel(V, d, seed)
    w = Workload("language_model", K, model.D, dtype, [float(t) for t in taus], [], seed)
    workspace, tdtype = model.new_workspace(T), torch.float32 if dtype == "f32" else torch.bfloat16
    for k in range(K):
        flat = torch.zeros(model.D, dtype=tdtype, device=model.device)
        tokens = model.tokens(T, seed * 1000 + 2 * k)
        model.micro_gradient(tokens, model.tokens(T, seed * 1000 + 2 * k + 1).clamp(min=0), flat, workspace)
        w.grads.append(flat)
    if binding.gaf_read_status(workspace) & binding.GAF_STATUS_TIMEOUT:
        raise RuntimeError("a bounded wait of a weight gradient ran out: the micro-gradients are not valid")
    return w
