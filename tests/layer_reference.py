"""The layers' operators from their definitions, in binary64 (plain torch, any device), and how far a kernel may be off.

Every bound counts roundings: U = 2^-24 for one binary32 operation, half a step of the result's type for the last one."""
import torch

U = 2.0 ** -24
BLOCK = 128
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LAST = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}     # torch.finfo(t).eps / 2


def blocks(d):
    return (d + BLOCK - 1) // BLOCK


def exponents(x):
    """Exponent of every block of a binary64 matrix."""
    T, d = x.shape
    a = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x))
    a = torch.nn.functional.pad(a, (0, blocks(d) * BLOCK - d)).reshape(T, blocks(d), BLOCK).amax(dim=2)
    e = torch.full_like(a, -120)
    for k in range(-119, 121):                  # the smallest e with a <= 448 * 2^e
        e = torch.where(a > 448.0 * 2.0 ** (k - 1), torch.full_like(e, k), e)
    return e


def codes(x):
    """(values / 2^e, e) of the checkpoint of a binary64 matrix: what a code stands for, NaN where x is not finite."""
    T, d = x.shape
    e = exponents(x)
    wide = e.repeat_interleave(BLOCK, dim=1)[:, :d]
    q = x * torch.exp2(-wide)
    step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
    step = torch.where(torch.isfinite(step), step, torch.ones_like(step))
    r = torch.round(q / step) * step            # (round: half to even)
    most = torch.where(wide == 120, 240.0, 448.0).to(r)
    r = torch.minimum(torch.maximum(r, -most), most)
    return torch.where(torch.isfinite(x), r, torch.full_like(r, float("nan"))), e


def values(x):
    r, e = codes(x)
    return r * torch.exp2(e).repeat_interleave(BLOCK, dim=1)[:, :x.shape[1]]


def checkpoint_values(checkpoint):
    """What a checkpoint's bytes stand for."""
    c, s = checkpoint
    v = c.contiguous().view(torch.float8_e4m3fn).to(torch.float64)
    return v * torch.exp2(s.to(torch.float64) - 127).repeat_interleave(BLOCK, dim=1)[:, :c.shape[1]]


def embedding(table, tokens, scale):
    out = torch.zeros(tokens.numel(), table.shape[1], dtype=torch.float64, device=table.device)
    for t, v in enumerate(tokens.flatten().tolist()):
        if 0 <= v < table.shape[0]:
            out[t] = table[v].to(torch.float64) * scale
    return out


def embedding_grad(dy, tokens, V, scale, base=None):
    """(grad, bound of a kernel's error before the last rounding)."""
    dy = dy.to(torch.float64)
    grad = torch.zeros(V, dy.shape[1], dtype=torch.float64, device=dy.device)
    size, n = torch.zeros_like(grad), torch.zeros(V, dtype=torch.float64, device=dy.device)
    t = tokens.flatten().to(torch.int64)
    at = torch.nonzero((t >= 0) & (t < V)).flatten()
    grad.index_add_(0, t[at], dy[at])
    size.index_add_(0, t[at], dy[at].abs())
    n.index_add_(0, t[at], torch.ones(at.numel(), dtype=torch.float64, device=dy.device))
    # n - 1 additions of terms whose sum of magnitudes is `size`, the scale's rounding, the product, the addition of base
    off = U * (n[:, None] + 3) * size * abs(scale)
    grad *= scale
    if base is not None:
        grad += base.to(torch.float64)
        off += U * (size * abs(scale) + base.to(torch.float64).abs())
    return grad, off


def rms_norm(x, residual, weight, eps, type_):
    """(h as stored, r, unrounded y)."""
    h = x if residual is None else (x.to(torch.float32) + residual.to(torch.float32)).to(type_)
    v = h.to(torch.float64)
    r = (v.square().mean(dim=1) + eps).rsqrt()
    return h, r, v * r[:, None] * weight.to(torch.float64)


# A thread adds up to 32 squares, its warp 5 times, then up to 16 warps: 53 roundings of positive terms, halved by the root; the
# division by d, eps, the root and the reciprocal one each.
RSTD = (53 / 2 + 5) * U


def rms_norm_grad(dy, h, weight, r, residual_grad=None, base=None):
    """(dx, dweight, bounds of a kernel's errors before the last rounding); h in binary64."""
    dy, w, r = dy.to(torch.float64), weight.to(torch.float64), r.to(torch.float64)[:, None]
    n = h * r
    q = dy * w * n
    mean = q.mean(dim=1, keepdim=True)
    dx = r * (dy * w - n * mean)
    # the mean: n, dy w and their product one rounding each, 53 additions, the division; then n * mean, the difference, r * it
    off_x = U * r * (3 * (dy * w).abs() + n.abs() * (60 * q.abs().mean(dim=1, keepdim=True) + 3 * mean.abs()))
    if residual_grad is not None:
        g = residual_grad.to(torch.float64)
        dx = dx + g
        off_x = off_x + U * (dx.abs() + g.abs())
    dw = (dy * n).sum(dim=0)
    off_w = U * (dy.shape[0] + 4) * (dy * n).abs().sum(dim=0)      # (a CTA's rows in binary32, four of them side by side)
    if base is not None:
        dw = dw + base.to(torch.float64)
        off_w = off_w + U * base.to(torch.float64).abs()
    return dx, dw, off_x, off_w


def weight_grad(dy, x, base=None):
    """(dW, bound): x the values of the codes, in binary64."""
    dy = dy.to(torch.float64)
    dw = dy.t() @ x
    size = dy.abs().t() @ x.abs()
    # A tensor core adds 16 products to its accumulator at a time, each of the 17 terms cut to 24 bits of the largest: 17 cuts of at most 2 U
    # of the magnitudes so far, which are half of the chain's on average, 32 times a chain: 16 * 17 * 2 U; then the chains, the parts of the
    # tokens, three terms of dy.
    off = (16 * 17 * 2 + dy.shape[0] / 256 * 3 + 300) * U * size
    if base is not None:
        dw = dw + base.to(torch.float64)
        off = off + U * (dw.abs() + base.to(torch.float64).abs())
    return dw, off


def assert_close(got, want, off, what=""):
    """got within off of want, and half a step of got's type."""
    want = want.to(got.device)
    far = (got.to(torch.float64) - want).abs()
    allowed = torch.as_tensor(off, dtype=torch.float64, device=got.device) * (1 + 2 ** -8) + LAST[got.dtype] * want.abs() + 1e-44
    worst = (far / allowed.clamp(min=1e-300)).max().item() if far.numel() else 0.0
    assert not torch.isnan(far).any() and worst <= 1.0, f"{what}: {worst:.3g} times what is allowed"
