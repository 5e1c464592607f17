"""Timed operators of a language model's layers, the part of a training step that makes a micro-gradient.

  lookup       gaf_embedding: rows of a table, scaled; tokens outside the table are padding and give zero rows
  table_grad   gaf_embedding_grad: the table's gradient, into its slice of the micro-gradient
  norm         gaf_rms_norm: addition of the residual and root-mean-square norm; with ``coded`` its result also in 8 bits
  norm_grad    gaf_rms_norm_grad: its backward pass; with ``coded`` from an 8-bit checkpoint of the norm's input
  checkpoint   gaf_checkpoint_pack and gaf_checkpoint_unpack: a matrix of activations into 8 bits and back
  weight_grad  gaf_linear_weight_grad: gradient of a linear layer's weight from an 8-bit checkpoint of its input

An 8-bit checkpoint holds e4m3 codes and, for every 128 consecutive elements of a row, the power of two that they are
multiplied with (as its exponent + 127 in a byte), so that the values that codes stand for are exact in bfloat16.

Sizes: T tokens (rows), d columns (weight_grad: M columns of the layer's input, N of its output), V rows of the table.
Outputs and workspace are allocated once and kept, as a training loop keeps them; every pass overwrites all outputs.
"""
import math

import torch

own = False

EPS = 1e-6
BLOCK = 128


def _case(op, T, d, dtype, V=0, N=0, coded=False, add=False, name=None):
    case = {"op": op, "T": T, "d": d, "dtype": dtype, "V": V, "N": N, "coded": coded, "add": add}
    return dict(case, name=name) if name else case


def listed():
    return [
        # the tokens of one step of generation, GPT-2-small's table: the call itself is most of the cost
        _case("lookup", 8, 768, "f32", V=50_257, name="lookup_f32_8"),
        # a large microbatch on a large table
        _case("lookup", 32_768, 4096, "bf16", V=100_000, name="lookup_bf16_32k"),
        # one sequence of GPT-2-small: nearly all rows of the gradient are zero
        _case("table_grad", 1000, 768, "f32", V=50_257, name="table_grad_f32_1000"),
        # a large microbatch, a table that is also the output layer's weight: added to that one's gradient
        _case("table_grad", 32_768, 2048, "bf16", V=100_000, add=True, name="table_grad_bf16_32k"),
        # one token, odd width, no residual
        _case("norm", 1, 1001, "f32", name="norm_f32_1"),
        # a large microbatch; the 8-bit result is kept for the backward pass and its values are what goes on
        _case("norm", 16_384, 4096, "bf16", coded=True, add=True, name="norm_bf16_16k_coded"),
        # one ragged sequence of GPT-2-small's width
        _case("norm_grad", 515, 768, "f32", name="norm_grad_f32_515"),
        # a large microbatch, from the 8-bit checkpoint, joined by the gradient that comes past the layer
        _case("norm_grad", 16_384, 4096, "bf16", coded=True, add=True, name="norm_grad_bf16_16k_coded"),
        # a short sequence of an odd width
        _case("checkpoint", 67, 1111, "f32", name="checkpoint_f32_67"),
        # the activations of a large microbatch
        _case("checkpoint", 32_768, 4096, "bf16", name="checkpoint_bf16_32k"),
        # one short sequence, a layer of GPT-2-small's width
        _case("weight_grad", 300, 768, "bf16", N=768, name="weight_grad_300"),
        # a large microbatch, a wide layer
        _case("weight_grad", 16_384, 4096, "bf16", N=4096, name="weight_grad_16k"),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["lookup", "table_grad", "norm", "norm_grad", "checkpoint", "weight_grad"])
    dtype = rng.choice(["f32", "bf16"])
    T = _log_uniform(rng, 1, {"lookup": 32_768, "table_grad": 32_768, "checkpoint": 32_768}.get(op, 16_384))
    d = _log_uniform(rng, 64, 4096)
    if rng.random() < 0.5:
        d = (d + 63) // 64 * 64                 # what most layers are; the others take any width
    if op == "lookup":
        return _case(op, T, d, dtype, V=_log_uniform(rng, 500, 100_000))
    if op == "table_grad":
        return _case(op, T, min(d, 2048), dtype, V=_log_uniform(rng, 500, 100_000), add=rng.random() < 0.5)
    if op == "weight_grad":
        N = _log_uniform(rng, 64, 4096)
        if dtype == "f32":
            T = min(T, 5000)
        return _case(op, T, d, dtype, N=N, add=rng.random() < 0.25)
    if op == "checkpoint":
        return _case(op, T, d, dtype)
    coded = rng.random() < 0.5
    if op == "norm" and coded:
        dtype = "bf16"                          # what keeps 8-bit activations computes in bfloat16
    return _case(op, T, d, dtype, coded=coded, add=rng.random() < 0.5)


def _blocks(d):
    return (d + BLOCK - 1) // BLOCK


def work(case):
    op, T, d, V, N = (case[k] for k in ("op", "T", "d", "V", "N"))
    e = 4 if case["dtype"] == "f32" else 2
    n, code = T * d, T * (d + _blocks(d))       # elements, bytes of their checkpoint
    if op == "lookup":
        return {"bytes": 2 * n * e + 8 * T, "flops": n}
    if op == "table_grad":
        return {"bytes": n * e + 8 * T + V * d * 4 * (2 if case["add"] else 1), "flops": 2 * n}
    if op == "norm":
        # x, the residual, h; y; the root; the checkpoint
        return {"bytes": n * e * (4 if case["add"] else 2) + 4 * T + (code if case["coded"] else 0), "flops": 6 * n}
    if op == "norm_grad":
        return {"bytes": n * e * (3 if case["add"] else 2) + (code if case["coded"] else n * e) + 4 * T, "flops": 11 * n}
    if op == "checkpoint":
        return {"bytes": 2 * (n * e + code), "flops": 4 * n}
    return {"bytes": T * N * e + code + N * d * 4 * (2 if case["add"] else 1), "flops": 2 * T * N * d}


# ------------------------------------------------------------------ inputs ----

def _normal(g, T, d, dtype, size=1.0, wide=False):
    """Normal values; ``wide``: some columns are much larger than the others, as in a residual stream."""
    x = torch.randn(T, d, generator=g, device="cuda")
    x *= size
    if wide:
        column = torch.exp(0.5 * torch.randn(d, generator=g, device="cuda"))
        column[torch.randint(0, d, (max(1, d // 200),), generator=g, device="cuda")] *= 20.0
        x *= column
    return x.to(torch.float32 if dtype == "f32" else torch.bfloat16)


def _exponents(x):
    """Exponent of the scale of every block of a [T, d] binary32 or binary64 matrix: int32 [T, blocks]."""
    T, d = x.shape
    a = torch.where(torch.isfinite(x), x.abs(), torch.zeros((), dtype=x.dtype, device=x.device))
    a = torch.nn.functional.pad(a, (0, _blocks(d) * BLOCK - d)).reshape(T, _blocks(d), BLOCK).amax(dim=2)
    m, q = torch.frexp(a)                       # a = m 2^q with m in [1/2, 1); 448 = 0.875 * 2^9
    e = torch.where(m > 0.875, q - 8, q - 9)
    return torch.where(a > 0, e, torch.full_like(e, -120)).clamp(-120, 120).to(torch.int32)


def _power(e, d, dtype):
    """2^e of every block, for each of the d columns."""
    p = ((e + 127) << 23).view(torch.float32).to(dtype)
    return p.repeat_interleave(BLOCK, dim=1)[:, :d]


def _pack(x):
    """Codes (e4m3, as their bytes) and scale bytes of a [T, d] matrix."""
    x = x.to(torch.float32)
    e = _exponents(x)
    q = x * _power(-e, x.shape[1], torch.float32)
    most = torch.where(e == 120, 240.0, 448.0).repeat_interleave(BLOCK, dim=1)[:, :x.shape[1]]
    q = torch.where(torch.isfinite(q), torch.minimum(torch.maximum(q, -most), most), torch.full_like(q, math.nan))
    return q.to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _values(codes, scales):
    """What codes stand for, in binary32 (exact)."""
    d = codes.shape[1]
    return codes.contiguous().view(torch.float8_e4m3fn).to(torch.float32) * _power(scales.to(torch.int32) - 127, d, torch.float32)


def prepare(case, seed):
    op, T, d, V, N, dtype = (case[k] for k in ("op", "T", "d", "V", "N", "dtype"))
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    s = dict(case)
    if op in ("lookup", "table_grad"):
        # Zipf's law: a few tokens make up much of the text; some positions are padding
        u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
        s["tokens"] = (torch.exp(u * math.log(V + 1)).to(torch.int64) - 1).clamp(0, V - 1)
        s["tokens"][torch.rand(T, generator=g, device="cuda") < 0.02] = -1
        s["scale"] = math.sqrt(d)
    if op == "lookup":
        s["table"] = _normal(g, V, d, dtype, 0.02)
        s["out"] = torch.empty(T, d, dtype=t, device="cuda")
    elif op == "table_grad":
        s["dy"] = _normal(g, T, d, dtype, 1e-3)
        s["base"] = _normal(g, V, d, "f32", 1e-3) if case["add"] else None
        s["grad"] = torch.empty(V, d, device="cuda")
    elif op == "norm":
        s["x"] = _normal(g, T, d, dtype)
        s["residual"] = _normal(g, T, d, dtype, 3.0, wide=True) if case["add"] else None
        s["weight"] = (1.0 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(t)
        s["y"], s["rstd"] = torch.empty(T, d, dtype=t, device="cuda"), torch.empty(T, device="cuda")
        s["h"] = torch.empty(T, d, dtype=t, device="cuda") if case["add"] else None
    elif op == "norm_grad":
        s["dy"] = _normal(g, T, d, dtype, 1e-3)
        s["h"] = _normal(g, T, d, dtype, 3.0, wide=True)
        s["residual_grad"] = _normal(g, T, d, dtype, 1e-3) if case["add"] else None
        s["weight"] = (1.0 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(t)
        s["rstd"] = torch.rsqrt(s["h"].to(torch.float64).square().mean(dim=1) + EPS).to(torch.float32)
        s["dx"], s["dweight"] = torch.empty(T, d, dtype=t, device="cuda"), torch.empty(d, device="cuda")
    elif op == "checkpoint":
        s["x"] = _normal(g, T, d, dtype, wide=True)
        s["out"] = torch.empty(T, d, dtype=t, device="cuda")
    else:
        s["x"] = _normal(g, T, d, "bf16", wide=True)
        s["dy"] = torch.zeros(T, (N + 7) // 8 * 8, dtype=t, device="cuda")[:, :N]
        s["dy"].copy_(_normal(g, T, N, dtype, 1e-3))
        s["base"] = _normal(g, N, d, "f32", 1e-2) if case["add"] else None
        s["dweight"] = torch.empty(N, d, device="cuda")
    if op == "checkpoint" or op == "weight_grad" or case["coded"]:
        # rows of codes start at multiples of 16 bytes
        s["codes"] = torch.zeros(T, (d + 15) // 16 * 16, dtype=torch.uint8, device="cuda")[:, :d]
        s["scales"] = torch.empty(T, _blocks(d), dtype=torch.uint8, device="cuda")
    if op == "weight_grad" or (op == "norm_grad" and case["coded"]):
        codes, scales = _pack(s.pop("x" if op == "weight_grad" else "h"))
        s["codes"].copy_(codes)
        s["scales"].copy_(scales)
    if own:
        import paper_2412_18052_b200 as gaf
        s["gaf"] = gaf
        if op in ("table_grad", "norm_grad", "weight_grad"):
            s["workspace"] = gaf.new_layer_workspace(T, max(d, N), gaf.GAF_F32 if dtype == "f32" else gaf.GAF_BF16, V=V)
    return s


# --------------------------------------------------------------- operators ----

def _run_own(s):
    gaf, op = s["gaf"], s["op"]
    if op == "lookup":
        return gaf.gaf_embedding(s["table"], s["tokens"], scale=s["scale"], out=s["out"])
    if op == "table_grad":
        return gaf.gaf_embedding_grad(s["dy"], s["tokens"], s["grad"], s["workspace"], scale=s["scale"], base=s["base"])
    if op == "norm":
        checkpoint = (s["codes"], s["scales"]) if s["coded"] else None
        y, h, rstd = gaf.gaf_rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS, y=s["y"], h=s["h"], rstd=s["rstd"],
                                      y_checkpoint=checkpoint, coded_y=s["coded"])
        return {"y": y, "h": h, "rstd": rstd}
    if op == "norm_grad":
        h = (s["codes"], s["scales"]) if s["coded"] else s["h"]
        dx, dweight = gaf.gaf_rms_norm_grad(s["dy"], h, s["weight"], s["rstd"], s["dweight"], s["workspace"],
                                            residual_grad=s["residual_grad"], dx=s["dx"])
        return {"dx": dx, "dweight": dweight}
    if op == "checkpoint":
        checkpoint = gaf.gaf_checkpoint_pack(s["x"], checkpoint=(s["codes"], s["scales"]))
        return gaf.gaf_checkpoint_unpack(checkpoint, out=s["out"])
    return gaf.gaf_linear_weight_grad(s["dy"], (s["codes"], s["scales"]), s["dweight"], s["workspace"], base=s["base"])


def _run_plain(s):
    op = s["op"]
    if op == "lookup":
        ok = (s["tokens"] >= 0) & (s["tokens"] < s["V"])
        rows = s["table"][torch.where(ok, s["tokens"], 0)].to(torch.float32) * s["scale"]
        return torch.where(ok[:, None], rows, 0.0).to(s["table"].dtype)
    if op == "table_grad":
        ok = (s["tokens"] >= 0) & (s["tokens"] < s["V"])
        dy = torch.where(ok[:, None], s["dy"].to(torch.float32), 0.0)
        total = torch.zeros(s["V"], s["d"], device=dy.device).index_add_(0, torch.where(ok, s["tokens"], 0), dy)
        total *= s["scale"]
        return total if s["base"] is None else total + s["base"]
    if op == "norm":
        h = s["x"]
        if s["residual"] is not None:
            h = (h.to(torch.float32) + s["residual"].to(torch.float32)).to(h.dtype)
        v = h.to(torch.float32)
        rstd = 1.0 / torch.sqrt(v.square().mean(dim=1) + EPS)
        y = v * rstd[:, None] * s["weight"].to(torch.float32)
        y = _values(*_pack(y)).to(h.dtype) if s["coded"] else y.to(h.dtype)
        return {"y": y, "h": None if s["residual"] is None else h, "rstd": rstd}
    if op == "norm_grad":
        h = _values(s["codes"], s["scales"]) if s["coded"] else s["h"].to(torch.float32)
        dy, r = s["dy"].to(torch.float32), s["rstd"][:, None]
        wdy, n = dy * s["weight"].to(torch.float32), h * r
        dx = r * (wdy - n * (wdy * n).mean(dim=1, keepdim=True))
        if s["residual_grad"] is not None:
            dx = dx + s["residual_grad"].to(torch.float32)
        return {"dx": dx.to(s["dy"].dtype), "dweight": (dy * n).sum(dim=0)}
    if op == "checkpoint":
        return _values(*_pack(s["x"])).to(s["x"].dtype)
    total = s["dy"].to(torch.float32).t() @ _values(s["codes"], s["scales"])
    return total if s["base"] is None else total + s["base"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


def exact(case, seed):
    """The same from the definitions, in 64 bits.  What is rounded to 8 bits after a sum has no such value: whether it falls
    on one side of a border or the other hangs on the last bit of that sum."""
    s, f = prepare(case, seed), torch.float64
    op = case["op"]
    if op == "lookup":
        out = torch.zeros(case["T"], case["d"], dtype=f, device="cuda")
        at = torch.nonzero((s["tokens"] >= 0) & (s["tokens"] < case["V"])).flatten()
        out[at] = s["table"][s["tokens"][at]].to(f) * s["scale"]
        return out
    if op == "table_grad":
        # sorted tokens, so that each row's terms are one run: the run's sum is a difference of running sums of its columns
        at = torch.nonzero((s["tokens"] >= 0) & (s["tokens"] < case["V"])).flatten()
        out = torch.zeros(case["V"], case["d"], dtype=f, device="cuda") if s["base"] is None else s["base"].to(f)
        if at.numel():
            tokens, order = torch.sort(s["tokens"][at], stable=True)
            rows, count = torch.unique_consecutive(tokens, return_counts=True)
            running = torch.cumsum(s["dy"][at[order]].to(f), dim=0)[count.cumsum(0) - 1]
            running[1:] -= running[:-1].clone()
            out[rows] += running * s["scale"]
        return out
    if op == "norm":
        h, h_exact = s["x"].to(f), None
        if s["residual"] is not None:
            # the stored sum is the definition's: the norm is of what is stored
            h_exact = h + s["residual"].to(f)
            h = h_exact.to(torch.float32).to(s["x"].dtype).to(f)
        rstd = (h.square().sum(dim=1) / case["d"] + EPS).rsqrt()
        y = None if case["coded"] else h * rstd[:, None] * s["weight"].to(f)[None, :]
        return {"y": y, "h": h_exact, "rstd": rstd}
    if op == "norm_grad":
        if case["coded"]:
            h = s["codes"].contiguous().view(torch.float8_e4m3fn).to(f)
            h *= torch.exp2(s["scales"].to(f) - 127.0).repeat_interleave(BLOCK, dim=1)[:, :case["d"]]
        else:
            h = s["h"].to(f)
        dy, r = s["dy"].to(f), s["rstd"].to(f)
        q = torch.einsum("tj,j,tj->t", dy, s["weight"].to(f), h)
        dx = (dy * s["weight"].to(f)) * r[:, None] - h * (r ** 3 * q / case["d"])[:, None]
        if s["residual_grad"] is not None:
            dx += s["residual_grad"].to(f)
        return {"dx": dx, "dweight": torch.einsum("tj,tj,t->j", dy, h, r)}
    if op == "checkpoint":
        x = s["x"].to(f)
        e = _exponents(x).to(f).repeat_interleave(BLOCK, dim=1)[:, :case["d"]]
        q = x * torch.exp2(-e)
        # e4m3: steps of an eighth of the power of two below |q|, of 2^-9 below 2^-6
        step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
        return torch.round(q / step) * step * torch.exp2(e)
    x = s["codes"].contiguous().view(torch.float8_e4m3fn).to(f)
    x *= torch.exp2(s["scales"].to(f) - 127.0).repeat_interleave(BLOCK, dim=1)[:, :case["d"]]
    out = s["dy"].to(f).t() @ x
    return out if s["base"] is None else out + s["base"].to(f)
