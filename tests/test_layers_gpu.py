"""The layers' operators on the GPU against their definitions in binary64 (``layer_reference``)."""
import math

import pytest
import torch

import paper_2412_18052_b200 as gaf
from oracle import gaf_oracle as orc
from paper_2412_18052_b200 import workloads
import layer_reference as ref
from layer_reference import TYPES, assert_close

pytestmark = pytest.mark.gpu

GUARD = 64          # elements before and behind a slice of a flat gradient that a call must leave alone


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype=torch.float32, size=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * size).to(dtype)


def strided(x, pad):
    """The same matrix with rows `pad` elements further apart (what lies between them is NaN: it must not be read into a result)."""
    room = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=x.dtype, device=x.device)
    room[:, :x.shape[1]] = x
    return room[:, :x.shape[1]]


class Slice:
    """A weight's place in a flat micro-gradient, between guards."""
    def __init__(self, shape, dtype):
        n = math.prod(shape)
        self.flat = torch.full((GUARD + (n + 7) // 8 * 8 + GUARD,), 12345.0, dtype=dtype, device="cuda")
        self.view = self.flat[GUARD:GUARD + n].view(shape)
        self.n = n

    def check_guards(self):
        assert bool((self.flat[:GUARD] == 12345.0).all()) and bool((self.flat[GUARD + self.n:] == 12345.0).all())


def workspace(T, width, dtype, V=0):
    """Filled with ones: what a workspace holds must not matter."""
    ws = gaf.new_layer_workspace(T, width, gaf.GAF_F32 if dtype == torch.float32 else gaf.GAF_BF16, V=V)
    ws.fill_(255)
    return ws


# -------------------------------------------------------------- embedding ----

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (1, 50, 8), (7, 3, 100), (33, 1000, 768), (130, 77, 1001), (257, 5000, 1032), (64, 40, 5000)])
def test_embedding(dtype, T, V, d):
    t, g = TYPES[dtype], gen(T + d)
    table, scale = randn(g, V, d, dtype=t), 1.5
    tokens = torch.randint(0, V, (T,), generator=g, device="cuda")
    tokens[::5] = -1                            # padding, on either side of the table
    tokens[3::7] = V
    for tok in (tokens, tokens.to(torch.int32)):
        for tb in (table, strided(table, 8), strided(table, 3)):
            out = torch.full((T, d), float("nan"), dtype=t, device="cuda")
            got = gaf.gaf_embedding(tb, tok, scale=scale, out=out)
            assert got.data_ptr() == out.data_ptr()
            assert_close(got, ref.embedding(table, tokens, scale), 0.0)
            assert bool((got[(tokens < 0) | (tokens >= V)] == 0).all())
    # tokens of any shape, a slice of them that starts anywhere, numbers beyond 32 bits
    far = torch.cat([torch.tensor([2 ** 40, -2 ** 40], device="cuda"), tokens])
    got = gaf.gaf_embedding(table, far[1:])
    assert bool((got[0] == 0).all())
    assert_close(got[1:], ref.embedding(table, tokens, 1.0), 0.0)
    assert gaf.gaf_embedding(table, tokens.view(1, T)).shape == (1, T, d)


def test_embedding_of_nothing():
    table = torch.zeros(0, 64, device="cuda")
    assert bool((gaf.gaf_embedding(table, torch.zeros(5, dtype=torch.int64, device="cuda")) == 0).all())
    assert gaf.gaf_embedding(table, torch.zeros(0, dtype=torch.int64, device="cuda")).shape == (0, 64)


def zipf(g, T, V):
    u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
    return (torch.exp(u * math.log(V + 1)).to(torch.int64) - 1).clamp(0, V - 1)


@pytest.mark.parametrize("grad_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,d", [(0, 5, 64), (1, 1, 1), (31, 1, 64), (32, 1, 1000), (33, 1, 1001), (200, 300, 768), (1000, 3, 520), (5000, 700, 96),
                                   (4099, 9000, 1300)])
def test_embedding_grad(dtype, grad_dtype, T, V, d):
    t, gt, g = TYPES[dtype], TYPES[grad_dtype], gen(T + V + d)
    dy, scale = randn(g, T, d, dtype=t), 0.75
    tokens = zipf(g, T, V)
    tokens[::11] = -1
    tokens[5::13] = V + 3
    ws = workspace(T, d, t, V=V)
    for base_is in ("none", "other", "itself"):
        for d_y, tok in ((dy, tokens), (strided(dy, 5), tokens.to(torch.int32))):
            place = Slice((V, d), gt)
            base = None if base_is == "none" else randn(g, V, d, dtype=gt, size=3.0)
            want, off = ref.embedding_grad(dy, tokens, V, scale, base)
            if base_is == "itself":
                place.view.copy_(base)
                base = place.view
            else:
                place.view.fill_(float("nan"))
            gaf.gaf_embedding_grad(d_y, tok, place.view, ws, scale=scale, base=base)
            assert_close(place.view, want, off, base_is)
            place.check_guards()


@pytest.mark.parametrize("kind", ["all the same", "all padding", "all different", "two by turns"])
def test_embedding_grad_of_unusual_texts(kind):
    T, V, d, g = 20000, 30000, 264, gen(4)
    dy = randn(g, T, d, dtype=torch.bfloat16)
    at = torch.arange(T, device="cuda")
    tokens = {"all the same": torch.full_like(at, 123), "all padding": torch.full_like(at, -7), "all different": torch.randperm(V, generator=g, device="cuda")[:T],
              "two by turns": torch.where(at % 2 == 0, 5, V - 1)}[kind]
    ws = workspace(T, d, torch.bfloat16, V=V)
    want, off = ref.embedding_grad(dy, tokens, V, 1.0)
    first = gaf.gaf_embedding_grad(dy, tokens, torch.full((V, d), float("nan"), device="cuda"), ws)
    assert_close(first, want, off)
    for _ in range(3):                          # bitwise reproducible, whatever order the counters handed out
        again = gaf.gaf_embedding_grad(dy, tokens, torch.empty(V, d, device="cuda"), ws)
        assert torch.equal(first, again)


def test_embedding_grad_beyond_one_bitmap():
    """More positions than one CTA's bitmap holds at once (262,144)."""
    T, V, d, g = 600_001, 12, 8, gen(6)
    dy = randn(g, T, d, dtype=torch.bfloat16)
    tokens = torch.randint(0, V, (T,), generator=g, device="cuda")
    ws = workspace(T, d, torch.bfloat16, V=V)
    want, off = ref.embedding_grad(dy, tokens, V, 1.0)
    first = gaf.gaf_embedding_grad(dy, tokens, torch.empty(V, d, device="cuda"), ws)
    assert_close(first, want, off)
    assert torch.equal(first, gaf.gaf_embedding_grad(dy, tokens, torch.empty(V, d, device="cuda"), ws))


def test_embedding_far_into_a_table():
    """Rows of a table, and of its gradient, beyond 2^31 elements."""
    V, d = 600_000, 4096
    table = torch.empty(V, d, dtype=torch.bfloat16, device="cuda")
    tokens = torch.tensor([0, V - 1, 555_555, 524_288, 524_287], device="cuda")
    table[tokens] = randn(gen(1), 5, d, dtype=torch.bfloat16)
    assert torch.equal(gaf.gaf_embedding(table, tokens), table[tokens])
    dy = randn(gen(2), 5, d, dtype=torch.bfloat16)
    gaf.gaf_embedding_grad(dy, tokens, table, workspace(5, d, torch.bfloat16, V=V))
    assert torch.equal(table[tokens], dy)
    table[tokens] = 0
    for lo in range(0, V, 100_000):
        assert not bool(table[lo:lo + 100_000].any())


# ------------------------------------------------------------- checkpoints ----

def awkward(g, T, d, t):
    """Values of many sizes: blocks of zeros, subnormal and huge numbers, ties, one large among small, infinities and NaN."""
    x = torch.randn(T, d, generator=g, device="cuda", dtype=torch.float64) * torch.exp2(torch.randint(-30, 30, (T, 1), generator=g, device="cuda").double())
    rows = torch.arange(T, device="cuda") % 11
    x[rows == 1] = 0.0
    x[rows == 2] *= 2.0 ** -100
    x[rows == 3] = torch.sign(x[rows == 3]) * 3.0e38
    x[rows == 4] = torch.randint(-1000, 1000, (int((rows == 4).sum()), d), generator=g, device="cuda").double() / 16
    x[rows == 5, ::3] = float("inf")
    x[rows == 6, 1::5] = float("nan")
    x[rows == 7, 0] = 1e30
    x[rows == 8] = -float("inf")
    x[rows == 9] = 448.0 * 2.0 ** 5
    x[rows == 10] = 1e-42
    return x.to(t)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,d", [(1, 1), (3, 8), (40, 100), (22, 127), (22, 128), (33, 129), (55, 256), (66, 1111), (44, 4096), (13, 8200)])
def test_checkpoint(dtype, T, d):
    t = TYPES[dtype]
    x = awkward(gen(d), T, d, t)
    want = ref.values(x.to(torch.float64))
    _, e = ref.codes(x.to(torch.float64))
    for m in (x, strided(x, 8), strided(x, 5)):
        ck = gaf.gaf_checkpoint_pack(m)
        assert torch.equal(ck[1].to(torch.float64), e + 127)
        got = ref.checkpoint_values(ck)
        assert torch.equal(got.nan_to_num(nan=7e77), want.nan_to_num(nan=7e77))
        for out_t in (torch.float32, torch.bfloat16):
            for room in (torch.empty(T, d, dtype=out_t, device="cuda"), torch.empty(T, d + 5, dtype=out_t, device="cuda")[:, :d]):
                v = gaf.gaf_checkpoint_unpack(ck, out=room)
                assert torch.equal(v.to(torch.float64).nan_to_num(nan=7e77), want.nan_to_num(nan=7e77))
    # half a step of e4m3: 2^-4 of the value, and of the smallest step below
    fine = torch.isfinite(x) & (x.abs() < 2.0 ** 126)
    far = (want - x.to(torch.float64)).abs()
    step = 2.0 ** -10 * torch.exp2(e).repeat_interleave(128, dim=1)[:, :d]
    assert bool((far <= torch.maximum(2.0 ** -4 * x.to(torch.float64).abs(), step))[fine].all())


def test_checkpoint_leaves_the_space_between_rows():
    x = randn(gen(3), 20, 100)
    codes = torch.full((20, 128), 77, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(20, 1, dtype=torch.uint8, device="cuda")
    gaf.gaf_checkpoint_pack(x, (codes[:, :100], scales))
    assert bool((codes[:, 100:] == 77).all())
    out = torch.full((20, 128), 5.0, device="cuda")
    gaf.gaf_checkpoint_unpack((codes[:, :100], scales), out=out[:, :100])
    assert bool((out[:, 100:] == 5.0).all())


def test_checkpoint_of_every_code():
    """Every byte with every scale that a checkpoint can have, back to its value."""
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(241, 1)
    scales = (torch.arange(-120, 121, device="cuda") + 127).to(torch.uint8)[:, None].repeat(1, 2)
    got = gaf.gaf_checkpoint_unpack((codes, scales), dtype=torch.float32)
    want = codes.view(torch.float8_e4m3fn).to(torch.float64) * torch.exp2(scales[:, :1].to(torch.float64) - 127)
    want = want.to(torch.float32)               # (256 * 2^120 and above are infinite: pack writes no such code)
    assert torch.equal(got.nan_to_num(nan=1.0), want.nan_to_num(nan=1.0))


# -------------------------------------------------------------------- norm ----

WIDTHS = [1, 8, 100, 256, 768, 1001, 1024, 1032, 2048, 3000, 4096, 5001, 8192, 12000, 16384]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_rms_norm(dtype, d):
    t, g, eps = TYPES[dtype], gen(d), 1e-5
    for T in (1, 5, 131):
        x, res, w = randn(g, T, d, dtype=t), randn(g, T, d, dtype=t, size=4.0), randn(g, d, dtype=t)
        for residual in (None, res):
            for pad in (0, 8, 3):
                xs, rs = strided(x, pad), None if residual is None else strided(residual, pad)
                h_want, r, y = ref.rms_norm(x, residual, w, eps, t)
                yc, hc = gaf.new_checkpoint(T, d), gaf.new_checkpoint(T, d)
                got, h, rstd = gaf.gaf_rms_norm(xs, w, residual=rs, eps=eps, y_checkpoint=yc, h_checkpoint=hc)
                assert_close(rstd, r, ref.RSTD * r, "rstd")
                assert_close(got, y, (ref.RSTD + 2 * ref.U) * y.abs(), "y")
                if residual is None:
                    assert h is None
                else:
                    assert torch.equal(h, h_want)
                # the checkpoint of h is that of a known matrix; that of y is of a value that may be RSTD off before it is rounded: half a step more
                # than that, and a whole step where that crosses a border
                assert torch.equal(ref.checkpoint_values(hc), ref.values(h_want.to(torch.float64)))
                step = torch.exp2(yc[1].to(torch.float64) - 127 - 10).repeat_interleave(128, dim=1)[:, :d]
                far = (ref.checkpoint_values(yc) - y).abs()
                assert bool((far <= torch.maximum(2.0 ** -4 * y.abs(), step) * (1 + 2 ** -10) + 4 * ref.RSTD * y.abs()).all())
                # values of the codes instead of y
                coded, _, _ = gaf.gaf_rms_norm(xs, w, residual=rs, eps=eps, y_checkpoint=yc, coded_y=True)
                assert torch.equal(coded.to(torch.float64), ref.checkpoint_values(yc))


def test_rms_norm_in_place_and_optional_outputs():
    g = gen(9)
    for d in (768, 1001):
        x, res, w = randn(g, 50, d), randn(g, 50, d), randn(g, d)
        want_h, _, want = ref.rms_norm(x, res, w, 1e-6, torch.float32)
        for into in ("residual", "x"):
            a, b = x.clone(), res.clone()
            y, h, _ = gaf.gaf_rms_norm(a, w, residual=b, h=b if into == "residual" else a)
            assert torch.equal(h, want_h) and h.data_ptr() == (b if into == "residual" else a).data_ptr()
            assert_close(y, want, (ref.RSTD + 2 * ref.U) * want.abs())
        y, h, rstd = gaf.gaf_rms_norm(x, w, want_y=False)
        assert y is None and h is None
        ck = gaf.new_checkpoint(50, d)
        y, _, _ = gaf.gaf_rms_norm(x, w, want_y=False, y_checkpoint=ck)
        full = gaf.new_checkpoint(50, d)
        gaf.gaf_rms_norm(x, w, y_checkpoint=full)
        assert y is None and torch.equal(ck[0], full[0]) and torch.equal(ck[1], full[1])
    x3, w3 = randn(g, 2, 5, 64), randn(g, 64)
    y, _, rstd = gaf.gaf_rms_norm(x3, w3)
    assert y.shape == (2, 5, 64) and rstd.shape == (2, 5)
    y, _, rstd = gaf.gaf_rms_norm(x3[:, :0], w3)
    assert y.shape == (2, 0, 64)


def test_rms_norm_rows_are_alone():
    """Zeros, infinities and NaN stay in their rows."""
    x, w = randn(gen(2), 9, 512), randn(gen(3), 512)
    x[2] = 0
    x[4, 7] = float("inf")
    x[6, 9] = float("nan")
    clean = [0, 1, 3, 5, 7, 8]
    y, _, rstd = gaf.gaf_rms_norm(x, w, eps=1e-6)
    _, r, want = ref.rms_norm(x, None, w, 1e-6, torch.float32)
    assert_close(y[clean], want[clean], (ref.RSTD + 2 * ref.U) * want[clean].abs())
    assert bool((y[2] == 0).all()) and abs(rstd[2].item() - 1000.0) < 1e-3
    assert rstd[4].item() == 0 and bool(torch.isnan(y[4, 7])) and bool((y[4, :7] == 0).all()) and bool(torch.isnan(y[6]).all())


@pytest.mark.parametrize("grad_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_rms_norm_grad(dtype, grad_dtype, d):
    t, gt, g = TYPES[dtype], TYPES[grad_dtype], gen(d + 1)
    for T in (0, 1, 3, 6, 2500 if d <= 1032 else 700):
        dy, h, w, res = randn(g, T, d, dtype=t), randn(g, T, d, dtype=t, size=3.0), randn(g, d, dtype=t), randn(g, T, d, dtype=t)
        rstd = (h.double().square().mean(dim=1) + 1e-6).rsqrt().float()
        ck = gaf.gaf_checkpoint_pack(h)
        ws = workspace(T, d, t)
        base = randn(g, d, dtype=gt)
        for coded in (False, True):
            for pad, residual, b in ((0, None, None), (8, res, base), (3, res, None)):
                hv = ref.checkpoint_values(ck) if coded else h.double()
                place = Slice((d,), gt)
                place.view.fill_(float("nan"))
                dx, _ = gaf.gaf_rms_norm_grad(strided(dy, pad), ck if coded else strided(h, pad), w, rstd, place.view, ws,
                                              residual_grad=None if residual is None else strided(residual, pad), base=b)
                want_x, want_w, off_x, off_w = ref.rms_norm_grad(dy, hv, w, rstd, residual, b)
                assert_close(dx, want_x, off_x, "dx")
                assert_close(place.view, want_w, off_w, "dweight")
                place.check_guards()


def test_rms_norm_grad_in_place():
    g = gen(12)
    for d in (256, 4096, 1001):
        dy, h, w, res, base = randn(g, 333, d), randn(g, 333, d), randn(g, d), randn(g, 333, d), randn(g, d)
        rstd, ws = (h.double().square().mean(dim=1)).rsqrt().float(), workspace(333, d, torch.float32)
        want, want_w = gaf.gaf_rms_norm_grad(dy, h, w, rstd, torch.empty(d, device="cuda"), ws, residual_grad=res, base=base)
        for into in ("dy", "res"):
            a, b, c = dy.clone(), res.clone(), base.clone()
            dx, dw = gaf.gaf_rms_norm_grad(a, h, w, rstd, c, ws, residual_grad=b, dx=a if into == "dy" else b, base=c)
            assert torch.equal(dx, want) and torch.equal(dw, want_w)


def test_rms_norm_grad_against_differences():
    """dx and dw against central differences of the norm in binary64."""
    T, d, g, eps = 3, 40, gen(5), 1e-3
    x, w, dy = (randn(g, *s).double() for s in ((T, d), (d,), (T, d)))

    def loss(x, w):
        return (dy * x * (x.square().mean(dim=1, keepdim=True) + eps).rsqrt() * w).sum()
    y, _, rstd = gaf.gaf_rms_norm(x.float(), w.float(), eps=eps)
    dw = torch.empty(d, device="cuda")
    dx, _ = gaf.gaf_rms_norm_grad(dy.float(), x.float(), w.float(), rstd, dw, workspace(T, d, torch.float32))
    # step 1e-4 in binary64: the third derivative leaves about 1e-8, rounding 1e-12 / 1e-4; the kernel's own error is of the order of 1e-6
    s = 1e-4
    for t in range(T):
        for j in range(0, d, 7):
            e = torch.zeros_like(x)
            e[t, j] = s
            assert abs((loss(x + e, w) - loss(x - e, w)).item() / (2 * s) - dx[t, j].item()) < 2e-5
    for j in range(0, d, 5):
        e = torch.zeros_like(w)
        e[j] = s
        assert abs((loss(x, w + e) - loss(x, w - e)).item() / (2 * s) - dw[j].item()) < 2e-5


# ------------------------------------------------------------ weight grad ----

@pytest.mark.parametrize("T,N,M", [(1, 1, 1), (16, 64, 128), (64, 256, 128), (65, 8, 130), (300, 768, 768), (1000, 100, 1111), (513, 1024, 64), (2100, 257, 384),
                                   (3000, 40, 40)])
def test_linear_weight_grad_of_whole_numbers(T, N, M):
    """Small whole numbers: every product and sum is exact, so that the result is too (a wrong place, scale or token would show)."""
    g = gen(T)
    x = torch.randint(-3, 4, (T, M), generator=g, device="cuda").float() * torch.exp2(torch.randint(0, 4, (T, 1), generator=g, device="cuda").float())
    dy = torch.randint(-4, 5, (T, N), generator=g, device="cuda").float()
    ck = gaf.gaf_checkpoint_pack(x)
    assert torch.equal(ref.checkpoint_values(ck), x.double())
    want = (dy.double().t() @ x.double()).float()
    for t in (torch.bfloat16, torch.float32):
        ws = workspace(T, max(N, M), t)
        for d_y in (strided(dy.to(t), -N % 8 + 8), strided(dy.to(t), 1), dy.to(t)):
            place = Slice((N, M), torch.float32)
            place.view.fill_(float("nan"))
            gaf.gaf_linear_weight_grad(d_y, ck, place.view, ws)
            assert gaf.gaf_read_status(ws) == 0
            assert torch.equal(place.view, want), t
            place.check_guards()


@pytest.mark.parametrize("grad_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,M", [(0, 5, 7), (1, 9, 200), (100, 130, 257), (777, 768, 640), (5000, 384, 130), (4096, 1000, 1100)])
def test_linear_weight_grad(dtype, grad_dtype, T, N, M):
    t, gt, g = TYPES[dtype], TYPES[grad_dtype], gen(T + N)
    x = randn(g, T, M) * torch.exp2(torch.randint(-20, 20, (T, 1), generator=g, device="cuda").float())
    ck = gaf.gaf_checkpoint_pack(x)
    xv = ref.checkpoint_values(ck)
    dy = torch.zeros(T, (N + 7) // 8 * 8, dtype=t, device="cuda")[:, :N]
    dy.copy_(randn(g, T, N) * torch.exp2(torch.randint(-10, 10, (T, 1), generator=g, device="cuda").float()))
    ws = workspace(T, max(N, M), t)
    for base_is in ("none", "other", "itself"):
        place = Slice((N, M), gt)
        base = None if base_is == "none" else randn(g, N, M, dtype=gt)
        want, off = ref.weight_grad(dy, xv, base)
        if base_is == "itself":
            place.view.copy_(base)
            base = place.view
        else:
            place.view.fill_(float("nan"))
        gaf.gaf_linear_weight_grad(dy, ck, place.view, ws, base=base)
        assert gaf.gaf_read_status(ws) == 0
        assert_close(place.view, want, off, base_is)
        place.check_guards()


def test_linear_weight_grad_scales_and_special_values():
    """Every scale, subnormal codes, NaN codes and infinite gradients: what reaches one entry reaches no other."""
    T, N, M, g = 241, 72, 256, gen(8)
    codes = torch.randint(0, 256, (T, M), generator=g, device="cuda").to(torch.uint8)
    codes[(codes & 127) == 127] = 1
    scales = (torch.arange(-120, 121, device="cuda") + 127).to(torch.uint8)[:, None].repeat(1, 2)
    ck = (codes, scales)
    # each token has one column of its own of dy, so that each entry is one product
    for lo in range(0, T, N):
        dy = torch.zeros(T, N, dtype=torch.bfloat16, device="cuda")
        n = min(N, T - lo)
        dy[torch.arange(lo, lo + n), torch.arange(n)] = 1.0
        got = gaf.gaf_linear_weight_grad(dy, ck, torch.empty(N, M, device="cuda"), workspace(T, M, torch.bfloat16))
        want = ref.checkpoint_values((codes[lo:lo + n], scales[lo:lo + n])).float()
        # 256 * 2^120 and above are infinite in a product's operand, and infinity times the other tokens' zeros is NaN: pack writes no such code
        fine = (want.abs() < 2.0 ** 127) & (want.abs() >= 2.0 ** -126)
        bad_columns = (ref.checkpoint_values(ck).abs() >= 2.0 ** 128).any(dim=0)
        fine[:, bad_columns] = False
        assert torch.equal(got[:n][fine], want[fine])
    x = randn(g, T, M)
    x[5, 7], x[100, 200] = float("nan"), float("inf")
    dy = randn(g, T, N, dtype=torch.bfloat16)
    dy[9, 3] = float("inf")
    got = gaf.gaf_linear_weight_grad(dy, gaf.gaf_checkpoint_pack(x), torch.empty(N, M, device="cuda"), workspace(T, M, torch.bfloat16))
    bad = torch.zeros(N, M, dtype=torch.bool, device="cuda")
    bad[:, 7] = bad[:, 200] = bad[3] = True
    assert not bool(torch.isfinite(got)[bad].any()) and bool(torch.isfinite(got)[~bad].all())


def test_linear_weight_grad_accuracy():
    """Long sums: no further from binary64 than 1e-6 of the result's norm.  A chain has 32 steps of the tensor core, each of which cuts off up
    to 2 U of the sum so far, half of that on average, and the sum so far is half of the chain's on average where all terms agree (less for others):
    16 U for a chain; then up to 64 chains rounded to nearest, whose errors do not add up: under 16 U = 9.6e-7."""
    g = gen(31)
    for T, N, M in ((16384, 256, 256), (8192, 512, 1024)):
        ck, dy = gaf.gaf_checkpoint_pack(randn(g, T, M)), randn(g, T, N, dtype=torch.bfloat16)
        for shift in (0.0, 2.0):                # terms of either sign, and a sum that grows steadily
            d_y = (dy.float() + shift).to(torch.bfloat16)
            c = ck if shift == 0 else gaf.gaf_checkpoint_pack(randn(g, T, M).abs())
            got = gaf.gaf_linear_weight_grad(d_y, c, torch.empty(N, M, device="cuda"), workspace(T, M, torch.bfloat16)).double()
            want = d_y.double().t() @ ref.checkpoint_values(c)
            assert ((got - want).norm() / want.norm()).item() < 16 * ref.U


def test_linear_weight_grad_bounded_waits():
    """An awaited copy that never counts as complete: the call ends, says so, and the next one is right."""
    g = gen(14)
    ck, dy = gaf.gaf_checkpoint_pack(randn(g, 700, 300)), randn(g, 700, 520, dtype=torch.bfloat16)
    ws, dw = workspace(700, 520, torch.bfloat16), torch.empty(520, 300, device="cuda")
    gaf.gaf_test_set_wait_fault(50, 1)
    try:
        gaf.gaf_linear_weight_grad(dy, ck, dw, ws)
        assert gaf.gaf_read_status(ws) & gaf.GAF_STATUS_TIMEOUT
    finally:
        gaf.gaf_test_set_wait_fault(0, False)
    gaf.gaf_linear_weight_grad(dy, ck, dw, ws)
    assert gaf.gaf_read_status(ws) == 0
    assert_close(dw, *ref.weight_grad(dy, ref.checkpoint_values(ck)))


# ---------------------------------------------------------------- together ----

class Model(workloads.LanguageModel):
    def check(self, s, flat):
        """Every gradient against binary64, from the activations and gradients that the step itself had."""
        g = self.views(flat)
        v = ref.checkpoint_values
        dx, dw, ox, ow = ref.rms_norm_grad(s["dy2"], v(s["h2c"]), self.w2, s["r2"])
        assert_close(s["dh2"], dx, ox, "dh2")
        assert_close(g["w2"], dw, ow, "w2")
        dx, dw, ox, ow = ref.rms_norm_grad(s["dy1"], v(s["h1c"]), self.w1, s["r1"], s["dh2"])
        assert_close(s["de"], dx, ox, "de")
        assert_close(g["w1"], dw, ow, "w1")
        assert_close(g["lin"], *ref.weight_grad(s["dh2"], v(s["y1c"])), "lin")
        out_layer, o1 = ref.weight_grad(s["dlogits"], v(s["y2c"]))
        table, o2 = ref.embedding_grad(s["de"], s["tokens"], self.V, math.sqrt(self.d))
        assert_close(g["table"], out_layer + table, o1 + o2 + 4 * ref.U * (out_layer.abs() + table.abs()), "table")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [600, 301])
def test_micro_gradients_of_a_language_model_are_filtered(V, dtype):
    K, T, d = 4, 200, 264
    m = Model(V, d, 3, dtype=TYPES[dtype])
    ws = m.new_workspace(T)
    flats, g = [torch.zeros(m.D, device="cuda") for _ in range(K)], gen(77)
    for k, flat in enumerate(flats):
        m.check(m.micro_gradient(m.tokens(T, k), torch.randint(0, V, (T,), generator=g, device="cuda"), flat, ws), flat)
    filter_ws = gaf.new_workspace(K, m.D, gaf.GAF_F32)
    macro, mask, dist, count = gaf.gaf_filter_accumulate(flats, 0.97, filter_ws)
    want = orc.filter_accumulate([workloads.as_numpy_bits(f) for f in flats], 0.97)
    near = abs(want.dist - 0.97) < 1e-5
    assert not near.any() and mask.cpu().numpy().tolist() == want.mask.tolist() and int(count.item()) == want.count
    assert float(abs(dist.cpu().numpy() - want.dist).max()) < 1e-5


def test_language_model_workload():
    """The workload's micro-gradients, in both types, through the filter and its bucketed form."""
    for dtype, code in (("f32", gaf.GAF_F32), ("bf16", gaf.GAF_BF16)):
        w = workloads.language_model(3, 500, 128, 150, seed=2, dtype=dtype)
        want = orc.filter_accumulate([workloads.as_numpy_bits(f) for f in w.grads], 0.97)
        ws = gaf.new_workspace(w.K, w.D, code)
        macro, mask, dist, count = gaf.gaf_filter_accumulate(w.grads, 0.97, ws)
        assert float(abs(dist.cpu().numpy() - want.dist).max()) < 1e-5 and mask.cpu().numpy().tolist() == want.mask.tolist()
        offsets = workloads.LanguageModel(500, 128, 2).offsets
        _, m, _, c = gaf.gaf_filter_accumulate_bucketed(w.grads, 0.97, offsets, ws)
        assert m.shape == (4, 3) and bool((c >= 1).all())


def test_one_workspace_serves_layers_and_filter():
    """The layers leave alone what the filter keeps in a workspace from call to call."""
    K, T, V, d = 4, 150, 300, 128
    m = Model(V, d, 5)
    n = max(gaf.gaf_layer_workspace_bytes(T, V, gaf.GAF_BF16, V), gaf.gaf_workspace_bytes(K, m.D, gaf.GAF_F32))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    gaf.gaf_workspace_init(ws)
    alone = gaf.new_workspace(K, m.D, gaf.GAF_F32)
    g = gen(78)
    flats = [torch.zeros(m.D, device="cuda") for _ in range(K)]
    for round_ in range(4):
        for flat in flats:
            m.micro_gradient(zipf(g, T, V), torch.randint(0, V, (T,), generator=g, device="cuda"), flat, ws)
        for k in (2, 3, 4):
            got = gaf.gaf_filter_accumulate(flats[:k], 0.97, ws)
            want = gaf.gaf_filter_accumulate(flats[:k], 0.97, alone)
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_captured_and_on_another_stream():
    """The whole microbatch captured into a graph, replayed on new inputs; and issued on a stream of its own."""
    T, V, d = 300, 500, 256
    m = Model(V, d, 6)
    g = gen(79)
    ws = gaf.new_layer_workspace(T, max(V, d), gaf.GAF_BF16, V=V)
    batches = [(zipf(g, T, V), torch.randint(0, V, (T,), generator=g, device="cuda")) for _ in range(3)]
    want = []
    for tokens, targets in batches:
        flat = torch.zeros(m.D, device="cuda")
        m.micro_gradient(tokens, targets, flat, ws)
        want.append(flat)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for (tokens, targets), w in zip(batches, want):
            flat = torch.zeros(m.D, device="cuda")
            m.micro_gradient(tokens, targets, flat, ws)
            side.synchronize()
            assert torch.equal(flat, w)
    torch.cuda.synchronize()
    tokens, targets, flat = batches[0][0].clone(), batches[0][1].clone(), torch.zeros(m.D, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.micro_gradient(tokens, targets, flat, ws)
    for (a, b), w in list(zip(batches, want)) * 2:
        tokens.copy_(a)
        targets.copy_(b)
        flat.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(flat, w)


def test_binding_refusals():
    x, w, ws = randn(gen(1), 4, 64), randn(gen(2), 64), workspace(4, 64, torch.float32, V=10)
    tokens, bf = torch.zeros(4, dtype=torch.int64, device="cuda"), randn(gen(3), 4, 64, dtype=torch.bfloat16)
    ck = gaf.gaf_checkpoint_pack(x)
    for call in (lambda: gaf.gaf_embedding(x, tokens[None, ::2]), lambda: gaf.gaf_embedding(x[None], tokens), lambda: gaf.gaf_embedding(x, tokens, out=bf),
                 lambda: gaf.gaf_embedding(x, tokens, out=x[:3]), lambda: gaf.gaf_embedding_grad(x, tokens[:3], x.clone(), ws),
                 lambda: gaf.gaf_embedding_grad(x, tokens, torch.zeros(10, 63, device="cuda"), ws),
                 lambda: gaf.gaf_embedding_grad(x, tokens, torch.zeros(10, 64, device="cuda"), ws, base=torch.zeros(9, 64, device="cuda")),
                 lambda: gaf.gaf_rms_norm(x, w[:63]), lambda: gaf.gaf_rms_norm(bf, w), lambda: gaf.gaf_rms_norm(x, w, residual=bf),
                 lambda: gaf.gaf_rms_norm(x.t(), w[:4]), lambda: gaf.gaf_rms_norm(x, w, h=x.clone()), lambda: gaf.gaf_rms_norm(x, w, y=bf),
                 lambda: gaf.gaf_rms_norm(x, w, y_checkpoint=(ck[0][:3], ck[1])), lambda: gaf.gaf_rms_norm_grad(x, None, w, w[:4], w.clone(), ws),
                 lambda: gaf.gaf_rms_norm_grad(x, bf, w, w[:4], w.clone(), ws), lambda: gaf.gaf_rms_norm_grad(x, x, w, w[:3], w.clone(), ws),
                 lambda: gaf.gaf_linear_weight_grad(x, ck, torch.zeros(64, 63, device="cuda"), ws),
                 lambda: gaf.gaf_linear_weight_grad(x[:3], ck, torch.zeros(64, 64, device="cuda"), ws), lambda: gaf.gaf_checkpoint_unpack(ck, out=x[:3])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: gaf.gaf_embedding(x, tokens.float()), lambda: gaf.gaf_embedding(x.double(), tokens), lambda: gaf.gaf_rms_norm(x.half(), w.half()),
                 lambda: gaf.gaf_checkpoint_pack(x, (ck[0].int(), ck[1])), lambda: gaf.gaf_linear_weight_grad(x.half(), ck, torch.zeros(64, 64, device="cuda"), ws)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: gaf.gaf_rms_norm(x[:1].expand(4, 64), w), lambda: gaf.gaf_embedding_grad(x, tokens, torch.zeros(10, 64, device="cuda"), ws[:256]),
                 lambda: gaf.gaf_embedding(x.flatten()[1:65].view(1, 64), tokens), lambda: gaf.gaf_checkpoint_pack(x, (ck[0].flatten()[:4 * 40].view(4, 40), ck[1]))):
        with pytest.raises((gaf.GafError, ValueError)):
            call()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nothing_is_written_outside_a_workspace(dtype):
    """A workspace of exactly the size asked for: what lies before and behind it, and what the filter keeps in it, stays as it was."""
    t, g = TYPES[dtype], gen(40)
    code = gaf.GAF_F32 if dtype == "f32" else gaf.GAF_BF16
    for T, width, V in ((1, 1, 1), (40, 300, 20), (3000, 264, 50), (700, 1000, 3000)):
        n = gaf.gaf_layer_workspace_bytes(T, width, code, V)
        room = torch.full((n + 4096,), 77, dtype=torch.uint8, device="cuda")
        ws = room[1024:1024 + n]
        d = width
        dy, tokens = randn(g, T, d, dtype=t), zipf(g, T, V)
        gaf.gaf_embedding_grad(dy, tokens, torch.empty(V, d, device="cuda"), ws)
        h, w = randn(g, T, d, dtype=t), randn(g, d, dtype=t)
        gaf.gaf_rms_norm_grad(dy, h, w, torch.ones(T, device="cuda"), torch.empty(d, device="cuda"), ws)
        gaf.gaf_linear_weight_grad(dy, gaf.gaf_checkpoint_pack(h), torch.empty(d, d, device="cuda"), ws)
        assert gaf.gaf_read_status(ws) == 0
        assert bool((room[:1024] == 77).all()) and bool((room[1024 + n:] == 77).all())
        kept = room[1024:1024 + 53248 + 138240]          # control block, partial sums, words that CTAs exchange
        assert int((kept != 77).sum()) <= 4              # (the status word)
        with pytest.raises(gaf.GafError):
            gaf.gaf_embedding_grad(dy, tokens, torch.empty(V, d, device="cuda"), ws[:1024])


def test_two_streams_and_two_graphs_at_once():
    """The same work on two streams side by side, and two captured graphs replayed together, each with a workspace of its own."""
    T, V, d = 700, 900, 520
    m = Model(V, d, 8)
    g = gen(80)
    batches = [(m.tokens(T, 50 + k), torch.randint(0, V, (T,), generator=g, device="cuda")) for k in range(2)]
    spaces = [m.new_workspace(T) for _ in range(2)]
    want = []
    for tokens, targets in batches:
        flat = torch.zeros(m.D, device="cuda")
        m.micro_gradient(tokens, targets, flat, spaces[0])
        want.append(flat)
    torch.cuda.synchronize()
    streams, flats = [torch.cuda.Stream() for _ in range(2)], [torch.zeros(m.D, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                flats[k].zero_()
                m.micro_gradient(*batches[k], flats[k], spaces[k])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(flats, want))
    graphs = []
    for k in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            m.micro_gradient(*batches[k], flats[k], spaces[k])
        graphs.append(graph)
    for _ in range(3):
        for f in flats:
            f.zero_()
        torch.cuda.synchronize()
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                graphs[k].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(flats, want))


def test_everything_is_reproducible():
    """Bit for bit, call after call, whatever ran in between."""
    g = gen(90)
    T, d, V, N = 3000, 776, 400, 520
    dy, h, w, tokens = randn(g, T, d, dtype=torch.bfloat16), randn(g, T, d, dtype=torch.bfloat16), randn(g, d, dtype=torch.bfloat16), zipf(g, T, V)
    dyn, rstd, ck = randn(g, T, N, dtype=torch.bfloat16), torch.ones(T, device="cuda"), gaf.gaf_checkpoint_pack(h)
    ws = workspace(T, d, torch.bfloat16, V=V)

    def run():
        a = gaf.gaf_embedding_grad(dy, tokens, torch.empty(V, d, device="cuda"), ws)
        b = gaf.gaf_rms_norm_grad(dy, ck, w, rstd, torch.empty(d, device="cuda"), ws)
        c = gaf.gaf_linear_weight_grad(dyn, ck, torch.empty(N, d, device="cuda"), ws)
        return [a, *b, c]
    first = run()
    for _ in range(5):
        ws.random_()
        assert all(torch.equal(x, y) for x, y in zip(run(), first))


def test_dense_neighbours_of_every_alignment():
    """Weights' slices at every place of a flat gradient that the library takes: multiples of 16 bytes that are none of 32."""
    g = gen(91)
    T, d, V = 300, 264, 120
    dy, tokens = randn(g, T, d), zipf(g, T, V)
    h, w, rstd, ck = randn(g, T, d), randn(g, d), torch.ones(T, device="cuda"), gaf.gaf_checkpoint_pack(randn(g, T, d))
    ws = workspace(T, d, torch.float32, V=V)
    for gt, shift in ((torch.float32, 4), (torch.float32, 8), (torch.bfloat16, 8), (torch.bfloat16, 24)):
        flat = torch.full((V * d + 2 * d * d + 200,), 7.0, dtype=gt, device="cuda")
        a, b = flat[shift:shift + V * d].view(V, d), flat[V * d + 40 + shift:V * d + 40 + shift + d]
        c = flat[V * d + d + 80 + shift:V * d + d + 80 + shift + d * d].view(d, d)
        gaf.gaf_embedding_grad(dy, tokens, a, ws)
        assert_close(a, *ref.embedding_grad(dy, tokens, V, 1.0))
        _, dw = gaf.gaf_rms_norm_grad(dy, h, w, rstd, b, ws)
        _, want, _, off = ref.rms_norm_grad(dy, h.double(), w, rstd)
        assert_close(b, want, off)
        gaf.gaf_linear_weight_grad(dy, ck, c, ws)
        assert_close(c, *ref.weight_grad(dy, ref.checkpoint_values(ck)))
        used = torch.zeros_like(flat, dtype=torch.bool)
        for v in (a, b, c):
            lo = (v.data_ptr() - flat.data_ptr()) // flat.element_size()
            used[lo:lo + v.numel()] = True
        assert bool((flat[~used] == 7.0).all())
    # matrices whose rows are 16 bytes, not 32, from a boundary
    x = torch.zeros(T * (d + 4) + 4, device="cuda")[4:].view(T, d + 4)[:, :d]
    x.copy_(h)
    y, _, _ = gaf.gaf_rms_norm(x, w)
    _, _, want = ref.rms_norm(h, None, w, 1e-6, torch.float32)
    assert_close(y, want, (ref.RSTD + 2 * ref.U) * want.abs())


@pytest.mark.parametrize("grad_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,d", [(5000, 1), (3001, 3), (4096, 7), (2050, 33), (1000, 64), (999, 250), (700, 257), (515, 1030)])
def test_embedding_grad_of_rows_that_do_not_occur(V, d, grad_dtype):
    """Runs of absent rows of every length, at every alignment: zeros, or base, and nothing else."""
    g, gt = gen(V + d), TYPES[grad_dtype]
    T = 60
    dy = randn(g, T, d, dtype=torch.bfloat16)
    tokens = torch.randint(0, V, (T,), generator=g, device="cuda")
    tokens[:8] = torch.tensor([0, 1, 31, 32, 33, V // 2, V // 2 - 1, V - 1], device="cuda")
    ws = workspace(T, d, torch.bfloat16, V=V)
    for base in (None, randn(g, V, d, dtype=gt)):
        place = Slice((V, d), gt)
        place.view.fill_(float("nan"))
        gaf.gaf_embedding_grad(dy, tokens, place.view, ws, base=base)
        absent = torch.ones(V, dtype=torch.bool, device="cuda")
        absent[tokens] = False
        want = torch.zeros(V, d, dtype=gt, device="cuda") if base is None else base
        assert torch.equal(place.view[absent], want[absent])
        assert_close(place.view, *ref.embedding_grad(dy, tokens, V, 1.0, base))
        place.check_guards()
