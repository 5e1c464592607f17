"""What the layers' calls leave for later calls to find, and what they do at the edges of their arguments: status words, values that are not finite,
arguments of odd kinds, long texts."""
import math
import weakref

import pytest
import torch

import paper_2412_18052_b200 as gaf
from paper_2412_18052_b200 import workloads
import layer_reference as ref
from layer_reference import TYPES, assert_close

pytestmark = pytest.mark.gpu


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype=torch.float32, size=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * size).to(dtype)


class Layers:
    """One call of each of the gradients on a workspace."""
    T, d, V = 200, 264, 300

    def __init__(self, seed=1):
        g = gen(seed)
        self.dy, self.h, self.w = randn(g, self.T, self.d), randn(g, self.T, self.d), randn(g, self.d)
        self.rstd, self.ck = torch.ones(self.T, device="cuda"), gaf.gaf_checkpoint_pack(self.h)
        self.tokens = torch.randint(0, self.V, (self.T,), generator=g, device="cuda")

    def bytes(self):
        return gaf.gaf_layer_workspace_bytes(self.T, self.d, gaf.GAF_F32, self.V)

    def embedding(self, ws):
        return gaf.gaf_embedding_grad(self.dy, self.tokens, torch.empty(self.V, self.d, device="cuda"), ws)

    def norm(self, ws):
        return gaf.gaf_rms_norm_grad(self.dy, self.h, self.w, self.rstd, torch.empty(self.d, device="cuda"), ws)

    def linear(self, ws):
        return gaf.gaf_linear_weight_grad(self.dy, self.ck, torch.empty(self.d, self.d, device="cuda"), ws)

    def calls(self):
        return [self.embedding, self.norm, self.linear]


# ------------------------------------------------------------------ status ----

@pytest.mark.parametrize("which", [0, 1, 2])
def test_layers_between_the_arrivals_of_a_stream(which):
    """A filter that takes its gradients one at a time, the layers making the next one in between on the same workspace: what an arrival left
    in the status is still there at the end, and decisions and distances are those of a workspace of its own."""
    L, D = Layers(), 4096
    n = max(L.bytes(), gaf.gaf_workspace_bytes(4, D, gaf.GAF_F32))
    shared, alone = torch.empty(n, dtype=torch.uint8, device="cuda"), gaf.new_workspace(4, D, gaf.GAF_F32)
    gaf.gaf_workspace_init(shared)
    for bad, bit in ((0.0, gaf.GAF_STATUS_ZERO_NORM), (float("nan"), gaf.GAF_STATUS_NONFINITE)):
        grads = [randn(gen(k), D) for k in range(4)]
        grads[1].fill_(bad)
        got = []
        for ws, between in ((shared, True), (alone, False)):
            acc = torch.empty(D, device="cuda")
            gaf.gaf_stream_begin(grads[0], acc, ws)
            for t in (1, 2, 3):
                gaf.gaf_stream_push(grads[t], t, 0.97, acc, ws)
                if between:
                    L.calls()[which](ws)
            got.append((acc, *gaf.gaf_stream_end(4, acc, ws)))
            assert gaf.gaf_read_status(ws) & bit, between
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(*got))      # (bits: a distance may be NaN)


def test_a_wait_that_ran_out_is_told_after_later_calls():
    """GAF_STATUS_TIMEOUT of a weight gradient stays, through the calls that follow it on the workspace, until it has been read."""
    L, D = Layers(), 4096
    n = max(L.bytes(), gaf.gaf_workspace_bytes(2, D, gaf.GAF_F32))
    grads = [randn(gen(k), D) for k in range(2)]
    for after in (L.calls(), [L.linear], [L.norm], [L.embedding], [lambda ws: gaf.gaf_filter_accumulate(grads, 2.0, ws)]):
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        gaf.gaf_workspace_init(ws)
        gaf.gaf_test_set_wait_fault(50, 1)
        try:
            L.linear(ws)
        finally:
            gaf.gaf_test_set_wait_fault(0, False)
        for call in after:
            call(ws)
        assert gaf.gaf_read_status(ws) == gaf.GAF_STATUS_TIMEOUT
        assert gaf.gaf_read_status(ws) == 0                      # (told once)
        for call in after:
            call(ws)
        assert gaf.gaf_read_status(ws) == 0


@pytest.mark.parametrize("fill", [0, 1, 4, 15, 0x4D4D4D4D, -1])
def test_status_of_a_workspace_that_held_anything(fill):
    """A workspace for the layers alone says nothing of what the memory held before."""
    L = Layers()
    old = torch.full((L.bytes() // 4,), fill, dtype=torch.int32, device="cuda")
    del old                                                      # (the allocator hands the same memory out again)
    ws = gaf.new_layer_workspace(L.T, L.d, gaf.GAF_F32, V=L.V)
    for call in L.calls():
        call(ws)
    assert gaf.gaf_read_status(ws) == 0


def test_workload_with_a_wait_that_ran_out_is_refused():
    gaf.gaf_test_set_wait_fault(50, 1)
    try:
        with pytest.raises(RuntimeError, match="ran out"):
            workloads.language_model(2, 300, 128, 100)
    finally:
        gaf.gaf_test_set_wait_fault(0, False)
    assert len(workloads.language_model(2, 300, 128, 100).grads) == 2


# --------------------------------------------------------------- arguments ----

class NoTruth:
    def __bool__(self):
        raise ArithmeticError("neither")


def test_flags_that_have_no_truth_value():
    """What a flag's own conversion raises reaches the caller, and nothing is written."""
    x, w = randn(gen(1), 5, 64), torch.ones(64, device="cuda")
    for name in ("want_y", "coded_y"):
        y, ck = torch.full((5, 64), 7.0, device="cuda"), gaf.new_checkpoint(5, 64)
        ck[0].zero_()
        with pytest.raises(ArithmeticError):
            gaf.gaf_rms_norm(x, w, y=y, y_checkpoint=ck, **{name: NoTruth()})
        assert bool((y == 7.0).all()) and not bool(ck[0].any())


class MadeWhenAsked:
    """A pair whose items are made as they are asked for, and which notes how many launches the latest call had made when each was let go."""
    def __init__(self, *pair):
        self.pair, self.made, self.gone = pair, 0, {}

    def __len__(self):
        return 2

    def __getitem__(self, i):
        t = self.pair[i].view(self.pair[i].shape)               # (an object of its own)
        weakref.finalize(t, lambda k: self.gone.__setitem__(k, gaf.gaf_last_launch_count()), self.made)
        self.made += 1
        return t


def test_a_checkpoint_is_held_until_the_launch():
    L = Layers()
    ws, out = gaf.new_layer_workspace(L.T, L.d, gaf.GAF_F32), torch.empty(L.d, L.d, device="cuda")
    other, third = gaf.new_checkpoint(L.T, L.d), gaf.new_checkpoint(L.T, L.d)

    def norm(pair):
        gaf.gaf_rms_norm(L.h, L.w, y_checkpoint=pair, h_checkpoint=third)
        assert torch.equal(third[0], L.ck[0]) and torch.equal(third[1], L.ck[1])
    for call, launches, pair in ((lambda p: gaf.gaf_linear_weight_grad(L.dy, p, out, ws), 3, L.ck),
                                 (lambda p: gaf.gaf_checkpoint_unpack(p, out=torch.empty(L.T, L.d, device="cuda")), 1, L.ck),
                                 (lambda p: gaf.gaf_checkpoint_pack(L.h, p), 1, other), (norm, 1, other)):
        made = MadeWhenAsked(*pair)
        gaf.gaf_embedding_grad(L.dy, L.tokens, torch.empty(L.V, L.d, device="cuda"), gaf.new_layer_workspace(L.T, L.d, gaf.GAF_F32, V=L.V))
        assert gaf.gaf_last_launch_count() == 2
        call(made)
        assert gaf.gaf_last_launch_count() == launches
        # (the first item is asked for once more to begin with, to see whether the pair can be indexed)
        assert made.made >= 3 and all(made.gone[k] == launches for k in range(1, 3)), made.gone


# -------------------------------------------------------------- long texts ----

def time_of(call, n=3):
    call()
    best = math.inf
    for _ in range(n):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


def test_embedding_grad_of_two_tokens_grows_with_the_text():
    """Two tokens that make up a text of a million and more positions (segment numbers, say): four times the text takes about four times as long, not sixteen."""
    V, d, ms = 2, 8, {}
    for T in (1 << 19, 1 << 21):
        dy = randn(gen(3), T, d, dtype=torch.bfloat16)
        tokens = torch.randint(0, V, (T,), generator=gen(4), device="cuda")
        ws, grad = gaf.new_layer_workspace(T, d, gaf.GAF_BF16, V=V), torch.empty(V, d, device="cuda")
        ms[T] = time_of(lambda: gaf.gaf_embedding_grad(dy, tokens, grad, ws))
    print("ms", ms)
    assert ms[1 << 21] < 8 * ms[1 << 19], ms


@pytest.mark.parametrize("T,V,d", [(32_768, 3, 8), (32_769, 3, 8), (65_536, 2, 5), (98_310, 700, 24), (200_000, 5000, 8), (16_777_217, 3, 1), (17_000_000, 2, 1)])
def test_embedding_grad_of_long_texts(T, V, d):
    """Texts of one window of the ordering (32,768 positions), of several, and of more than 512: whole numbers, whose sums are exact; and the same bits again
    and again for others, whatever order the counters handed out."""
    g = gen(T + V)
    tokens = torch.randint(-1, V, (T,), generator=g, device="cuda")
    ws = gaf.new_layer_workspace(T, d, gaf.GAF_BF16, V=V)
    whole = torch.randint(-1, 2, (T, d), generator=g, device="cuda").to(torch.bfloat16)
    want = torch.zeros(V + 1, d, dtype=torch.float64, device="cuda").index_add_(0, torch.where(tokens < 0, V, tokens), whole.double())[:V]
    assert bool((want.abs() < 2 ** 24).all())
    assert torch.equal(gaf.gaf_embedding_grad(whole, tokens, torch.empty(V, d, device="cuda"), ws).double(), want)
    dy = randn(g, T, d, dtype=torch.bfloat16)
    first = gaf.gaf_embedding_grad(dy, tokens, torch.empty(V, d, device="cuda"), ws)
    for _ in range(3):
        assert torch.equal(first, gaf.gaf_embedding_grad(dy, tokens, torch.empty(V, d, device="cuda"), ws))


# ---------------------------------------------------- values not finite ----

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [264, 1001])
def test_embedding_grad_of_values_that_are_not_finite(dtype, d):
    """They reach their own column of their own token's row, in short and in long stretches; padding's reach nothing."""
    t, g, T, V = TYPES[dtype], gen(d), 500, 40
    dy = randn(g, T, d, dtype=t)
    tokens = torch.randint(2, V, (T,), generator=g, device="cuda")
    tokens[100:300] = 1                             # a long stretch
    tokens[[3, 400]] = torch.tensor([0, -1], device="cuda")
    dy[3, 5], dy[250, 7], dy[400] = float("nan"), float("inf"), float("nan")
    dy[251, 9], dy[252, 9] = float("inf"), -float("inf")
    base = randn(g, V, d)
    base[2, 11], base[V - 1, 0] = float("nan"), -float("inf")
    ws = gaf.new_layer_workspace(T, d, gaf.GAF_F32 if dtype == "f32" else gaf.GAF_BF16, V=V)
    for b in (None, base):
        got = gaf.gaf_embedding_grad(dy, tokens, torch.empty(V, d, device="cuda"), ws, scale=0.5, base=b)
        want, off = ref.embedding_grad(dy, tokens, V, 0.5, b)
        assert bool(torch.isnan(want[0, 5])) and bool(torch.isnan(want[1, 9])) and want[1, 7].item() == math.inf
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
        fine = torch.isfinite(want)
        assert torch.equal(got[torch.isinf(want)].double(), want[torch.isinf(want)])
        assert_close(got[fine], want[fine], off[fine])


@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [264, 1001, 4096])
def test_rms_norm_grad_of_values_that_are_not_finite(d, dtype, coded):
    """They reach their own row of dx, through its mean, and the columns of dweight that they stand in."""
    t, g, T = TYPES[dtype], gen(d + 1), 40
    dy, h, w, res = randn(g, T, d, dtype=t), randn(g, T, d, dtype=t), randn(g, d, dtype=t), randn(g, T, d, dtype=t)
    rstd = (h.double().square().mean(dim=1) + 1e-6).rsqrt().float()
    dy[3, 5], dy[9, 100], h[20, 7], res[30, 8] = float("nan"), float("inf"), float("nan"), float("inf")
    ck = gaf.gaf_checkpoint_pack(h)
    hv = ref.checkpoint_values(ck) if coded else h.double()
    dw = torch.empty(d, device="cuda")
    ws = gaf.new_layer_workspace(T, d, gaf.GAF_F32 if dtype == "f32" else gaf.GAF_BF16)
    dx, _ = gaf.gaf_rms_norm_grad(dy, ck if coded else h, w, rstd, dw, ws, residual_grad=res)
    want, want_w, off, off_w = ref.rms_norm_grad(dy, hv, w, rstd, res)
    rows = torch.ones(T, dtype=torch.bool, device="cuda")
    rows[[3, 9, 20, 30]] = False
    columns = torch.ones(d, dtype=torch.bool, device="cuda")
    columns[[5, 7, 100]] = False
    assert_close(dx[rows], want[rows], off[rows])
    assert_close(dw[columns], want_w[columns], off_w[columns])
    assert not bool(torch.isfinite(dw[~columns]).any()) and not bool(torch.isfinite(dx[[3, 9, 20]]).any())
    assert dx[30, 8].item() == math.inf and bool(torch.isfinite(dx[30, :8]).all()) and bool(torch.isfinite(dx[30, 9:]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layers_between_filter_calls_of_every_kind(dtype):
    """One workspace for the layers and for filters that keep tags, hints and tickets in it from call to call: what a workspace of its own gives, bit for bit."""
    L, D, code = Layers(), 50_000, gaf.GAF_F32 if dtype == "f32" else gaf.GAF_BF16
    g = gen(7)
    common = randn(g, D)
    grads = [(common + randn(g, D)).to(TYPES[dtype]) for _ in range(40)]
    shared = torch.empty(max(L.bytes(), gaf.gaf_workspace_bytes(40, D, code)), dtype=torch.uint8, device="cuda")
    gaf.gaf_workspace_init(shared)
    alone = gaf.new_workspace(40, D, code)
    calls = [lambda ws, K=K: gaf.gaf_filter_accumulate(grads[:K], 0.6, ws) for K in (2, 3, 8, 9, 17, 40)]
    calls += [lambda ws, K=K, s=s: gaf.gaf_filter_accumulate(grads[:K], 0.6, ws, schedule=s) for K in (2, 4) for s in (gaf.binding.GAF_SCHED_STEPWISE, gaf.binding.GAF_SCHED_GRAM)]
    calls += [lambda ws, K=K: gaf.gaf_pairwise_cosdist(grads[:K], ws) for K in (2, 8, 17)]
    calls += [lambda ws: gaf.gaf_filter_accumulate_bucketed(grads[:4], 0.6, [0, 16_000, 40_000, D], ws), lambda ws: gaf.gaf_filter_accumulate_any_seed(grads[:3], 0.6, ws)]
    for turn in range(2):
        for k, call in enumerate(calls):
            for layer in L.calls():
                layer(shared)
            got, want = call(shared), call(alone)
            assert all(torch.equal(a, b) for a, b in zip(got, want) if torch.is_tensor(a)), (turn, k)
            assert gaf.gaf_read_status(shared) == gaf.gaf_read_status(alone), (turn, k)
