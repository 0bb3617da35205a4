"""The RMS norm in front of a quantized linear: refusals without a GPU, codes, scales and bf16 rows against a plain 64-bit form on one."""
import ctypes

import pytest
import torch

import lowbit_reference as ref
import paper_2606_14598_b200 as w8
from paper_2606_14598_b200 import norm

INVALID, ALIGNMENT = 1, 2
P = ctypes.c_void_p
NAN = float("nan")


def test_refusals():
    f = norm._lib.int8_rmsnorm
    names = ["x", "ldx", "res", "ldr", "w", "wt", "eps", "M", "K", "sum", "lds", "qa", "s", "y", "ldy", "stream"]
    ok = dict(zip(names, [P(4096), 64, P(8192), 64, P(4096), 0, 1e-6, 3, 64, P(16384), 64, P(4096), P(4096), P(4096), 64, None]))

    def status(**change):
        return f(*{**ok, **change}.values())

    for name in ("x", "w", "qa", "s"):
        assert status(**{name: None}) == INVALID, name
    assert status(qa=None, s=None, y=None) == INVALID
    assert status(M=-1) == INVALID and status(K=0) == INVALID and status(K=(1 << 24) + 8) == INVALID and status(wt=2) == INVALID
    for eps in (0.0, -1e-6, NAN, float("inf")):
        assert status(eps=eps) == INVALID, eps
    for name in ("ldx", "ldr", "lds", "ldy"):
        assert status(**{name: 56}) == INVALID and status(**{name: 68}) == ALIGNMENT, name
    for name in ("x", "res", "w", "sum", "qa", "y"):
        assert status(**{name: P(4104)}) == ALIGNMENT, name
    assert status(s=P(4098)) == ALIGNMENT and status(K=60) == ALIGNMENT
    assert status(sum=P(4096), lds=128) == INVALID and status(sum=P(8192), lds=128) == INVALID       # in place, but shifted
    # what is not there needs neither stride nor alignment; nothing to do needs no addresses
    assert status(res=None, ldr=0, sum=None, lds=0, y=None, ldy=0) not in (INVALID, ALIGNMENT)
    assert status(qa=None, s=None) not in (INVALID, ALIGNMENT)
    assert status(M=0, x=None, qa=None, s=None, y=None) not in (INVALID, ALIGNMENT)


def test_python_refusals():
    x, w = torch.zeros(3, 64, dtype=torch.bfloat16), torch.ones(64)
    for call in (w8.int8_rmsnorm, w8.rmsnorm):
        with pytest.raises(TypeError):
            call(x.float(), w)
        with pytest.raises(TypeError):
            call(x[0], w)
        with pytest.raises(TypeError):
            call(x, w.half())
        with pytest.raises(ValueError):
            call(x, w[:32])
        with pytest.raises(TypeError):
            call(x.t().contiguous().t(), w)
        with pytest.raises(ValueError):
            call(x, w, residual=x[:2])
        with pytest.raises(TypeError):
            call(x, w, residual=x.float())
        with pytest.raises(ValueError):
            call(x, w, sum_out=x[:2])
        with pytest.raises(ValueError):
            call(x, w, out=x[:, :32])
        with pytest.raises(ValueError):
            call(x, w)                                          # no CPU fallback
    with pytest.raises(ValueError):
        w8.int8_rmsnorm(x, w, qa=torch.zeros(3, 32, dtype=torch.int8))
    with pytest.raises(ValueError):
        w8.int8_rmsnorm(x, w, s_tok=torch.zeros(4))


# ------------------------------------------------------------------------------------------------ on the GPU

def single(x):
    return x.float().double()


def form(x, weight, eps, residual=None):
    """(h, codes, scales, normed rows) in 64 bits, rounded where the definition rounds."""
    h = x.double() if residual is None else single(x.double() + residual.double()).float().to(torch.bfloat16).double()
    u = single(h * weight.double())
    squares = (h * h).sum(-1)
    r = 1 / torch.sqrt(squares / x.shape[1] + eps)
    bad = ~torch.isfinite(u).all(-1) | (squares > torch.finfo(torch.float32).max)
    codes, c = ref.int8_quantize(torch.where(bad[:, None], torch.zeros_like(u), u))
    r = torch.where(bad, torch.full_like(r, NAN), r)
    s = torch.where((u == 0).all(-1), torch.ones_like(r), c * r)
    return h, codes, s, u * r[:, None]


def slack(k):
    """Relative error of the factor r and of the products with it: the roundings of the sum (a thread adds at most k / 1024 + 24 squares one after
    another, then ten steps of halving), halved by the root, then quotient, sum, root and product."""
    return (k / 1024 + 40) * 2.0 ** -24


def near(got, want, tolerance):
    got = got.double()
    same = torch.isnan(got) == torch.isnan(want)
    return bool(same.all()) and bool(((got - want).abs() <= want.abs() * tolerance)[~torch.isnan(want)].all())


def check(x, weight, eps=1e-6, residual=None, **kw):
    h, codes, s, y = form(x, weight, eps, residual)
    out = torch.full(x.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    qa, s_tok, total = w8.int8_rmsnorm(x, weight, eps, residual=residual, out=out, **kw)
    assert ref.same_values(total, h)
    assert torch.equal(qa.long(), codes)
    assert near(s_tok, s, slack(x.shape[1]))
    assert near(out, y, 2.0 ** -8 + slack(x.shape[1]))
    return qa, s_tok, total, out


def inputs(m, k, seed=0):
    gen = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn(m, k, generator=gen, device="cuda")
    x[:, torch.randperm(k, generator=gen, device="cuda")[: max(1, k // 100)]] *= 20
    residual = torch.randn(m, k, generator=gen, device="cuda") * 3
    return x.to(torch.bfloat16), residual.to(torch.bfloat16), 1 + 0.2 * torch.randn(k, generator=gen, device="cuda")


@pytest.mark.gpu
@pytest.mark.parametrize("m", [1, 2, 7, 300])
@pytest.mark.parametrize("k", [8, 16, 248, 256, 264, 1056, 2056, 4104, 4608, 8192, 12288, 24576, 24584, 66560])
def test_rows(m, k):
    x, residual, weight = inputs(m, k, m + k)
    a = check(x, weight, residual=residual)
    b = w8.rmsnorm(x, weight, residual=residual)
    assert torch.equal(a[3], b[0]) and torch.equal(a[2], b[1])
    check(x, weight.to(torch.bfloat16))
    again = w8.int8_rmsnorm(x, weight, residual=residual)
    assert torch.equal(a[0], again[0]) and torch.equal(a[1], again[1])


@pytest.mark.gpu
def test_many_rows():
    x, residual, weight = inputs(70001, 72, 5)
    check(x, weight, residual=residual)


@pytest.mark.gpu
@pytest.mark.parametrize("k", [264, 4608, 66560])
def test_in_place_and_strides(k):
    x, residual, weight = inputs(33, k + 24, 3)
    want = form(x[:, :k], weight[:k], 1e-5, residual[:, :k])
    plain = w8.int8_rmsnorm(x[:, :k].contiguous(), weight[:k].contiguous(), 1e-5, residual=residual[:, :k].contiguous())
    for target in ("x", "residual"):
        xs, rs = x.clone(), residual.clone()
        to = (xs if target == "x" else rs)[:, :k]
        y = torch.full((33, k + 8), 5.0, dtype=torch.bfloat16, device="cuda")
        got = w8.int8_rmsnorm(xs[:, :k], weight[:k].contiguous(), 1e-5, residual=rs[:, :k], sum_out=to, out=y[:, :k])
        assert got[2].data_ptr() == to.data_ptr() and ref.same_values(to, want[0])
        assert torch.equal(got[0], plain[0]) and torch.equal(got[1], plain[1])
        assert bool((y[:, k:] == 5).all()) and near(y[:, :k], want[3], 2.0 ** -8 + slack(k))
        assert torch.equal((xs if target == "x" else rs)[:, k:], (x if target == "x" else residual)[:, k:])      # beside the rows: left alone


@pytest.mark.gpu
@pytest.mark.parametrize("k", [256, 4608, 40000])
def test_extremes(k):
    """Rows of zeros, single spikes, huge, tiny and non-finite elements, each among ordinary rows that must not notice."""
    x, residual, weight = inputs(16, k, 9)
    x[1], residual[1] = 0, 0
    x[2], residual[2] = 0, 0
    x[2, k - 1] = -3
    x[3, 5], x[4, 0], x[5, k - 1] = NAN, float("inf"), -float("inf")
    residual[6, 7], residual[7, k // 2] = NAN, float("inf")
    x[8], residual[8] = 2.0 ** 100, 0                           # squares past fp32
    x[9], residual[9] = 2.0 ** -60, 2.0 ** -61                  # squares vanish beside eps
    x[10], residual[10] = 2.0 ** -133, 0                        # subnormal
    x[11], residual[11] = x[12], -x[12]                         # cancels
    x[13], residual[13] = 2.0 ** 60, 2.0 ** 59
    qa, s_tok, _, out = check(x, weight, residual=residual)
    for row in (3, 4, 5, 6, 7, 8):
        assert bool(torch.isnan(s_tok[row])) and not qa[row].any() and bool(torch.isnan(out[row]).all())
    assert s_tok[1] == 1 and not qa[1].any() and not out[1].any()
    # an infinite weight, or a product past fp32, makes its rows NaN and nothing else
    weight[3] = float("inf")
    check(x[:3], weight, residual=residual[:3])


@pytest.mark.gpu
def test_codes_go_into_the_linear():
    x, residual, weight = inputs(77, 1056, 4)
    w = torch.randn(256, 1056, device="cuda") * 0.03
    qw, s_ch = w8.int8_quantize_weight_per_channel(w)
    qa, s_tok, _ = w8.int8_rmsnorm(x, weight, residual=residual)
    out = w8.int8_linear_fused(qa, qw, s_ch, None, s_tok=s_tok)
    want = (qa.double() @ qw.double().t()) * s_tok.double()[:, None] * s_ch.double()
    assert near(out, want, 2.0 ** -8 + 3 * 2.0 ** -24)


@pytest.mark.gpu
def test_graph_stream_and_no_rows():
    x, residual, weight = inputs(5, 512, 2)
    want = w8.int8_rmsnorm(x, weight, residual=residual)
    qa, s_tok, total = (torch.zeros_like(t) for t in want)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        w8.int8_rmsnorm(x, weight, residual=residual, sum_out=total, qa=qa, s_tok=s_tok)
    for _ in range(2):
        for t in (qa, s_tok, total):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(qa, want[0]) and torch.equal(s_tok, want[1]) and torch.equal(total, want[2])
    qa, s_tok, total = w8.int8_rmsnorm(x[:0], weight, residual=residual[:0])
    assert qa.shape == (0, 512) and s_tok.shape == (0,) and total.shape == (0, 512)
    assert w8.rmsnorm(x[:0], weight)[0].shape == (0, 512)
