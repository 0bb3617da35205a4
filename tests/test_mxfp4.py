"""The MXFP4 linear, its quantizer and its inverse: refusals without a GPU, values against plain 64-bit forms on one."""
import ctypes

import pytest
import torch

import lowbit_reference as ref
import paper_2606_14598_b200 as w8
from paper_2606_14598_b200 import mxfp4

OK, INVALID, ALIGNMENT, WORKSPACE = 0, 1, 2, 4
P = ctypes.c_void_p


# ------------------------------------------------------------------------------------------ without a GPU

def test_sizes():
    assert mxfp4._lib.mxfp4_scale_bytes(1, 32) == 512
    assert mxfp4._lib.mxfp4_scale_bytes(128, 128) == 512
    assert mxfp4._lib.mxfp4_scale_bytes(129, 160) == 4 * 512
    assert mxfp4._lib.mxfp4_scale_bytes(0, 32) == 0 and mxfp4._lib.mxfp4_scale_bytes(4, 48) == 0
    assert w8.mxfp4_linear_workspace_bytes(77, 2048, 1056) >= 256 + 9 * 512 + 77 * 528
    assert w8.mxfp4_linear_workspace_bytes(77, 0, 1056) == 0 and w8.mxfp4_linear_workspace_bytes(77, 8, 1050) == 0


def test_quantize_refusals():
    q = mxfp4._lib.mxfp4_quantize
    ok = [P(4096), 0, 4, 64, 64, P(8192), P(16384), None]

    def status(**change):
        a = list(ok)
        for i, v in change.items():
            a[int(i[1:])] = v
        return q(*a)

    assert status(_0=None) == INVALID and status(_5=None) == INVALID and status(_6=None) == INVALID
    assert status(_1=2) == INVALID and status(_1=-1) == INVALID
    assert status(_2=0) == INVALID and status(_2=(1 << 30) + 1) == INVALID and status(_3=0) == INVALID and status(_3=(1 << 24) + 32) == INVALID
    assert status(_4=32) == INVALID
    assert status(_3=48) == ALIGNMENT and status(_4=68) == ALIGNMENT
    assert status(_0=P(4104)) == ALIGNMENT and status(_5=P(8196)) == ALIGNMENT and status(_6=P(16388)) == ALIGNMENT
    d = mxfp4._lib.mxfp4_dequantize
    assert d(P(4096), P(8192), 4, 64, None, 0, 64, None) == INVALID
    assert d(P(4096), P(8192), 4, 64, P(16384), 3, 64, None) == INVALID
    assert d(P(4096), P(8192), 4, 64, P(16384), 0, 60, None) == INVALID
    assert d(P(4096), P(8192), 4, 64, P(16384), 0, 68, None) == ALIGNMENT
    assert d(P(4096), P(8192), 4, 64, P(16392), 0, 64, None) == ALIGNMENT


def test_linear_refusals():
    f = mxfp4._lib.mxfp4_linear_fused
    names = ["A", "a_dtype", "lda", "a_scales", "qw", "sw", "bias", "out", "ldo", "M", "N", "K", "ws", "ws_bytes", "stream"]
    ok = dict(zip(names, [P(4096), 0, 64, None, P(8192), P(8192), None, P(4096), 16, 4, 16, 64, P(4096), 1 << 20, None]))

    def status(**change):
        return f(*{**ok, **change}.values())

    for name in ("A", "qw", "sw", "out"):
        assert status(**{name: None}) == INVALID, name
    assert status(a_dtype=1) == INVALID and status(a_dtype=7) == INVALID
    assert status(a_scales=P(4096)) == INVALID and status(a_dtype=2) == INVALID          # scales go with codes, codes with scales
    for name in ("M", "N", "K"):
        assert status(**{name: 0}) == INVALID and status(**{name: -8}) == INVALID
    assert status(M=(1 << 30) + 1) == INVALID
    assert status(lda=56) == INVALID and status(ldo=8) == INVALID
    assert status(K=48) == ALIGNMENT and status(N=12) == ALIGNMENT and status(lda=68) == ALIGNMENT and status(ldo=20) == ALIGNMENT
    for name in ("A", "qw", "sw", "out"):
        assert status(**{name: P(4104)}) == ALIGNMENT, name
    assert status(bias=P(4104)) == ALIGNMENT
    assert status(ws=None) == WORKSPACE and status(ws=P(4096 + 128)) == WORKSPACE and status(ws_bytes=256) == WORKSPACE


def test_unknown_configurations_are_refused():
    """Ids other than -1 (automatic) and those of the kernels; the few-token kernel with too many tokens. Refused before the device is looked at."""
    f = mxfp4._lib.mxfp4_linear_fused

    def status(config, m):
        old = w8.mxfp4_force_config(config)
        try:
            return f(P(4096), 0, 64, None, P(8192), P(8192), None, P(4096), 16, m, 16, 64, P(4096), 1 << 20, None)
        finally:
            assert w8.mxfp4_force_config(old) == config

    for config in (-2, -1000, w8.MXFP4_NUM_CONFIGS + 1, 1000):
        assert status(config, 4) == INVALID, config
    assert status(w8.MXFP4_NUM_CONFIGS, 65) == INVALID


def test_workspace_whose_memory_is_smaller_than_its_shape_is_refused(monkeypatch):
    """An expanded or strided tensor counts more bytes than it owns in one piece. (The call is recorded: no GPU.)"""
    seen = []
    monkeypatch.setattr(mxfp4, "call", lambda fn, where, dev, *args: seen.append(args))
    x, codes, scales = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(16, 32, dtype=torch.uint8), torch.zeros(1, 1, 512, dtype=torch.uint8)
    need = w8.mxfp4_linear_workspace_bytes(4, 16, 64)
    for workspace in (torch.zeros(1, dtype=torch.uint8).expand(need), torch.zeros(2 * need, dtype=torch.uint8)[::2], torch.zeros(4, need, dtype=torch.uint8).t()):
        with pytest.raises(TypeError):
            w8.mxfp4_linear_fused(x, codes, scales, workspace=workspace)
    assert not seen
    w8.mxfp4_linear_fused(x, codes, scales, workspace=torch.zeros(need + 64, dtype=torch.uint8))
    assert seen[0][-1] == need + 64


def test_stream_and_device_without_the_short_ways_to_them():
    """A torch without the two private functions: calls go through its public ones. In a process of its own, with a stand-in for the library's call."""
    import os
    import subprocess
    import sys
    code = """if True:
        import torch
        for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
            if hasattr(torch._C, name):
                delattr(torch._C, name)
        from types import SimpleNamespace
        torch.cuda.current_device = lambda: 3
        torch.cuda.current_stream = lambda device: SimpleNamespace(cuda_stream=1000 + device)
        from paper_2606_14598_b200 import mxfp4
        seen = []
        mxfp4.call(lambda *args: seen.append(args) or 0, "here", 3, 7, 8)
        assert seen == [(7, 8, 1003)], seen
        print("called")
    """
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "called" in r.stdout, r.stdout + r.stderr


def test_python_refusals():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        w8.mxfp4_quantize(x.half())
    with pytest.raises(TypeError):
        w8.mxfp4_quantize(x.t())
    with pytest.raises(ValueError):
        w8.mxfp4_quantize(x, scales=torch.zeros(1, 2, 512, dtype=torch.uint8))
    with pytest.raises(ValueError):
        w8.mxfp4_quantize(x)                                     # no CPU fallback
    codes, scales = torch.zeros(16, 32, dtype=torch.uint8), torch.zeros(1, 1, 512, dtype=torch.uint8)
    with pytest.raises(TypeError):
        w8.mxfp4_dequantize(codes, scales, dtype=torch.float16)
    with pytest.raises(ValueError):
        w8.mxfp4_linear_fused(torch.zeros(4, 96, dtype=torch.bfloat16), codes, scales)
    with pytest.raises(TypeError):
        w8.mxfp4_linear_fused(x.float(), codes, scales)
    with pytest.raises(TypeError):
        w8.mxfp4_linear_fused(x, codes, scales, torch.zeros(8))
    with pytest.raises(TypeError):
        w8.mxfp4_linear_fused(x, codes, scales, out=torch.zeros(4, 16))
    with pytest.raises(ValueError):
        w8.mxfp4_linear_fused(x, codes, scales)


def test_reference_grid():
    """The reference's own rounding on hand-made values: every tie goes to the even code, 7 saturates."""
    x = torch.zeros(1, 32, dtype=torch.float64)
    x[0, :14] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, -0.25, -0.75, 5.001, 0.2501, 4.0], dtype=torch.float64)
    codes, scale = ref.mx_quantize(x)
    assert scale.item() == 127 and codes[0, :14].tolist() == [0, 2, 2, 4, 4, 6, 6, 7, 7, 8, 10, 7, 1, 6]


# ------------------------------------------------------------------------------------------ quantizer

def check_quantized(x):
    codes, scales = w8.mxfp4_quantize(x)
    want_codes, want_bytes = ref.mx_quantize(x)
    assert torch.equal(scales, ref.tile(want_bytes))                 # zero bytes past the end included
    assert torch.equal(codes, ref.pack(want_codes))
    for dtype in (torch.bfloat16, torch.float32):
        out = w8.mxfp4_dequantize(codes, scales, dtype=dtype)
        assert out.dtype == dtype and ref.same_values(out, ref.mx_values(want_codes, want_bytes))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,k", [(1, 32), (1, 4608), (3, 64), (127, 96), (128, 128), (129, 160), (7, 1056), (300, 992), (33, 12288), (1000, 224)])
def test_quantizer(m, k, dtype):
    g = torch.Generator("cuda").manual_seed(m * 1000 + k)
    x = torch.randn(m, k, generator=g, device="cuda") * torch.exp2(torch.randint(-20, 20, (m, 1), generator=g, device="cuda").float())
    check_quantized(x.to(dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantizer_of_more_rows_than_the_grid_holds(dtype):
    """A launch holds 75776 warps of two rows (fp32 to codes: one): more rows go round its loop."""
    check_quantized(torch.randn(160001, 64, generator=torch.Generator("cuda").manual_seed(9), device="cuda").to(dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantizer_strides(dtype):
    x = torch.randn(70, 3, 352, device="cuda").to(dtype)
    check_quantized(x[:, 1])                                         # a slice of a fused buffer
    check_quantized(x.view(70, 1056)[:, 32:32 + 320])
    wide = torch.full((40, 512), 7.0, device="cuda", dtype=dtype)
    codes, scales = w8.mxfp4_quantize(x.view(70, 1056)[:40, :256])
    w8.mxfp4_dequantize(codes, scales, out=wide[:, 128:384])
    assert (wide[:, :128] == 7).all() and (wide[:, 384:] == 7).all()
    assert torch.equal(wide[:, 128:384], w8.mxfp4_dequantize(codes, scales, dtype=dtype))


@pytest.mark.gpu
def test_quantizer_special_values():
    x = torch.zeros(12, 64, device="cuda")
    x[1] = -0.0
    x[2, 0] = 2.0 ** -133                      # bf16 subnormal: the scale clamps at 2^-127
    x[2, 1] = 2.0 ** -128
    x[2, 40] = 2.0 ** -126
    x[3, 5] = float("inf")                     # first block bad, second untouched
    x[3, 40] = 3.0
    x[4, 33] = float("nan")
    x[4, 0] = -5.0
    x[5, 63] = float("-inf")
    x[6] = torch.finfo(torch.bfloat16).max
    x[7, ::2] = -torch.finfo(torch.bfloat16).max
    x[8, :9] = torch.tensor([4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0])
    x[9] = -x[8] * 2.0 ** 100
    x[10, 0], x[10, 1] = 1.0, 2.0 ** -120      # far below the block's largest
    x[11, :2] = torch.tensor([7.96875, 6.96875])
    check_quantized(x.bfloat16())
    x[2, 2] = 2.0 ** -149                      # fp32 subnormals
    x[6] = torch.finfo(torch.float32).max
    check_quantized(x)


@pytest.mark.gpu
def test_quantizer_every_finite_bf16_value():
    """Every finite bf16 value in blocks led by a value 0 to 9 powers of two above it."""
    bits = torch.arange(1 << 16, device="cuda", dtype=torch.int32)
    v = bits.to(torch.int16).view(torch.bfloat16)
    v = v[torch.isfinite(v)]
    for up in range(10):
        x = torch.zeros(v.numel() // 31 + 1, 32, device="cuda", dtype=torch.bfloat16)
        x[:, 1:].reshape(-1)
        flat = torch.zeros(x.shape[0] * 31, device="cuda", dtype=torch.bfloat16)
        flat[: v.numel()] = v
        x[:, 1:] = flat.view(-1, 31)
        lead = x.float().abs().amax(1) * 2.0 ** up
        x[:, 0] = torch.where(torch.isfinite(lead.bfloat16()), lead, torch.zeros_like(lead)).bfloat16()
        check_quantized(x)


@pytest.mark.gpu
def test_dequantize_all_codes_and_scales():
    codes = torch.arange(16, device="cuda").repeat(256, 2)
    rows = torch.arange(256, device="cuda")[:, None]
    got = w8.mxfp4_dequantize(ref.pack(codes), ref.tile(rows), dtype=torch.float32)
    want = ref.mx_values(codes, rows)
    want[254][want[254].abs() > torch.finfo(torch.bfloat16).max] *= float("inf")     # 2^127 * 2 and above: past bf16 and fp32
    want[253][want[253].abs() > torch.finfo(torch.bfloat16).max] *= float("inf")
    assert ref.same_values(got, want)


# ------------------------------------------------------------------------------------------ linear

def operands(m, n, k, seed=0, loud=True):
    g = torch.Generator("cuda").manual_seed(seed + 7 * m + 11 * n + 13 * k)
    a = torch.randn(m, k, generator=g, device="cuda")
    if loud:
        a[:, torch.randperm(k, generator=g, device="cuda")[: max(1, k // 100)]] *= 20
    w = torch.randn(n, k, generator=g, device="cuda") * 0.02
    bias = torch.randn(n, generator=g, device="cuda") * 0.01
    return a.bfloat16(), w, bias


def check_linear(out, a, w, bias):
    """out against the 64-bit product of the quantized values. Tolerance: half an ulp of bf16 (8 significant bits: at most 2^-8 of the result), and for the
    fp32 accumulation at most 2^-22 of the sum of the products' magnitudes for each step of 32 along K."""
    av, wv = ref.mx_values(*ref.mx_quantize(a)), ref.mx_values(*ref.mx_quantize(w))
    want = av @ wv.t() + (0 if bias is None else bias.double())
    size = av.abs() @ wv.abs().t() + (0 if bias is None else bias.double().abs())
    tol = want.abs() * 2.0 ** -8 + (a.shape[1] // 32 + 2) * 2.0 ** -22 * size + 2.0 ** -133
    assert out.dtype == torch.bfloat16 and out.shape == want.shape
    worst = ((out.double() - want).abs() / tol).max().item()
    assert worst <= 1.0, worst


SHAPES = [(1, 8, 32), (1, 4608, 4608), (1, 136, 96), (2, 27648, 1056), (3, 1000, 160), (4, 256, 12288), (7, 264, 64), (8, 128, 256), (9, 2048, 1056),
          (15, 24, 544), (16, 512, 512), (17, 120, 2048), (31, 264, 288), (32, 128, 4128), (33, 136, 1024), (64, 1160, 768), (65, 384, 96),
          (77, 2048, 1056), (100, 4616, 4608), (127, 128, 128), (128, 256, 256), (129, 264, 320), (200, 16, 3008), (255, 520, 1088),
          (257, 248, 224), (300, 328, 384), (513, 1032, 1184), (1000, 2056, 736), (1200, 4608, 2336), (2305, 1000, 512)]


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_linear(m, n, k):
    a, w, bias = operands(m, n, k)
    qw, sw = w8.mxfp4_quantize(w)
    ws = w8.mxfp4_alloc_workspace(m, n, k)
    ws.fill_(255)
    out = w8.mxfp4_linear_fused(a, qw, sw, bias, workspace=ws)
    assert w8.int8_check_status(ws) == 0
    check_linear(out, a, w, bias)
    plain = w8.mxfp4_linear_fused(a, qw, sw)
    check_linear(plain, a, w, None)
    codes, scales = w8.mxfp4_quantize(a)
    again = w8.mxfp4_linear_fused(codes, qw, sw, bias, a_scales=scales, workspace=ws)
    assert torch.equal(again, out)                                   # the same kernel on the same codes: the same bits
    for _ in range(3):
        assert torch.equal(w8.mxfp4_linear_fused(a, qw, sw, bias, workspace=ws), out)


@pytest.mark.gpu
@pytest.mark.parametrize("m", [1, 5, 40, 150, 700])
def test_linear_strides_and_guards(m):
    n, k = 264, 416
    a, w, bias = operands(m, n, k)
    qw, sw = w8.mxfp4_quantize(w)
    want = w8.mxfp4_linear_fused(a, qw, sw, bias)
    wide = torch.full((m + 2, 3 * k), float("nan"), device="cuda", dtype=torch.bfloat16)      # neighbours must not be read
    wide[1:-1, k:2 * k] = a
    buf = torch.full((m + 2, n + 32), 9.0, device="cuda", dtype=torch.bfloat16)
    w8.mxfp4_linear_fused(wide[1:-1, k:2 * k], qw, sw, bias, out=buf[1:-1, 16:16 + n])
    assert torch.equal(buf[1:-1, 16:16 + n], want)
    buf[1:-1, 16:16 + n] = 9.0
    assert (buf == 9.0).all()
    codes, scales = w8.mxfp4_quantize(a)
    padded = torch.full((m, k // 2 + 48), 255, device="cuda", dtype=torch.uint8)
    padded[:, 16:16 + k // 2] = codes
    assert torch.equal(w8.mxfp4_linear_fused(padded[:, 16:16 + k // 2], qw, sw, bias, a_scales=scales), want)


@pytest.mark.gpu
@pytest.mark.parametrize("m", [2, 20, 130, 300])
def test_linear_non_finite_rows_stay_apart(m):
    n, k = 144, 352
    a, w, bias = operands(m, n, k)
    qw, sw = w8.mxfp4_quantize(w)
    want = w8.mxfp4_linear_fused(a, qw, sw, bias)
    a[1, k - 1] = float("nan")
    out = w8.mxfp4_linear_fused(a, qw, sw, bias)
    assert torch.isnan(out[1]).all()
    keep = [i for i in range(m) if i != 1]
    assert torch.equal(out[keep], want[keep])
    w[7, 3] = float("inf")
    qw, sw = w8.mxfp4_quantize(w)
    out = w8.mxfp4_linear_fused(a, qw, sw, bias)
    assert torch.isnan(out[:, 7]).all() and torch.equal(out[keep][:, :7], want[keep][:, :7]) and torch.equal(out[keep][:, 8:], want[keep][:, 8:])


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(1, 128, 256), (24, 128, 512), (200, 256, 256)])
def test_linear_scale_range(m, n, k):
    """Scales from the smallest to ones whose products nearly overflow fp32; zero rows and columns."""
    g = torch.Generator("cuda").manual_seed(5)
    a = torch.randn(m, k, generator=g, device="cuda") * torch.exp2(torch.randint(-60, 50, (m, 1), generator=g, device="cuda").float())
    w = torch.randn(n, k, generator=g, device="cuda") * torch.exp2(torch.randint(-60, 50, (n, 1), generator=g, device="cuda").float())
    a[0], w[3], w[5] = a[0] if m == 1 else 0, 0, torch.zeros(k, device="cuda")
    a = a.bfloat16()
    qw, sw = w8.mxfp4_quantize(w)
    check_linear(w8.mxfp4_linear_fused(a, qw, sw), a, w, None)


@pytest.mark.gpu
def test_linear_on_another_stream_and_in_a_graph():
    n, k = 520, 1056
    for m in (1, 12, 300):
        a, w, bias = operands(m, n, k)
        qw, sw = w8.mxfp4_quantize(w)
        want = w8.mxfp4_linear_fused(a, qw, sw, bias)
        ws, out = w8.mxfp4_alloc_workspace(m, n, k), torch.zeros_like(want)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            w8.mxfp4_linear_fused(a, qw, sw, bias, out=out, workspace=ws)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, want)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            w8.mxfp4_linear_fused(a, qw, sw, bias, out=out, workspace=ws)
            w8.mxfp4_linear_fused(a, qw, sw, bias, out=out, workspace=ws)
        a2 = operands(m, n, k, seed=99)[0]
        a.copy_(a2)
        graph.replay()
        assert torch.equal(out, w8.mxfp4_linear_fused(a2, qw, sw, bias))


@pytest.mark.gpu
@pytest.mark.parametrize("config", range(w8.MXFP4_NUM_CONFIGS))
def test_linear_every_configuration(config):
    """Shapes of several tiles for a CTA, odd numbers of k-blocks, ragged edges, on each kernel configuration."""
    try:
        for m, n, k in [(1, 8, 32), (130, 264, 96), (129, 136, 288), (300, 520, 1056), (700, 1000, 800), (2305, 4104, 544), (1500, 9224, 3104)]:
            a, w, bias = operands(m, n, k)
            qw, sw = w8.mxfp4_quantize(w)
            w8.mxfp4_force_config(config)
            ws = w8.mxfp4_alloc_workspace(m, n, k)
            out = w8.mxfp4_linear_fused(a, qw, sw, bias, workspace=ws)
            assert w8.int8_check_status(ws) == 0
            check_linear(out, a, w, bias)
            for _ in range(3):
                assert torch.equal(w8.mxfp4_linear_fused(a, qw, sw, bias, workspace=ws), out)
    finally:
        w8.mxfp4_force_config(-1)


@pytest.mark.gpu
@pytest.mark.parametrize("config", range(w8.MXFP4_NUM_CONFIGS))
def test_linear_wait_runs_out_and_the_kernel_returns(config):
    a, w, bias = operands(600, 1032, 2080)
    qw, sw = w8.mxfp4_quantize(w)
    ws = w8.mxfp4_alloc_workspace(600, 1032, 2080)
    want = w8.mxfp4_linear_fused(a, qw, sw, bias, workspace=ws)
    try:
        w8.mxfp4_force_config(config)
        want = w8.mxfp4_linear_fused(a, qw, sw, bias, workspace=ws)
        w8.debug_set_wait_limit_ns(3_000_000)
        w8.debug_set_starve(1)
        w8.mxfp4_linear_fused(a, qw, sw, bias, workspace=ws)
        assert w8.int8_check_status(ws) == 7 and w8.int8_sticky_status() == 7
    finally:
        w8.debug_set_starve(0)
        w8.debug_set_wait_limit_ns(0)
    try:
        again = w8.mxfp4_linear_fused(a, qw, sw, bias, workspace=ws)
    finally:
        w8.mxfp4_force_config(-1)
    assert w8.int8_check_status(ws) == 0 and w8.int8_sticky_status() == 0 and torch.equal(again, want)


SKINNY = [(1, 8, 32), (2, 136, 96), (3, 4608, 1024), (16, 128, 2048), (5, 264, 4352), (7, 1000, 6176), (13, 40, 12288), (1, 20000, 544), (16, 256, 24608), (4, 24, 49152),
          (1, 20000, 4608), (2, 28000, 9216), (3, 19008, 3488), (9, 30000, 2560), (16, 27656, 4384), (11, 8, 65536),
          (17, 264, 2080), (32, 1024, 4608), (33, 136, 12288), (48, 2056, 1312), (49, 4608, 4608), (60, 136, 8224), (64, 1032, 4640), (64, 24, 544),
          (63, 20000, 800)]


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", SKINNY)
def test_linear_few_tokens(m, n, k):
    """Every way the few-token kernel cuts K (1 to 8 parts), odd numbers of k-blocks, ragged edges; bf16 and codes agree."""
    a, w, bias = operands(m, n, k)
    qw, sw = w8.mxfp4_quantize(w)
    codes, scales = w8.mxfp4_quantize(a)
    ws = w8.mxfp4_alloc_workspace(m, n, k)
    w8.mxfp4_force_config(w8.MXFP4_NUM_CONFIGS)
    try:
        out = w8.mxfp4_linear_fused(a, qw, sw, bias, workspace=ws)
        assert w8.int8_check_status(ws) == 0
        check_linear(out, a, w, bias)
        for _ in range(5):
            assert torch.equal(w8.mxfp4_linear_fused(codes, qw, sw, bias, a_scales=scales, workspace=ws), out)
            assert torch.equal(w8.mxfp4_linear_fused(a, qw, sw, bias, workspace=ws), out)
    finally:
        w8.mxfp4_force_config(-1)


@pytest.mark.gpu
def test_linear_few_tokens_refuses_many():
    a, w, bias = operands(65, 64, 64)
    qw, sw = w8.mxfp4_quantize(w)
    w8.mxfp4_force_config(w8.MXFP4_NUM_CONFIGS)
    try:
        with pytest.raises(w8.W8A8Error):
            w8.mxfp4_linear_fused(a, qw, sw, bias)
    finally:
        w8.mxfp4_force_config(-1)


@pytest.mark.gpu
@pytest.mark.parametrize("m", [3, 9, 30, 60])
def test_linear_few_tokens_wait_runs_out(m):
    a, w, bias = operands(m, 1032, 4128)
    qw, sw = w8.mxfp4_quantize(w)
    ws = w8.mxfp4_alloc_workspace(m, 1032, 4128)
    want = w8.mxfp4_linear_fused(a, qw, sw, bias, workspace=ws)
    try:
        w8.debug_set_wait_limit_ns(3_000_000)
        w8.debug_set_starve(1)
        w8.mxfp4_linear_fused(a, qw, sw, bias, workspace=ws)
        assert w8.int8_check_status(ws) == 7 and w8.int8_sticky_status() == 7
    finally:
        w8.debug_set_starve(0)
        w8.debug_set_wait_limit_ns(0)
    again = w8.mxfp4_linear_fused(a, qw, sw, bias, workspace=ws)
    assert w8.int8_check_status(ws) == 0 and w8.int8_sticky_status() == 0 and torch.equal(again, want)


@pytest.mark.gpu
@pytest.mark.parametrize("writer", ["quantize", "kernel"])
@pytest.mark.parametrize("m,config", [(1, -1), (6, -1), (14, -1), (40, -1), (300, 0), (300, 1), (300, 2)])
def test_linear_reads_weights_written_just_ahead(m, config, writer):
    """Weights rewritten by the kernel directly ahead of every call, through the quantizer or another kernel, bf16 tokens and codes: each call
    sees its own weights, eagerly and in a graph."""
    n, k = 4608, 2080
    a, w, bias = operands(m, n, k)
    both = [w, w.flip(0).contiguous()]
    made = [w8.mxfp4_quantize(x) for x in both]
    codes, scales = w8.mxfp4_quantize(a)
    ws = w8.mxfp4_alloc_workspace(m, n, k)
    qw, sw = (torch.zeros_like(t) for t in made[0])
    mask = torch.zeros_like(qw), torch.zeros_like(sw)
    w8.mxfp4_force_config(config)
    try:
        want = [w8.mxfp4_linear_fused(a, *made[i], bias, workspace=ws) for i in range(2)]
        torch.cuda.synchronize()
        outs = torch.zeros(24, m, n, dtype=torch.bfloat16, device="cuda")

        def calls():
            for i, out in enumerate(outs):
                if writer == "quantize":
                    w8.mxfp4_quantize(both[i % 2], codes=qw, scales=sw)
                else:
                    torch.bitwise_xor(made[i % 2][1], mask[1], out=sw)
                    torch.bitwise_xor(made[i % 2][0], mask[0], out=qw)
                if i % 4 < 2:
                    w8.mxfp4_linear_fused(a, qw, sw, bias, out=out, workspace=ws)
                else:
                    w8.mxfp4_linear_fused(codes, qw, sw, bias, a_scales=scales, out=out, workspace=ws)

        for _ in range(4):
            outs.zero_()
            calls()
            assert all(torch.equal(out, want[i % 2]) for i, out in enumerate(outs))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls()
        for _ in range(4):
            outs.zero_()
            graph.replay()
            assert all(torch.equal(out, want[i % 2]) for i, out in enumerate(outs))
        assert w8.int8_check_status(ws) == 0
    finally:
        w8.mxfp4_force_config(-1)


@pytest.mark.gpu
def test_linear_random_shapes():
    import random
    r = random.Random(3)
    for _ in range(60):
        m, n, k = r.choice([r.randint(1, 40), r.randint(1, 300), r.randint(1, 1200)]), 8 * r.randint(1, 160), 32 * r.randint(1, 60)
        a, w, bias = operands(m, n, k, seed=r.randint(0, 999))
        qw, sw = w8.mxfp4_quantize(w)
        check_linear(w8.mxfp4_linear_fused(a, qw, sw, bias), a, w, bias)


# ------------------------------------------------------------------------------------------ operator, module, example

def test_operator_traces_without_a_gpu():
    from torch._subclasses.fake_tensor import FakeTensorMode
    from paper_2606_14598_b200 import torch_op
    with FakeTensorMode():
        out = torch_op.mxfp4_linear(torch.empty(2, 5, 64, dtype=torch.bfloat16), torch.empty(24, 32, dtype=torch.uint8),
                                    torch.empty(1, 1, 512, dtype=torch.uint8), None)
    assert out.shape == (2, 5, 24) and out.dtype == torch.bfloat16


@pytest.mark.gpu
def test_module():
    from paper_2606_14598_b200.torch_op import MXFP4Linear
    a, w, bias = operands(70, 136, 96)
    layer = MXFP4Linear.from_float(w, bias)
    x = a.view(2, 35, 96)
    want = w8.mxfp4_linear_fused(a, *w8.mxfp4_quantize(w), bias)
    assert torch.equal(layer(x).view(70, 136), want)
    assert torch.equal(layer(x.transpose(0, 1)).transpose(0, 1).reshape(70, 136), want)      # rows in another order, copied
    assert layer(x[:, :0]).shape == (2, 0, 136)
    assert torch.equal(torch.compile(layer, fullgraph=True, backend="eager")(x).view(70, 136), want)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
def test_example_block(fmt):
    """The example's block stays near its fp32 form. Each MXFP4 matrix is off by about a tenth of its norm (a step of 0.5 to 2 in 6,
    uniform within a step), a linear by about 0.14 of its output; the residual stream, as large as what the three linears of a step
    add to it, keeps the result of three steps within a cosine of 0.9."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "mxfp4_block.py")
    spec = importlib.util.spec_from_file_location("mxfp4_block", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    four, full = module.run(fmt)
    assert four.shape == full.shape and torch.isfinite(four).all()
    assert torch.nn.functional.cosine_similarity(four.flatten(), full.flatten(), dim=0) > 0.9


@pytest.mark.gpu
def test_chained_with_the_int8_kernels():
    """Launches that follow one another closely (programmatic dependent launch, shared tensor memory): int8 linears of one, a few dozen and
    many tokens between 4-bit ones of every kind and cache calls, eagerly and as a graph, against each one run by itself."""
    g = torch.Generator("cuda").manual_seed(21)
    calls, alone = [], []
    for m, n, k in [(1, 1024, 512), (6, 2048, 768), (40, 512, 1024), (30, 256, 512), (200, 384, 768), (700, 1032, 1056)]:
        a, w, bias = operands(m, n, k, seed=m)
        qw4, sw4 = w8.mxfp4_quantize(w)
        qw8, s8 = w8.int8_quantize_weight_per_channel(w)
        ws4, ws8 = w8.mxfp4_alloc_workspace(m, n, k), w8.alloc_workspace(m, n, k)
        out4, out8 = (torch.empty(m, n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        calls.append((lambda a=a, q=qw8, s=s8, b=bias, o=out8, ws=ws8: w8.int8_linear_fused(a, q, s, b, out=o, workspace=ws), out8))
        calls.append((lambda a=a, q=qw4, s=sw4, b=bias, o=out4, ws=ws4: w8.mxfp4_linear_fused(a, q, s, b, out=o, workspace=ws), out4))
    x = torch.randn(200, 4, 64, generator=g, device="cuda").bfloat16()
    cache = w8.QuantKVCache.empty(13, 16, 4, 64, "mxfp4")
    table, cu = torch.arange(13, dtype=torch.int32, device="cuda")[None], torch.tensor([0, 200], dtype=torch.int32, device="cuda")
    k_out, v_out, slots = torch.empty_like(x), torch.empty_like(x), torch.arange(200, device="cuda")

    def cached():
        w8.kv_cache_write(cache, x, x, slots)
        w8.kv_cache_read(cache, table, cu, 200, k_out=k_out, v_out=v_out)

    calls.insert(5, (cached, k_out))
    for call, out in calls:
        call()
        torch.cuda.synchronize()
        alone.append(out.clone())
    order = list(range(len(calls))) * 3 + list(range(len(calls)))[::-1] * 2 + [0, 3, 0, 3, 1, 1, 3, 3, 5, 4, 5, 4, 7, 6, 7, 12, 3, 12, 0]
    for _ in range(10):
        for i in order:
            calls[i][0]()
    torch.cuda.synchronize()
    assert all(torch.equal(out, want) for (_, out), want in zip(calls, alone))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for i in order:
            calls[i][0]()
    for _, out in calls:
        out.zero_()
    for _ in range(10):
        graph.replay()
    assert all(torch.equal(out, want) for (_, out), want in zip(calls, alone)) and w8.int8_sticky_status() == 0
