"""The Python entry points of the int8 linear refuse tensors that the kernels would read or write past: wrong sizes, other devices, workspaces
that own less than their shape says. No GPU: the library's entry points are replaced by recorders, so a call that gets through is seen, not run."""
import pytest
import torch

import paper_2606_14598_b200 as w8
from paper_2606_14598_b200 import binding

M, N, K = 16, 24, 32


class Recorder:
    """Notes compute calls; sizes are still the library's."""

    def __init__(self, lib):
        self.lib, self.calls = lib, []

    def __getattr__(self, name):
        if "workspace_" in name:
            return getattr(self.lib, name)
        return lambda *args: self.calls.append(name) or 0


@pytest.fixture
def lib(monkeypatch):
    r = Recorder(binding._lib)
    monkeypatch.setattr(binding, "_lib", r)
    yield r
    assert not r.calls, r.calls                                       # nothing got through to the kernels


def tensors():
    return dict(A=torch.zeros(M, K, dtype=torch.bfloat16), qw=torch.zeros(N, K, dtype=torch.int8), s_ch=torch.ones(N))


def bad_sizes():
    """Keyword, value, and what the refusal names."""
    bf16 = dict(dtype=torch.bfloat16)
    yield "out", torch.zeros(1, N, **bf16), "out"
    yield "out", torch.zeros(M, N - 8, **bf16), "out"
    yield "bias", torch.zeros(N - 1), "bias"
    yield "workspace", torch.zeros(1, dtype=torch.uint8).expand(1 << 20), "workspace"


@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("entry", ["int8_linear_fused", "int8_linear_fused_rowmax", "int8_linear_fused_smooth", "int8_linear_fused_static"])
def test_sizes(lib, entry, which):
    name, value, names = list(bad_sizes())[which]
    if entry == "int8_linear_fused_static" and name == "workspace":
        return
    t = tensors()
    args = (t["A"], torch.ones(K), t["qw"], t["s_ch"]) if entry == "int8_linear_fused_smooth" else (t["A"], t["qw"], t["s_ch"])
    with pytest.raises((TypeError, ValueError), match=names):
        getattr(w8, entry)(*args, **{name: value})


def test_scales_and_codes(lib):
    t = tensors()
    codes = torch.zeros(M, K, dtype=torch.int8)
    for entry in (w8.int8_linear_fused, w8.int8_linear_fused_rowmax):
        with pytest.raises(ValueError, match="s_tok"):
            entry(codes, t["qw"], t["s_ch"], s_tok=torch.ones(M - 1))
    with pytest.raises(ValueError, match="qa"):
        w8.int8_quantize_act_per_token(t["A"], qa=codes[:4])
    with pytest.raises(TypeError, match="qa"):
        w8.int8_quantize_act_per_token(t["A"], qa=torch.zeros(M, 2 * K, dtype=torch.int8)[:, :K])
    with pytest.raises(ValueError, match="s_tok"):
        w8.int8_quantize_act_per_token(t["A"], s_tok=torch.ones(M - 1))
    with pytest.raises(ValueError, match="shape"):
        w8.int8_gemm_i32_debug(codes, torch.zeros(N, K // 2, dtype=torch.int8))


def test_host_entry(lib):
    t = tensors()
    ok = dict(A_host=t["A"], d_A=t["A"].clone(), qw=t["qw"], s_ch=t["s_ch"], bias=torch.zeros(N), d_out=torch.zeros(M, N, dtype=torch.bfloat16),
              out_host=torch.zeros(M, N, dtype=torch.bfloat16), workspace=torch.zeros(1 << 16, dtype=torch.uint8))
    for name in ("d_A", "s_ch", "bias", "d_out", "out_host"):
        with pytest.raises(ValueError, match=name):
            w8.int8_linear_fused_host(**{**ok, name: ok[name][:-1].contiguous()})


def test_host_memory_is_not_handed_to_the_kernels(lib):
    """No CPU fallback, and no host address where the kernels expect a device's."""
    t = tensors()
    codes, s_tok = torch.zeros(M, K, dtype=torch.int8), torch.ones(M)
    for call in (lambda: w8.int8_linear_fused(t["A"], t["qw"], t["s_ch"]), lambda: w8.int8_linear_fused(codes, t["qw"], t["s_ch"], s_tok=s_tok),
                 lambda: w8.int8_linear_fused_rowmax(t["A"], t["qw"], t["s_ch"]), lambda: w8.int8_linear_fused_static(t["A"], t["qw"], t["s_ch"]),
                 lambda: w8.int8_linear_fused_smooth(t["A"], torch.ones(K), t["qw"], t["s_ch"]),
                 lambda: w8.int8_quantize_act_per_token(t["A"]), lambda: w8.int8_quantize_weight_per_channel(torch.zeros(N, K)),
                 lambda: w8.int8_quantize_act_per_token_smooth(t["A"], torch.ones(K)), lambda: w8.int8_gemm_i32_debug(codes, t["qw"]),
                 lambda: w8.int8_quantize_weight_per_channel_smooth(torch.zeros(N, K), torch.ones(K)),
                 lambda: w8.int8_quantize_act_per_token_given_absmax(t["A"], torch.ones(M))):
        with pytest.raises(ValueError, match="CUDA device"):
            call()


@pytest.mark.gpu
def test_tensors_of_the_host_beside_the_device():
    a, w, bias = (torch.randn(*s, device="cuda") for s in ((M, K), (N, K), (N,)))
    qw, s_ch = w8.int8_quantize_weight_per_channel(w)
    for change in (dict(bias=bias.cpu()), dict(out=torch.zeros(M, N, dtype=torch.bfloat16)), dict(workspace=torch.zeros(1 << 16, dtype=torch.uint8)),
                   dict(s_ch=s_ch.cpu()), dict(qw=qw.cpu())):
        with pytest.raises(ValueError, match="devices"):
            w8.int8_linear_fused(**{**dict(A=a.bfloat16(), qw=qw, s_ch=s_ch), **change})
