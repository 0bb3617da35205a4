"""Operands written directly ahead of an int8 linear on its stream: the linear reads them after the work ahead is complete, although its
kernels are set up while that work is still running."""
import pytest
import torch

import paper_2606_14598_b200 as w8
from paper_2606_14598_b200 import binding


@pytest.mark.gpu
@pytest.mark.parametrize("last", ["quantizer", "qw", "s_ch", "bias"])
@pytest.mark.parametrize("m,n,k", [(3, 4608, 2048), (32, 512, 512), (64, 1024, 256), (200, 1024, 8192), (300, 4608, 2048), (2100, 2560, 1024)])
def test_weights_written_just_ahead(m, n, k, last):
    """Two sets of weights in turn, whatever operand the kernel directly ahead writes; tokens as bf16 and as codes, eagerly and in a graph."""
    g = torch.Generator("cuda").manual_seed(m + n + k)
    a = torch.randn(m, k, generator=g, device="cuda").bfloat16()
    plain = [torch.randn(n, k, generator=g, device="cuda") * 0.02 * (i + 1) for i in range(2)]
    biases = [torch.randn(n, generator=g, device="cuda") for _ in range(2)]
    made = [w8.int8_quantize_weight_per_channel(w) for w in plain]
    codes, s_tok = w8.int8_quantize_act_per_token(a)
    ws, ws_codes = w8.alloc_workspace(m, n, k), w8.alloc_workspace(m, n, k, binding.ACT_INT8)
    want = [w8.int8_linear_fused(a, *made[i], biases[i], workspace=ws) for i in range(2)]
    assert not torch.equal(want[0], want[1])
    qw, s_ch, bias = torch.zeros_like(made[0][0]), torch.zeros_like(made[0][1]), torch.zeros_like(biases[0])
    zero, mask = torch.zeros_like(bias), torch.zeros_like(qw)
    outs = torch.zeros(16, m, n, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()

    def write(i):
        steps = {"qw": lambda: torch.bitwise_xor(made[i][0], mask, out=qw), "s_ch": lambda: torch.add(made[i][1], zero, out=s_ch),
                 "bias": lambda: torch.add(biases[i], zero, out=bias)}
        if last == "quantizer":
            steps["bias"]()
            stream = torch.cuda.current_stream().cuda_stream
            assert binding._lib.int8_quantize_weight_per_channel(plain[i].data_ptr(), n, k, k, qw.data_ptr(), s_ch.data_ptr(), stream) == 0
            return
        for name in sorted(steps, key=lambda x: x == last):
            steps[name]()

    def calls():
        for i, out in enumerate(outs):
            write(i % 2)
            if i % 4 < 2:
                w8.int8_linear_fused(a, qw, s_ch, bias, out=out, workspace=ws)
            else:
                w8.int8_linear_fused(codes, qw, s_ch, bias, s_tok=s_tok, out=out, workspace=ws_codes)

    for _ in range(3):
        outs.zero_()
        calls()
        assert all(torch.equal(out, want[i % 2]) for i, out in enumerate(outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(3):
        outs.zero_()
        graph.replay()
        assert all(torch.equal(out, want[i % 2]) for i, out in enumerate(outs))
    assert w8.int8_check_status(ws) == 0 and w8.int8_check_status(ws_codes) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("k", [256, 4608, 66560])
def test_quantizer_inputs_written_just_ahead(k):
    """Activations, weights and SmoothQuant factors written by the kernel directly ahead of their quantizers, for rows of every kind (the longest
    go through the kernel without a ring)."""
    rows = 40
    g = torch.Generator("cuda").manual_seed(k)
    both = [torch.randn(rows, k, generator=g, device="cuda") * (i + 1) for i in range(2)]
    mults = [torch.rand(k, generator=g, device="cuda") + 0.5 + i for i in range(2)]
    acts = [x.bfloat16() for x in both]
    quantizers = {"act": lambda a, w, m: w8.int8_quantize_act_per_token(a), "weight": lambda a, w, m: w8.int8_quantize_weight_per_channel(w),
                  "act_smooth": lambda a, w, m: w8.int8_quantize_act_per_token_smooth(a, m),
                  "weight_smooth": lambda a, w, m: w8.int8_quantize_weight_per_channel_smooth(w, m)}
    a, w, m = torch.zeros_like(acts[0]), torch.zeros_like(both[0]), torch.zeros_like(mults[0])
    for name, quantize in quantizers.items():
        want = [quantize(acts[i], both[i], mults[i]) for i in range(2)]
        torch.cuda.synchronize()
        got = []
        for i in range(20):
            for last in (False, True):
                if name.endswith("smooth") == last:
                    torch.mul(mults[i % 2], 1.0, out=m)
                else:
                    torch.mul(acts[i % 2], 1.0, out=a)
                    torch.mul(both[i % 2], 1.0, out=w)
            got.append(quantize(a, w, m))
        for i, (q, s) in enumerate(got):
            assert torch.equal(q, want[i % 2][0]) and torch.equal(s, want[i % 2][1]), (name, i)
