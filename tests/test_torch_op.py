"""The fused linear as a PyTorch custom operator: shape-only tracing without a GPU, and, on a GPU, a small MLP of
two such linears traced as ONE graph (no graph break at the quantized linears) and replayed from a CUDA graph,
checked against the oracle."""
import numpy as np
import pytest
import torch

import oracle
from paper_2606_14598_b200 import inputs as synth


def test_operator_is_registered_and_traces_with_fake_tensors():
    from torch._subclasses.fake_tensor import FakeTensorMode

    from paper_2606_14598_b200 import torch_op
    assert hasattr(torch.ops.w8a8_b200, "linear_fused")
    with FakeTensorMode():
        A = torch.empty((3, 50, 64), dtype=torch.bfloat16)
        qw = torch.empty((24, 64), dtype=torch.int8)
        s_ch = torch.empty((24,), dtype=torch.float32)
        out = torch_op.linear_fused(A, qw, s_ch, None)          # the shape-only implementation: no kernel runs
        assert out.shape == (3, 50, 24) and out.dtype == torch.bfloat16
        with pytest.raises(Exception):
            torch_op.linear_fused(A.float(), qw, s_ch, None)


@pytest.mark.gpu
def test_compiled_mlp_has_no_graph_break_and_matches_the_oracle():
    import paper_2606_14598_b200 as w8
    from paper_2606_14598_b200.torch_op import W8A8Linear
    dev = "cuda:0"
    up, down = synth.LinearSpec("op_up", 300, 256, 512), synth.LinearSpec("op_down", 300, 512, 264)
    tu, td = synth.make_linear(up), synth.make_linear(down)

    class Mlp(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.up = W8A8Linear.from_float(tu["W"].to(dev), tu["bias"].to(dev))
            self.down = W8A8Linear.from_float(td["W"].to(dev), td["bias"].to(dev))

        def forward(self, x):
            return self.down(torch.relu(self.up(x)))        # an activation that is exact in bf16 (max with zero)

    mlp = Mlp()
    x = tu["A"].to(dev)
    eager = mlp(x)
    # the oracle's chain: linear, relu on the bf16 values, linear
    qwu, scu = oracle.quantize_weight_per_channel(tu["W"].numpy())
    qwd, scd = oracle.quantize_weight_per_channel(td["W"].numpy())
    h = oracle.linear_fused_bf16(synth.bf16_bits(tu["A"]), qwu, scu, tu["bias"].numpy())["out"]
    h_relu = np.where(h & 0x8000, 0, h).astype(np.uint16)
    ref = oracle.linear_fused_bf16(h_relu, qwd, scd, td["bias"].numpy())["out"]
    assert np.array_equal(synth.bf16_bits(eager.cpu()), ref)
    # one graph, no break at the quantized linears
    explanation = torch._dynamo.explain(mlp)(x)
    assert explanation.graph_break_count == 0 and explanation.graph_count == 1, str(explanation)
    compiled = torch.compile(mlp, fullgraph=True, backend="aot_eager")
    assert torch.equal(compiled(x), eager)
    # the calls allocate through torch only and enqueue on the current stream: replay from a CUDA graph
    static_x = x.clone()
    g = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        mlp(static_x)                                       # warm-up on the side stream
    torch.cuda.current_stream().wait_stream(s)
    with torch.cuda.graph(g):
        y = mlp(static_x)
    static_x.copy_(synth.make_activations(up, seed=3).to(dev))
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, mlp(static_x))
    assert w8.int8_sticky_status(clear=True) == 0


def modules(device, n=24, k=64):
    from paper_2606_14598_b200.torch_op import MXFP4Linear, W8A8Linear
    g = torch.Generator(device).manual_seed(2)
    bias = torch.randn(n, generator=g, device=device)
    int8 = W8A8Linear(torch.randint(-127, 128, (n, k), generator=g, device=device, dtype=torch.int8), torch.rand(n, generator=g, device=device) + 0.1, bias.clone())
    mx = MXFP4Linear(torch.randint(0, 256, (n, k // 2), generator=g, device=device, dtype=torch.uint8),
                     torch.full(((n + 127) // 128, (k + 127) // 128, 512), 120, device=device, dtype=torch.uint8), bias.clone())
    return int8, mx


@pytest.mark.parametrize("cast", [lambda m: m.bfloat16(), lambda m: m.half(), lambda m: m.to(torch.bfloat16), lambda m: m.double(), lambda m: m.cpu(),
                                  lambda m: torch.nn.Sequential(m).bfloat16()[0]])
def test_casting_a_model_leaves_scales_and_bias_as_they_are(cast):
    for module in modules("cpu"):
        before = {name: b.clone() for name, b in module.named_buffers()}
        after = dict(cast(module).named_buffers())
        assert after.keys() == before.keys()
        assert all(after[name].dtype == b.dtype and torch.equal(after[name], b) for name, b in before.items())


@pytest.mark.gpu
def test_inputs_of_any_strides():
    """Expanded rows, slices off 16-byte boundaries, odd row strides, other orders, single rows of them: as their dense copies."""
    for module in modules("cuda"):
        k = module.qw.shape[1] * (2 if module.qw.dtype == torch.uint8 else 1)
        wide = torch.randn(12, 5, k + 7, device="cuda").bfloat16()
        inputs = [wide[0, 0, :k].expand(9, k), wide[:, :1, :k].expand(12, 5, k), wide[..., 1:k + 1], wide[..., :k], wide[::2, 1, 3:k + 3], wide[0, 0, 5:k + 5],
                  wide[:1, :1, 1:k + 1], wide[0, 0, :k].expand(1, k), wide[..., :k].transpose(0, 1), wide.permute(2, 0, 1)[:k].permute(1, 2, 0), wide[:0, :, :k]]
        for x in inputs:
            want = module(x.clone(memory_format=torch.contiguous_format))
            got = module(x)
            assert got.shape == (*x.shape[:-1], 24) and torch.equal(got, want)


@pytest.mark.gpu
def test_forward_after_a_cast():
    x = torch.randn(10, 64, device="cuda").bfloat16()
    for module in modules("cuda"):
        want = module(x)
        assert torch.equal(module.bfloat16()(x), want) and torch.equal(module.cpu().half().cuda()(x), want)
