"""Tensor memory of a CTA pair: tcgen05.alloc with cta_group::2 is waited for without limit, so its order is checked in the source (no GPU),
and by many back-to-back calls whose quantizer shares the SMs with the pairs that are being set up."""
import os
import re
import time

import pytest
import torch

import paper_2606_14598_b200 as w8

CSRC = os.path.join(os.path.dirname(os.path.abspath(w8.__file__)), "csrc")
PAIR_KERNELS = sorted(f for f in os.listdir(CSRC) if f.endswith(".cu") and "tmem_alloc_pair(" in open(os.path.join(CSRC, f)).read())


def test_the_kernels_that_allocate_for_a_pair():
    assert PAIR_KERNELS == ["gemm_tc.cu", "mxfp4_gemm.cu"]


@pytest.mark.parametrize("name", PAIR_KERNELS)
def test_barriers_around_what_concerns_the_pair(name):
    """An operation on a pair needs both CTAs: a barrier of the cluster before the allocation (the peer has begun), one between it and the return of
    the permit (no CTA may allocate after that), one before memory is freed (the peer uses it no more) and one after (neither has left)."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    steps = re.findall(r"tmem_alloc_pair\(|cluster_sync_all\(\)|tmem_relinquish_pair\(|tmem_dealloc_pair\(", text)
    assert [x.split("(")[0] for x in steps] == ["cluster_sync_all", "tmem_alloc_pair", "cluster_sync_all", "tmem_relinquish_pair", "cluster_sync_all",
                                                "tmem_dealloc_pair", "cluster_sync_all"]


def test_no_store_into_a_cta_that_may_not_have_begun():
    """The one-kernel path of the int8 linear writes into the other CTAs' shared memory: behind a barrier of the cluster."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "small_fused.cu")).read())
    body = text[text.index("small_fused_kernel(const SmallArgs p)"):]
    arrive, wait = body.index("cluster_arrive()"), body.index("cluster_wait()")
    assert arrive < wait < min(body.index("st_cluster_f32(s_remote"), body.index("st_cluster_v2(a_remote"))


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(5125, 10592, 1504), (4110, 4608, 1056), (2100, 13824, 512), (8192, 2048, 288)])
def test_many_calls_back_to_back(m, n, k):
    """Short k-loops on many rows: a pair is set up every few dozen microseconds beside the CTAs of the quantizer ahead of it."""
    g = torch.Generator("cuda").manual_seed(k)
    a, w = torch.randn(m, k, generator=g, device="cuda").bfloat16(), torch.randn(n, k, generator=g, device="cuda")
    qw, sw = w8.mxfp4_quantize(w)
    sets = [(w8.mxfp4_alloc_workspace(m, n, k), torch.empty(m, n, dtype=torch.bfloat16, device="cuda")) for _ in range(3)]
    want = w8.mxfp4_linear_fused(a, qw, sw)
    try:
        for config in (0, 1):
            w8.mxfp4_force_config(config)
            for _ in range(10):
                for i in range(200):
                    w8.mxfp4_linear_fused(a, qw, sw, workspace=sets[i % 3][0], out=sets[i % 3][1])
                done, began = torch.cuda.Event(), time.monotonic()
                done.record()
                while not done.query():
                    assert time.monotonic() - began < 60, "the calls do not end"
                    time.sleep(0.001)
                assert all(w8.int8_check_status(ws) == 0 for ws, _ in sets)
            assert all(torch.allclose(out.float(), want.float(), rtol=2 ** -7, atol=1e-3 * k ** 0.5) for _, out in sets)
    finally:
        w8.mxfp4_force_config(-1)
