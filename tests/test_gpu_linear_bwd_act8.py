"""gws_linear_bwd_w_act8: the weight gradient with the linear's input kept in 8 bits, against 64 bits on the decoded input."""
import numpy as np
import pytest
import torch

import gated_ref as ref
import oracle
import paper_2505_11170_amd as gws
from paper_2505_11170_amd import synth
from gpu_util import DEV, assert_dbt_close, ensure_built

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


def inputs(M, K, N, pad=0, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed + 1000 * M + K + N)
    x = (torch.randn(M, K, generator=gen, device=DEV) * torch.exp(torch.randn(1, K, generator=gen, device=DEV))).bfloat16()
    x[M // 3] = 0.0
    codes = torch.full((M, K + 8 * pad), 0x7F, dtype=torch.uint8, device=DEV)
    scales = torch.full((M, K // 32 + pad), 255, dtype=torch.uint8, device=DEV)
    a = gws.Act8(codes[:, :K], scales[:, :K // 32])
    gws.gws_act8_encode(x, a)
    dy = torch.full((M, N + 8 * pad), float("nan"), dtype=torch.bfloat16, device=DEV)
    dy[:, :N] = (torch.randn(M, N, generator=gen, device=DEV) * 1e-3).bfloat16()
    return a, dy[:, :N]


@pytest.mark.parametrize("room", ["least", "all"])
@pytest.mark.parametrize("M,K,N,nk,pad", [(64, 256, 256, False, 0), (64, 256, 512, True, 1), (960, 768, 2304, False, 0), (2048, 1024, 512, True, 5),
                                          (4096, 768, 768, False, 0), (512, 2048, 5632, True, 0)])
def test_weight_gradient(M, K, N, nk, pad, room):
    a, dy = inputs(M, K, N, pad)
    rows, cols = (N, K) if nk else (K, N)
    w = synth.make_tensor(17, rows, cols, with_grad=False)
    seed, step = gws.gws_derive_seed(3, 4), 9
    _, scale = oracle.sample_fwd(synth.bits(w["w"]), w["bt"].numpy(), oracle.FMT_BF16, seed, step)
    scale = torch.as_tensor(scale).to(DEV)
    dw, dbt = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV), torch.zeros(rows // 32, cols // 32, device=DEV)
    d = gws.TensorDesc(rows=rows, cols=cols, seed=seed, dw=dw, dbt=dbt, scale=scale)
    need = -(-2 * M * K // 256) * 256
    most = gws.gws_linear_bwd_w_act8_workspace_bytes(d, M, w_is_nk=nk)
    assert most >= need
    ws = torch.full(((need if room == "least" else most) + 256,), 0x5A, dtype=torch.uint8, device=DEV)
    gws.gws_linear_bwd_w_act8(a, dy, d, step, ws[:-256], w_is_nk=nk)
    torch.cuda.synchronize()
    assert (ws[-256:] == 0x5A).all()
    x = ref.decode(a.codes, a.xscale)
    p, q = (dy.double(), x) if nk else (x, dy.double())
    want, bound = p.t().contiguous() @ q, M * ref.ULP * (p.abs().t().contiguous() @ q.abs())
    ref.assert_within(dw, want, ref.BF16 * want.abs() + bound + 1e-38, "dw")
    _, ref_dbt, asum = oracle.sample_bwd(synth.bits(dw.cpu()), scale.cpu().numpy(), seed, step)   # on the gradient as it was rounded
    assert_dbt_close(dbt.cpu().numpy(), ref_dbt, asum)
    # and without dL/db_t the same gradient
    again = torch.zeros_like(dw)
    gws.gws_linear_bwd_w_act8(a, dy, gws.TensorDesc(rows=rows, cols=cols, seed=seed, dw=again), step, ws[:-256], w_is_nk=nk)
    torch.cuda.synchronize()
    assert torch.equal(again, dw)


def test_a_nan_block_reaches_its_own_rows_of_the_gradient():
    M, K, N = 128, 256, 256
    a, dy = inputs(M, K, N)
    a.xscale[5, 2] = 255
    dw = torch.zeros(K, N, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(2 * M * K, dtype=torch.uint8, device=DEV)
    gws.gws_linear_bwd_w_act8(a, dy, gws.TensorDesc(rows=K, cols=N, seed=1, dw=dw), 0, ws)
    torch.cuda.synchronize()
    want = np.zeros((K, N), bool)
    want[64:96] = True
    assert np.array_equal(torch.isnan(dw).cpu().numpy(), want)
