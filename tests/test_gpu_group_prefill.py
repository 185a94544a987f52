"""Causal attention of packed prompts with grouped heads against the oracle (float64).

Tolerance of an output o = sum_j w_j v_j, with W = sum_j w_j |v_j| and A = scale * max_j sum |q| |k_j|.  bfloat16: its own rounding, 2^-8 |o|;
probabilities rounded to bfloat16, off by half a step, 2^-8 of each at most: 2^-8 W; scores, exponentials and their sums in float32, twice
(Dh + 16) 2^-23 A and 2 n 2^-23.  float32: no first two terms, and 2^-22 |o| for the last division and product."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2412_00876_amd as P
from oracle import mx_ref as R

DEV = "cuda:0"
CODE = {torch.float32: P.F32, torch.bfloat16: P.BF16}


def f64(t):
    return t.double().cpu().numpy()


def run_and_check(lens, Hq, Hkv, Dh, dtype, fused, seed=0, extra=0, scale=None):
    rs = np.random.default_rng(seed + Hq + Dh)
    scale = Dh ** -0.5 if scale is None else scale
    rows, n = sum(lens), (Hq + 2 * Hkv) * Dh
    off = torch.tensor(np.cumsum([0] + lens), dtype=torch.int32, device=DEV)
    x = torch.from_numpy(rs.standard_normal((rows + extra + 1, n))).to(DEV, dtype)
    Q, K, V = x[:, :Hq * Dh], x[:, Hq * Dh:(Hq + Hkv) * Dh], x[:, (Hq + Hkv) * Dh:]
    if not fused:
        Q, K, V = (t.contiguous() for t in (Q, K, V))
    O = torch.full((rows + extra + 1, Hq, Dh), 3.0, dtype=dtype, device=DEV)
    P.dllava_group_prefill_attn(Q, Q.stride(0), K, V, K.stride(0), len(lens), off, rows + extra, Hq, Hkv, Dh, scale, O, CODE[dtype])
    assert (O[rows:] == 3.0).all()                           # rows behind the last sequence
    r0 = 0
    for m in lens:
        if m:
            q, k, v = (f64(t[r0:r0 + m]).reshape(m, -1, Dh) for t in (Q, K, V))
            want, W, A = R.attention(q, k, v, scale, causal=True)
            err = np.abs(f64(O[r0:r0 + m]) - want)
            tol = (2 * (Dh + 16) * 2.0 ** -23 * A[..., None] + 2 * m * 2.0 ** -23) * W
            tol = tol + (2.0 ** -8 * (np.abs(want) + W) if dtype == torch.bfloat16 else 2.0 ** -22 * np.abs(want))
            bad = ~(err <= tol)
            assert not bad.any(), (m, bad.sum(), np.argwhere(bad)[:4], err.max())
        r0 += m


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,Dh", [(1, 1, 64), (4, 2, 128), (7, 1, 64), (14, 2, 64), (8, 8, 128), (6, 1, 128), (24, 4, 64), (16, 2, 128)])
@pytest.mark.parametrize("fused", [False, True])
def test_ragged(Hq, Hkv, Dh, dtype, fused):
    run_and_check([5, 0, 1, 16, 33, 64, 0, 127, 130, 1], Hq, Hkv, Dh, dtype, fused)


@pytest.mark.parametrize("blocks", [3, 16])
@pytest.mark.parametrize("waves", [1, 2, 4])
@pytest.mark.parametrize("Dh", [64, 128])
def test_every_launch_shape(Dh, waves, blocks):
    P.dllava_set_launch_override(P.LAUNCH_PREFILL_WAVES, waves)
    P.dllava_set_launch_override(P.LAUNCH_PREFILL_BLOCKS, blocks)
    try:
        run_and_check([1, 100, 257, 31], 4, 2, Dh, torch.bfloat16, True)
        run_and_check([1, 100, 257, 31], 8, 2, Dh, torch.bfloat16, True)
    finally:
        P.dllava_set_launch_override(P.LAUNCH_PREFILL_WAVES, 0)
        P.dllava_set_launch_override(P.LAUNCH_PREFILL_BLOCKS, 0)


def test_long_and_many():
    run_and_check([900, 3], 4, 1, 128, torch.bfloat16, False)
    run_and_check([(7 * i) % 40 for i in range(80)], 4, 2, 64, torch.bfloat16, True)      # more than 64 sequences
    run_and_check([(5 * i) % 37 for i in range(70)], 16, 4, 64, torch.bfloat16, False)    # the same, heads in eights
    run_and_check([1500, 700], 40, 8, 64, torch.bfloat16, True)                           # several rounds of items to a block
    run_and_check([200], 8, 2, 128, torch.bfloat16, True, extra=37)                       # rows is an upper bound
    run_and_check([150, 20], 4, 2, 128, torch.bfloat16, True, scale=1.5)                  # sharp softmax


def test_one_query_head_per_head_against_prefill_attn():
    """The same as dllava_prefill_attn's, whose probabilities have 16 bits (off by 2^-14 at most), but for both outputs' rounding and the one
    probabilities': W <= max |v|."""
    rs = np.random.default_rng(5)
    lens, H, Dh = [300, 1, 77], 4, 128
    rows = sum(lens)
    off = torch.tensor(np.cumsum([0] + lens), dtype=torch.int32, device=DEV)
    Q, K, V = (torch.from_numpy(rs.standard_normal((rows, H, Dh))).to(DEV, torch.bfloat16) for _ in range(3))
    a, b = torch.zeros_like(Q), torch.zeros_like(Q)
    P.dllava_group_prefill_attn(Q, H * Dh, K, V, H * Dh, 3, off, rows, H, H, Dh, 0.09, a, P.BF16)
    P.dllava_prefill_attn(Q, K, V, None, 3, off, rows, H, Dh, 0.09, b, P.BF16)
    top = V.double().abs().amax((0, 2))[None, :, None]
    assert ((a.double() - b.double()).abs() <= 2.0 ** -8 * (a.double().abs() + b.double().abs()) + (2.0 ** -8 + 2.0 ** -13) * top).all()


def test_captured():
    rs = np.random.default_rng(6)
    lens, Hq, Hkv, Dh = [40, 0, 130], 6, 2, 64
    rows = sum(lens)
    off = torch.tensor(np.cumsum([0] + lens), dtype=torch.int32, device=DEV)
    new = lambda h: torch.from_numpy(rs.standard_normal((rows, h, Dh))).to(DEV, torch.bfloat16)
    Q, K, V, O = new(Hq), new(Hkv), new(Hkv), torch.zeros((rows, Hq, Dh), dtype=torch.bfloat16, device=DEV)
    call = lambda: P.dllava_group_prefill_attn(Q, Hq * Dh, K, V, Hkv * Dh, 3, off, rows, Hq, Hkv, Dh, 0.125, O, P.BF16)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        Q.copy_(new(Hq))
        call()
        eager = O.clone()
        O.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, eager)
