"""A decoder layer on the calls of include/dllava_mx.h, as a program runs it: prompts through products in 4 bits and grouped-head attention,
the kept rows' keys and values into the paged cache in 4 bits, then decode steps over it.  Every call's output is compared with the
oracle (float64) on the inputs that the call was given; the tolerances are those of the calls' own tests."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2412_00876_amd as P
from oracle import mx_ref as R

DEV = "cuda:0"
HIDDEN, HQ, H, DH, FFN = 512, 8, 2, 64, 704
QKV, SCALE = (HQ + 2 * H) * DH, DH ** -0.5


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    return t if dtype is None else t.to(dtype)


def f64(t):
    return t.double().cpu().numpy()


def i32(a):
    return dev(np.asarray(a, np.int32))


def close(y, want, mag, extra):
    bad = ~(np.abs(f64(y) - want) <= 2.0 ** -8 * np.abs(want) + extra * mag)
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:4])


class Weights:
    """A matrix [N, K], packed on the device, and the values that it stands for."""

    def __init__(self, rs, N, K):
        w = dev(rs.standard_normal((N, K)) * K ** -0.5).bfloat16()
        self.N, self.K = N, K
        self.q = torch.empty(P.dllava_mx_bytes(N, K), dtype=torch.uint8, device=DEV)
        P.dllava_mx_quantize(w, K, N, K, self.q, P.BF16)
        self.w = R.dequantize(*R.quantize(f64(w)))

    def rows(self, x, act=0, residual=None, few=False):
        """act(x W^T) (+ | *) residual, checked."""
        M, N, K = x.shape[0], self.N, self.K
        x2 = x.reshape(M, K)
        y = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device=DEV)
        if few:
            P.dllava_mx_linear_few(x2, K, M, K, self.q, None, N, act, residual, y, N, P.BF16)
            values = f64(x2)
        else:
            xq = torch.empty(P.dllava_mx_bytes(M, K), dtype=torch.uint8, device=DEV)
            P.dllava_mx_quantize(x2, K, M, K, xq, P.BF16)
            P.dllava_mx_linear(xq, M, K, self.q, None, N, act, residual, y, N, P.BF16)
            values = R.dequantize(*R.quantize(f64(x2)))
        want, mag = R.linear(values, self.w, None, act, None if residual is None else f64(residual))
        close(y, want, mag, (K + 8) * 2.0 ** -23)
        return y


def feed_forward(ws, x, few):
    gate = ws["gate"].rows(x, few=few)
    return ws["down"].rows(ws["up"].rows(x, act=2, residual=gate, few=few), residual=x, few=few)


@pytest.mark.parametrize("lens,steps", [([40, 1, 77, 0, 130], 3), ([5], 18)])
def test_prompts_then_decode_steps(lens, steps):
    rs = np.random.default_rng(len(lens))
    B, rows = len(lens), sum(lens)
    ws = {n: Weights(rs, N, K) for n, N, K in (("qkv", QKV, HIDDEN), ("out", HIDDEN, HQ * DH), ("gate", FFN, HIDDEN), ("up", FFN, HIDDEN), ("down", HIDDEN, FFN))}
    off = np.cumsum([0] + lens)
    x = dev(rs.standard_normal((rows, HIDDEN))).bfloat16()

    # prompts: the projection's output is passed as it is, strided
    qkv = ws["qkv"].rows(x)
    q, k, v = qkv[:, :HQ * DH], qkv[:, HQ * DH:(HQ + H) * DH], qkv[:, (HQ + H) * DH:]
    o = torch.full((rows, HQ, DH), float("nan"), dtype=torch.bfloat16, device=DEV)
    P.dllava_group_prefill_attn(q, QKV, k, v, QKV, B, i32(off), rows, HQ, H, DH, SCALE, o, P.BF16)
    for b, n in enumerate(lens):
        if n:
            at = slice(off[b], off[b + 1])
            want, W, A = R.attention(*(f64(t[at]).reshape(n, -1, DH) for t in (q, k, v)), SCALE, causal=True)
            close(o[at], want, W, 2.0 ** -8 + (2 * (DH + 16) * A[..., None] + 2 * n) * 2.0 ** -23)
    feed_forward(ws, ws["out"].rows(o, residual=x), few=False)

    # half of the rows are kept: theirs go to the cache
    kept = [np.sort(rs.permutation(n)[:(n + 1) // 2]) for n in lens]
    kept_off = np.cumsum([0] + [len(i) for i in kept])
    pages_each = (max(lens) + 1) // 2 // 16 + 3
    table = rs.permutation(B * pages_each + 2)[:B * pages_each].reshape(B, pages_each).astype(np.int32)
    ref = R.Cache(np.full((B * pages_each + 2, H, 17 * DH), 0xFF, np.uint8), table, np.zeros(B))
    pages, cache_len, err = dev(ref.pages), torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    cache = P.KVCache(pages, dev(table), cache_len)
    P.dllava_mx_cache_store(k, v, QKV, B, i32(kept_off), None, int(kept_off[-1]), i32(off), i32(np.concatenate(kept)), cache, err, P.BF16)
    K, V = (f64(t).reshape(rows, H, DH) for t in (k, v))
    for b in range(B):
        for i, r in enumerate(kept[b]):
            ref.put(b, i, K[off[b] + r], V[off[b] + r])
        ref.lens[b] = len(kept[b])
    assert np.array_equal(pages.cpu().numpy(), ref.pages)

    # decode steps: one row a sequence
    ws_step = torch.zeros(P.dllava_mx_decode_workspace(B, HQ, H, DH, pages_each), dtype=torch.uint8, device=DEV)
    x = dev(rs.standard_normal((B, HIDDEN))).bfloat16()
    for step in range(steps):
        qkv = ws["qkv"].rows(x, few=True)
        q, k, v = (t.contiguous() for t in (qkv[:, :HQ * DH], qkv[:, HQ * DH:(HQ + H) * DH], qkv[:, (HQ + H) * DH:]))
        logits, keep = dev(rs.standard_normal((B, 2)).astype(np.float32)), torch.empty(B, dtype=torch.uint8, device=DEV)
        o = torch.full((B, HQ, DH), float("nan"), dtype=torch.bfloat16, device=DEV)
        P.dllava_mx_decode_attn_append(q, k, v, B, HQ, logits, 0.0, None, cache, SCALE, o, keep, err, ws_step)
        lg = logits.cpu().numpy()
        decided = lg[:, 1] > lg[:, 0]
        for b in range(B):
            n = int(ref.lens[b])
            kb, vb = ref.rows(b, n)
            own = [f64(t[b]).reshape(1, -1, DH) for t in (q, k, v)]
            want, W, A = R.attention(own[0], np.concatenate([kb, own[1]]), np.concatenate([vb, own[2]]), SCALE)
            close(o[b:b + 1], want, W, 2.0 ** -8 + (2 * (DH + 16) * A[..., None] + 2 * (n + 1)) * 2.0 ** -23)
            if decided[b] and n < ref.cap:
                ref.put(b, n, own[1][0], own[2][0])
                ref.lens[b] += 1
        assert np.array_equal(keep.cpu().numpy(), decided.astype(np.uint8))
        assert np.array_equal(pages.cpu().numpy(), ref.pages) and cache_len.tolist() == ref.lens.tolist()
        x = feed_forward(ws, ws["out"].rows(o, residual=x, few=True), few=True)
        x = (x.float() / x.float().square().mean(1, keepdim=True).sqrt()).bfloat16()
    assert int(err) == 0
