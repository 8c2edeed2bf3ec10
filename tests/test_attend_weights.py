"""The softmax weights' precision in md_attend_cache over a cache in eight bits, seen where values cancel.

Logits that are exact until they meet their factor: one channel of the queries and keys is not 0.  Two
tokens share the weight, and their values nearly cancel, so that the output's own rounding (2^-8 of
the output) leaves the weights' errors in sight.  Of sum p |v|, a weight and the sum of weights may be off by
  a logit's two roundings and that of its distance to the base, at most 8: 2^-22 + 2^-23, x ln 2; exp2 2^-22:
  2^-20.8 together, twice for the quotient                                                        2^-19.8
  two f16 terms of a weight 2^-22; 18 roundings at 2^-24 in each of two matrix instructions      2^-18.6
  merges of warps, CTAs and parts, the sums of weights, the division: 32 x 2^-24 at most          2^-19
2^-17.5 in all, taken as 2^-17.  One f16 term would be off by up to 2^-11."""
import math

import numpy as np
import pytest

import paper_2607_10582_gb300 as md
from paper_2607_10582_gb300 import build as mdbuild

torch = pytest.importorskip("torch")
D = 128
mdbuild.build()
gpu = pytest.mark.gpu


def build_case(n, seed, L=2, Hkv=2, G=8, ps=16):
    """Codes and scales of one sequence, queries, and the reference: everything on the CPU, in 64 bits."""
    r = np.random.default_rng(seed)
    P = -(-n // ps)
    codes = torch.zeros((L, P, Hkv, 2, ps, D))
    codes[:, :, :, 0, :, 0] = -448.0                              # logits of -39 and less: no weight to speak of
    codes[:, :, :, 1] = torch.from_numpy(r.choice([-8.0, -2.0, 1.0, 5.0], (L, P, Hkv, ps, D))).float()
    q = torch.zeros((1, L, Hkv * G, D))
    q[..., 0] = torch.from_numpy(1 + r.integers(0, 128, q.shape[:3]) / 128).float()   # 8 bits, as bf16 has
    two = r.choice(n, 2, replace=False)
    for l in range(L):
        for h in range(Hkv):
            k = r.choice(np.arange(0, 16), 2, replace=False) / 4
            v = r.integers(8, 16, D) * 2.0 ** r.integers(-3, 3, D) * r.choice([-1, 1], D)
            x = float(q[0, l, h * G, 0]) * (k[0] - k[1]) / math.sqrt(D)     # of the group's first head
            other = torch.from_numpy(-v * math.exp(x)).float().to(torch.float8_e4m3fn).float()
            for t, kk, vv in ((two[0], k[0], torch.from_numpy(v).float()), (two[1], k[1], other)):
                codes[l, t // ps, h, 0, t % ps, 0] = kk
                codes[l, t // ps, h, 1, t % ps] = vv
    pool = codes.to(torch.float8_e4m3fn)
    assert torch.equal(pool.float(), codes)
    kv = codes.double().permute(0, 2, 3, 1, 4, 5).reshape(L, Hkv, 2, P * ps, D)[:, :, :, :n]
    x = torch.einsum("lhgd,lhnd->lhgn", q[0].double().view(L, Hkv, G, D), kv[:, :, 0]) / math.sqrt(D)
    p = torch.softmax(x, -1)
    ref = torch.einsum("lhgn,lhnd->lhgd", p, kv[:, :, 1])
    size = torch.einsum("lhgn,lhnd->lhgd", p, kv[:, :, 1].abs())
    return pool, q.bfloat16(), ref.reshape(q.shape), size.reshape(q.shape)


SIZES = [2, 31, 40, 257, 700, 2089, 20011]


@pytest.mark.parametrize("n", SIZES[:4])
def test_the_values_cancel(n):
    """A part of the channels ends below 2^-6 of the sizes that went into it: one f16 term would show there."""
    _, _, ref, size = build_case(n, n)
    assert float((ref.abs() < 2.0 ** -6 * size).double().mean()) > 0.05


@gpu
@pytest.mark.parametrize("workspace", [False, True])
@pytest.mark.parametrize("n", SIZES)
def test_weights_have_more_bits_than_the_output_shows(n, workspace):
    if not torch.cuda.is_available():  # pragma: no cover
        pytest.skip("needs a CUDA GPU")
    pool, q, ref, size = build_case(n, n)
    L, P, Hkv, _, ps, _ = pool.shape
    q, out = q.cuda(), torch.empty_like(q, device="cuda")
    ws = torch.empty(md.MD_ATTEND_WORKSPACE, dtype=torch.uint8, device="cuda") if workspace else None
    scales = torch.ones((L, P, Hkv, 2, ps // 16), device="cuda")
    many = 1 if n > 700 else 64                                   # a warp, a CTA or a cluster per row
    table = torch.arange(P, dtype=torch.int32, device="cuda")
    for batch in {1, many}:
        out = torch.empty((batch,) + q.shape[1:], dtype=torch.bfloat16, device="cuda")
        md.md_attend_cache(q.expand(batch, -1, -1, -1).contiguous(), pool.cuda(), table.expand(batch, -1).contiguous(), [n] * batch,
                           out, scales=scales, workspace=ws)
        err = (out.cpu().double() - ref).abs() / (2.0 ** -8 * ref.abs() + 2.0 ** -17 * size)
        assert float(err.max()) <= 1, float(err.max())
