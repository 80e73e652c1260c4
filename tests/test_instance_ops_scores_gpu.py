"""Attention where scores lie far apart or are very large, on the GPU against
the formula in 64 bits.  Tolerances are those of test_instance_ops_gpu."""
import math

import pytest

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402
from test_instance_ops_gpu import BF, HF, check_decode, check_prefill, decode_case, device, gen, prefill_case, randn  # noqa: E402, F401

pytestmark = pytest.mark.gpu


# A score above all others whose value is zero: the result is what the others
# leave, each with a weight of e^-16 to e^-18.  Weights are off by at most 2^-35
# (float16) of the largest, n of them by n 2^-35 = 3e-6 v at 100,000: within
# the tolerance of 2^-10 of their sum, n e^-17 v = 4e-3 v.
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("n,heads", [(300, 16), (20000, 16), (100000, 16), (20000, 128)])
def test_decode_many_small_weights(n, heads, dtype):
    q, cache, table, lengths = decode_case([n, 40], 1, heads, 512, 64, 16, dtype, seed=n)
    g = gen(n)
    rows = cache.view(-1, 576)
    rows[:, :512] = randn(g, rows.shape[0], 512).abs().to(dtype)
    rows[:, 512:] = 0
    rows[:, 513] = torch.rand(rows.shape[0], generator=g, device="cuda").to(dtype)
    q[..., :512] = 0
    q[..., 512:514] = torch.tensor([18.0, 2.0], device="cuda", dtype=dtype)
    cache[int(table[0, n // 32]), 3] = 0
    cache[int(table[0, n // 32]), 3, 512] = 1.0
    out, lse = ops.latent_decode(q, cache, table, lengths, scale=1.0)
    check_decode(q, cache, table, lengths, 512, 1.0, out, lse)
    assert float(out[0].max()) > 0


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("nq,nk,heads", [(3, 380, 2), (3, 20000, 1), (200, 20000, 80)])
def test_prefill_many_small_weights(nq, nk, heads, dtype):
    q, key, shared, value, qo, ko = prefill_case([nq], [nk], heads, 128, 64, 128, dtype, seed=nk)
    value.abs_()
    key.zero_(), shared.zero_(), q.zero_()
    key[:, :, 1] = torch.rand(nk, heads, generator=gen(nk), device="cuda").to(dtype)
    shared[nk // 3, 0] = 1.0
    key[nk // 3], value[nk // 3] = 0, 0
    q[..., 1], q[..., 128] = 2.0, 18.0
    out, lse = ops.latent_prefill(q, key, shared, value, qo, ko, scale=1.0, longest=nq)
    check_prefill(q, key, shared, value, qo, ko, 1.0, out, lse)
    assert float(out.max()) > 0


# Scores of 1e6 and more, far apart: all of the weight is on the largest.  The
# result is its value, rounded once; a score's 32-bit sum is good to 1e-6 of the
# products' absolute sum, which is about five times the largest score.
def one_hot(s, value, out, lse):
    assert torch.allclose(lse.double(), s.amax(1), rtol=1e-5)
    alone = torch.topk(s, 2).values.diff()[:, 0].abs() > 1e-5 * s.abs().max()  # no two compete
    assert alone.double().mean() > 0.99
    want = value[s.argmax(1)].double()[alone]
    assert ((out[alone].double() - want).abs() <= 2.0 ** -8 * want.abs()).all()
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("dtype,size", [(BF, 1e5), (BF, 2e3), (HF, 1e4), (HF, 1e3)])
@pytest.mark.parametrize("n,heads", [(90, 16), (700, 16), (700, 128), (5000, 16)])
def test_decode_very_large_scores(n, heads, dtype, size):
    q, cache, table, lengths = decode_case([n, 40], 1, heads, 512, 64, 16, dtype, seed=n)
    q, cache = (q.float() * size).to(dtype), (cache.float() * size).to(dtype)
    out, lse = ops.latent_decode(q, cache, table, lengths, scale=0.1)
    for b, m in enumerate((n, 40)):
        rows = cache[table[b, :-(-m // 16)].long()].reshape(-1, 576)[:m]
        one_hot(q[b, 0].double() @ rows.double().T * 0.1, rows[:, :512], out[b, 0], lse[b, 0])


@pytest.mark.parametrize("dtype,size", [(BF, 1e5), (BF, 2e3), (HF, 1e4), (HF, 1e3)])
@pytest.mark.parametrize("nq,nk,heads", [(100, 100, 2), (130, 3000, 1), (300, 700, 40)])
def test_prefill_very_large_scores(nq, nk, heads, dtype, size):
    args = prefill_case([nq], [nk], heads, 128, 64, 128, dtype, seed=nk)
    q, key, shared, value = [(t.float() * size).to(dtype) for t in args[:4]]
    out, lse = ops.latent_prefill(q, key, shared, value, *args[4:], scale=0.1, longest=nq, causal=False)
    for h in range(heads):
        s = q[:, h].double() @ torch.cat((key[:, h], shared), 1).double().T * 0.1
        one_hot(s, value[:, h], out[:, h], lse[:, h])
