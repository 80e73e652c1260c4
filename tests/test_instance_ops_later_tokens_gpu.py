"""Infinities and NaN in tokens that a row does not see: the row is as if they
were not there, to the bit, wherever the tiles of keys end."""

import pytest

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402
from test_instance_ops_gpu import BF, HF, decode_case, device, prefill_case  # noqa: E402, F401

pytestmark = pytest.mark.gpu
JUNK = [float("nan"), float("inf"), float("-inf")]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("nq,nk,heads,value_dim", [
    ([200], [200], 2, 128), ([64, 100], [64, 100], 3, 72), ([300, 5], [301, 77], 2, 64),  # short prompts
    ([1000], [1000], 80, 128), ([700, 513], [900, 2600], 40, 104),                         # two tiles a block
    ([257], [5000], 1, 128), ([513, 300], [1300, 3001], 3, 40), ([700, 0], [600, 5000], 2, 8)])  # keys shared by blocks
def test_prefill_later_values_do_not_count(nq, nk, heads, value_dim, dtype):
    q, key, shared, value, qo, ko = prefill_case(nq, nk, heads, 128, 64, value_dim, dtype, seed=sum(nk))
    want, lse = ops.latent_prefill(q, key, shared, value, qo, ko, scale=0.1, longest=max(nq))
    junk = value.clone()
    first = {}  # the first query row of each request that sees each of the bad values
    for b, (a, n) in enumerate(zip(nq, nk)):
        for i, back in enumerate((1, 2, 3, 50, 130, 131, 190, 256)):
            j = n - back
            if j < 0 or a == 0:
                continue
            e = (7 * i + b) % value_dim
            junk[int(ko[b]) + j, i % heads, e] = JUNK[i % 3]
            first[b, i % heads, e, i] = (max(j - (n - a), 0), JUNK[i % 3])
    out, lse2 = ops.latent_prefill(q, key, shared, junk, qo, ko, scale=0.1, longest=max(nq))
    assert torch.equal(lse2, lse)
    hit = {}
    for (b, h, e, _), (row, x) in first.items():
        for r in range(row, nq[b]):
            hit.setdefault((int(qo[b]) + r, h, e), []).append(x)
    same = torch.ones_like(out, dtype=torch.bool)
    for at, xs in hit.items():
        same[at] = False
    assert torch.equal(out[same], want[same])
    at = torch.tensor(list(hit), device="cuda")
    expect = torch.tensor([sum(xs) for xs in hit.values()], device="cuda")
    assert torch.equal(torch.nan_to_num(out[at[:, 0], at[:, 1], at[:, 2]].float(), nan=0.5), torch.nan_to_num(expect, nan=0.5))
    again, _ = ops.latent_prefill(q, key, shared, junk, qo, ko, scale=0.1, longest=max(nq))
    assert torch.equal(torch.nan_to_num(again), torch.nan_to_num(out))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lengths,new,heads,rank,block", [
    ([64, 65, 66, 130], 4, 16, 512, 16), ([1, 2, 3, 0, 5], 5, 3, 512, 16), ([700, 64], 2, 64, 256, 24), ([90, 33], 3, 40, 128, 7),
    ([3000], 3, 16, 512, 16), ([4100, 2500], 7, 10, 192, 33), ([300, 128], 2, 128, 512, 64)])
def test_decode_later_rows_do_not_count(lengths, new, heads, rank, block, dtype):
    """Each of the last new - 1 cached rows in turn holds something that is no number: the new tokens before it are untouched."""
    q, cache, table, n = decode_case(lengths, new, heads, rank, 64, block, dtype, seed=rank + heads)
    q = torch.where(q == 0, torch.ones_like(q), q)
    want, lse = ops.latent_decode(q, cache, table, n, scale=0.05, out=torch.empty(len(lengths), new, heads, rank, device="cuda", dtype=dtype))
    for back in range(new - 1):
        junk = cache.clone()
        for b, m in enumerate(lengths):
            j = m - 1 - back
            if j >= 0:
                for e in (5 + b, 70, rank - 1):
                    junk[int(table[b, j // block]), j % block, e] = JUNK[(b + e) % 3]
        out, lse2 = ops.latent_decode(q, junk, table, n, scale=0.05, out=torch.empty_like(want))
        before = new - 1 - back  # new tokens that come before the bad row
        assert torch.equal(out[:, :before], want[:, :before]) and torch.equal(lse2[:, :before], lse[:, :before])
        for b, m in enumerate(lengths):
            if m - 1 - back >= 0:
                assert not torch.isfinite(out[b, before:, :, [5 + b, 70, rank - 1]]).any()
            else:
                assert torch.equal(out[b], want[b]) and torch.equal(lse2[b], lse[b])
