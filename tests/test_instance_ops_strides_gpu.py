"""Tensors that repeat a row (a stride of zero, as ``expand`` gives) and dimensions
of one element whose stride says nothing: the bits of the contiguous copies."""
import pytest

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402
from test_instance_ops_gpu import BF, F32, HF, decode_case, device, gen, prefill_case, randn  # noqa: E402, F401

pytestmark = pytest.mark.gpu


def same(call, args, changed, **rest):
    """The call with some arguments replaced equals the call with their contiguous copies."""
    got = call(*[changed.get(i, t) for i, t in enumerate(args)], **rest)
    want = call(*[changed[i].contiguous() if i in changed else t for i, t in enumerate(args)], **rest)
    got, want = ([r] if torch.is_tensor(r) else r for r in (got, want))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def odd(t, dim, stride):
    """The same elements with that stride for a dimension of size one."""
    assert t.shape[dim] == 1
    strides = list(t.stride())
    strides[dim] = stride
    return t.as_strided(t.shape, strides)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("nq,nk,heads", [([200, 33], [200, 90], 4), ([700], [3000], 2), ([600] * 8, [600] * 8, 40)])
def test_prefill_expanded(nq, nk, heads, dtype):
    args = prefill_case(nq, nk, heads, 128, 64, 128, dtype, seed=1)
    rest = dict(scale=0.1, longest=max(nq))
    q, key, shared, value = args[:4]
    one = lambda t: t[:, :1].expand(t.shape)
    for changed in ({1: one(key)}, {3: one(value)}, {0: one(q)}, {1: one(key), 3: one(value)}, {2: shared[:1].expand(shared.shape)},
                    {0: q[:1].expand(q.shape)}, {1: key[:1].expand(key.shape), 3: value[:1].expand(value.shape)}):
        same(ops.latent_prefill, args, changed, **rest)


def test_prefill_one_row_or_head():
    for nq, heads in ((1, 4), (50, 1), (1, 1)):
        args = prefill_case([nq], [nq], heads, 128, 64, 128, BF, seed=2)
        for i in (0, 1, 3):
            for dim in range(2):
                if args[i].shape[dim] == 1:
                    same(ops.latent_prefill, args, {i: odd(args[i], dim, 77)}, scale=0.1, longest=nq)
        if nq == 1:
            same(ops.latent_prefill, args, {2: odd(args[2], 0, 33)}, scale=0.1, longest=nq)
            out = torch.empty(1, heads, 128, device="cuda", dtype=BF)
            want, _ = ops.latent_prefill(*args, scale=0.1, longest=1)
            assert torch.equal(ops.latent_prefill(*args, scale=0.1, longest=1, out=odd(out, 0, 5))[0], want)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("requests,new,heads,block", [(3, 1, 16, 16), (2, 2, 40, 16), (2, 3, 16, 12), (1, 1, 128, 64)])
def test_decode_expanded(requests, new, heads, block, dtype):
    q, cache, table, n = decode_case([300, 70, 5][:requests], new, heads, 512, 64, block, dtype, seed=3, junk=0.0)
    args = (q, cache, table, n)
    for changed in ({0: q[:, :, :1].expand(q.shape)}, {0: q[:1].expand(q.shape)}, {0: q[:, :1].expand(q.shape)},
                    {1: cache[:1].expand(cache.shape)}, {2: table[:1].expand(table.shape)}):
        same(ops.latent_decode, args, changed, scale=0.05)


def test_decode_one_of_each():
    q, cache, table, n = decode_case([9], 1, 1, 512, 64, 16, BF, seed=4, junk=0.0)
    args = (q, cache, table, n)
    for changed in ({0: odd(q, 0, 3)}, {0: odd(q, 1, 3)}, {0: odd(q, 2, 3)}, {1: odd(cache[:1], 0, 7)}, {2: odd(table, 0, 1)}):
        same(ops.latent_decode, args, changed, scale=0.05)
    q, cache, table, n = decode_case([9], 1, 4, 512, 64, 1, BF, seed=4, junk=0.0)
    same(ops.latent_decode, (q, cache, table, n), {1: odd(cache, 1, 7)}, scale=0.05)
    out = torch.empty(1, 1, 4, 512, device="cuda", dtype=BF)
    want, _ = ops.latent_decode(q, cache, table, n, scale=0.05)
    assert torch.equal(ops.latent_decode(q, cache, table, n, scale=0.05, out=odd(odd(out, 0, 9), 1, 9))[0], want)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rotary_append_sample_expanded(dtype):
    g = gen(5)
    f, pos = ops.rotary_frequencies(64), torch.arange(7, device="cuda")
    x = randn(g, 7, 4, 128, dtype=dtype)
    for v in (x[:, :1].expand(x.shape), x[:1].expand(x.shape), odd(x[:1, :1], 0, 3), odd(x[:1, :1], 1, 3)):
        same(ops.rotary, (v, pos[:len(v)], f), {0: v}, offset=64)
    latent, key, slots = randn(g, 7, 512, dtype=dtype), randn(g, 7, 64, dtype=dtype), torch.arange(7, device="cuda")
    for changed in ({0: latent[:1].expand(7, 512)}, {1: key[:1].expand(7, 64)}):
        cache = [torch.zeros(1, 16, 576, device="cuda", dtype=dtype) for _ in range(2)]
        for c, same_as in zip(cache, (lambda t: t, lambda t: t.contiguous())):
            ops.latent_append(*[same_as(changed[i]) if i in changed else t for i, t in enumerate((latent, key))], pos, f, slots, c)
        assert torch.equal(*cache)
    logits, u = randn(g, 5, 4000, dtype=dtype), torch.rand(5, generator=g, device="cuda")
    same(ops.sample, (logits[:1].expand(5, 4000), u), {0: logits[:1].expand(5, 4000)})
    same(ops.sample, (odd(logits[:1], 0, 1), u[:1]), {0: odd(logits[:1], 0, 1)})
