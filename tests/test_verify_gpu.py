"""Verification of drafted tokens on the GPU against its definition in 64 bits.

Tokens are whole numbers: they must be equal wherever the numbers that decide are
further from a border than 32-bit weights can move them (a probability is good to 4e-7 of itself, a
sum of them to that of its terms), and the other side of the border else.  A log-probability is
one of a weight of 2^-22 and a sum: 1e-6 and 1e-6 of itself are allowed."""
import math

import pytest

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402

pytestmark = pytest.mark.gpu

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
NEAR = 4e-7


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    yield
    assert ops.faults() == 0


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def chances(row, t):
    """softmax(row / t) in 64 bits (zeros: no logit above -infinity), and its logarithm."""
    x = row.double()
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    top = x.max()
    if top == -math.inf:
        return torch.zeros_like(x), torch.full_like(x, -math.inf)
    if not t > 0:
        p = torch.zeros_like(x)
        p[int((x == top).nonzero()[0])] = 1.0
        return p, torch.log(p)
    x = (x == math.inf).double().log() if top == math.inf else torch.where(x == -math.inf, x, (x - top) / t)
    x = torch.where(x < -126 * math.log(2), torch.full_like(x, -math.inf), x)  # (weights that 32 bits do not hold are none)
    w = torch.exp(x)
    return w / w.sum(), x - torch.log(w.sum())


def check(target, tokens, uniform, draft, temperature, drafted, out, count, logprob):
    b, places, vocab = target.shape
    d = places - 1
    for r in range(b):
        t = 1.0 if temperature is None else float(temperature[r])
        n = d if drafted is None else min(max(int(drafted[r]), 0), d)
        got, kept = out[r].tolist(), int(count[r])
        u = uniform[r].double().tolist()
        assert 1 <= kept <= n + 1
        for i in range(kept):
            p, logs = chances(target[r, i], t)
            q = None
            if i < n:
                x = int(tokens[r, i])
                q = torch.zeros_like(p)
                if draft is not None:
                    q = chances(draft[r, i], t)[0]
                elif 0 <= x < vocab:
                    q[x] = 1.0
                px, qx = (float(p[x]), float(q[x])) if 0 <= x < vocab else (0.0, 0.0)
                border = abs(u[i] * qx - px) <= NEAR * (px + qx)
                assert border or (u[i] * qx < px) == (i < kept - 1), (r, i, u[i] * qx, px)
            if i < kept - 1:
                assert got[i] == x
            else:
                weight = (p - q).clamp_min(0) if i < n else p
                if not float(weight.sum()) > 0:
                    weight = p
                total = float(weight.sum())
                if total == 0:
                    assert got[i] == -1 and float(logprob[r, i]) == -math.inf
                    continue
                sums = weight.cumsum(0)
                v = got[i]
                assert 0 <= v < vocab
                slack = NEAR * (float(p.sum()) + float(q.sum() if q is not None else 0)) + 1e-12
                below = float(sums[v]) - float(weight[v])
                assert below - slack <= u[d] * total <= float(sums[v]) + slack, (r, i, below, u[d] * total, float(sums[v]))
                assert float(p[v]) > 0
            lp = float(logs[got[i]])
            assert abs(float(logprob[r, i]) - lp) <= 1e-6 + 1e-6 * abs(lp), (r, i)
        assert got[kept:] == [-1] * (places - kept) and (logprob[r, kept:] == -math.inf).all()


def case(b, d, vocab, dtype, seed, spread=2.0, apart=0.5, known=True):
    g = gen(seed)
    target = (torch.randn(b, d + 1, vocab, generator=g, device="cuda") * spread)
    draft = (target[:, :d] + apart * torch.randn(b, d, vocab, generator=g, device="cuda")).to(dtype)
    noise = -torch.log(-torch.log(torch.rand(draft.shape, generator=g, device="cuda").clamp(1e-30, 1 - 1e-7)))
    tokens = (draft.float() + noise).argmax(-1) if known else draft.argmax(-1)
    return target.to(dtype), tokens, torch.rand(b, d + 1, generator=g, device="cuda"), draft if known else None


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("known", [True, False])
@pytest.mark.parametrize("b,d,vocab", [(1, 1, 1), (1, 0, 7), (3, 2, 5), (1, 4, 32000), (9, 3, 1023), (5, 8, 4097), (40, 5, 333), (2, 64, 100),
                                       (3, 2, 131075), (1, 1, 1 << 20), (200, 1, 64), (7, 10, 2048), (2, 3, 50001), (160, 2, 8192)])
def test_verify(b, d, vocab, known, dtype):
    target, tokens, uniform, draft = case(b, d, vocab, dtype, seed=b + d + vocab, known=known)
    check(target, tokens, uniform, draft, None, None, *ops.verify(target, tokens, uniform, draft=draft))
    temperature = torch.linspace(0.3, 1.7, b, device="cuda")
    temperature[::4] = 0.0
    drafted = torch.randint(0, d + 1, (b,), generator=gen(1), device="cuda", dtype=torch.int32)
    rest = dict(draft=draft, temperature=temperature, drafted=drafted)
    got = ops.verify(target, tokens, uniform, **rest)
    check(target, tokens, uniform, draft, temperature, drafted, *got)
    assert all(torch.equal(x, y) for x, y in zip(got, ops.verify(target, tokens, uniform, **rest)))  # the same bits


@pytest.mark.parametrize("b,d,dtype", [(310, 1, BF), (160, 0, F32), (90, 2, HF), (40, 1, BF), (21, 1, HF)])
def test_verify_more_requests_than_blocks_of_threads(b, d, dtype):
    """Every size of cluster, down to one block with more steps a warp than are kept."""
    for known in (True, False):
        target, tokens, uniform, draft = case(b, d, 70001, dtype, seed=b, known=known)
        check(target, tokens, uniform, draft, None, None, *ops.verify(target, tokens, uniform, draft=draft))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_ends_of_the_uniform_numbers(dtype):
    """0 accepts whatever the target can give and draws the first token; just below 1 the last."""
    target, tokens, uniform, draft = case(6, 3, 777, dtype, seed=2)
    target[..., :5], target[..., 770:] = -math.inf, -math.inf
    for u in (0.0, 1.0 - 2.0 ** -24, 0.5):
        uniform.fill_(u)
        for drafted in (None, torch.tensor([0, 1, 2, 3, -5, 99], dtype=torch.int32, device="cuda")):
            got = ops.verify(target, tokens, uniform, draft=draft, drafted=drafted)
            check(target, tokens, uniform, draft, None, drafted, *got)
    uniform.fill_(0.0)
    tokens.fill_(300)
    out, count, _ = ops.verify(target, tokens, uniform, draft=draft)
    assert (count == 4).all() and (out[:, :3] == 300).all() and (out[:, 3] == 5).all()


@pytest.mark.parametrize("u,as_if", [(1.0, 1.0 - 2.0 ** -24), (7.5, 1.0 - 2.0 ** -24), (math.inf, 1.0 - 2.0 ** -24), (-0.5, 0.0), (-math.inf, 0.0), (math.nan, 0.0)])
def test_a_draw_by_a_number_outside_its_range(u, as_if):
    """Every request gets a token, that of the nearest number in the range (NaN: of 0)."""
    for vocab in (9, 70001):
        target, tokens, uniform, _ = case(3, 0, vocab, BF, seed=4, spread=0.1)
        got = ops.verify(target, tokens, uniform.fill_(u), out=torch.full((3, 1), -7, device="cuda"), count=torch.zeros(3, dtype=torch.int32, device="cuda"))
        assert (got[1] == 1).all() and all(torch.equal(x, y) for x, y in zip(got, ops.verify(target, tokens, uniform.fill_(as_if))))


@pytest.mark.parametrize("known", [True, False])
def test_greedy(known):
    """A temperature of zero (or NaN, or below): the largest logit of lowest index, and tokens are accepted while they are it."""
    target, tokens, uniform, draft = case(4, 3, 500, BF, seed=3, known=known)
    target[:, :, 40], target[:, :, 90], target[:, :, 300] = 20.0, 20.0, 20.0
    tokens[:] = 40
    tokens[1, 0], tokens[2, 2] = 90, 41
    t = torch.tensor([0.0, -1.0, math.nan, 0.0], device="cuda")
    for kind in (BF, HF, F32):
        args = target.to(kind), tokens, uniform
        got = ops.verify(*args, draft=None if draft is None else draft.to(kind), temperature=t)
        check(*args, None if draft is None else draft.to(kind), t, None, *got)
        assert got[1].tolist() == [4, 1, 3, 4] and got[0][1].tolist() == [40, -1, -1, -1] and got[0][2].tolist() == [40, 40, 40, -1]
        assert (got[2][0] == 0).all()


def test_logits_that_are_none():
    """NaN counts as -infinity, +infinity takes the probability, rows of nothing refuse and give -1."""
    target, tokens, uniform, draft = case(8, 2, 300, F32, seed=4)
    target[0, 0], draft[1, 0] = -math.inf, -math.inf
    target[2, 2] = math.nan
    target[3, 0, [7, 250]] = math.inf
    tokens[3, 0] = 250
    draft[4, 0, [7, 250]] = math.inf
    tokens[4, 0] = 7
    target[5, :, ::3] = math.nan
    draft[5, :, 1::3] = math.nan
    target[6] = -math.inf
    tokens[7, 0], tokens[7, 1] = -1, 300
    uniform[2:4, :2] = 0.0
    for d in (draft, None):
        for t in (None, torch.full((8,), 0.5, device="cuda"), torch.zeros(8, device="cuda")):
            check(target, tokens, uniform, d, t, None, *ops.verify(target, tokens, uniform, draft=d, temperature=t))


@pytest.mark.parametrize("t", [1e-30, 1e-3, 1e6, math.inf])
def test_extreme_temperatures(t):
    target, tokens, uniform, draft = case(5, 2, 1000, F32, seed=5)
    target[..., ::50] = -math.inf
    temperature = torch.full((5,), t, device="cuda")
    check(target, tokens, uniform, draft, temperature, None, *ops.verify(target, tokens, uniform, draft=draft, temperature=temperature))


def test_equal_distributions_accept_everything():
    """p = q: u q < p for every u below one, and logits far from zero or apart do not matter."""
    target, tokens, uniform, _ = case(20, 4, 900, F32, seed=6)
    target = target * 10 + 3000.0
    draft = target[:, :4].contiguous()
    tokens = draft.argmax(-1)
    out, count, _ = ops.verify(target, tokens, uniform, draft=draft)
    assert (count == 5).all() and torch.equal(out[:, :4], tokens)
    tokens[:] = draft.argmin(-1)  # of almost no probability: refused where the draft could not have drawn it
    check(target, tokens, uniform, draft, None, None, *ops.verify(target, tokens, uniform, draft=draft))


@pytest.mark.parametrize("known", [True, False])
def test_the_target_distribution_comes_out(known):
    """Over many draws the first token has the target's distribution, whatever the draft's: every frequency within five standard deviations."""
    n, vocab = 40000, 12
    g = gen(7)
    target = torch.randn(1, 2, vocab, generator=g, device="cuda")
    draft = torch.randn(1, 1, vocab, generator=g, device="cuda")
    q = torch.softmax(draft[0, 0].double(), 0)
    tokens = torch.multinomial(q, n, replacement=True, generator=g)[:, None] if known else torch.randint(0, vocab, (n, 1), generator=g, device="cuda")
    out, _, _ = ops.verify(target.expand(n, 2, vocab), tokens, torch.rand(n, 2, generator=g, device="cuda"),
                           draft=draft.expand(n, 1, vocab) if known else None)
    p = torch.softmax(target[0, 0].double(), 0)
    got = torch.bincount(out[:, 0], minlength=vocab).double() / n
    assert ((got - p).abs() <= 5 * torch.sqrt(p * (1 - p) / n)).all()


@pytest.mark.parametrize("dtype", [BF, HF, F32])
def test_strides_and_alignment(dtype):
    """Rows off a vector's place and behind one another with gaps (sums are split by the vectors' places, so
    that log-probabilities may differ in their last bits), rows that repeat."""
    near = lambda x, y: torch.equal(x[0], y[0]) and torch.equal(x[1], y[1]) and torch.allclose(x[2], y[2], rtol=1e-6, atol=1e-6)
    for vocab in (1000, 4097):
        target, tokens, uniform, draft = case(6, 2, vocab, dtype, seed=8)
        want = ops.verify(target, tokens, uniform, draft=draft)
        for gap, first in ((1, 0), (16, 3), (24, 8), (5, 1), (2, 6)):
            store = torch.full((6, 3, vocab + gap + first), 99.0, device="cuda", dtype=dtype)
            other = torch.full((2, 6, vocab + gap + first + 1), 99.0, device="cuda", dtype=dtype)
            a, b = store[:, :, first:first + vocab], other.transpose(0, 1)[:, :, first:first + vocab]
            a.copy_(target), b.copy_(draft)
            got = ops.verify(a, tokens, uniform, draft=b)
            assert near(want, got)
            check(target, tokens, uniform, draft, None, None, *got)
        got = ops.verify(target[:1].expand(target.shape), tokens, uniform, draft=draft[:, :1].expand(draft.shape))
        want = ops.verify(target[:1].expand(target.shape).contiguous(), tokens, uniform, draft=draft[:, :1].expand(draft.shape).contiguous())
        assert near(got, want)


def test_given_outputs_streams_and_graphs():
    target, tokens, uniform, draft = case(9, 3, 5000, BF, seed=9)
    out = torch.full((9, 4), 77, device="cuda"), torch.full((9,), 77, device="cuda", dtype=torch.int32), torch.full((9, 4), 7.0, device="cuda")
    call = lambda: ops.verify(target, tokens, uniform, draft=draft, out=out[0], count=out[1], logprob=out[2])
    want = [t.clone() for t in ops.verify(target, tokens, uniform, draft=draft)]
    before = [t._version for t in out]
    assert all(x is y for x, y in zip(call(), out)) and all(torch.equal(x, y) for x, y in zip(out, want))
    assert all(t._version > v for t, v in zip(out, before))
    s, late = torch.cuda.Stream(), torch.zeros_like(target)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        late.copy_(target)
        got = ops.verify(late, tokens, uniform, draft=draft)
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    target.copy_(target.flip(0)), uniform.mul_(0.5)
    want = [t.clone() for t in ops.verify(target, tokens, uniform, draft=draft)]
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(out, want))
    assert all(t.shape[0] == 0 for t in ops.verify(target[:0], tokens[:0], uniform[:0], draft=draft[:0]))
    for k in ("target", "draft"):
        args = dict(target=target, tokens=tokens, uniform=uniform, draft=draft)
        args[k] = args[k].clone().requires_grad_()
        with pytest.raises(ValueError, match="forward only"):
            ops.verify(**args)
