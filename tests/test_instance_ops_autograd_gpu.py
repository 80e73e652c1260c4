"""What autograd sees of the operators: writes into the caller's tensors count
as changes in place, and tensors that ask for a gradient are refused."""
import pytest

torch = pytest.importorskip("torch")
import torch.autograd.forward_ad as forward_ad  # noqa: E402

from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, device="cuda", dtype=dtype)


def calls():
    """{name: (call, its input tensors by keyword, the tensors that it writes by keyword)}"""
    i32, i64, f32 = torch.int32, torch.int64, torch.float32
    f = ops.rotary_frequencies(64)
    offsets = torch.tensor([0, 5], device="cuda", dtype=i32)
    return {
        "rotary": (ops.rotary, dict(x=zeros(3, 2, 64), positions=zeros(3, dtype=i32), frequencies=f), dict(out=zeros(3, 2, 64)), {}),
        "latent_append": (ops.latent_append, dict(latent=zeros(3, 512), key=zeros(3, 64), positions=zeros(3, dtype=i32), frequencies=f,
                                                  slots=torch.arange(3, device="cuda")), dict(cache=zeros(2, 16, 576)), {}),
        "latent_decode": (ops.latent_decode, dict(q=zeros(1, 1, 4, 576), cache=zeros(2, 16, 576), table=zeros(1, 2, dtype=i32),
                                                  lengths=torch.full((1,), 5, device="cuda", dtype=i32)),
                          dict(out=zeros(1, 1, 4, 512), lse=zeros(1, 1, 4, dtype=f32)), dict(scale=1.0)),
        "latent_prefill": (ops.latent_prefill, dict(q=zeros(5, 2, 192), key=zeros(5, 2, 128), shared=zeros(5, 64), value=zeros(5, 2, 128),
                                                    q_offsets=offsets, k_offsets=offsets),
                           dict(out=zeros(5, 2, 128), lse=zeros(5, 2, dtype=f32)), dict(scale=1.0, longest=5)),
        "sample": (ops.sample, dict(logits=zeros(2, 100), uniform=zeros(2, dtype=f32), temperature=zeros(2, dtype=f32) + 1,
                                    top_p=zeros(2, dtype=f32) + 0.9, min_p=zeros(2, dtype=f32), top_k=zeros(2, dtype=i32)),
                   dict(out=zeros(2, dtype=i64), logprob=zeros(2, dtype=f32)), {}),
    }


NAMES = ["rotary", "latent_append", "latent_decode", "latent_prefill", "sample"]


@pytest.mark.parametrize("name", NAMES)
def test_writes_raise_the_version(name):
    call, given, written, rest = calls()[name]
    before = {k: t._version for k, t in {**given, **written}.items()}
    call(**given, **written, **rest)
    assert all(t._version > before[k] for k, t in written.items())
    assert all(t._version == before[k] for k, t in given.items())
    with torch.inference_mode():
        made = {k: torch.zeros_like(t) for k, t in written.items()}
    call(**given, **made, **rest)  # tensors without a version are written as before
    with torch.inference_mode():
        call(**given, **made, **rest)


def test_a_backward_pass_sees_the_change():
    w = torch.ones(3, 2, 64, device="cuda", requires_grad=True)
    x = torch.randn(3, 2, 64, device="cuda")
    loss = (x * w).sum()  # keeps x
    with torch.no_grad():
        ops.rotary(x, torch.arange(3, device="cuda"), ops.rotary_frequencies(64), out=x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


@pytest.mark.parametrize("name", NAMES)
def test_gradients_are_refused(name):
    call, given, written, rest = calls()[name]
    for k in [k for k, t in {**given, **written}.items() if t.is_floating_point()]:
        args = {**given, **written}
        args[k] = args[k].clone().requires_grad_()
        with pytest.raises(ValueError, match="forward only"):
            call(**args, **rest)
        with torch.no_grad():
            call(**args, **rest)
        with forward_ad.dual_level():
            args[k] = forward_ad.make_dual(args[k].detach(), torch.ones_like(args[k]))
            with pytest.raises(ValueError, match="tangent"):
                call(**args, **rest)
            call(**{**args, k: forward_ad.unpack_dual(args[k]).primal}, **rest)
