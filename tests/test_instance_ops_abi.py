"""The operators' boundary without a GPU: include/mtsim_ops.h compiles as
strict C and C++, the packed argument structs have the C compiler's layout,
every declared symbol is exported, and bad arguments are refused on the host."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2608_16336_gb300 import _build, mtsim

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402

HEADER = os.path.join(_build.INCLUDE, "mtsim_ops.h")
STRUCTS = {"sim_op_rotary_t": ops.ROTARY, "sim_op_latent_append_t": ops.APPEND, "sim_op_latent_decode_t": ops.DECODE,
           "sim_op_latent_prefill_t": ops.PREFILL, "sim_op_sample_t": ops.SAMPLE}


def _text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def _fields(name):
    """[(type, field)] of a struct in the header, in order."""
    body = re.search(r"typedef struct \{([^}]*)\}\s*%s;" % name, _text()).group(1)
    out = []
    for decl in body.split(";"):
        decl = decl.strip()
        if decl:
            kind, names = re.match(r"((?:const )?\w+(?: \*)?)\s*(.*)", decl, flags=re.S).groups()
            out += [(kind, n.strip().lstrip("*")) for n in names.split(",")]
    return out


@pytest.fixture(scope="module")
def L():
    _build.build_mtsim()
    return ops.lib()


@pytest.mark.parametrize("std,lang,cc", [("c99", "c", "gcc"), ("c11", "c", "gcc"), ("c++11", "c++", "g++")])
def test_header_is_strict(std, lang, cc):
    if shutil.which(cc) is None:
        pytest.skip("no compiler")
    subprocess.run([cc, "-std=" + std, "-Wall", "-Wextra", "-Werror", "-I", _build.INCLUDE, "-fsyntax-only", "-x", lang, HEADER],
                   check=True)


def test_exports(L):
    declared = sorted(set(re.findall(r"\b(sim_op_[a-z_]+)\s*\(", _text())))
    assert declared == sorted(ops.EXPORTS)
    for name in declared:
        assert hasattr(L, name), name


@pytest.mark.parametrize("name", sorted(STRUCTS))
def test_packed_structs_have_the_compilers_layout(name, tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no compiler")
    fields = _fields(name)
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "mtsim_ops.h"', "int main(void) {",
             '    printf("%%zu\\n", sizeof(%s));' % name]
    lines += ['    printf("%%zu\\n", offsetof(%s, %s));' % (name, f) for _, f in fields]
    src, exe = tmp_path / "s.c", tmp_path / "s"
    src.write_text("\n".join(lines + ["    return 0;", "}"]) + "\n")
    subprocess.run(["gcc", "-std=c99", "-I", _build.INCLUDE, str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    st = STRUCTS[name]
    codes = st.format.lstrip("@").replace("0q", "")
    codes = "".join(c for c in codes)
    assert len(codes) == len(fields)
    import struct as S
    want, kinds = [], {"int64_t": "q", "int32_t": "i", "float": "f", "size_t": "N"}
    for i, (kind, _) in enumerate(fields):
        assert codes[i] == ("P" if "*" in kind or kind.startswith("const") or kind == "void" else kinds[kind]), fields[i]
        want.append(S.calcsize("@" + codes[:i] + "0" + codes[i]))
    assert got == [st.size] + want


def _args(name, **over):
    """Plausible arguments with fake device pointers (the refusals come before any use), some replaced."""
    sizes = dict(tokens=4, x_token=256, x_head=64, out_token=256, out_head=64, heads=4, dim=64, rot_dim=32, rot_offset=0,
                 latent_token=512, key_token=64, cache_block=16 * 576, cache_row=576, blocks=8, block_tokens=16, rank=512,
                 key_dim=64, workspace_bytes=1 << 40, requests=2, new_tokens=1, table_blocks=4, table_row=4, q_request=2304, q_token=2304,
                 q_head=576, out_request=2048, head_dim=128, value_dim=128, longest=8, q_rows=8, k_rows=8, q_row=768,
                 key_row=512, key_head=128, shared_row=64, value_row=512, value_head=128, out_row=512, rows=2, vocab=100,
                 logits_row=100, causal=1, scale=1.0, amplitude=1.0)
    if name == "sim_op_latent_decode":
        sizes.update(out_token=2048, out_head=512)
    if name == "sim_op_latent_prefill":
        sizes.update(q_head=192, out_head=128)
    vals = []
    for kind, f in _fields(name + "_t"):
        pointer = "*" in kind or kind.startswith("const") or kind == "void"
        vals.append(over.get(f, 0x10000 if pointer else sizes.get(f, 0)))
    return STRUCTS[name + "_t"].pack(*vals)


BAD = [
    ("sim_op_rotary", dict(type=3)), ("sim_op_rotary", dict(layout=2)), ("sim_op_rotary", dict(tokens=-1)),
    ("sim_op_rotary", dict(rot_dim=31)), ("sim_op_rotary", dict(rot_dim=0)), ("sim_op_rotary", dict(rot_dim=258, dim=512)),
    ("sim_op_rotary", dict(rot_offset=33)), ("sim_op_rotary", dict(rot_offset=-1)), ("sim_op_rotary", dict(x=0)),
    ("sim_op_rotary", dict(frequencies=0)), ("sim_op_rotary", dict(out_token=128)),
    ("sim_op_latent_append", dict(type=-1)), ("sim_op_latent_append", dict(block_tokens=0)), ("sim_op_latent_append", dict(rank=0)),
    ("sim_op_latent_append", dict(rot_dim=3)), ("sim_op_latent_append", dict(slots=0)), ("sim_op_latent_append", dict(blocks=-1)),
    ("sim_op_latent_decode", dict(type=2)), ("sim_op_latent_decode", dict(rank=96)), ("sim_op_latent_decode", dict(rank=576)),
    ("sim_op_latent_decode", dict(rank=0)), ("sim_op_latent_decode", dict(key_dim=72)), ("sim_op_latent_decode", dict(key_dim=4)),
    ("sim_op_latent_decode", dict(requests=-1)), ("sim_op_latent_decode", dict(block_tokens=0)),
    ("sim_op_latent_decode", dict(scale=float("nan"))), ("sim_op_latent_decode", dict(scale=float("inf"))),
    ("sim_op_latent_decode", dict(q=0)), ("sim_op_latent_decode", dict(q=0x10008)), ("sim_op_latent_decode", dict(cache_row=580)),
    ("sim_op_latent_decode", dict(out_head=516)), ("sim_op_latent_decode", dict(workspace=0)),
    ("sim_op_latent_decode", dict(workspace_bytes=0)), ("sim_op_latent_decode", dict(heads=1 << 30, new_tokens=4)),
    ("sim_op_latent_prefill", dict(type=2)), ("sim_op_latent_prefill", dict(head_dim=136)), ("sim_op_latent_prefill", dict(head_dim=4)),
    ("sim_op_latent_prefill", dict(key_dim=65)), ("sim_op_latent_prefill", dict(value_dim=0)), ("sim_op_latent_prefill", dict(causal=2)),
    ("sim_op_latent_prefill", dict(scale=float("-inf"))), ("sim_op_latent_prefill", dict(key=0)),
    ("sim_op_latent_prefill", dict(value=0x10004)), ("sim_op_latent_prefill", dict(value_head=132)),
    ("sim_op_latent_prefill", dict(requests=70000)), ("sim_op_latent_prefill", dict(longest=-1)),
    ("sim_op_sample", dict(type=5)), ("sim_op_sample", dict(rows=-1)), ("sim_op_sample", dict(vocab=0)),
    ("sim_op_sample", dict(vocab=(1 << 20) + 1)), ("sim_op_sample", dict(token=0)), ("sim_op_sample", dict(uniform=0)),
]


@pytest.mark.parametrize("name,over", BAD, ids=lambda v: v if isinstance(v, str) else "-".join("%s=%s" % i for i in v.items()))
def test_refusals(L, name, over):
    assert getattr(L, name)(_args(name, **over), None) == mtsim.SIM_ERR_ARG
    assert L.sim_op_last_error()


@pytest.mark.parametrize("name", sorted(n[:-2] for n in STRUCTS))
def test_null_and_empty(L, name):
    assert getattr(L, name)(None, None) == mtsim.SIM_ERR_ARG
    empty = {"sim_op_rotary": "tokens", "sim_op_latent_append": "tokens", "sim_op_latent_decode": "requests",
             "sim_op_latent_prefill": "requests", "sim_op_sample": "rows"}[name]
    assert getattr(L, name)(_args(name, **{empty: 0}), None) == mtsim.SIM_OK


def test_binding_refuses_on_the_host():
    f = ops.rotary_frequencies(32, device="cpu")
    x = torch.zeros(4, 2, 64)
    pos = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        ops.rotary(x, pos, f)
    with pytest.raises(ValueError, match="do not lie"):
        ops.rotary(x, pos, f, offset=40)
    with pytest.raises(TypeError, match="int32"):
        ops.rotary(x, pos.float(), f)
    with pytest.raises(ValueError, match="float64"):
        ops.rotary(x, pos, f.float())
    with pytest.raises(TypeError, match="bfloat16"):
        ops.rotary(x.double(), pos, f)
    with pytest.raises(ValueError, match="contiguous"):
        ops.rotary(torch.zeros(4, 64, 40).transpose(1, 2), pos, f)
    with pytest.raises(ValueError, match="rank"):
        ops.latent_decode(torch.zeros(1, 1, 4, 100), torch.zeros(2, 16, 100), torch.zeros(1, 2, dtype=torch.int32),
                          torch.zeros(1, dtype=torch.int32), scale=1.0)
    with pytest.raises(ValueError, match="vocabulary"):
        ops.sample(torch.zeros(2, 0), torch.zeros(2))
    with pytest.raises(TypeError, match="top_k"):
        ops.sample(torch.zeros(2, 8), torch.zeros(2), top_k=torch.zeros(2))
    with pytest.raises(ValueError, match="head"):
        ops.latent_prefill(torch.zeros(4, 2, 100), torch.zeros(4, 2, 64), torch.zeros(4, 32), torch.zeros(4, 2, 64),
                           torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), scale=1.0, longest=4)


@pytest.mark.parametrize("scaling,factor", [(None, 1.0), ("linear", 4.0), ("base", 8.0), ("ramp", 8.0)])
def test_frequencies(scaling, factor):
    f = ops.rotary_frequencies(64, 10000.0, scaling=scaling, factor=factor, trained=4096, device="cpu")
    plain = 10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)
    assert f.dtype is torch.float64 and f.shape == (32,)
    ratio = f / plain
    if scaling is None:
        assert torch.equal(f, plain)
    elif scaling == "linear":
        assert torch.allclose(ratio, torch.full_like(f, 1 / factor), rtol=1e-14)
    elif scaling == "base":
        assert abs(ratio[0] - 1) < 1e-14 and abs(ratio[-1] * factor - 1) < 1e-12 and (ratio.diff() < 0).all()
    else:
        turns = 4096 * plain / (2 * torch.pi)
        assert (ratio[turns > 32] == 1).all() and (ratio[turns < 1] == 1 / factor).all() and (ratio.diff() <= 0).all()
    for bad in (dict(rot_dim=7), dict(rot_dim=64, base=0.0), dict(rot_dim=64, scaling="other"), dict(rot_dim=64, scaling="ramp")):
        with pytest.raises(ValueError):
            ops.rotary_frequencies(device="cpu", **bad)
    assert ops.ramp_amplitude(1.0) == 1.0 and abs(ops.ramp_amplitude(8.0) - 1.2079441541679836) < 1e-12
