"""The boundary of the 8-bit cache's, the drafts' and the blocks' operators
without a GPU: packed argument structs, refusals in C and in the binding."""
import re
import shutil
import struct as S
import subprocess

import pytest

from paper_2608_16336_gb300 import _build, mtsim

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402
from test_instance_ops_abi import _fields  # noqa: E402

STRUCTS = {"sim_op_quantized_append": ops.QUANTIZED_APPEND, "sim_op_quantized_decode": ops.QUANTIZED_DECODE,
           "sim_op_verify": ops.VERIFY, "sim_op_block_copy": ops.BLOCK_COPY}
EMPTY = {"sim_op_quantized_append": "tokens", "sim_op_quantized_decode": "requests", "sim_op_verify": "requests", "sim_op_block_copy": "pairs"}


@pytest.fixture(scope="module")
def L():
    _build.build_mtsim()
    return ops.lib()


@pytest.mark.parametrize("name", sorted(STRUCTS))
def test_packed_structs_have_the_compilers_layout(name, tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no compiler")
    fields = _fields(name + "_t")
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "mtsim_ops.h"', "int main(void) {",
             '    printf("%%zu\\n", sizeof(%s_t));' % name]
    lines += ['    printf("%%zu\\n", offsetof(%s_t, %s));' % (name, f) for _, f in fields]
    src, exe = tmp_path / "s.c", tmp_path / "s"
    src.write_text("\n".join(lines + ["    return 0;", "}"]) + "\n")
    subprocess.run(["gcc", "-std=c99", "-I", _build.INCLUDE, str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    codes = STRUCTS[name].format.lstrip("@").replace("0q", "")
    kinds = {"int64_t": "q", "int32_t": "i", "float": "f", "size_t": "N"}
    assert len(codes) == len(fields)
    for code, (kind, f) in zip(codes, fields):
        assert code == ("P" if "*" in kind or kind.startswith("const") or kind == "void" else kinds[kind]), f
    assert got == [STRUCTS[name].size] + [S.calcsize("@" + codes[:i] + "0" + codes[i]) for i in range(len(codes))]


def test_limits_are_the_headers():
    text = open(_build.INCLUDE + "/mtsim_ops.h").read()
    assert int(re.search(r"#define SIM_OP_MAX_DRAFTS (\d+)", text).group(1)) == ops.MAX_DRAFTS


def _args(name, **over):
    """Plausible arguments with fake device pointers (the refusals come before any use), some replaced."""
    sizes = dict(tokens=4, latent_token=512, key_token=64, cache_block=16 * 576, cache_row=576, table_row=4, blocks=8, requests=2,
                 table_blocks=4, block_tokens=16, rank=512, rot_dim=64, key_dim=64, amplitude=1.0, workspace_bytes=1 << 40, q_request=2304,
                 q_token=2304, q_head=576, out_request=2048, out_token=2048, out_head=512, new_tokens=1, heads=4, scale=1.0,
                 target_request=500, target_row=100, draft_request=400, draft_row=100, drafts=4, vocab=100, row_bytes=576,
                 source_layer=8 * 9216, source_block=9216, source_row=576, destination_layer=8 * 9216, destination_block=9216,
                 destination_row=576, source_blocks=8, destination_blocks=8, layers=2, rows=16, pairs=3)
    if name == "sim_op_verify":
        sizes["tokens"] = 0x10000
    vals = []
    for kind, f in _fields(name + "_t"):
        pointer = "*" in kind or kind.startswith("const") or kind == "void"
        vals.append(over.get(f, 0x10000 if pointer else sizes.get(f, 0)))
    return STRUCTS[name].pack(*vals)


A, D, V, C = "sim_op_quantized_append", "sim_op_quantized_decode", "sim_op_verify", "sim_op_block_copy"
BAD = [
    (A, dict(type=3)), (A, dict(layout=2)), (A, dict(tokens=-1)), (A, dict(requests=-1)), (A, dict(block_tokens=0)), (A, dict(rank=0)),
    (A, dict(rot_dim=0)), (A, dict(rot_dim=7)), (A, dict(rot_dim=258)), (A, dict(blocks=-2)), (A, dict(table_blocks=-1)),
    (A, dict(scales=0)), (A, dict(offsets=0)), (A, dict(cache=0)), (A, dict(amplitude=float("nan"))), (A, dict(tokens=1 << 31)),
    (A, dict(table_blocks=1 << 28)), (A, dict(rank=0x7FFFFFFF)),
    (D, dict(type=2)), (D, dict(rank=96)), (D, dict(rank=0)), (D, dict(rank=576)), (D, dict(key_dim=8)), (D, dict(key_dim=80)),
    (D, dict(key_dim=-16)), (D, dict(requests=-1)), (D, dict(block_tokens=0)), (D, dict(scale=float("inf"))), (D, dict(q=0)),
    (D, dict(scales=0)), (D, dict(q=0x10008)), (D, dict(cache=0x10008)), (D, dict(cache_row=580)), (D, dict(cache_block=9224)),
    (D, dict(cache_row=560)), (D, dict(cache_block=9216 + 16)), (D, dict(out_head=516)), (D, dict(workspace=0)), (D, dict(workspace_bytes=0)),
    (D, dict(workspace=0x10010)), (D, dict(heads=1 << 30, new_tokens=4)), (D, dict(table_blocks=1 << 28)),
    (V, dict(type=-1)), (V, dict(requests=-1)), (V, dict(drafts=-1)), (V, dict(drafts=65)), (V, dict(vocab=0)), (V, dict(vocab=(1 << 20) + 1)),
    (V, dict(target=0)), (V, dict(tokens=0)), (V, dict(uniform=0)), (V, dict(out=0)), (V, dict(count=0)), (V, dict(requests=(1 << 24) + 1)), (V, dict(workspace=0)),
    (V, dict(workspace=0x10010)), (V, dict(workspace_bytes=0)),
    (C, dict(layers=-1)), (C, dict(rows=-1)), (C, dict(pairs=-1)), (C, dict(row_bytes=-4)), (C, dict(source_blocks=-1)),
    (C, dict(source=0)), (C, dict(destination=0)), (C, dict(from_blocks=0)), (C, dict(to_blocks=0)), (C, dict(destination_row=570)),
]


@pytest.mark.parametrize("name,over", BAD, ids=lambda v: v if isinstance(v, str) else "-".join("%s=%s" % i for i in v.items()))
def test_refusals(L, name, over):
    assert getattr(L, name)(_args(name, **over), None) == mtsim.SIM_ERR_ARG
    assert L.sim_op_last_error()


@pytest.mark.parametrize("name", sorted(STRUCTS))
def test_null_and_empty(L, name):
    assert getattr(L, name)(None, None) == mtsim.SIM_ERR_ARG
    assert getattr(L, name)(_args(name, **{EMPTY[name]: 0}), None) == mtsim.SIM_OK


def zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


I32, I64, F32, E4 = torch.int32, torch.int64, torch.float32, torch.float8_e4m3fn


def append_args(**over):
    f = ops.rotary_frequencies(32, device="cpu")
    return {**dict(latent=zeros(5, 64), key=zeros(5, 32), frequencies=f, offsets=zeros(3, dtype=I32), table=zeros(2, 4, dtype=I32),
                   lengths=zeros(2, dtype=I32), cache=zeros(6, 16, 96, dtype=E4), scales=zeros(6, 2, dtype=F32)), **over}


def decode_args(**over):
    return {**dict(q=zeros(2, 1, 4, 576), cache=zeros(6, 16, 576, dtype=E4), scales=zeros(6, 2, dtype=F32), table=zeros(2, 3, dtype=I32),
                   lengths=zeros(2, dtype=I32), scale=1.0), **over}


def verify_args(**over):
    return {**dict(target=zeros(2, 4, 50), tokens=zeros(2, 3, dtype=I64), uniform=zeros(2, 4, dtype=F32), draft=zeros(2, 3, 50)), **over}


def copy_args(**over):
    return {**dict(source=zeros(2, 6, 16, 64), destination=zeros(2, 9, 16, 64), from_blocks=zeros(3, dtype=I32), to_blocks=zeros(3, dtype=I32)), **over}


CALLS = {"quantized_append": append_args, "quantized_decode": decode_args, "verify": verify_args, "block_copy": copy_args}
REFUSED = [
    ("quantized_append", dict(), ValueError, "CUDA"),
    ("quantized_append", dict(latent=zeros(5, 64, 1)), ValueError, "latent must be"),
    ("quantized_append", dict(key=zeros(5, 30)), ValueError, "key"),
    ("quantized_append", dict(cache=zeros(6, 16, 96)), TypeError, "float8_e4m3fn"),
    ("quantized_append", dict(cache=zeros(6, 16, 98, dtype=E4)), ValueError, "cache"),
    ("quantized_append", dict(scales=zeros(6, 1, dtype=F32)), ValueError, "scales"),
    ("quantized_append", dict(scales=zeros(6, 2)), TypeError, "scales must be float32"),
    ("quantized_append", dict(offsets=zeros(2, dtype=I32)), ValueError, "offsets"),
    ("quantized_append", dict(offsets=zeros(3, dtype=I64)), TypeError, "int32"),
    ("quantized_append", dict(lengths=zeros(3, dtype=I32)), ValueError, "lengths"),
    ("quantized_append", dict(table=zeros(2, 4, dtype=I64)), TypeError, "table"),
    ("quantized_append", dict(latent=zeros(5, 64, dtype=F32)), TypeError, "same type"),
    ("quantized_append", dict(layout="other"), ValueError, "CUDA|layout"),
    ("quantized_decode", dict(), ValueError, "CUDA"),
    ("quantized_decode", dict(q=zeros(2, 1, 4, 584)), ValueError, "rank"),
    ("quantized_decode", dict(q=zeros(2, 1, 4, 576, dtype=F32)), TypeError, "bfloat16 or float16"),
    ("quantized_decode", dict(cache=zeros(6, 16, 576)), TypeError, "float8_e4m3fn"),
    ("quantized_decode", dict(cache=zeros(6, 16, 592, dtype=E4)), ValueError, "cache"),
    ("quantized_decode", dict(scales=zeros(5, 2, dtype=F32)), ValueError, "scales"),
    ("quantized_decode", dict(lengths=zeros(2, dtype=I64)), TypeError, "lengths"),
    ("quantized_decode", dict(table=zeros(3, 3, dtype=I32)), ValueError, "table"),
    ("quantized_decode", dict(lse=zeros(2, 1, 4)), TypeError, "lse"),
    ("quantized_decode", dict(out=zeros(2, 1, 4, 480)), ValueError, "rank"),
    ("verify", dict(), ValueError, "CUDA"),
    ("verify", dict(target=zeros(2, 50)), ValueError, "target must be"),
    ("verify", dict(target=zeros(2, 66, 5)), ValueError, "1 to 65 rows"),
    ("verify", dict(target=zeros(2, 0, 5)), ValueError, "1 to 65 rows"),
    ("verify", dict(target=zeros(2, 4, 0)), ValueError, "vocabulary"),
    ("verify", dict(tokens=zeros(2, 3, dtype=I32)), TypeError, "int64"),
    ("verify", dict(tokens=zeros(2, 4, dtype=I64)), ValueError, "tokens"),
    ("verify", dict(uniform=zeros(2, 3, dtype=F32)), ValueError, "uniform"),
    ("verify", dict(draft=zeros(2, 4, 50)), ValueError, "draft"),
    ("verify", dict(draft=zeros(2, 3, 50, dtype=F32)), TypeError, "same type"),
    ("verify", dict(temperature=zeros(2)), TypeError, "temperature"),
    ("verify", dict(drafted=zeros(3, dtype=I32)), ValueError, "drafted"),
    ("verify", dict(out=zeros(2, 4, dtype=I32)), TypeError, "out must be"),
    ("block_copy", dict(), ValueError, "CUDA"),
    ("block_copy", dict(source=zeros(2, 6)), ValueError, "source and destination"),
    ("block_copy", dict(source=zeros(2, 6, 64)), ValueError, "source and destination"),
    ("block_copy", dict(source=zeros(2, 6, 16, 64, dtype=F32)), TypeError, "same type"),
    ("block_copy", dict(source=zeros(3, 6, 16, 64)), ValueError, "destination"),
    ("block_copy", dict(source=zeros(2, 6, 16, 60)), ValueError, "destination"),
    ("block_copy", dict(from_blocks=zeros(3, dtype=I64)), TypeError, "from_blocks"),
    ("block_copy", dict(to_blocks=zeros(2, dtype=I32)), ValueError, "to_blocks"),
    ("block_copy", dict(destination=zeros(2, 9, 64, 16).transpose(2, 3)), ValueError, "contiguous"),
]


@pytest.mark.parametrize("name,over,error,match", REFUSED, ids=lambda v: v if isinstance(v, str) else None)
def test_binding_refuses_on_the_host(name, over, error, match):
    with pytest.raises(error, match=match):
        getattr(ops, name)(**CALLS[name](**over))
