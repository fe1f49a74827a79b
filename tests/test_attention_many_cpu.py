"""Attention's kernel of many rows without a GPU: which calls reach it, and what stands
between the reading and the writing of its tiles."""

import os
import re
import subprocess

import pytest
import torch

from paper_2607_16305_amd import build
from paper_2607_16305_amd import lookme as lk
from tests import attention as A
from tests import attention_many as M


@pytest.mark.parametrize("dtype,d", M.MANY)
@pytest.mark.parametrize("name", list(M.CALLS))
def test_the_calls_reach_the_kernel_of_many_rows(name, dtype, d):
    p = M.of(name, dtype, d)
    assert p.tiles == 0 and p.block == (128 if (dtype, d) == ("bf16", 128) else 64)
    assert (p.target == 0) == M.CALLS[name][4]


def _bundle(obj, to):
    """the gfx950 code of one of this library's objects"""
    tools = "/opt/rocm/llvm/bin/"
    if not os.path.exists(obj) or not os.path.exists(tools + "llvm-objdump"):
        pytest.skip("needs the objects of a build and the toolchain's llvm-objdump")
    section, code = os.path.join(to, "fat"), os.path.join(to, "code")
    subprocess.run([tools + "llvm-objcopy", f"--dump-section=.hip_fatbin={section}", obj,
                    os.path.join(to, "copy.o")], check=True, capture_output=True)
    subprocess.run([tools + "clang-offload-bundler", "--type=o", "--unbundle",
                    f"--targets=hipv4-amdgcn-amd-amdhsa--{build.ARCH}", f"--input={section}",
                    f"--output={code}"], check=True, capture_output=True)
    return subprocess.run([tools + "llvm-objdump", "-d", "--no-show-raw-insn", code], check=True,
                          capture_output=True, text=True).stdout


def test_no_tile_is_written_where_the_first_scores_read(tmp_path):
    """The operands of k of the first two tiles lie in the two halves of a buffer, turn 0
    writes those of the third over the first: between the workgroup's first barrier (they
    have come) and its second (their scores are done) nothing is written."""
    text = _bundle(os.path.join(build.BUILD, "attend.hip.o"), str(tmp_path))
    kernels = re.split(r"\n[0-9a-f]+ <", text)
    many = [k for k in kernels if "attend_many_kernel" in k.split(">")[0]]
    assert len(many) == len(M.MANY)
    for k in many:
        steps = re.findall(r"\b(ds_read|ds_write|s_barrier)", k)
        first = steps.index("s_barrier")
        second = steps.index("s_barrier", first + 1)
        assert "ds_write" in steps[:first]
        assert set(steps[first + 1:second]) == {"ds_read"}, k.split(">")[0]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_form_of_all_rows_is_the_form_of_each(dtype, causal):
    g = torch.Generator().manual_seed(0)
    for m, n in ((5, 9), (9, 5), (1, 1), (3, 0)):
        q = torch.randn((m, 6, 64), generator=g).to(dtype)
        k, v = (torch.randn((n, 2, 64), generator=g, dtype=torch.float64) for _ in range(2))
        for got, want in zip(M.attention(q, k, v, 0.2, causal), A.attention(q, k, v, 0.2, causal)):
            assert (got - want).abs().max() <= 1e-12
        keep = torch.arange(n) % 3 != 1
        if not causal and n:
            got = M.attention(q, k, v, 0.2, False, keep)
            want = A.attention(q, k[keep], v[keep], 0.2, False)
            assert (got[0] - want[0]).abs().max() <= 1e-12


def test_the_largest_scale():
    args = [1, 0, 0, 4, 2, 128, 0, 512, 0, 0, 0, 3, 8, 64, 0, None, 1, 0, 512, 0, 0]
    for scale, status in ((2.0 ** 126, None), (2.0 ** 127, lk.LOOKME_ERR_INVALID),
                          (1.0001 * 2.0 ** 126, lk.LOOKME_ERR_INVALID), (1e-45, None)):
        args[15] = scale
        if status is None:
            lk.lookme_cache_attention(*args, stream=0)
        else:
            with pytest.raises(lk.LookmeError) as e:
                lk.lookme_cache_attention(*args, stream=0)
            assert e.value.status == status
