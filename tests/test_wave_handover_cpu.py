"""LDS that one lane of a wave writes and another reads, without a barrier of the
workgroup, is handed over by a fence and a wave barrier that the compiler has to keep
(no GPU needed: the kernels' code as the compiler has it before it picks instructions)."""
import os
import re
import subprocess

import pytest

from paper_2607_00466_amd import build

pytestmark = pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="needs hipcc")

STAGED = """
#include "attn_tile.hpp"
using namespace eldr;
extern "C" __global__ void staged(const char* in, u32x4* out, int steps) {
  __shared__ __attribute__((aligned(16))) char lds[StagedKeys<128, false>::kBytes];
  StagedKeys<128, false> keys;
  for (int k = 0; k < steps; ++k) {
    keys.load<false>(0, in + k * keys.kBytes);
    keys.load<false>(1, in + k * keys.kBytes + keys.kTileBytes);
    keys.put(lds);
    for (int i = 0; i < 4; ++i) out[(k * 4 + i) * 64 + threadIdx.x] = keys.get(lds, i & 1, i, threadIdx.x % 16, threadIdx.x / 16);
  }
}
"""


def _ir(source, tmp_path):
    out = str(tmp_path / "code.ll")
    flags = [f for f in build.FLAGS if f != "-fPIC"]
    r = subprocess.run([build.HIPCC, *flags, "--offload-device-only", "-S", "-emit-llvm", str(source), "-o", out],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    return open(out).read()


def _events(text):
    """Per function: w and r for LDS written and read, | for a whole hand-over."""
    found = {}
    for name, body in re.findall(r"^define [^@]*@(\S+?)\(.*?\{\n(.*?)^\}", text, re.M | re.S):
        seen = ""
        for line in body.splitlines():
            if re.search(r"\bstore\b.*addrspace\(3\)", line):
                seen += "w"
            elif re.search(r"\bload\b.*addrspace\(3\)", line):
                seen += "r"
            elif 'fence syncscope("wavefront") release' in line:
                seen += "<"
            elif "call void @llvm.amdgcn.wave.barrier" in line:
                seen += "="
            elif 'fence syncscope("wavefront") acquire' in line:
                seen += ">"
        found[name] = seen.replace("<=>", "|")
    return found


def test_staged_keys_are_handed_over_both_ways(tmp_path):
    src = tmp_path / "staged.hip"
    src.write_text(STAGED)
    seen = _events(_ir(src, tmp_path))["staged"]
    # written after a hand-over (the step before has been read), read after another
    assert re.fullmatch(r"(\|w+\|r+)+", seen), seen


@pytest.mark.parametrize("source", ["attn_decode.hip", "attn_weights.hip"])
def test_the_kernels_keep_them(source, tmp_path):
    seen = _events(_ir(os.path.join(build.CSRC, source), tmp_path))
    kernels = [k for k in seen if re.search("attn_(decode|weights)_kernel", k)]
    assert len(kernels) == 6
    for k in kernels:
        assert "|" in seen[k] and not re.search("[<=>]", seen[k]), (k, seen[k])
