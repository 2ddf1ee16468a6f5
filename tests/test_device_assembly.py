"""What the compiler makes of the inline assembly that moves rows from memory into LDS: a register of the hardware's (m0) says where to, and
the compiler has to know that it does.  Compiles one small kernel for gfx950; runs without a GPU."""
import os
import re
import subprocess

from paper_2202_04305_amd import build

KERNEL = """
#include "attention_tiles.h"
__global__ __launch_bounds__(256) void three_rows(const float4 *p, float *out)
{
    extern __shared__ float lds[];
    const unsigned to = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(attn_lds_f32 *)lds + threadIdx.x / 64 * 1024);
    for (int k = 0; k < 3; ++k) attn_to_lds(p + k * 256 + threadIdx.x, to + k * 4096);
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
    __syncthreads();
    out[threadIdx.x] = lds[threadIdx.x];
}
"""


def test_loads_to_lds_take_their_place_from_an_operand(tmp_path):
    src, asm = tmp_path / "rows.hip", tmp_path / "rows.s"
    src.write_text(KERNEL)
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
    p = subprocess.run(["hipcc", "-S", "--cuda-device-only", str(src), "-o", str(asm), "-I", os.path.join(build.ROOT, "include"),
                        "-I", os.path.join(build.HERE, "csrc")] + flags, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0, p.stdout
    assert "reserved registers" not in p.stdout and "m0" not in p.stdout, p.stdout
    lines = [l.split(";")[0].strip() for l in asm.read_text().splitlines()]
    lines = [l for l in lines if l and not l.startswith(".") and not l.endswith(":")]
    loads = [k for k, l in enumerate(lines) if l.startswith("global_load_lds_dwordx4")]
    assert len(loads) == 3
    for k in loads:
        assert lines[k - 1] == "s_nop 0"                 # a cycle between a write to m0 and the load
        writes = [l for l in lines[:k] if re.match(r"\S+\s+m0\b", l)]
        assert writes and writes[-1].startswith("s_"), writes        # by the scalar unit: a vector one would need five
