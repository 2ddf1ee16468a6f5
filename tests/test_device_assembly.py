"""What the compiler makes of the kernels of attention, without a GPU.  The inline assembly that moves rows from memory into LDS, whose place a
register of the hardware's (m0) says: the compiler has to know that it does.  And kernels that need more registers than there are."""
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


OBJDUMP = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")


def lost_registers(assembly):
    """{kernel: [what it keeps aside and never fetches]} of disassembled device code: accumulation registers that moves write and nothing
    reads, words of scratch that are stored and never loaded."""
    lost, body = {}, None

    def ended():
        if body is not None:
            moved, read, stored, loaded = body
            rest = sorted("a%d" % r for r in moved - read) + sorted("scratch + %d" % o for o in stored - loaded)
            if rest:
                lost[name] = rest
    for line in assembly:
        m = re.match(r"[0-9a-f]+ <(\S+)>:", line)
        if m:
            ended()
            name, body = m.group(1), (set(), set(), set(), set())
            continue
        op, _, rest = line.split("//")[0].strip().partition(" ")
        if body is None or not op:
            continue
        moved, read, stored, loaded = body
        if op.startswith("scratch_"):
            at = int((re.search(r"offset:(\d+)", rest) or [0, 0])[1])
            words = range(at, at + 4 * {"x2": 2, "x3": 3, "x4": 4}.get(op[-2:], 1), 4)
            (stored if "store" in op else loaded).update(words)
        for k, field in enumerate(rest.split(",")):
            for lo, hi in re.findall(r"\ba\[?(\d+)(?::(\d+))?\b", field):
                regs = range(int(lo), int(hi or lo) + 1)
                if k > 0 or "store" in op or "write_b" in op and op.startswith("ds_"):
                    read.update(regs)
                elif op.startswith("v_accvgpr"):
                    moved.update(regs)
    ended()
    return lost


def test_lost_registers_are_found():
    kept = ["0000 <k>:", "\tv_accvgpr_write_b32 a133, v235  // 0", "\tscratch_store_dwordx2 off, v[2:3], off offset:8", "\tv_accvgpr_mov_b32 a35, a133",
            "\tscratch_load_dwordx2 a[2:3], off, off offset:8", "\tv_mfma_f32_32x32x2_f32 a[16:31], v3, a35, a[16:31]"]
    assert lost_registers(kept) == {}
    assert lost_registers(kept[:2] + kept[3:]) == {}
    assert lost_registers(kept[:3] + kept[4:5]) == {"k": ["a133"]}
    assert lost_registers(kept[:4] + ["\tscratch_load_dword a2, off, off offset:8"] + kept[5:]) == {"k": ["scratch + 12"]}


def test_no_kernel_of_attention_loses_what_it_keeps_aside(tmp_path):
    """The compiler has dropped one of four parts of an operand that it kept in accumulation registers and scratch (a gradient of f32 heads
    of 256, whose dQ was wrong by it); every part has to be fetched again."""
    lib = tmp_path / "lib.so"
    build.is_stale() and build.build()
    lib.write_bytes(open(build.LIB, "rb").read())
    subprocess.check_call([OBJDUMP, "--offloading", str(lib)], stdout=subprocess.DEVNULL, cwd=tmp_path)
    kernels = 0
    for part in sorted(tmp_path.glob("lib.so.*gfx950")):
        names = subprocess.run([OBJDUMP, "-t", str(part)], stdout=subprocess.PIPE, text=True, check=True).stdout
        if not re.search(r"(dq|dkv|forward)_kernel", names):
            continue
        asm = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(part)], stdout=subprocess.PIPE, text=True, check=True).stdout.splitlines()
        kernels += sum(bool(re.match(r"[0-9a-f]+ <\S*(dq|dkv|forward)_kernel", l)) for l in asm)
        assert lost_registers(asm) == {}
    assert kernels >= 60, kernels
