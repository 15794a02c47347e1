"""Matrix products of the cached attention and their first readers, checked in the compiled code (CPU only).

A vector instruction that reads a matrix product's result has to come some wait states after it; the hardware does not
hold it back. The compiler inserts them, but only between instructions that it knows: one inside inline assembly is opaque to
it, and then the result may be read before it is there. This test compiles kv_attention.hip for gfx950 with the library's
flags, follows every path from every matrix instruction of every kernel, and checks that no instruction touches the result
earlier than the compiler itself lets one in a kernel of two lines. The same holds for the exchanges between lanes that a
vector result goes into, so the file may have no instruction in inline assembly at all.
"""
import os
import re
import shutil
import subprocess

import pytest

from paper_2505_09142_amd import build as B

PROBE = r"""
#include <hip/hip_runtime.h>
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
extern "C" __global__ void probe(const bf16x8* a, float* out) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#if defined(__HIP_DEVICE_COMPILE__)
    s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[threadIdx.x], a[threadIdx.x], s, 0, 0, 0);
#endif
    out[threadIdx.x] = s[0] + s[1];
}
"""
MFMA = re.compile(r"v_mfma_\w+\s")
REG = re.compile(r"\bv(?:(\d+)|\[(\d+):(\d+)\])(?!\w)")
BRANCH = re.compile(r"(s_branch|s_cbranch_\w+)\s+(\S+)")


def compile_to_asm(src, out, extra=()):
    if not os.path.exists(B.HIPCC) and shutil.which("hipcc") is None:
        pytest.skip("hipcc not available")
    r = subprocess.run([B.HIPCC, *B.CFLAGS, *extra, "--cuda-device-only", "-S", str(src), "-o", str(out)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    return out.read_text().split("\n")


def regs(text):
    out = set()
    for one, lo, hi in REG.findall(text):
        out |= {int(one)} if one else set(range(int(lo), int(hi) + 1))
    return out


def kernels(lines):
    """name -> (instructions, label -> index of the instruction behind it)."""
    out, name = {}, None
    for line in lines:
        text = line.split(";")[0].strip()
        if re.match(r"\.Lfunc_end", text):
            name = None
        elif re.match(r"\w+:$", text) and not text.startswith("."):
            name = text[:-1]
            out[name] = ([], {})
        elif name is not None and text.endswith(":"):
            out[name][1][text[:-1]] = len(out[name][0])
        elif name is not None and text and not text.startswith("."):
            out[name][0].append(text)
    return {n: k for n, k in out.items() if any(x.startswith("s_endpgm") for x in k[0])}


def early_readers(ins, labels, need):
    """(matrix instruction, reader, wait states between) of every vector, LDS or memory instruction that touches a result too early."""
    bad = []
    for at, x in enumerate(ins):
        if not MFMA.match(x):
            continue
        dst, seen, todo = regs(x.split(",")[0]), {}, [(at + 1, 0)]
        while todo:
            i, waited = todo.pop()
            if i >= len(ins) or waited >= need or seen.get(i, need) <= waited:
                continue
            seen[i] = waited
            y = ins[i]
            if y.startswith("s_endpgm"):
                continue
            if not MFMA.match(y) and re.match(r"v_|ds_|buffer_|global_|flat_", y) and regs(y) & dst:
                bad.append((x, y, waited))
                continue
            b = BRANCH.match(y)
            waited += int(y.split()[1]) + 1 if y.startswith("s_nop") else 1
            if b:
                todo.append((labels[b.group(2)], waited))
            if not b or b.group(1) != "s_branch":
                todo.append((i + 1, waited))
    return bad


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("kv_isa")
    return compile_to_asm(os.path.join(B.CSRC, "kv_attention.hip"), tmp / "kv_attention.s", B.EXTRA["kv_attention.hip"])


@pytest.fixture(scope="module")
def need(tmp_path_factory):
    """Wait states that the compiler keeps between such a product and an ordinary addition."""
    tmp = tmp_path_factory.mktemp("probe")
    (tmp / "probe.hip").write_text(PROBE)
    (ins, labels), = kernels(compile_to_asm(tmp / "probe.hip", tmp / "probe.s", B.EXTRA["kv_attention.hip"])).values()
    for n in range(1, 64):
        if early_readers(ins, labels, n):
            return n - 1
    raise AssertionError("no reader found")


def test_no_product_is_read_early(code, need):
    assert need >= 4, need
    ks = {n: k for n, k in kernels(code).items() if "kv_attention" in n}
    assert len(ks) > 16 and all(any(MFMA.match(x) for x in ins) for ins, _ in ks.values())
    bad = {n: early_readers(*k, need) for n, k in ks.items()}
    assert not any(bad.values()), {n: b[:2] for n, b in bad.items() if b}


def test_no_instruction_in_inline_assembly(code):
    inside, found = False, []
    for line in code:
        if "#ASMSTART" in line or "#ASMEND" in line:
            inside = "#ASMSTART" in line
        elif inside and line.split(";")[0].strip():
            found.append(line.strip())
    assert not found, found[:3]
