"""The wide operators' device code as it is compiled for gfx950 (CPU only, nothing runs): what the
compiler is told about the instructions that are written out, and what orders a wave's LDS accesses."""
import concurrent.futures as cf
import os
import re
import subprocess

import pytest

from paper_1812_04352_amd import build as B

SOURCE = """
#include "lp_mm.h"
using namespace lp::mm;
template <int R, int NT, bool COLS>
static __device__ void request(const void* p, long ld, int rows, int k1, unsigned char* lds) {
  Stage<bf16, R, 128, NT, COLS> s;
  s.start(p, ld, 0, rows, 0, k1);
  s.load(lds, 0);
}
__global__ void k_load(const void* p, long ld, int rows, int k1) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[256 * 128];
  request<256, 512, false>(p, ld, rows, k1, lds);
  request<256, 512, true>(p, ld, rows, k1, lds);
  request<64, 256, false>(p, ld, rows, k1, lds);
  request<64, 256, true>(p, ld, rows, k1, lds);
}
__global__ void k_block(bf16* a, long ld, Place c) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[WAVE_LDS];
  f32x4 v[4] = {};
  BlockIO<bf16>::quads(BlockIO<bf16>::fetch(a, ld, c, 0, 0), lds, c, v);
  BlockIO<bf16>::store(a, ld, c, 0, 0, lds, v, [](int m) { return m; });
  c.meet<1>();
}
"""


@pytest.fixture(scope="module")
def ir(tmp_path_factory):
    """The source's device code, before optimisation."""
    if not os.path.exists(B.HIPCC):
        pytest.skip("no compiler")
    d = tmp_path_factory.mktemp("ir")
    (d / "t.hip").write_text(SOURCE)
    flags = [f for f in B.FLAGS if f != "-O3"]
    r = subprocess.run([B.HIPCC, *flags, "-O1", "-Xclang", "-disable-llvm-passes", "--offload-device-only", "-S", "-emit-llvm",
                        "-x", "hip", str(d / "t.hip"), "-o", str(d / "t.ll")], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    return (d / "t.ll").read_text()


def test_loads_to_lds_declare_what_they_change(ir):
    """m0 and memory; and they keep a wait state between m0 and the load."""
    calls = re.findall(r'asm sideeffect "([^"]*buffer_load_dwordx4[^"]*)", "([^"]*)"', ir)
    assert len(calls) >= 4
    for text, constraints in calls:
        assert "~{m0}" in constraints and "~{memory}" in constraints, constraints
        lines = [x.strip() for x in text.replace("\\09", "").split("\\0A")]
        assert [x.split()[0] for x in lines] == ["s_mov_b32", "s_nop", "buffer_load_dwordx4"] and " lds" in lines[2]


def test_exchanges_over_a_waves_lds_are_ordered(ir):
    """Every barrier of a wave alone stands between fences: the barrier itself does not keep the
    compiler from moving LDS accesses of one lane past those of another."""
    lines = [x.strip() for x in ir.split("\n")]
    at = [i for i, x in enumerate(lines) if re.search(r"call void @llvm\.amdgcn\.wave\.barrier", x)]
    assert at
    for i in at:
        assert lines[i - 1].startswith('fence syncscope("wavefront") release'), lines[i - 1]
        assert lines[i + 1].startswith('fence syncscope("wavefront") acquire'), lines[i + 1]


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    """Assembly of the operators' kernels and the compiler's remarks on their resources, by element type."""
    if not os.path.exists(B.HIPCC):
        pytest.skip("no compiler")
    d = tmp_path_factory.mktemp("asm")

    def compiled(t):
        r = subprocess.run([B.HIPCC, *B.FLAGS, "-Rpass-analysis=kernel-resource-usage", "--offload-device-only", "-S", "-x",
                            "hip", os.path.join(B.CSRC, f"lp_step_{t}.hip"), "-o", str(d / f"{t}.s")], capture_output=True, text=True,
                           timeout=600)
        assert r.returncode == 0, r.stderr[-2000:]
        return (d / f"{t}.s").read_text(), r.stderr

    types = ("bf16", "f16", "f32")
    with cf.ThreadPoolExecutor(3) as ex:
        return dict(zip(types, ex.map(compiled, types)))


CARRY = re.compile(r"v_(add|sub|subrev|addc|subb|subbrev)_co_|v_mad_[ui]64|v_div_scale")


def scalars(operand):
    """The scalar registers that an operand names."""
    m = re.match(r"s\[(\d+):(\d+)\]$|s(\d+)$", operand)
    return set() if not m else {int(m[3])} if m[3] else set(range(int(m[1]), int(m[2]) + 1))


def instructions(asm):
    """(labels in front, mnemonic, operands) of each kernel's instructions."""
    out, labels = [], []
    for line in asm.split("\n"):
        line = line.split(";")[0].strip()
        if not line:
            continue
        if line.endswith(":"):
            labels.append(line[:-1])
            if line.startswith("_Z"):
                if out:
                    yield out
                out = []
        elif re.match(r"[a-z]+_", line):
            name, *ops = line.split(None, 1)
            out.append((labels, name, [x.strip() for x in ops[0].split(",")] if ops else []))
            labels = []
    if out:
        yield out


def hazards(asm):
    """(loads to LDS, those within five wait states of a vector instruction that writes a scalar of their
    descriptor)."""
    loads, bad = 0, []
    for code in instructions(asm):
        at = {x: i for i, (ls, _, _) in enumerate(code) for x in ls}
        jumps = {}
        for i, (_, name, ops) in enumerate(code):
            if name.startswith(("s_branch", "s_cbranch")):
                jumps.setdefault(at.get(ops[0]), []).append(i)
        for i, (_, name, ops) in enumerate(code):
            if not (name.startswith("buffer_load") and ops[-1].endswith(" lds")):
                continue
            loads += 1
            need, todo, seen = scalars(ops[1]), [(i, 5)], set()
            assert len(need) == 4, ops
            while todo:
                j, left = todo.pop()
                before = list(jumps.get(j, [])) + ([j - 1] if j and code[j - 1][1] not in ("s_branch", "s_endpgm") else [])
                for k in before:
                    _, n, o = code[k]
                    writes = scalars(o[0]) if n.startswith("v_") else set()
                    if CARRY.match(n):
                        writes |= scalars(o[1])
                    if writes & need:
                        bad.append((name, ops, n, o))
                    rest = left - (int(o[0], 0) + 1 if n == "s_nop" else 1)
                    if rest > 0 and (k, rest) not in seen:
                        seen.add((k, rest))
                        todo.append((k, rest))
    return loads, bad


def test_the_check_for_hazards_sees_them():
    load = "\tbuffer_load_dwordx4 v1, s[4:7], 0 offen lds\n"
    head, mov = "_Zk:\n", "\ts_mov_b32 m0, s9\n\ts_nop 0\n"
    assert hazards(head + "\tv_readlane_b32 s6, v0, 3\n" + mov + load)[1]
    assert hazards(head + "\tv_readfirstlane_b32 s4, v0\n\ts_nop 2\n" + mov + load)[1] == []
    assert hazards(head + "\tv_readfirstlane_b32 s4, v0\n\ts_nop 1\n" + mov + load)[1]
    assert hazards(head + "\tv_readlane_b32 s8, v0, 3\n" + mov + load)[1] == []
    assert hazards(head + "\tv_mad_u64_u32 v[2:3], s[6:7], v0, v1, v[2:3]\n" + mov + load)[1]
    jump = "\tv_readlane_b32 s7, v0, 3\n\ts_branch .L1\n.L0:\n\ts_endpgm\n.L1:\n" + mov + load
    assert hazards(head + jump)[1] and hazards(head + jump)[0] == 1


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_descriptors_of_loads_to_lds_are_settled(code, t):
    """A vector memory instruction takes a scalar that a vector instruction wrote five wait states later
    at the earliest, and the compiler does not look into instructions that are written out."""
    loads, bad = hazards(code[t][0])
    assert loads >= 500 and not bad, (loads, bad[:3])


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_kernels_hardly_spill(code, t):
    """Registers kept in memory, as the compiler reports them: only the gradient's epilogue on the largest
    tiles has any (16-bit types 12 bytes a lane, floats 144), a step without one would show more."""
    use = re.findall(r"Function Name: (\S+).*?ScratchSize \[bytes/lane\]: (\d+)", code[t][1], re.S)
    assert len(use) >= 60
    spilled = {n: int(s) for n, s in use if int(s)}
    assert len(spilled) <= 1 and all(re.search(r"k_mm.*ShapeILi256.*EpGrad", n) for n in spilled), spilled
    assert sum(spilled.values()) <= (160 if t == "f32" else 16), spilled
