"""The device code of the gated layers and the orthogonalised updates as it is compiled for gfx950 (CPU only,
nothing runs): descriptors of the loads to LDS, which are written out, and registers kept in memory."""
import concurrent.futures as cf
import os
import re
import subprocess

import pytest

from paper_1812_04352_amd import build as B
from test_wide_code import hazards

UNITS = ("lp_gated_bf16", "lp_gated_f32", "lp_orth_f16", "lp_orth_f32", "lp_norm")


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    """Assembly and the compiler's remarks on the kernels' resources, by source."""
    if not os.path.exists(B.HIPCC):
        pytest.skip("no compiler")
    d = tmp_path_factory.mktemp("asm")

    def compiled(u):
        r = subprocess.run([B.HIPCC, *B.FLAGS, "-Rpass-analysis=kernel-resource-usage", "--offload-device-only", "-S", "-x", "hip",
                            os.path.join(B.CSRC, u + ".hip"), "-o", str(d / f"{u}.s")], capture_output=True, text=True, timeout=900)
        assert r.returncode == 0, r.stderr[-2000:]
        return (d / f"{u}.s").read_text(), r.stderr

    with cf.ThreadPoolExecutor(len(UNITS)) as ex:
        return dict(zip(UNITS, ex.map(compiled, UNITS)))


@pytest.mark.parametrize("u", UNITS[:4])
def test_descriptors_of_loads_to_lds_are_settled(code, u):
    """Five wait states from a vector instruction that writes a scalar to the load that takes it, and the
    descriptor in scalars at all (pairs of arrays have two)."""
    loads, bad = hazards(code[u][0])
    assert loads >= 100 and not bad, (loads, bad[:3])


@pytest.mark.parametrize("u", UNITS)
def test_kernels_do_not_spill(code, u):
    use = re.findall(r"Function Name: (\S+).*?ScratchSize \[bytes/lane\]: (\d+)", code[u][1], re.S)
    spilled = {n: int(s) for n, s in use if int(s)}
    assert len(use) >= 20 and not spilled, spilled


@pytest.mark.parametrize("u", UNITS[:4])
def test_written_out_reads_of_a_first_lane_wait(code, u):
    """The compiler does not see their hazards: a vector register may be read a wait state after a vector instruction
    wrote it, and the scalar that they write five later."""
    seen = 0
    for text in re.findall(r"#ASMSTART\n(.*?);;#ASMEND", code[u][0], re.S):
        if "v_readfirstlane" not in text:
            continue
        seen += 1
        names = [x.split()[:2] for x in text.split("\n") if x.split()]
        assert [n[0] for n in names] == ["s_nop", "v_readfirstlane_b32", "v_readfirstlane_b32", "s_nop"], text
        assert int(names[0][1]) >= 1 and int(names[3][1]) >= 4, text
    assert seen >= 10
