"""Properties of the compiled kernels of the quantised cache, read from the compiler's assembly (no GPU)."""
import re
import subprocess

import pytest

from paper_2606_00144_amd import build
from test_device_code import MIXED


def _assembly(src, out):
    r = subprocess.run([build.HIPCC, *build.FLAGS, "--offload-device-only", "-S", str(src), "-o", str(out)], capture_output=True,
                       text=True)
    assert r.returncode == 0, r.stderr
    return out.read_text()


@pytest.mark.parametrize("source,kernels", [("quant.hip", 7), ("qattn.hip", 32)])
def test_kernels_use_no_scratch_and_no_packed_floats(tmp_path, source, kernels):
    # the first access of a wave to scratch memory costs more than a small call's whole work
    text = _assembly(f"{build.CSRC}/{source}", tmp_path / "x.s")
    for field in ("private_segment_fixed_size", "vgpr_spill_count"):
        sizes = re.findall(rf"^ +\.{field}: +(\d+)", text, re.M)
        assert sizes == ["0"] * kernels, (field, sizes)
    assert not re.search(r"\bscratch_(load|store)|\bv_pk_(add|mul|fma)_f32", text)


def test_hidden_non_temporal_loads_leave_the_compilers_lds_base_alone(tmp_path):
    # as test_device_code has it for the other hidden loads
    for i, hidden in enumerate(["bd::dma16_nt_hidden(g + threadIdx.x * 8 + 4096, other)",
                                "bd::dma16_nt_hidden(g, off + 16 * threadIdx.x, other)", "bd::dma4_hidden(g + threadIdx.x * 2, other)"]):
        src = tmp_path / f"m{i}.hip"
        src.write_text(MIXED.replace("HIDDEN", hidden))
        text = _assembly(src, tmp_path / f"m{i}.s")
        ops = [line.split()[:2] for line in text.splitlines() if "m0" in line or "global_load_lds" in line]
        assert [op[1].rstrip(",") == "m0" for op in ops if op] == [True, False] * 3, ops
        assert ("nt" in text.split("global_load_lds_dwordx4")[2].splitlines()[0]) == ("nt_hidden" in hidden)
