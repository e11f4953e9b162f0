"""How many workgroups of the gated 8-bit quantizer a CU runs at once, as its launches count on, against what the compiler made of it; no GPU needed."""
import re
import subprocess

from paper_2506_04985_amd import build
from test_code_objects import code_objects, kernels  # noqa: F401


def test_launches_count_on_as_many_workgroups_as_a_cu_holds(kernels, tmp_path):  # noqa: F811
    """160 KB of LDS in pieces of 1280 bytes; a SIMD's 512 registers a lane in pieces of 8 and its 800 scalar registers in pieces of 16, shared by at most eight waves."""
    lines, seen = [], 0
    for name, notes in kernels.items():
        m = re.search(r"quantize8_kernelILi2ELi(\d+)ELi(\d+)ELb([01])ELb1E", name)
        if not m:
            continue
        waves, chunks, ragged = (int(v) for v in m.groups())
        number = lambda key: int(re.search(rf"\.{key}:\s+(\d+)", notes).group(1))
        held = min(8, 512 // (-(-number("vgpr_count") // 8) * 8), 800 // (-(-number("sgpr_count") // 16) * 16)) * 4 // max(waves, 4)
        fit = min(held, 160 * 1024 // (-(-number("group_segment_fixed_size") // 1280) * 1280))
        lines.append(f'static_assert(fptq::resident<{waves}, {chunks}, {"true" if ragged else "false"}>() == {fit}, "{waves} waves, {chunks} chunks, ragged {ragged}: {fit}");')
        seen += 1
    assert seen == 2 * 13
    path = tmp_path / "check.hip"
    path.write_text('#include "fptq_quant8.hip"\n' + "\n".join(lines) + "\n")
    p = subprocess.run([build.HIPCC, *build.FLAGS, "--offload-host-only", "-fsyntax-only", str(path)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0, p.stdout
