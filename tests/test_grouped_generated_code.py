"""What the compiler makes of the copies to LDS that the grouped kernels write as instructions (grouped.h): they set m0, which the
compiler is not told.  So nothing else in these kernels may use it: this reads the assembly of the sources, built as the library
builds them."""
import re
import subprocess

import pytest

from paper_2306_08367_amd import build


@pytest.mark.parametrize("source", ["grouped_product.hip", "grouped_gradient.hip"])
def test_nothing_but_the_copies_uses_m0(source, tmp_path):
    out = tmp_path / "grouped.s"
    r = subprocess.run([build.hipcc(), *build.FLAGS, "--offload-device-only", "-S", f"{build.CSRC}/{source}", "-o", str(out)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    lines = [line.split(";")[0].strip() for line in out.read_text().splitlines()]
    lines = [line for line in lines if line and not line.startswith((".", "//"))]
    copies = 0
    for i, line in enumerate(lines):
        if re.match(r"global_load_lds_dword", line):
            assert re.match(r"s_mov_b32 m0, s\d+$", lines[i - 2]) and lines[i - 1] == "s_nop 0", lines[i - 3:i + 1]
            copies += 1
        elif re.search(r"\bm0\b", line):
            assert re.match(r"global_load_lds_dword", lines[i + 2]), f"m0 is used by: {line}"
        # (indexed register moves and messages take m0 without naming it)
        assert not re.match(r"s_set_gpr_idx|v_movrel|s_movrel|s_sendmsg |ds_gws|buffer_load.* lds", line), line
    assert copies > 100
