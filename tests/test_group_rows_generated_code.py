"""What the compiler makes of the counts in LDS that the lanes of a wavefront read and change for each other (group_rows.hip).  LDS instructions
of a wavefront take effect in their order; loads through the flat path, which a pointer without its address space becomes, are not
among them.  So the placing kernels have no flat access, and every addition to a count stands between the two reads around it."""
import re
import subprocess

import pytest

from paper_2306_08367_amd import build


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = tmp_path_factory.mktemp("rows") / "group_rows.s"
    r = subprocess.run([build.hipcc(), *build.FLAGS, "--offload-device-only", "-S", f"{build.CSRC}/group_rows.hip", "-o", str(out)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    found, body = {}, None
    for line in out.read_text().splitlines():
        line = line.split(";")[0].strip()
        if re.match(r"_Z\w+:$", line):
            body = found.setdefault(line[:-1], [])
        elif line.startswith(".end_amdhsa_kernel"):
            body = None
        elif body is not None and line and line[0] not in ".#":
            body.append(line.split()[0])
    return {name: body for name, body in found.items() if re.search("group_(rows|place|count)_kernel", name)}


def test_counts_are_read_by_lds_instructions(kernels):
    assert len(kernels) == 6, sorted(kernels)
    for name, body in kernels.items():
        assert not [op for op in body if op.startswith("flat_")], name


def test_every_step_reads_its_counts_before_and_behind_the_addition(kernels):
    steps = 8                     # of the unrolled loop
    for name, body in kernels.items():
        if "count_kernel" in name:
            continue
        lds = "".join({"ds_read_b32": "r", "ds_add_u32": "a"}.get(op, "") for op in body if op.startswith("ds_"))
        few = "group_place_kernelILb1ELb1E" in name        # (one lane adds for all of its group and asks for no count behind it)
        assert len(re.findall("ra" if few else "rar", lds)) >= steps, (name, lds)
