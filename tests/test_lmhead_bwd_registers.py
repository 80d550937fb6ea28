"""How many workgroups of the LM head's gradient a CU holds: what its planner takes for granted against what the compiler made of the kernels (no GPU)."""
import os
import re
import subprocess

from paper_2604_04215_amd import build

SRC = os.path.join(build.CSRC, "lmhead_bwd.hip")
SHAPES = {(2, 2, 4, 4): (256, 256), (4, 1, 2, 4): (256, 128), (4, 1, 2, 2): (256, 64), (2, 2, 2, 2): (128, 128), (2, 2, 1, 1): (64, 64)}


def table():
    """{tile: (workgroups a CU, the same with sums in two floats)}"""
    with open(SRC) as f:
        rows = re.search(r"LMB_TILES\[\] = \{(.*)\};", f.read())[1]
    return {(int(i), int(j)): (int(a), int(b)) for i, j, a, b in re.findall(r"\{(\d+), (\d+), (\d+), (\d+)\}", rows)}


def test_workgroups_of_a_cu(tmp_path):
    asm = tmp_path / "lmhead_bwd.s"
    subprocess.check_call([os.environ.get("HIPCC", "hipcc"), *build.FLAGS, "--cuda-device-only", "-S", SRC, "-o", str(asm)], stderr=subprocess.DEVNULL)
    kernel, seen = None, {}
    for line in asm.read_text().splitlines():
        if line.startswith("_ZN3dlm") and line.split(":")[0].endswith("LmbParamsE"):
            kernel = line.split(":")[0]
        elif line.startswith("; Occupancy:") and kernel and "LmbShape" in kernel:
            seen[kernel] = int(line.split(":")[1])
    assert len(seen) >= 16
    tiles = table()
    assert set(tiles) == set(SHAPES.values())
    for name, occupancy in seen.items():                # wavefronts a SIMD: workgroups of four wavefronts a CU
        shapes = re.findall(r"LmbShapeILi(\d)ELi(\d)ELi(\d)ELi(\d)EEE?", name)
        blocks = re.search(r"lmb_dz_kernel.*ELi\dELi(\d)EEEv" if "lmb_dz" in name else r"lmb_grad_kernelILb\dELi(\d)E", name)[1]
        held = min(tiles[SHAPES[tuple(map(int, s))]][blocks != "0"] for s in shapes)
        assert occupancy == held, (name, occupancy, held)
