"""What msa_evict's kernels say they hold in registers is there: no scratch memory, and no LDS in those that move rows."""
import os
import re
import subprocess

import pytest

from paper_2603_23516_amd import build


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """What the compiler reports for every kernel of msa_evict.hip, by mangled name."""
    src = os.path.join(build.HERE, "csrc", "msa_evict.hip")
    obj = str(tmp_path_factory.mktemp("evict") / "evict.o")
    r = subprocess.run([build.HIPCC] + build.COMMON + ["-I", os.path.join(build.ROOT, "include"), "--cuda-device-only", "-c", src, "-o", obj,
                                                       "-Rpass-analysis=kernel-resource-usage"],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:]
    return {block.split()[0]: {key: int(re.search(key + r"[^:\n]*: (\d+)", block).group(1))
                               for key in ("ScratchSize", "VGPRs Spill", "LDS Size")}
            for block in r.stdout.split("Function Name: ")[1:]}


def test_rows_stay_in_registers(kernels):
    for kernel in ("evict_move_kernel", "evict_move_in_place_kernel"):
        of = {name: x for name, x in kernels.items() if kernel in name}
        assert len(of) == 2, sorted(kernels)          # 64 and 128 dims
        assert all(not any(x.values()) for x in of.values()), of


def test_weights_stay_in_registers(kernels):
    of = {name: x for name, x in kernels.items() if "evict_select_kernel" in name}
    assert len(of) == 4, sorted(kernels)              # 8, 16, 32 rows of a thread, and any number
    assert all(x["ScratchSize"] == 0 and x["VGPRs Spill"] == 0 for x in of.values()), of
