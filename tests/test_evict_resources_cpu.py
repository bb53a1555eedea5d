"""msa_evict's kernels that move rows hold them in registers: no scratch memory and no LDS."""
import os
import re
import subprocess

from paper_2603_23516_amd import build


def test_rows_stay_in_registers(tmp_path):
    src = os.path.join(build.HERE, "csrc", "msa_evict.hip")
    r = subprocess.run([build.HIPCC] + build.COMMON + ["-I", os.path.join(build.ROOT, "include"), "--cuda-device-only", "-c", src, "-o",
                                                       str(tmp_path / "evict.o"), "-Rpass-analysis=kernel-resource-usage"],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:]
    seen = {}
    for block in r.stdout.split("Function Name: ")[1:]:
        name = block.split()[0]
        seen[name] = {key: int(re.search(key + r"[^:\n]*: (\d+)", block).group(1)) for key in ("ScratchSize", "VGPRs Spill", "LDS Size")}
    for kernel in ("evict_move_kernel", "evict_move_in_place_kernel"):
        of = {name: x for name, x in seen.items() if kernel in name}
        assert len(of) == 2, sorted(seen)          # 64 and 128 dims
        assert all(not any(x.values()) for x in of.values()), of
