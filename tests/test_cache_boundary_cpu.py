"""Host code of the entry points around the life of a local cache, under sanitizers at extreme sizes."""
import os
import subprocess

import test_boundary_cpu as boundary


def test_host_sanitizers_on_extreme_sizes():
    """tests/csrc/cache_sanitize.cpp with the sanitized library that the other entry points' driver builds and links: up to 2^25
    tokens, 65535 heads, prefixes and caches of 2^28 rows.  No device is visible, so nothing can launch."""
    boundary.test_host_sanitizers_on_extreme_sizes()          # builds the library where it is older than its sources
    out_dir = os.path.join(boundary.ROOT, "tests", "_build")
    src, exe = os.path.join(boundary.ROOT, "tests", "csrc", "cache_sanitize.cpp"), os.path.join(out_dir, "cache_sanitize")
    san = []
    for f in ("-fsanitize=address", "-fsanitize=undefined", "-fsanitize=integer", "-fno-sanitize-recover=all"):
        san += ["-Xarch_host", f]
    r = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-arch=gfx950", "-O1", "-g", "-std=c++17"] + san +
                       ["-I", os.path.join(boundary.ROOT, "include"), src, "-L", out_dir, "-lmsa_san", "-Wl,-rpath," + out_dir,
                        "-o", exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:]
    env = dict(os.environ, HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="", ASAN_OPTIONS="detect_leaks=0")
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300, env=env)
    assert r.returncode == 0 and "cache_sanitize: ok" in r.stdout, r.stdout[-3000:]
