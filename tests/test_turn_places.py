"""Where the lanes of a rotation's work-group read (rsa_rotate.hip), on the host: never outside their own wave's LDS."""
import os

from test_sanitizers import ROOT, SAN, run


def test_lanes_read_their_own_rows(tmp_path):
    exe = str(tmp_path / "turns")
    run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-arch=gfx950", "-O1", "-std=c++17",
         "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_2105_13120_amd", "csrc"),
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument",
         "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all",
         "-x", "hip", os.path.join(SAN, "turn_driver.cpp"), "-o", exe])
    assert "TURNS_OK" in run([exe])
