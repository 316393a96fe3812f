"""The host code of csrc/kv_tree_api.hip under -fsanitize=address,undefined (host only), with stubs in place of the launchers."""
import os

from test_sanitizers import ENV, ROOT, SAN, _run


def test_kv_tree_host_side_under_sanitizers(tmp_path):
    exe = str(tmp_path / "kv_tree_san")
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    csrc = os.path.join(ROOT, "paper_2312_01712_amd", "csrc")
    _run([hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
          "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
          "-Xarch_host", "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "include"), "-I", csrc,
          os.path.join(csrc, "kv_tree_api.hip"), "-x", "hip", os.path.join(SAN, "kv_tree_driver.cpp"), "-o", exe])
    assert "kv_tree_driver: clean" in _run([exe], env=ENV)
