"""The host half of the calls on the key / value cache under AddressSanitizer and UndefinedBehaviorSanitizer (no GPU; GPU code is not instrumented):
argument checks, plans and workspace sizes over a spread of sizes up to the limits (tests/sanitize/abi_cache_paths.cpp). The units that plan
and launch are compiled for this, the others linked as built."""
import os
import shutil

import pytest

from tests.test_host_sanitizers import ENV, SAN, _clean, _run


@pytest.mark.skipif(shutil.which("hipcc") is None or not os.path.exists("/opt/rocm/llvm/bin/clang++"), reason="ROCm toolchain not found")
def test_cache_host_paths_under_address_and_undefined_sanitizers(tmp_path):
    from paper_2508_21058_amd import build as hb
    hb.build()
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined"]
    units, objs = ["moc_api", "moc_cache", "moc_cache_attn"], []
    for u in units:
        objs.append(str(tmp_path / (u + "_san.o")))
        _run(["hipcc", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", *san,
              "-c", os.path.join(hb.CSRC, u + ".hip"), "-o", objs[-1]])
    others = [os.path.join(hb.OBJ, u + ".o") for u in hb.UNITS if u not in units]
    exe, drv = str(tmp_path / "cache_san"), str(tmp_path / "abi_cache_paths.o")
    _run(["/opt/rocm/llvm/bin/clang++", "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
          "-c", os.path.join(SAN, "abi_cache_paths.cpp"), "-o", drv])
    _run(["hipcc", "--offload-arch=gfx950", *san, drv, *objs, *others, "-o", exe])
    r = _run([exe], env=ENV)
    _clean(r)
    assert r.stdout.startswith("ok ")
