"""Host code of the attention to other states under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only): tests/sanitize/cross_driver.cpp with host-sanitized
builds of its three sources; the other objects are linked as built."""
import os

import pytest

from tests.test_sanitizers import ENV, HIPCC, HOST_SAN, KERNEL_OBJS, ROOT, SAN, _run

SOURCES = ["cross_api", "cross_fwd", "cross_bwd"]


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")
def test_cross_host_code_under_sanitizers(tmp_path):
    objs = [os.path.join(ROOT, "_build", o + ".o") for o in KERNEL_OBJS + ["api"]]
    if not all(os.path.exists(o) for o in objs):
        from paper_2606_28560_amd.build import build
        build()
    inc = ["-I", os.path.join(ROOT, "include")]
    for s in SOURCES:
        _run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-fPIC", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
              "-packed-fp32-ops", *inc, *HOST_SAN, "-c",
              os.path.join(ROOT, "paper_2606_28560_amd", "csrc", s + ".hip"), "-o", str(tmp_path / (s + ".o"))])
        objs.append(str(tmp_path / (s + ".o")))
    drv, exe = str(tmp_path / "driver.o"), str(tmp_path / "cross_san")
    _run([HIPCC, "-O1", "-g", "-std=c++17", *inc, *HOST_SAN, "-c", os.path.join(SAN, "cross_driver.cpp"), "-o", drv])
    _run([HIPCC, "--offload-arch=gfx950", *HOST_SAN, "-o", exe, drv, *objs])
    r = _run([exe], env=ENV, timeout=300)
    assert r.stdout.strip().endswith("OK")
