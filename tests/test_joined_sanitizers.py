"""Host code of fibattn_backward_joined under AddressSanitizer and UndefinedBehaviorSanitizer
(CPU only): tests/sanitize/joined_driver.cpp with a host-sanitized build of api.hip."""
import os

import pytest

from tests.test_sanitizers import ENV, HIPCC, HOST_SAN, KERNEL_OBJS, ROOT, SAN, _run


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")
def test_joined_host_code_under_sanitizers(tmp_path):
    objs = [os.path.join(ROOT, "_build", o + ".o") for o in KERNEL_OBJS]
    if not all(os.path.exists(o) for o in objs):
        from paper_2606_28560_amd.build import build
        build()
    api, drv, exe = str(tmp_path / "api.o"), str(tmp_path / "driver.o"), str(tmp_path / "joined_san")
    inc = ["-I", os.path.join(ROOT, "include")]
    _run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-fPIC", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
          "-packed-fp32-ops", *inc, *HOST_SAN, "-c", os.path.join(ROOT, "paper_2606_28560_amd", "csrc", "api.hip"), "-o", api])
    _run([HIPCC, "-O1", "-g", "-std=c++17", *inc, *HOST_SAN, "-c", os.path.join(SAN, "joined_driver.cpp"), "-o", drv])
    _run([HIPCC, "--offload-arch=gfx950", *HOST_SAN, "-o", exe, drv, api, *objs])
    r = _run([exe], env=ENV, timeout=300)
    assert r.stdout.strip().endswith("OK")
