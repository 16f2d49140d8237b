"""Which calls of the norm go past the caches (tests/host/norm_host.cpp): built against the library's own objects; no kernel is launched."""
import os
import subprocess

from paper_2605_04569_amd import build as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_host_side_of_the_norm(tmp_path):
    hipcc = B._hipcc()
    objs = [os.path.join(B.HERE, "_build", s.replace(".hip", ".o")) for s in B.SOURCES]
    if not all(os.path.exists(o) for o in objs):
        B.build()
    obj, exe = str(tmp_path / "norm_host.o"), str(tmp_path / "norm_host")
    r = subprocess.run([hipcc, *B.FLAGS, "-x", "hip", "-c", os.path.join(ROOT, "tests", "host", "norm_host.cpp"), "-o", obj], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([hipcc, "--offload-arch=gfx950", obj, *objs, "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "host checks ok" in r.stdout, (r.stdout[-3000:], r.stderr[-3000:])
