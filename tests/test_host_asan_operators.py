"""The host code of every source that the library is built from under
AddressSanitizer, on the host side only (-Xarch_host, device code untouched):
the block-scaled FP8 operators, the losses and the two block scalings with
arguments out of contract (tests/host_validation_operators.c), and the calls of
tests/host_validation.c once more against the whole library.  No device is
used: every call in the drivers fails validation before any HIP call."""
import os
import re
import subprocess

import pytest

from paper_2607_24062_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TESTS = os.path.join(ROOT, "tests")
DRIVERS = ["host_validation.c", "host_validation_operators.c"]
HIPCC = "/opt/rocm/bin/hipcc"
ASAN = ["--offload-arch=gfx950", "-Xarch_host", "-fsanitize=address"]


def _all(commands):
    procs = [subprocess.Popen(c, stdout=subprocess.PIPE, stderr=subprocess.STDOUT) for c in commands]
    for pr in procs:
        out = pr.communicate(timeout=600)[0]
        assert pr.returncode == 0, out.decode(errors="replace")[-2000:]


@pytest.fixture(scope="module")
def objects(tmp_path_factory):
    """The library's objects, host code with AddressSanitizer."""
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    tmp = tmp_path_factory.mktemp("asan")
    objs = {src: str(tmp / (src + ".o")) for src in build.SOURCES}
    _all([[HIPCC, *ASAN, "-O1", "-fPIC", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-c",
           os.path.join(build.CSRC, src), "-o", obj] for src, obj in objs.items()])
    return list(objs.values())


@pytest.mark.parametrize("driver", DRIVERS)
def test_validation_paths(objects, driver, tmp_path):
    obj, exe = str(tmp_path / "driver.o"), str(tmp_path / "driver")
    _all([[HIPCC, "-Xarch_host", "-fsanitize=address", "-I", os.path.join(ROOT, "include"), "-x", "c", "-c",
           os.path.join(TESTS, driver), "-o", obj]])
    _all([[HIPCC, *ASAN, "-o", exe, obj, *objects]])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0 and r.stdout.startswith("0 unexpected results"), (r.stdout[-3000:] + r.stderr[-3000:])
    assert "ERROR: AddressSanitizer" not in r.stderr and "LeakSanitizer" not in r.stderr, r.stderr[-3000:]


def test_every_entry_point_has_a_driver():
    with open(os.path.join(ROOT, "include", "acrl.h")) as f:
        header = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    names = set(re.findall(r"\b(acrl_\w+)\(", header))
    calls = set()
    for d in DRIVERS:
        with open(os.path.join(TESTS, d)) as f:
            calls |= set(re.findall(r"\b(acrl_\w+)\(", f.read()))
    assert len(names) > 20 and names - calls == set()
