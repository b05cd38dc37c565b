"""The host code of beams, adapters and embedding under AddressSanitizer and UndefinedBehaviorSanitizer: argument checks and workspace
arithmetic at the ends of their ranges.  Built host-only, as test_sanitizers_cpu.py builds the sampler's."""
import os
import re
import shutil

import pytest

from .test_sanitizers_cpu import ROOT, SAN, _run


def test_host_side_of_beams_adapters_and_embedding(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    clang = "/opt/rocm/lib/llvm/bin/clang"
    if not (os.path.exists(hipcc) and os.path.exists(clang)):
        pytest.skip("no hipcc / clang")
    include = ["-I", os.path.join(ROOT, "include")]
    lib = str(tmp_path / "libsip_san.so")
    rc, out = _run([hipcc, "--cuda-host-only", "--offload-arch=gfx950", "-std=c++17", "-fPIC", "-shared", "-ffp-contract=off", *SAN,
                    "-fno-sanitize=enum", *include, "-o", lib, os.path.join(ROOT, "paper_2506_22033_amd", "csrc", "sip.hip")],
                   cwd=str(tmp_path))
    assert rc == 0, out
    m = re.search(r"__hip_fatbin_[0-9a-f]+", _run(["nm", "-D", "-u", lib])[1])       # an empty bundle stands in for the device code
    stub = tmp_path / "bundle_stub.cpp"
    stub.write_text("struct Bundle { char magic[24]; unsigned long long n; };\nextern \"C\" { extern const Bundle %s; }\n"
                    "alignas(4096) const Bundle %s = {{%s}, 0};\n" % (m.group(0), m.group(0), ",".join(
                        "'%s'" % c for c in "__CLANG_OFFLOAD_BUNDLE__")))
    exe = str(tmp_path / "search_san")
    rc, out = _run([clang + "++", "-std=c++17", *SAN, "-fno-sanitize=enum", *include, os.path.join(ROOT, "tests", "sanitize", "search_main.cpp"),
                    str(stub), "-o", exe, "-L", str(tmp_path), "-lsip_san", "-Wl,-rpath," + str(tmp_path), "-L/opt/rocm/lib", "-lamdhip64",
                    "-Wl,-rpath,/opt/rocm/lib"])
    assert rc == 0, out
    rc, out = _run([exe], env={**os.environ, "ASAN_OPTIONS": "detect_leaks=0"})
    assert rc == 0 and "ok" in out and "ERROR" not in out and "runtime error" not in out, out
