"""CPU sanitizer build (AddressSanitizer + UndefinedBehaviorSanitizer, no recovery) of the host code behind the row norm,
the gradient norm, clipping and the Adam update, linked against the host stand-in for the HIP runtime."""
import os
import re
import subprocess

from test_sanitize_cpu import CSRC, HIPCC, ROOT, SAN, SAN_FLAGS, _run


def test_update_host_code_under_sanitizers(tmp_path):
    objs = []
    for src in ("norm_host.cpp", "norm.hip", "update_host.cpp", "update.hip"):
        obj = str(tmp_path / (os.path.splitext(src)[0] + ".o"))
        subprocess.run([HIPCC, "-x", "hip", "--cuda-host-only", "-O1", "-g", "-std=c++17", "-fPIC", "-ffp-contract=off",
                        "-I", os.path.join(ROOT, "include"), "-Xarch_host", SAN_FLAGS[0], "-Xarch_host", SAN_FLAGS[1],
                        "-Xarch_host", SAN_FLAGS[2], "-c", os.path.join(CSRC, src), "-o", obj],
                       check=True, capture_output=True)
        objs.append(obj)
    nm = subprocess.run(["nm", "-u", *objs], check=True, capture_output=True, text=True).stdout
    names = tmp_path / "fatbin_names.cpp"
    names.write_text("".join(f'extern "C" const char {f}[16] = {{0}};\n'
                             for f in sorted(set(re.findall(r"\b(__hip_fatbin_[0-9a-f]+)\b", nm)))))
    exe = str(tmp_path / "update_driver")
    subprocess.run(["/opt/rocm/llvm/bin/clang++", "-O1", "-g", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I", os.path.join(ROOT, "include"), *SAN_FLAGS, os.path.join(SAN, "update_driver.cpp"),
                    os.path.join(SAN, "hip_host_stub.cpp"), str(names), *objs, "-o", exe], check=True)
    rc, out, err = _run([exe], timeout=600)
    assert rc == 0 and "update driver ok" in out, (out[-2000:], err[-4000:])
    assert "runtime error" not in err and "AddressSanitizer" not in err, err[-4000:]
