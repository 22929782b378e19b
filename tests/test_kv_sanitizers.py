"""The host code of the 4-bit key/value cache under AddressSanitizer and UBSan (no GPU): its three sources alone, driven by a small program that
brings what they take from the rest of the library.  Sanitizers run on host code only; nothing here launches a kernel."""
import subprocess
from pathlib import Path

from tests.test_sanitizers import ENV, ROOT, SAN


def test_host_code_of_the_cache_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    from paper_2603_09229_amd import build as fk_build
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=all", "-Xarch_host", "-fno-omit-frame-pointer"]
    flags = [f for f in fk_build.FLAGS if f not in ("-O3", "-shared")]
    sources = [s for s in fk_build.sources() if s.name.startswith("fk_kv")]
    assert len(sources) == 3
    objects = [tmp_path / (s.name + ".o") for s in sources]
    jobs = [subprocess.Popen([fk_build.HIPCC, *flags, "-O1", "-g", *san, "-c", str(s), "-o", str(o)], stderr=subprocess.PIPE, text=True)
            for s, o in zip(sources, objects)]
    for j in jobs:
        err = j.communicate()[1]
        assert j.returncode == 0, err[-3000:]
    rocm = Path(fk_build.HIPCC).resolve().parent.parent
    clangxx = rocm / "lib" / "llvm" / "bin" / "clang++"
    exe = tmp_path / "kv_san"
    cmd = [str(clangxx), "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__",
           f"-I{rocm / 'include'}", f"-I{ROOT / 'include'}", "-o", str(exe), str(SAN / "kv_driver.cpp"), *map(str, objects),
           f"-L{rocm / 'lib'}", "-lamdhip64", f"-Wl,-rpath,{rocm / 'lib'}"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    # (leak checking off: the HIP runtime keeps allocations of its own)
    env = dict(ENV, ASAN_OPTIONS=ENV["ASAN_OPTIONS"].replace("detect_leaks=1", "detect_leaks=0"))
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=600)
    assert r.returncode == 0 and "kv sanitizer run ok" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]
