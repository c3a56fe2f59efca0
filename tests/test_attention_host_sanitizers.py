"""The host half of the attention entry points under AddressSanitizer and UndefinedBehaviorSanitizer, with stand-in launchers."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = os.path.join(ROOT, "tests", "host_sanitize")
SAN = ["-g", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer"]
ENV = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
ENV.pop("LD_PRELOAD", None)


def test_random_calls_stay_inside_what_they_are_given(tmp_path):
    exe = str(tmp_path / "attention_san")
    csrc = os.path.join(ROOT, "paper_2507_17511_amd", "csrc")
    for cmd in (["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                 os.path.join(csrc, "cf_attn_api.cpp"), os.path.join(HERE, "attention_driver.cpp"), "-o", exe], [exe]):
        res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=ENV)
        assert res.returncode == 0, f"{' '.join(cmd)}\n{res.stdout[-4000:]}"
    assert "all calls hold" in res.stdout
