"""The host half of the entry points for the cache in 8 bits under AddressSanitizer and UndefinedBehaviorSanitizer, with stand-in launchers."""
import os
import subprocess

from test_attention_host_sanitizers import ENV, HERE, ROOT, SAN


def test_random_calls_stay_inside_what_they_are_given(tmp_path):
    exe = str(tmp_path / "cache8_san")
    csrc = os.path.join(ROOT, "paper_2507_17511_amd", "csrc")
    for cmd in (["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                 os.path.join(csrc, "cf_attn8_api.cpp"), os.path.join(HERE, "cache8_driver.cpp"), "-o", exe], [exe]):
        res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=ENV)
        assert res.returncode == 0, f"{' '.join(cmd)}\n{res.stdout[-4000:]}"
    assert "all calls hold" in res.stdout
