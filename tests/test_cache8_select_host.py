"""The arithmetic of the selection of pages, which the kernel shares with this build for the host, under AddressSanitizer and UndefinedBehaviorSanitizer."""
import os
import subprocess

from test_attention_host_sanitizers import ENV, HERE, ROOT, SAN


def test_as_many_scores_are_taken_as_there_are_to_take(tmp_path):
    """Infinite scores among them: the range of those that are left ends at the largest number there is."""
    exe = str(tmp_path / "select_san")
    for cmd in (["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"),
                 "-I", os.path.join(ROOT, "paper_2507_17511_amd", "csrc"), os.path.join(HERE, "select_driver.cpp"), "-o", exe], [exe]):
        res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=ENV)
        assert res.returncode == 0, f"{' '.join(cmd)}\n{res.stdout[-4000:]}"
    assert "all selections hold" in res.stdout
