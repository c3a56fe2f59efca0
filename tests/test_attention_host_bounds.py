"""The attention entry points at the largest numbers that their arguments hold: what a launch cannot count is refused by its size, before anything is enqueued."""
import ctypes

import pytest

import paper_2507_17511_amd as cf
from test_attention_host import MB, SHAPE, append, cache, desc, prompt, refused, rows
from test_attention_host_sanitizers import ENV, HERE, ROOT, SAN

import os
import subprocess


def test_nothing_overflows_and_launches_are_counted(tmp_path):
    exe = str(tmp_path / "attention_bounds_san")
    csrc = os.path.join(ROOT, "paper_2507_17511_amd", "csrc")
    for cmd in (["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                 os.path.join(csrc, "cf_attn_api.cpp"), os.path.join(HERE, "attention_bounds_driver.cpp"), "-o", exe], [exe]):
        res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=ENV)
        assert res.returncode == 0, f"{' '.join(cmd)}\n{res.stdout[-4000:]}"
    assert "all calls hold" in res.stdout


def test_calls_of_more_work_items_than_a_launch_counts():
    """2^32 and more threads, at strides of 0 that need no memory to speak of."""
    one = desc(q_heads=4, kv_heads=4)
    refused(SHAPE, cf.cf_kv_append, one, cache(v=512 * MB), append(n_tokens=1 << 27, k=rows(1 * MB, 0, 0), v=rows(2 * MB, 0, 0), q=rows(None, 0, 0), q_out=rows(None, 0, 0), rotary_dim=0))
    refused(SHAPE, cf.cf_attn_prompt, desc(), prompt(n_seqs=1 << 24))
    p = (ctypes.c_void_p * 64)(*[1 << 50] * 64)
    for parts, tokens in ((1, 1 << 28), (16, 1 << 26), (64, 1 << 24)):
        refused(SHAPE, cf.cf_attn_join, desc(q_heads=1, kv_heads=1), cf.cf_join(parts, cf.CF_BF16, tokens, p, p, rows(1 * MB, 128, 128), None))


@pytest.mark.parametrize("n_pages,stride", [(1 << 30, 1 << 40), ((1 << 31) - 1, 1 << 36)])
def test_caches_larger_than_an_address_says(n_pages, stride):
    refused(SHAPE, cf.cf_kv_append, desc(), cache(n_pages=n_pages, page_stride=stride, v=64 * MB + 8 * stride), append())
