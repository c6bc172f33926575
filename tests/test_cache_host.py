"""The host side of the operators over shared and bounded caches
(csrc/cache_api.cpp) built with a host compiler alone and linked with launchers
that launch nothing (tests/cache_launch_stub.cpp): which form a call takes, and,
under AddressSanitizer and UndefinedBehaviorSanitizer, that no refusal reaches a
launcher."""
import ctypes
import os
import subprocess
import sys
from pathlib import Path

import pytest

import paper_2609_33586_amd as pkg
from oracle import build as obuild

ROOT = Path(__file__).resolve().parent.parent
CSRC = ROOT / "paper_2609_33586_amd" / "csrc"
A = 0x100000  # never dereferenced


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    lib = tmp_path_factory.mktemp("cache_host") / "libh15cache_host.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-ffp-contract=off", "-Wall", "-Wextra", "-Werror",
                    f"-I{ROOT / 'include'}", f"-I{CSRC}", str(CSRC / "cache_api.cpp"),
                    str(ROOT / "tests" / "cache_launch_stub.cpp"), "-o", str(lib)], check=True)
    L = ctypes.CDLL(str(lib))
    P, I, F, S = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    L.attn_decode_prefix.argtypes = [P] * 8 + [I] * 10 + [F] + [I] * 4 + [P, S, P]
    L.attn_key_weights.argtypes = [P] * 5 + [I] * 8 + [F, F, I, P, S, P]
    L.attn_evict.argtypes = [P] * 9 + [I] * 9 + [P, S, P]
    L.attn_evict_workspace_bytes.restype = S
    return L


def prefix_form(L, B, Hq, Hkv, Sq, P, Sk, p_cut=0, cut=0, causal=1, lens=None):
    rc = L.attn_decode_prefix(A, A, A, A, A, lens, A, None, B, Hq, Hkv, Sq, P, P, Sk, Sk, 128, causal, 0.1, 0, 0, p_cut,
                              cut, A, 1 << 40, None)
    assert rc == pkg.ATTN_ELAUNCH
    names = ("p_parts", "o_parts", "p_rows", "p_groups", "o_groups", "p_split", "o_split", "causal", "chain", "longest")
    return {n: L.h15_stub_prefix(i) for i, n in enumerate(names)}


def test_prefix_forms(host):
    # up to 128 rows of a KV head over the batch: workgroups of 32 rows, else of 128
    f = prefix_form(host, 8, 8, 2, 1, 1000, 100)
    assert f["p_rows"] == 32 and f["p_groups"] == 2 and f["o_groups"] == 8 * 2
    f = prefix_form(host, 32, 32, 8, 1, 1000, 100, 512, 0)
    assert f["p_rows"] == 32 and f["p_groups"] == 8 * 2 * 4
    f = prefix_form(host, 33, 32, 8, 1, 1000, 100, 512, 0)
    assert f["p_rows"] == 128 and f["p_parts"] == 2 and f["o_parts"] == 1 and f["p_groups"] == 8 * 2 * 2
    assert f["o_groups"] == 33 * 8 and f["o_split"] == 128 and f["p_split"] == 512
    assert prefix_form(host, 33, 32, 8, 1, 1000, 0)["p_rows"] == 32  # a single part writes O itself
    f = prefix_form(host, 2, 12, 2, 16, 0, 300, 0, 128)
    assert f["p_groups"] == 0 and f["o_groups"] == 2 * 2 * 3 * 3  # 96 rows a sequence: three blocks
    # one query row sees its whole cache with or without a causal mask
    assert prefix_form(host, 2, 4, 2, 1, 10, 10)["causal"] == 0 and prefix_form(host, 2, 4, 2, 2, 10, 10)["causal"] == 1


def test_prefix_before_own_caches(host):
    # a prefix of two rounds (of 128 BF16 keys, d = 128) in one part, own caches in one part
    f = prefix_form(host, 8, 8, 2, 1, 256, 100)
    assert f["chain"] == 1 and f["p_groups"] == 0 and f["o_groups"] == 8 * 2
    assert prefix_form(host, 8, 8, 2, 1, 257, 100)["chain"] == 0
    assert prefix_form(host, 8, 8, 2, 1, 256, 100, 128, 0)["chain"] == 0
    assert prefix_form(host, 8, 8, 2, 1, 256, 300, 0, 128)["chain"] == 0
    assert prefix_form(host, 8, 8, 2, 1, 256, 0)["chain"] == 0 and prefix_form(host, 8, 8, 2, 1, 0, 100)["chain"] == 0
    # more than 512 own caches take it only with full blocks of 32 rows
    assert prefix_form(host, 64, 32, 8, 1, 256, 100)["chain"] == 1
    assert prefix_form(host, 65, 32, 8, 1, 256, 100)["chain"] == 0
    assert prefix_form(host, 65, 32, 8, 8, 256, 100)["chain"] == 1


def test_long_caches_first(host):
    # 256 slots next to 256 prefix workgroups or more, 512 less those there are
    many = (1, 32768, 100, 1024, 0)  # Sq, P, Sk and cuts: 32 parts of 8 heads
    assert prefix_form(host, 32, 32, 8, *many, lens=A)["longest"] == 0
    assert prefix_form(host, 33, 32, 8, *many, lens=A)["longest"] == 1
    assert prefix_form(host, 33, 32, 8, *many)["longest"] == 0  # all alike
    assert prefix_form(host, 256, 2, 2, 1, 0, 100, lens=A)["longest"] == 0
    assert prefix_form(host, 256, 3, 3, 1, 0, 100, lens=A)["longest"] == 1
    assert prefix_form(host, 257, 3, 3, 1, 0, 100, lens=A)["longest"] == 0  # more than a workgroup's threads
    assert prefix_form(host, 1, 64, 64, 1, 0, 4096, 0, 128, lens=A)["longest"] == 0


def test_weights_runs(host):
    def form(Hq, Hkv, Sq, Sk):
        rc = host.attn_key_weights(A, A, A, None, A, 1, Hq, Hkv, Sq, Sk, Sk, 128, 1, 0.1, 1.0, 0, A, 1 << 40, None)
        assert rc == pkg.ATTN_ELAUNCH
        return {n: host.h15_stub_weights(i) for i, n in enumerate(("heads", "hrows", "parts", "blocks", "causal"))}

    # up to 256 query rows of a KV head: one part, blocks of four waves with runs
    # of one to three units of 64 keys, about 512 workgroups
    assert form(8, 2, 1, 256) == {"heads": 1, "hrows": 4, "parts": 1, "blocks": 1, "causal": 0}
    assert form(8, 2, 31, 257) == {"heads": 1, "hrows": 124, "parts": 1, "blocks": 2, "causal": 1}
    assert form(8, 2, 64, 257)["heads"] == 4 and form(8, 2, 64, 257)["blocks"] == 2
    assert [form(8, 8, 1, 64 * 2048 * x // 8)["blocks"] for x in (1, 2, 3, 4)] == [64, 64, 64, 86]
    # beyond: blocks of 256 keys, runs of one head from 32 rows on, parts of at most 32 tiles of 64 rows
    assert form(16, 1, 31, 257) == {"heads": 1, "hrows": 496, "parts": 1, "blocks": 2, "causal": 1}
    assert form(16, 1, 32, 257) == {"heads": 16, "hrows": 32, "parts": 1, "blocks": 2, "causal": 1}
    assert form(8, 2, 512, 512)["parts"] == 1 and form(8, 2, 513, 512)["parts"] == 2
    assert form(64, 1, 65, 512)["parts"] == 2  # more heads than tiles: one tile of each


def test_evict_forms(host):
    def form(B, Hkv, Sk, keep, d=128):
        at = [0x100000 + (i << 46) for i in range(9)]
        rc = host.attn_evict(at[0], at[1], at[2], None, *at[3:8], B, Hkv, Sk, Sk, keep, d, keep, 0, 0, at[8],
                             host.attn_evict_workspace_bytes(B, Hkv, Sk), None)
        assert rc == pkg.ATTN_ELAUNCH
        return host.h15_stub_evict(0), host.h15_stub_evict(1)

    # (parts of 4096 keys, whether the selecting workgroup copies the rows: up to 4096 chunks of 16 bytes)
    assert form(1, 2, 300, 100) == (1, 1) and form(1, 2, 300, 256) == (1, 1) and form(1, 2, 300, 257) == (1, 0)
    assert form(1, 2, 5 * 4096, 100) == (1, 1) and form(1, 2, 5 * 4096 + 1, 100) == (6, 0)
    assert form(4, 8, 32768, 1000) == (8, 0) and form(11, 3, 32768, 1000) == (1, 0)
    assert form(8, 8, 32769, 100) == (9, 0) and form(13, 5, 32769, 100) == (1, 1)


def evict_parts(host, heads, Sk):
    at = [0x100000 + (i << 46) for i in range(9)]
    rc = host.attn_evict(at[0], at[1], at[2], None, *at[3:8], 1, heads, Sk, Sk, 100, 64, 100, 0, 1, at[8],
                         host.attn_evict_workspace_bytes(1, heads, Sk), None)
    assert rc == pkg.ATTN_ELAUNCH
    return host.h15_stub_evict(0)


@pytest.mark.parametrize("heads", [1, 2, 7, 8, 20, 21, 32, 33, 64, 65, 256])
def test_evict_parts_stay_few(host, heads):
    # every workgroup adds up what its head's parts counted: their number is bounded as caches grow
    for Sk in (1, 20480, 20481, 32769, 100003, 131072, 1 << 18, 10 ** 6, 1 << 20):
        n = evict_parts(host, heads, Sk)
        # (a part counts up to 61440 keys in 16 bits)
        assert n == 1 or -(-Sk // 61440) <= n <= max(-(-Sk // 61440), min(32, 640 // heads))
        assert (n > 1) == (host.attn_evict_workspace_bytes(1, heads, Sk) > 0)


def test_evict_parts_of_the_longest_caches_fit_a_launch(host):
    assert evict_parts(host, 64, 2 ** 31 - 8193) * 64 <= 2 ** 22 - 1
    assert host.attn_evict_workspace_bytes(1, 64, 2 ** 31 - 8193) > 2 ** 31


def test_checks_under_sanitizers(tmp_path):
    lib = tmp_path / "libh15cache_san.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-fPIC", "-shared", "-ffp-contract=off",
                    "-Dh15_stub_launches=h15_forward_stub_launches", f"-I{ROOT / 'include'}", f"-I{CSRC}",
                    str(CSRC / "attn_api.cpp"), str(ROOT / "tests" / "sanitize_launch_stub.cpp"), "-c"], cwd=tmp_path,
                   check=True)
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-fPIC", "-shared", "-ffp-contract=off", f"-I{ROOT / 'include'}",
                    f"-I{CSRC}", str(CSRC / "cache_api.cpp"), str(ROOT / "tests" / "cache_launch_stub.cpp"),
                    str(tmp_path / "attn_api.o"), str(tmp_path / "sanitize_launch_stub.o"), "-o", str(lib)], check=True)
    env = dict(os.environ, LD_PRELOAD=obuild.sanitizer_preload(), ASAN_OPTIONS="detect_leaks=0:abort_on_error=0",
               UBSAN_OPTIONS="print_stacktrace=1", H15ATTN_LIB=str(lib))
    code = ("import sys, pytest; rc = pytest.main(['tests/test_cache_api.py', '-q', '-p', 'no:cacheprovider']); "
            "import paper_2609_33586_amd as p; assert p.lib()._name == %r and p.lib().h15_stub_launches() == 0; "
            "sys.exit(rc)" % str(lib))
    res = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    out = res.stdout + res.stderr
    assert "AddressSanitizer" not in out and "runtime error" not in out, out[-4000:]
    assert res.returncode == 0 and " passed" in out, out[-4000:]
