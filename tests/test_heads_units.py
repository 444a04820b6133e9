"""The forward of the head preparation sums a row over lanes of a warp inside a branch that depends on the tensor (V is only moved): the
groups of a warp must never belong to different tensors.  The kernel's own mapping, compiled for the CPU."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_12128_b200", "csrc")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    at = tmp_path_factory.mktemp("units")
    (at / "units.cpp").write_text('#include "hla_heads_units.h"\n'
                                  'extern "C" uint32_t all(uint32_t tokens, uint32_t runs, int log_lanes) { return hla::heads::units_of(tokens, runs, log_lanes).all; }\n'
                                  'extern "C" int unit(uint32_t tokens, uint32_t runs, int log_lanes, uint32_t i, uint32_t* run, uint32_t* token) {\n'
                                  '    const hla::heads::Unit u = hla::heads::unit_of(hla::heads::units_of(tokens, runs, log_lanes), i);\n'
                                  '    *run = u.run; *token = u.token; return u.live; }\n')
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(at / "units.cpp"), "-o", str(at / "units.so")], check=True)
    return ctypes.CDLL(str(at / "units.so"))


@pytest.mark.parametrize("log_lanes", range(6))
@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 7, 31, 32, 33, 41, 64, 105])
def test_a_warp_has_one_run_and_every_token_is_taken_once(lib, log_lanes, tokens):
    groups, run, token = 256 >> log_lanes, ctypes.c_uint32(), ctypes.c_uint32()
    for runs in (1, 2, 3, 5, 12):
        every = lib.all(tokens, runs, log_lanes)
        blocks = (every + groups - 1) // groups
        seen = []
        for warp in range(blocks * 8):
            of_warp = set()
            for g in range(32 >> log_lanes):
                live = lib.unit(tokens, runs, log_lanes, warp * (32 >> log_lanes) + g, ctypes.byref(run), ctypes.byref(token))
                assert run.value < runs and token.value < tokens
                of_warp.add(run.value)
                if live:
                    seen.append((run.value, token.value))
            assert len(of_warp) == 1
        assert sorted(seen) == [(r, t) for r in range(runs) for t in range(tokens)]


def test_the_largest_number_of_tokens(lib):
    """2^28 tokens of three tensors in groups of one lane: the units stay within 32 bits, the last one is a token."""
    run, token = ctypes.c_uint32(), ctypes.c_uint32()
    tokens = (1 << 28) - 1
    lib.all.restype = ctypes.c_uint32
    every = lib.all(tokens, 3, 0)
    assert every == 3 << 28
    assert lib.unit(tokens, 3, 0, every - 2, ctypes.byref(run), ctypes.byref(token)) and (run.value, token.value) == (2, tokens - 1)
    assert not lib.unit(tokens, 3, 0, every - 1, ctypes.byref(run), ctypes.byref(token)) and not lib.unit(tokens, 3, 0, every, ctypes.byref(run), ctypes.byref(token))
