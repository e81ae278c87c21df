"""Host-only checks of the prompt operators: exports, sizes, refusals before any GPU call, wait states of the matrix instructions."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2505_22179_amd import binding as B
from paper_2505_22179_amd import build
from tests import test_matrix_hazards_host as hazards
from tests.test_kv8_host import A, EALIGN, EINVAL, ENULL, EUNSUP, EWS, INF, NAN, refusals

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BIG = 1 << 40


def caller(lib, name, **defaults):
    f = getattr(lib, name)

    def call(**changed):
        assert not set(changed) - set(defaults)
        return f(*{**defaults, **changed}.values(), None)
    return call


def test_w8a8_symbols_are_exported():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "w8a8.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(w8a8_\w+)\s*\(", text)))
    assert names == sorted(B.EXPORTS_W8A8)
    for n in names:
        assert hasattr(B.load_w8a8(), n), n


def test_rope_table_refuses():
    call = caller(B.load(), "rope_table", cos=A, sin=A, first=0, n=64, R=128, theta=1e4, scaling=B.ROPE_BY_TURNS, factor=8.0, low=1.0, high=4.0, original=8192.0, amplitude=1.0)
    refusals(call, {
        EINVAL: [dict(first=-1), dict(n=0), dict(R=0), dict(R=7), dict(theta=1.0), dict(theta=NAN), dict(theta=INF), dict(scaling=-1), dict(scaling=4),
                 dict(factor=0.0), dict(factor=NAN), dict(factor=INF), dict(low=0.0), dict(low=4.0), dict(high=INF), dict(high=NAN), dict(original=0.0), dict(original=INF),
                 dict(amplitude=NAN), dict(amplitude=INF), dict(scaling=B.ROPE_BY_INDEX, high=0.5), dict(scaling=B.ROPE_LINEAR, factor=-1.0)],
        EUNSUP: [dict(R=1026), dict(first=2 ** 28), dict(n=2 ** 28 + 1)],
        ENULL: [dict(cos=None), dict(sin=None)], EALIGN: [dict(cos=A + 4), dict(sin=A + 8)],
    })


def test_rope_prompt_refuses():
    call = caller(B.load(), "rope_prompt", qkv=A, pos=A, cos=A, sin=A, n_pos=64, R=64, interleaved=0, slot=A, cache_rows=100, q=A, k=A, v=A, rows=10, Hq=8, Hkv=2, D=128)
    refusals(call, {
        EINVAL: [dict(n_pos=0), dict(R=0), dict(R=130), dict(R=63), dict(interleaved=2), dict(cache_rows=0), dict(rows=0), dict(Hq=0), dict(Hkv=0), dict(D=0), dict(D=100)],
        EUNSUP: [dict(D=520), dict(rows=2 ** 23 + 1), dict(Hq=2 ** 16 + 1), dict(Hkv=2 ** 16 + 1)],
        ENULL: [{n: None} for n in ("qkv", "pos", "cos", "sin", "q", "k", "v")],
        EALIGN: [{n: A + 8} for n in ("qkv", "cos", "sin", "q", "k", "v")] + [dict(pos=A + 2), dict(slot=A + 1)],
    })


def test_prompt_attn_refuses_and_states_its_scratch():
    size = B.w4a16_prompt_attn_workspace_bytes
    call = caller(B.load(), "w4a16_prompt_attn", q=A, k=A, v=A, q_start=A, k_start=A, k_len=A, out=A, batch=3, rows=100, k_rows=1000, max_q=50, max_k=700,
                  Hq=8, Hkv=2, D=128, scale=ctypes.c_float(0.1), ws=A, nbytes=BIG)
    shape = [dict(rows=0), dict(batch=0), dict(max_q=0), dict(max_k=0), dict(Hq=0), dict(Hkv=0), dict(Hq=9), dict(D=0)]
    unsupported = [dict(D=96), dict(D=256), dict(batch=4097), dict(rows=2 ** 23 + 1), dict(Hq=130), dict(Hkv=2048, Hq=2048), dict(max_q=2 ** 23 + 1), dict(max_k=2 ** 30 + 1),
                   dict(rows=2 ** 23, Hq=128, Hkv=2)]
    refusals(call, {
        EINVAL: shape + [dict(k_rows=0)] + [dict(scale=ctypes.c_float(s)) for s in (0.0, -1.0, NAN, INF)], EUNSUP: unsupported,
        ENULL: [{n: None} for n in ("q", "k", "v", "q_start", "out", "k_start", "k_len")],
        EALIGN: [{n: A + 8} for n in ("q", "k", "v", "out")] + [{n: A + 2} for n in ("q_start", "k_start", "k_len")] + [dict(ws=A + 16)],
        EWS: [dict(ws=None), dict(nbytes=100), dict(nbytes=size(100, 3, 50, 700, 8, 2, 128) - 1)],
    })
    assert size(100, 3, 50, 700, 8, 2, 128) >= 16384 and size(100, 3, 50, 700, 8, 2, 96) == 0 and size(0, 3, 50, 700, 8, 2, 128) == 0


def test_w8a8_refuses():
    lib = B.load_w8a8()
    assert lib.w8a8_packed_bytes(17, 100 * 16) == 2 * 26 * 1024 and lib.w8a8_packed_bytes(16, 64) == 2048
    assert lib.w8a8_packed_bytes(0, 64) == lib.w8a8_packed_bytes(1, 72) == lib.w8a8_packed_bytes(1, 65552) == 0
    for name in ("w8a8_pack", "w8a8_unpack"):
        call = caller(lib, name, a=A, b=A, rows=16, K=64)
        refusals(call, {EINVAL: [dict(rows=0), dict(K=0), dict(K=24)], EUNSUP: [dict(K=65552), dict(rows=2 ** 24 + 1)], ENULL: [dict(a=None), dict(b=None)],
                        EALIGN: [dict(a=A + 8), dict(b=A + 4)]})
    f = ctypes.c_float
    inputs = {EINVAL: [dict(pre=-1), dict(pre=3), dict(eps=f(-1.0)), dict(eps=f(NAN)), dict(pre=B.W8A8_PLAIN), dict(pre=B.W8A8_SILU_MUL)],
              ENULL: [dict(x=None), dict(gamma=None)], EALIGN: [dict(x=A + 8), dict(gamma=A + 2)]}
    call = caller(lib, "w8a8_quantize", x=A, pre=B.W8A8_RMS_NORM, gamma=A, eps=f(1e-5), codes=A, scale=A, M=4, K=64)
    refusals(call, inputs)
    refusals(call, {EINVAL: [dict(M=0), dict(K=0), dict(K=40)], EUNSUP: [dict(K=65552), dict(M=2 ** 20 + 1)], ENULL: [dict(codes=None), dict(scale=None)],
                    EALIGN: [dict(codes=A + 8), dict(scale=A + 4)]})
    sizes = {EINVAL: [dict(M=0), dict(N=0), dict(N=12), dict(K=0), dict(K=24)], EUNSUP: [dict(K=65552), dict(N=2 ** 20 + 8), dict(M=2 ** 20 + 1)],
             ENULL: [{n: None} for n in ("packed", "w_scale", "y")], EALIGN: [{n: A + 8} for n in ("packed", "w_scale", "y", "residual")] + [dict(ws=A + 16)],
             EWS: [dict(ws=None), dict(nbytes=lib.w8a8_workspace_bytes(4, 64, 64) - 1)]}
    shared = dict(packed=A, w_scale=A, residual=A, y=A, M=4, N=64, K=64, ws=A, nbytes=BIG)
    call = caller(lib, "w8a8_gemm", codes=A, scale=A, **shared)
    refusals(call, sizes)
    refusals(call, {ENULL: [dict(codes=None), dict(scale=None)], EALIGN: [dict(codes=A + 8), dict(scale=A + 4)]})
    call = caller(lib, "w8a8_linear", x=A, pre=B.W8A8_RMS_NORM, gamma=A, eps=f(1e-5), **shared)
    refusals(call, sizes)
    refusals(call, inputs)
    assert lib.w8a8_workspace_bytes(4, 60, 64) == lib.w8a8_workspace_bytes(0, 64, 64) == 0
    assert lib.w8a8_workspace_bytes(100, 4096, 4096) <= lib.w8a8_workspace_bytes(200, 4096, 4096)


# passes + 4: 16x16x64 of int8 takes four passes, as its fp16 form does
PASSES = {"v_mfma_i32_16x16x64_i8": 8, "v_mfma_i32_32x32x32_i8": 12}


@pytest.mark.parametrize("library, kernels", [("w4a16", "prompt_"), ("w8a8", "w8a8_")])
def test_no_result_of_a_matrix_instruction_is_touched_too_early(library, kernels, tmp_path, monkeypatch):
    if not os.path.exists(hazards.OBJDUMP):
        pytest.skip("no llvm-objdump")
    monkeypatch.setattr(hazards, "NEEDED", {**hazards.NEEDED, **PASSES})
    path, bad, matrix = tmp_path / "object", [], 0
    for obj in hazards.code_objects(build.build(force=False) if library == "w4a16" else build.build_w8a8(force=False)):
        path.write_bytes(obj)
        listing = subprocess.run([hazards.OBJDUMP, "-d", str(path)], capture_output=True, text=True, check=True).stdout
        if kernels not in listing:
            continue
        found, code = hazards.violations(listing.splitlines())
        bad += [b for b in found if kernels in b.split(":")[0]]
        matrix += sum(n.startswith("v_mfma") and kernels in k for n, k in zip(code.name, code.kernel))
    assert matrix > 50 and not bad, "\n".join(bad[:40])


def test_rope_table_refuses_factors_that_lead_out_of_its_range():
    call = caller(B.load(), "rope_table", cos=A, sin=A, first=0, n=64, R=128, theta=1e4, scaling=B.ROPE_LINEAR, factor=0.1249, low=1.0, high=4.0, original=8192.0, amplitude=1.0)
    refusals(call, {EUNSUP: [dict(), dict(scaling=B.ROPE_BY_TURNS), dict(scaling=B.ROPE_BY_INDEX), dict(factor=1e-300)]})
