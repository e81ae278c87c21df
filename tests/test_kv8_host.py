"""Host-only checks of the entry points around the 8-bit cache: bad arguments are refused before any GPU call."""
import ctypes

import numpy as np
import pytest

from paper_2505_22179_amd import binding as B

A = 0x1000   # fake, aligned, never dereferenced: every call below fails validation first
EINVAL, ENULL, EALIGN, EUNSUP, EWS = -1, -2, -3, -4, -5
NAN, INF = float("nan"), float("inf")


def caller(name, **defaults):
    f = getattr(B.load(), name)

    def call(**changed):
        assert not set(changed) - set(defaults)
        return f(*{**defaults, **changed}.values(), None)
    return call


def refusals(call, table):
    for code, changes in table.items():
        for change in changes:
            assert call(**change) == code, (code, change)


APPEND = dict(qkv=A, q_gamma=A, k_gamma=A, eps=1e-6, pos=A, cos=A, sin=A, n_pos=64, q=A, k=A, v=A)
SIZES = dict(M=4, P=10, Hq=8, Hkv=2, D=128)
APPEND_REFUSALS = {
    EINVAL: [dict(M=0), dict(P=-1), dict(Hq=0), dict(Hkv=0), dict(D=0), dict(D=4), dict(D=100), dict(n_pos=0), dict(eps=-1.0), dict(eps=NAN)],
    EUNSUP: [dict(M=65536), dict(D=520), dict(P=2 ** 30 + 1), dict(Hq=2 ** 21), dict(Hkv=2 ** 21)],
    ENULL: [dict(qkv=None), dict(pos=None), dict(cos=None), dict(sin=None), dict(q=None), dict(k=None), dict(v=None), dict(q_gamma=None), dict(k_gamma=None)],
    EALIGN: [dict(qkv=A + 8), dict(q_gamma=A + 2), dict(k_gamma=A + 8), dict(pos=A + 2), dict(cos=A + 4), dict(sin=A + 8), dict(q=A + 8), dict(k=A + 8),
             dict(v=A + 4)],
}


def test_rope_append_qk_norm_refuses():
    call = caller("rope_append_qk_norm", **APPEND, **SIZES)
    refusals(call, APPEND_REFUSALS)
    assert call(q_gamma=None, k_gamma=None) == ENULL


def test_rope_append_kv8_refuses():
    call = caller("rope_append_kv8", **APPEND, ks=A, vs=A, format=B.KV8_INT8, **SIZES)
    refusals(call, APPEND_REFUSALS)
    refusals(call, {EINVAL: [dict(format=0), dict(format=3), dict(format=-1)], ENULL: [dict(ks=None), dict(vs=None)], EALIGN: [dict(ks=A + 2), dict(vs=A + 8)]})


def test_w4a16_kv8_read_refuses():
    call = caller("w4a16_kv8_read", k=A, v=A, ks=A, vs=A, format=B.KV8_E4M3, first=3, rows=5, Hkv=2, D=128, k_out=A, v_out=A)
    refusals(call, {
        EINVAL: [dict(format=0), dict(first=-1), dict(rows=-1), dict(Hkv=0), dict(D=0), dict(D=12)],
        EUNSUP: [dict(D=1024), dict(first=2 ** 30 + 1), dict(rows=2 ** 30 + 1), dict(Hkv=2 ** 21)],
        ENULL: [{n: None} for n in ("k", "v", "ks", "vs", "k_out", "v_out")],
        EALIGN: [{n: A + 8} for n in ("k", "v", "ks", "vs", "k_out", "v_out")],
    })
    assert call(rows=0) == 0   # nothing to do


def test_tree_verify_attn_kv8_refuses():
    call = caller("tree_verify_attn_kv8", q=A, k=A, v=A, ks=A, vs=A, format=B.KV8_INT8, mask=A, out=A, M=60, P=2048, Hq=64, Hkv=8, D=128, scale=0.1, ws=A,
                  bytes=1 << 30)
    refusals(call, {
        EINVAL: [dict(format=0), dict(format=5), dict(M=0), dict(P=-1), dict(Hq=0), dict(Hkv=0), dict(Hkv=7), dict(scale=0.0), dict(scale=-0.1), dict(scale=NAN),
                 dict(scale=INF)],
        EUNSUP: [dict(D=64), dict(M=65), dict(Hkv=4), dict(Hq=8192, Hkv=8192), dict(P=2 ** 30 + 1)],
        ENULL: [{n: None} for n in ("q", "k", "v", "ks", "vs", "mask", "out")],
        EALIGN: [{n: A + 8} for n in ("q", "k", "v", "ks", "vs", "out")] + [dict(ws=A + 128)],
        EWS: [dict(ws=None), dict(bytes=0), dict(bytes=B.tree_verify_attn_kv8_workspace_bytes(60, 2048, 64, 8, 128) - 1)],
    })


def test_tree_accept_kv8_refuses():
    call = caller("tree_accept_kv8", parent=A, token=A, target=A, M=60, path=A, result=A, k=A, v=A, ks=A, vs=A, P=2048, Hkv=8, D=128)
    refusals(call, {
        EINVAL: [dict(M=0), dict(P=-1), dict(Hkv=0), dict(D=0), dict(D=20)],
        EUNSUP: [dict(M=65), dict(D=520), dict(P=2 ** 30 + 1), dict(Hkv=2 ** 21)],
        ENULL: [{n: None} for n in ("parent", "token", "target", "path", "result", "k", "v", "ks", "vs")],
        EALIGN: [{n: A + 2} for n in ("parent", "token", "target", "path", "result", "k", "v", "ks", "vs")],
    })


@pytest.mark.parametrize("Hq,Hkv", [(64, 8), (32, 8), (8, 8), (28, 4), (4096, 512), (7, 1)])
def test_workspace_serves_every_smaller_call(Hq, Hkv):
    sizes = [(M, P) for M in (1, 2, 7, 16, 33, 60, 64) for P in (0, 31, 500, 2048, 20000, 131072, 2 ** 30)]
    most = B.tree_verify_attn_kv8_workspace_bytes(64, 2 ** 30, Hq, Hkv, 128)
    for M, P in sizes:
        assert 0 < B.tree_verify_attn_kv8_workspace_bytes(M, P, Hq, Hkv, 128) <= most
    assert B.tree_verify_attn_kv8_workspace_bytes(65, 10, Hq, Hkv, 128) == 0


def test_lm_head_sample_refuses():
    call = caller("lm_head_sample", logits=A, M=4, V=1000, temperature=A, top_k=A, top_p=A, min_p=A, uniform=A, token=A, prob=A, ws=A, bytes=1 << 30)
    refusals(call, {
        EINVAL: [dict(M=0), dict(V=0), dict(V=-1)],
        EUNSUP: [dict(M=65), dict(V=262145)],
        ENULL: [{n: None} for n in ("logits", "uniform", "token", "prob")],
        EALIGN: [dict(logits=A + 4), dict(ws=A + 128)] + [{n: A + 2} for n in ("temperature", "top_k", "top_p", "min_p", "uniform", "token", "prob")],
        EWS: [dict(ws=None), dict(bytes=B.lm_head_sample_workspace_bytes(4, 1000) - 1)],
    })
    assert B.lm_head_sample_workspace_bytes(65, 1000) == 0 and B.lm_head_sample_workspace_bytes(1, 262145) == 0
    for M in (1, 7, 64):
        for V in (1, 1000, 128256, 262144):
            assert 0 < B.lm_head_sample_workspace_bytes(M, V) <= B.lm_head_sample_workspace_bytes(64, 262144)


def test_sample_workspace_serves_every_smaller_call():
    Vs = (1, 511, 513, 4096, 4097, 8192, 32000, 65537, 128256, 200001, 262144)
    sizes = np.array([[B.lm_head_sample_workspace_bytes(M, V) for V in Vs] for M in range(1, 65)])
    assert (np.diff(sizes, axis=0) >= 0).all() and (np.diff(sizes, axis=1) >= 0).all()


@pytest.mark.parametrize("M,V,K,top_k", [(1, 1, 128, 1), (1, 32000, 4096, 10), (60, 128256, 8192, 1), (64, 262144, 4096, 16)])
def test_the_lm_heads_workspace_has_a_ticket_area(M, V, K, top_k):
    """16384 bytes at its start, behind which it keeps statistics of 64 tokens each: the tickets of other calls on the same workspace stay at zero"""
    assert B.lm_head_workspace_bytes(M, V, K, top_k) >= 16384 + M * -(-V // 64) * 8


def plan(M, P, Hq, Hkv, fmt):
    return B.tree_verify_attn_kv8_plan_describe(M, P, Hq, Hkv, 128, fmt)


def test_attn_kv8_plan_describe_refuses():
    f, out = B.load().tree_verify_attn_kv8_plan_describe, (ctypes.c_int * 5)()
    assert f(60, 2048, 64, 8, 128, B.KV8_INT8, out) == 0 and f(60, 2048, 64, 8, 128, B.KV8_INT8, None) == ENULL
    for sizes in ((0, 1, 8, 8, 128), (1, -1, 8, 8, 128), (1, 1, 9, 8, 128)):
        assert f(*sizes, B.KV8_E4M3, out) == EINVAL
    assert f(60, 2048, 64, 8, 128, 0, out) == EINVAL
    for sizes in ((65, 1, 8, 8, 128), (1, 1, 8, 8, 64), (1, 2 ** 30 + 1, 8, 8, 128), (1, 1, 72, 8, 128), (1, 1, 4097, 4097, 128)):
        assert f(*sizes, B.KV8_E4M3, out) == EUNSUP


@pytest.mark.parametrize("fmt", [B.KV8_INT8, B.KV8_E4M3])
def test_attn_kv8_plans_cover_the_call(fmt):
    """every row in a tile, every key step in a range, partial results within the workspace, tickets within their area"""
    for Hq, Hkv in ((1, 1), (7, 1), (8, 8), (28, 4), (64, 8), (128, 128), (512, 64), (4096, 512), (4096, 4096)):
        for M in (1, 2, 5, 17, 33, 64):
            for P in (0, 31, 100, 2048, 16001, 131072, 2 ** 30):
                rows, tiles, ranges, fused, tall = plan(M, P, Hq, Hkv, fmt)
                pairs, pad = Hq // Hkv * M, 128 if tall else 32
                assert 1 <= rows <= pad and (tiles - 1) * rows < pairs <= tiles * rows
                assert 1 <= ranges <= min(32, -(-(P + M) // 32))
                assert ranges == 1 or Hkv * tiles * ranges <= 256
                assert not fused or (ranges > 1 and not tall and Hkv * tiles <= 4096)


@pytest.mark.parametrize("fmt", [B.KV8_INT8, B.KV8_E4M3])
@pytest.mark.parametrize("M,P,Hq,Hkv", [(64, 0, 512, 64), (64, 16001, 256, 32), (64, 16001, 512, 64), (64, 3000, 1024, 128), (24, 4000, 1024, 256), (64, 100, 192, 192)])
def test_more_row_tiles_than_compute_units_go_in_turns(M, P, Hq, Hkv, fmt):
    """LDS holds one workgroup per compute unit: tiles of 32 rows would take two to eight turns, tiles of 128 take one or two"""
    pairs = Hq // Hkv * M
    assert Hkv * -(-pairs // 32) > 256
    assert plan(M, P, Hq, Hkv, fmt)[4] == 1
