"""Host-only checks of w4a16_prompt_attn: the scales that it takes."""
import ctypes

from paper_2505_22179_amd import binding as B
from tests.test_kv8_host import A, EINVAL, EUNSUP, EWS, refusals
from tests.test_prompt_host import caller


def test_prompt_attn_refuses_scales_whose_scores_leave_fp32():
    call = caller(B.load(), "w4a16_prompt_attn", q=A, k=A, v=A, q_start=A, k_start=A, k_len=A, out=A, batch=3, rows=100, k_rows=1000, max_q=50, max_k=700,
                  Hq=8, Hkv=2, D=128, scale=ctypes.c_float(0.1), ws=A, nbytes=0)
    f = ctypes.c_float
    refusals(call, {EUNSUP: [dict(scale=f(s)) for s in (1.0001 * 2.0 ** 60, 2.0 ** 61, 3e38)], EINVAL: [dict(scale=f(s)) for s in (0.0, -1e-30)],
                    EWS: [dict(scale=f(s)) for s in (2.0 ** 60, 1.0, 1e-38)]})
