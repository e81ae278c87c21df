"""GPU: the prompt operators together, as a program runs them: packed prompts through a decoder layer of W8A8 linears into a cache, then single
tokens of the batch through the same layer; and the cache that they leave read by tree_verify_attn."""
import numpy as np
import pytest
import torch

from oracle import reference as R
from paper_2505_22179_amd import binding as B
from paper_2505_22179_amd import inputs as I
from tests.test_gpu_prompt_attn import close
from tests.test_gpu_w8a8 import plain_codes, quantised

pytestmark = pytest.mark.gpu
DEV = "cuda"
dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
half = lambda *shape: torch.empty(*shape, dtype=torch.float16, device=DEV)
H, HQ, HKV, D, FFN, EPS, N_POS = 512, 8, 2, 128, 1024, 1e-5, 256


class Layer:
    def __init__(self, seed):
        rng = np.random.default_rng(seed)
        self.w, self.t, self.packed = {}, {}, {}
        for name, N, K in (("qkv", (HQ + 2 * HKV) * D, H), ("o", H, HQ * D), ("gate_up", 2 * FFN, H), ("down", H, FFN)):
            self.w[name] = np.clip(np.rint(rng.standard_normal((N, K)) * 30), -127, 127).astype(np.int8)
            self.t[name] = (rng.uniform(0.5, 1.5, N) / (30 * np.sqrt(K))).astype(np.float32)
            self.packed[name] = torch.empty(B.w8a8_packed_bytes(N, K), dtype=torch.uint8, device=DEV)
            B.w8a8_pack(dev(self.w[name]), self.packed[name], N, K)
        self.g1, self.g2 = I.make_gamma(seed, H), I.make_gamma(seed + 1, H)
        self.cos, self.sin = torch.empty(N_POS, D // 2, device=DEV), torch.empty(N_POS, D // 2, device=DEV)
        B.rope_table(self.cos, self.sin, 0, N_POS, D, 500000.0, B.ROPE_BY_TURNS, 8.0, 1.0, 4.0, 128.0)

    def run(self, h, pos, slot, q_start, k_start, k_len, k, v, most):
        """the layer, enqueued without a stop; copies of its input and every intermediate result"""
        M, Bn = h.shape[0], len(q_start) - 1
        ws = B.new_workspace(max(B.w8a8_workspace_bytes(M, *s) for s in (((HQ + 2 * HKV) * D, H), (H, HQ * D), (2 * FFN, H), (H, FFN))))
        aws = B.new_workspace(B.w4a16_prompt_attn_workspace_bytes(M, Bn, *most, HQ, HKV, D))
        t = {n: dev(x) for n, x in self.t.items()}
        lin = lambda name, x, pre, gamma, res, y, N, K: B.w8a8_linear(x, pre, gamma, EPS, self.packed[name], t[name], res, y, M, N, K, ws)
        qkv, q, a, gu = half(M, (HQ + 2 * HKV) * D), half(M, HQ, D), half(M, HQ, D), half(M, 2 * FFN)
        h0, k0, v0 = h.clone(), k.clone(), v.clone()
        lin("qkv", h, B.W8A8_RMS_NORM, dev(self.g1), None, qkv, (HQ + 2 * HKV) * D, H)
        B.rope_prompt(qkv, dev(pos), self.cos, self.sin, N_POS, D, False, dev(slot), k.shape[0], q, k, v, M, HQ, HKV, D)
        B.w4a16_prompt_attn(q, k, v, dev(q_start), dev(k_start), dev(k_len), a, Bn, M, k.shape[0], *most, HQ, HKV, D, D ** -0.5, aws)
        lin("o", a, B.W8A8_PLAIN, None, h, h, H, HQ * D)
        h1 = h.clone()
        lin("gate_up", h, B.W8A8_RMS_NORM, dev(self.g2), None, gu, 2 * FFN, H)
        lin("down", gu, B.W8A8_SILU_MUL, None, h, h, H, FFN)
        return {n: x.cpu().numpy() for n, x in dict(h0=h0, k0=k0, v0=v0, qkv=qkv, q=q, k=k, v=v, a=a, h1=h1, gu=gu, h2=h).items()}

    def check(self, g, pos, slot, q_start, k_start, k_len):
        """each step against the oracle on what the step before it left, so that one operator's roundings count at a time (a code that is a
        neighbour behind one rounding moves everything behind it)"""
        M = g["h0"].shape[0]

        def linear(name, x, pre, gamma, res, got):
            N, K = self.w[name].shape
            codes, s = quantised(x, pre, gamma, EPS, M, K)
            codes = plain_codes(codes, M, K)
            exact = R.w8a8_input(x, pre, gamma, EPS)   # the bounds of the quantisation's own tests
            near = (2.0 ** -11 + (2.0 ** -16 if pre else 0.0)) * np.abs(exact) + 2.0 ** -25
            assert (np.abs(codes * s[:, None].astype(np.float64) - exact) <= s[:, None] / 2 * (1 + 1e-12) + near).all(), name
            ref = R.w8a8_gemm(codes, s, self.w[name], self.t[name], res)
            size = np.abs(R.w8a8_gemm(codes, s, self.w[name], self.t[name])) + (0.0 if res is None else np.abs(res.astype(np.float64)))
            assert (np.abs(got.astype(np.float64) - ref) <= 2.0 ** -11 * np.abs(ref) + 2.0 ** -25 + 2.0 ** -22 * size).all(), name
        linear("qkv", g["h0"], B.W8A8_RMS_NORM, self.g1, None, g["qkv"])
        q, k, v = R.rope_prompt(g["qkv"], pos, self.cos.cpu().numpy(), self.sin.cpu().numpy(), D, False, slot, np.zeros((M, HQ, D)), g["k0"], g["v0"])
        np.testing.assert_array_equal(g["v"], v.astype(np.float16))
        most = 2 * np.abs(g["qkv"].astype(np.float64)).max()
        for name, ref in (("q", q), ("k", k)):
            assert (np.abs(g[name].astype(np.float64) - ref) <= 2.0 ** -11 * np.abs(ref) + 2.0 ** -25 + 2.0 ** -23 * most).all(), name
        ref, spread = R.prompt_attn(g["q"], g["k"], g["v"], q_start, k_start, k_len, D ** -0.5, np.zeros((M, HQ, D)))
        close(g["a"], ref, spread, int(k_len.max()), D ** 0.5 * np.abs(g["q"].astype(np.float64)).max() * np.abs(g["k"].astype(np.float64)).max())
        linear("o", g["a"].reshape(M, -1), B.W8A8_PLAIN, None, g["h0"], g["h1"])
        linear("gate_up", g["h1"], B.W8A8_RMS_NORM, self.g2, None, g["gu"])
        linear("down", g["gu"], B.W8A8_SILU_MUL, None, g["h1"], g["h2"])


@pytest.mark.parametrize("lens", [[1], [5, 40, 1, 100], [130]])
def test_prompts_then_single_tokens(lens):
    layer, rows = Layer(31), 200 * len(lens)
    room = rows // len(lens)                                  # cache rows of a sequence
    k_start = (np.arange(len(lens)) * room + 3).astype(np.int32)
    kd, vd = (torch.zeros(rows, HKV, D, dtype=torch.float16, device=DEV) for _ in range(2))
    for step in range(3):                                     # the prompts, then two tokens of each
        new = lens if step == 0 else [1] * len(lens)
        before = [0] * len(lens) if step == 0 else [n + step - 1 for n in lens]
        q_start = np.cumsum([0] + new).astype(np.int32)
        k_len = np.array([a + b for a, b in zip(new, before)], dtype=np.int32)
        pos = np.concatenate([np.arange(b, b + n) for n, b in zip(new, before)]).astype(np.int32)
        slot = np.concatenate([s + np.arange(b, b + n) for n, b, s in zip(new, before, k_start)]).astype(np.int32)
        print(f"layer: step {step} of {lens}", flush=True)
        got = layer.run(dev(I.make_hidden(70 + step, len(pos), H, 2)), pos, slot, q_start, k_start, k_len, kd, vd, (max(new), int(k_len.max())))
        layer.check(got, pos, slot, q_start, k_start, k_len)
    q = dev(got["q"])
    # one more reader of the cache: a verification pass over the first sequence, whose last row is the token just decoded
    P = int(k_len[0]) - 1
    out, one = half(1, HQ, D), half(1, HQ, D)
    ws = B.new_workspace(max(B.tree_verify_attn_workspace_bytes(1, P, HQ, HKV, D), B.w4a16_prompt_attn_workspace_bytes(1, 1, 1, P + 1, HQ, HKV, D)))
    cut = slice(int(k_start[0]), int(k_start[0]) + P + 1)
    B.tree_verify_attn(q[:1], kd[cut].contiguous(), vd[cut].contiguous(), torch.ones(1, 1, dtype=torch.uint8, device=DEV), out, 1, P, HQ, HKV, D, D ** -0.5, ws)
    B.w4a16_prompt_attn(q[:1], kd, vd, dev(np.array([0, 1], dtype=np.int32)), dev(k_start[:1]), dev(k_len[:1]), one, 1, 1, rows, 1, P + 1, HQ, HKV, D, D ** -0.5, ws)
    torch.cuda.synchronize()
    ref, spread = R.prompt_attn(got["q"][:1], got["k"], got["v"], [0, 1], k_start[:1], k_len[:1], D ** -0.5, np.zeros((1, HQ, D)))
    for reader in (one, out):
        close(reader.cpu().numpy(), ref, spread, P + 1, D ** 0.5 * np.abs(got["q"].astype(np.float64)).max() * np.abs(got["k"].astype(np.float64)).max())
