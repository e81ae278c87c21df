"""GPU: W8A8 linears -- codes and scales exactly the oracle's, integer products exact, one rounding behind them."""
import numpy as np
import pytest
import torch

from oracle import reference as R
from paper_2505_22179_amd import binding as B
from paper_2505_22179_amd import inputs as I

pytestmark = pytest.mark.gpu
DEV = "cuda"
dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
SENTINEL = 1234.0


def quantised(x, pre, gamma, eps, M, K):
    codes = torch.full((B.w8a8_packed_bytes(M, K),), 0x5A, dtype=torch.uint8, device=DEV)
    scale = torch.full((M + 1,), 9.0, device=DEV)
    print(f"w8a8_quantize M {M} K {K} pre {pre}", flush=True)
    B.w8a8_quantize(dev(x), pre, dev(gamma), eps, codes, scale, M, K)
    torch.cuda.synchronize()
    scale = scale.cpu().numpy()
    assert scale[M] == 9.0
    return codes, scale[:M]


def plain_codes(codes, M, K):
    """codes [M, K] of the packed ones; padding of k is zero, rows beyond the last untouched"""
    full = np.ascontiguousarray(codes.cpu().numpy().view(np.int8).reshape((M + 15) // 16, -1, 4, 16, 16).transpose(0, 3, 1, 2, 4)).reshape((M + 15) // 16 * 16, -1)
    assert not full[:M, K:].any() and (full[M:] == 0x5A).all()
    return full[:M, :K]


@pytest.mark.parametrize("rows, K", [(1, 16), (16, 64), (17, 128), (8, 208), (40, 1040), (3, 65536)])
def test_pack_and_back(rows, K):
    w = np.random.default_rng(rows + K).integers(-128, 128, (rows, K)).astype(np.int8)
    packed = torch.full((B.w8a8_packed_bytes(rows, K),), 0x77, dtype=torch.uint8, device=DEV)
    B.w8a8_pack(dev(w), packed, rows, K)
    np.testing.assert_array_equal(packed.cpu().numpy().view(np.int8), R.w8a8_layout(w))
    back = torch.zeros(rows, K, dtype=torch.int8, device=DEV)
    B.w8a8_unpack(packed, back, rows, K)
    np.testing.assert_array_equal(back.cpu().numpy(), w)


@pytest.mark.parametrize("M, K", [(1, 16), (2, 48), (5, 4096), (17, 1040), (33, 8208), (3, 14336), (2, 28672), (2, 65536), (1, 32784)])
def test_codes_of_plain_rows_are_exact(M, K):
    rng = np.random.default_rng(M + K)
    x = I.make_hidden(M + K, M, K) if K > 64 else rng.standard_normal((M, K)).astype(np.float16)
    codes, scale = quantised(x, B.W8A8_PLAIN, None, 0.0, M, K)
    want_codes, want_scale = R.w8a8_quantise(x)
    np.testing.assert_array_equal(scale, want_scale)
    np.testing.assert_array_equal(plain_codes(codes, M, K), want_codes)


def test_every_magnitude_next_to_every_border():
    """for each row maximum of a spread, all fp16 numbers up to it: among them every one next to a half step, and the ties"""
    tops = np.array([0x0001, 0x0003, 0x007F, 0x00FE, 0x0400, 0x2C01, 0x3BF0, 0x3C00, 0x57F0, 0x5BF0, 0x6400, 0x7BFF], dtype=np.uint16)
    K = 65536
    x = np.zeros((len(tops), K), dtype=np.float16)
    for m, t in enumerate(tops):
        mags = np.arange(int(t) + 1, dtype=np.uint16)[-32768:]
        x[m, :len(mags)], x[m, len(mags):2 * len(mags)] = mags.view(np.float16), -mags.view(np.float16)
    codes, scale = quantised(x, B.W8A8_PLAIN, None, 0.0, len(tops), K)
    want_codes, want_scale = R.w8a8_quantise(x)
    np.testing.assert_array_equal(scale, want_scale)
    np.testing.assert_array_equal(plain_codes(codes, len(tops), K), want_codes)


def test_rows_of_zeros_and_rows_that_are_no_numbers():
    M, K, N = 6, 256, 24
    x = np.random.default_rng(1).standard_normal((M, K)).astype(np.float16)
    x[0], x[2, 7], x[3, 255], x[5, 0] = 0, np.nan, np.inf, -np.inf
    codes, scale = quantised(x, B.W8A8_PLAIN, None, 0.0, M, K)
    assert scale[0] == 0 and np.isnan(scale[[2, 3, 5]]).all() and not plain_codes(codes, M, K)[[0, 2, 3, 5]].any()
    lin = Linear(3, M, N, K, B.W8A8_PLAIN, True)
    lin.x = x
    y = lin.linear()
    assert np.isnan(y[[2, 3, 5]]).all()
    np.testing.assert_array_equal(y[0], lin.residual[0])
    np.testing.assert_array_equal(np.isfinite(y[[1, 4]]), True)


@pytest.mark.parametrize("pre", [B.W8A8_RMS_NORM, B.W8A8_SILU_MUL])
@pytest.mark.parametrize("M, K", [(1, 16), (3, 4096), (20, 1040), (2, 14336), (2, 28672), (1, 65536)])
def test_codes_behind_a_norm_or_a_gate(M, K, pre):
    x = np.random.default_rng(K).standard_normal((M, K * (2 if pre == B.W8A8_SILU_MUL else 1))).astype(np.float16) * np.float16(1.5)
    gamma, eps = (I.make_gamma(K, K), 1e-5) if pre == B.W8A8_RMS_NORM else (None, 0.0)
    codes, scale = quantised(x, pre, gamma, eps, M, K)
    exact = R.w8a8_input(x, pre, gamma, eps)
    # what is quantised is fp16: half a step of it, and fp32 arithmetic (a sum of squares: 2^-24 times the adds of a thread and of the joins, below 2^-16; else 2^-21)
    near = 2.0 ** -11 * np.abs(exact) + 2.0 ** -25 + 2.0 ** -16 * np.abs(exact)
    top = np.abs(exact).max(-1)
    assert (np.abs(scale * 127.0 - top) <= near.max(-1) + 2.0 ** -23 * top).all()
    s = scale.astype(np.float64)[:, None]
    assert (np.abs(plain_codes(codes, M, K) * s - exact) <= s / 2 * (1 + 1e-12) + near).all()


class Linear:
    def __init__(self, seed, M, N, K, pre=B.W8A8_PLAIN, residual=False, full=False):
        rng = np.random.default_rng(seed)
        self.M, self.N, self.K, self.pre, self.eps = M, N, K, pre, 1e-5
        self.x = (rng.standard_normal((M, K * (2 if pre == B.W8A8_SILU_MUL else 1))) * 1.5).astype(np.float16)
        self.gamma = I.make_gamma(seed, K) if pre == B.W8A8_RMS_NORM else None
        self.w = rng.integers(-128, 128, (N, K)).astype(np.int8) if not full else np.full((N, K), -128, dtype=np.int8)
        self.t = (rng.uniform(0.5, 1.5, N) / (40 * np.sqrt(K))).astype(np.float32)
        self.residual = rng.standard_normal((M, N)).astype(np.float16) if residual else None

    def packed(self):
        out = torch.empty(B.w8a8_packed_bytes(self.N, self.K), dtype=torch.uint8, device=DEV)
        B.w8a8_pack(dev(self.w), out, self.N, self.K)
        return out

    def workspace(self):
        ws = B.new_workspace(B.w8a8_workspace_bytes(self.M, self.N, self.K))
        ws[16384:].fill_(0x6B)
        return ws

    def linear(self, ws=None, y=None):
        M, N, K = self.M, self.N, self.K
        y = torch.full((M + 1, N), SENTINEL, dtype=torch.float16, device=DEV) if y is None else y
        print(f"w8a8_linear M {M} N {N} K {K} pre {self.pre}", flush=True)
        B.w8a8_linear(dev(self.x), self.pre, dev(self.gamma), self.eps, self.packed(), dev(self.t), dev(self.residual), y, M, N, K, self.workspace() if ws is None else ws)
        torch.cuda.synchronize()
        y = y.cpu().numpy()
        assert (y[M:] == SENTINEL).all()
        return y[:M]

    def gemm(self, codes, scale):
        M, N, K = self.M, self.N, self.K
        y = torch.full((M + 1, N), SENTINEL, dtype=torch.float16, device=DEV)
        print(f"w8a8_gemm M {M} N {N} K {K}", flush=True)
        B.w8a8_gemm(codes, dev(scale), self.packed(), dev(self.t), dev(self.residual), y, M, N, K, self.workspace())
        torch.cuda.synchronize()
        y = y.cpu().numpy()
        assert (y[M:] == SENTINEL).all()
        return y[:M]

    def check(self):
        codes, scale = quantised(self.x, self.pre, self.gamma, self.eps, self.M, self.K)
        y = self.gemm(codes, scale)
        plain = plain_codes(codes, self.M, self.K)
        ref = R.w8a8_gemm(plain, scale, self.w, self.t, self.residual)
        size = np.abs(R.w8a8_gemm(plain, scale, self.w, self.t)) + (0 if self.residual is None else np.abs(self.residual.astype(np.float64)))
        # half an fp16 step; fp32: the sum's conversion, two products, the residual: four roundings of 2^-24
        assert (np.abs(y.astype(np.float64) - ref) <= 2.0 ** -11 * np.abs(ref) + 2.0 ** -25 + 2.0 ** -22 * size).all()
        np.testing.assert_array_equal(self.linear().view(np.uint16), y.view(np.uint16))   # the same bits in one call


@pytest.mark.parametrize("M", [1, 2, 7, 16, 17, 31, 32, 33, 48, 64, 65, 100, 128, 129, 200, 257])
def test_linears_of_any_number_of_tokens(M):
    N, K = [(8, 16), (264, 1040), (1000, 336), (520, 2064), (4096, 512)][M % 5]
    Linear(M, M, N, K, M % 3, M % 2 == 1).check()


@pytest.mark.parametrize("M, N, K", [(1, 4096, 4096), (1, 28672, 4096), (4, 1024, 14336), (16, 16, 65536), (60, 1032, 8192), (64, 8, 128), (300, 4104, 1024), (520, 3000, 272), (1, 24, 28672),
                                     (777, 1024, 2048), (2000, 2056, 384), (130, 10248, 640)])
@pytest.mark.parametrize("residual", [False, True])
def test_linears_of_different_shapes(M, N, K, residual):
    Linear(M + N + K, M, N, K, B.W8A8_PLAIN, residual).check()


@pytest.mark.parametrize("M", [1, 40, 70])
def test_the_largest_sums_stay_exact(M):
    """every product at its largest: 65536 * 127 * 128 is just below 2^30"""
    lin = Linear(5, M, 16, 65536, full=True)
    lin.x = np.where(np.arange(65536) % 65536 < 65536, 3.0, 0).astype(np.float16)[None].repeat(M, 0)
    lin.t[:] = 2.0 ** -30
    lin.check()


def test_residual_in_place():
    for M in (3, 90):
        lin = Linear(6, M, 512, 512, B.W8A8_PLAIN, True)
        want = lin.linear()
        y = torch.full((M + 1, 512), SENTINEL, dtype=torch.float16, device=DEV)
        y[:M] = dev(lin.residual)
        B.w8a8_linear(dev(lin.x), lin.pre, None, 0.0, lin.packed(), dev(lin.t), y, y, M, 512, 512, lin.workspace())
        np.testing.assert_array_equal(y[:M].cpu().numpy(), want)


def test_norm_and_gate_are_those_of_the_rest_of_the_library():
    """rms_norm, then the plain linear, against the normed one: the sums of squares are joined in another order, so a few fp16 numbers may be neighbours"""
    M, N, K = 9, 256, 4096
    lin = Linear(7, M, N, K, B.W8A8_RMS_NORM)
    y = lin.linear().astype(np.float64)
    h = torch.empty(M, K, dtype=torch.float16, device=DEV)
    B.rms_norm(dev(lin.x), dev(lin.gamma), h, M, K, lin.eps)
    two = Linear(7, M, N, K)
    two.w, two.t, two.x = lin.w, lin.t, h.cpu().numpy()
    other = two.linear().astype(np.float64)
    assert np.linalg.norm(y - other) <= 2.0 ** -10 * np.linalg.norm(other)


@pytest.mark.parametrize("M", [1, 60, 300])
def test_graph_replays_on_a_shared_workspace(M):
    a, b = Linear(8, M, 1024, 2048, B.W8A8_RMS_NORM, True), Linear(9, M, 520, 4096, B.W8A8_SILU_MUL)
    want = [a.linear(), b.linear()]
    ws = B.new_workspace(max(B.w8a8_workspace_bytes(M, l.N, l.K) for l in (a, b)))
    held = [(dev(l.x), dev(l.gamma), l.packed(), dev(l.t), dev(l.residual), torch.empty(M, l.N, dtype=torch.float16, device=DEV), l) for l in (a, b)]

    def call(x, gamma, packed, t, residual, y, l):
        B.w8a8_linear(x, l.pre, gamma, l.eps, packed, t, residual, y, M, l.N, l.K, ws)
    for h in held:
        call(*h)
    torch.cuda.synchronize()
    graphs = []
    for h in held:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(*h)
        graphs.append(g)
    for _ in range(3):
        for h in held:
            h[5].zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for h, w in zip(held, want):
            np.testing.assert_array_equal(h[5].cpu().numpy(), w)
        call(*held[0])


@pytest.mark.parametrize("M, N, K", [(1, 1024, 14336), (20, 4096, 4096), (60, 8192, 2048), (64, 128, 8208), (65, 520, 2064), (100, 264, 256), (128, 520, 2048), (300, 1000, 400), (1000, 2000, 16),
                                     (777, 4096, 2000), (2048, 8192, 1040)])
def test_operands_that_arrive_late(M, N, K):
    """caches emptied before every call: a product that does not wait for its operands uses what was there before"""
    case = Linear(M + N, M, N, K)
    codes, scale = quantised(case.x, case.pre, None, 0.0, M, K)
    scale, packed, t, ws = dev(scale), case.packed(), dev(case.t), case.workspace()
    other = torch.zeros(1 << 28, dtype=torch.int32, device=DEV)   # 1 GiB
    first = None
    for call in range(12):
        y = torch.full((M, N), SENTINEL, dtype=torch.float16, device=DEV)
        if call:
            other.add_(1)
        B.w8a8_gemm(codes, scale, packed, t, None, y, M, N, K, ws)
        if first is None:
            first = y
        assert torch.equal(y, first), call


@pytest.mark.parametrize("pre", [B.W8A8_PLAIN, B.W8A8_RMS_NORM, B.W8A8_SILU_MUL])
def test_rows_are_quantised_alike_however_many_they_are(pre):
    M, K = 530, 9216
    x = np.random.default_rng(3).standard_normal((M, K * (2 if pre == B.W8A8_SILU_MUL else 1))).astype(np.float16)
    gamma = I.make_gamma(4, K) if pre == B.W8A8_RMS_NORM else None
    codes, scale = quantised(x, pre, gamma, 1e-5, M, K)
    few, few_scale = quantised(x[:32], pre, gamma, 1e-5, 32, K)
    plain, some = plain_codes(codes, M, K), plain_codes(few, 32, K)
    if pre != B.W8A8_RMS_NORM:   # its sum of squares is taken in another order
        np.testing.assert_array_equal(plain[:32], some)
        np.testing.assert_array_equal(scale[:32], few_scale)
    exact = R.w8a8_input(x, pre, gamma, 1e-5)   # bounds as in the other tests of codes
    near = (2.0 ** -11 + (2.0 ** -16 if pre else 0.0)) * np.abs(exact) + 2.0 ** -25
    assert (np.abs(plain * scale[:, None].astype(np.float64) - exact) <= scale[:, None].astype(np.float64) / 2 * (1 + 1e-12) + near).all()


@pytest.mark.parametrize("M, K, pre", [(1, 512, B.W8A8_PLAIN), (1, 256, B.W8A8_SILU_MUL), (3, 512, B.W8A8_RMS_NORM), (70, 512, B.W8A8_PLAIN)])
def test_input_in_place(M, K, pre):
    lin = Linear(M + 5, M, 512, K, pre)
    want = lin.linear()
    buffer = torch.full((M + 1, 512), SENTINEL, dtype=torch.float16, device=DEV)
    buffer[:M] = dev(lin.x)
    B.w8a8_linear(buffer, pre, dev(lin.gamma), lin.eps, lin.packed(), dev(lin.t), None, buffer, M, 512, K, lin.workspace())
    torch.cuda.synchronize()
    np.testing.assert_array_equal(buffer[:M].cpu().numpy().view(np.uint16), want.view(np.uint16))


@pytest.mark.parametrize("M, N, K", [(1900, 8072, 1168), (25, 6152, 1040), (60, 6152, 528)])
def test_linears_whose_tiles_end_outside(M, N, K):
    """tiles of 256 x 256, and two tiles of channels to a wavefront"""
    Linear(M, M, N, K, B.W8A8_RMS_NORM, True).check()
