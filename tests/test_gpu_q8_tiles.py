"""q8_linear kernel by kernel: the streamed ones and every tile, on rows that start on 16-byte borders and on rows that do not.  Every test asserts which kernel its sizes reach, so
that a moved line cannot empty it.  Bounds are those of test_gpu_q8_linear."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2111_01264_amd as P
from tests.gpu_kernels import kernels_of
from tests.test_gpu_q8_linear import TYPES, check, gen, levels, run, wanted

# kernel: M, N, K that reach it on rows of their own length, padded to 16 bytes where `aligned`
SIZES = {
    "q8_stream_kernel 16 4 4": (9, 1000, 700), "q8_stream_kernel 16 4 8": (5, 500, 4100), "q8_stream_kernel 32 8 8": (500, 512, 300),
    "q8_tile_kernel 64 256 1": (1000, 1003, 200), "q8_tile_kernel 64 256 0": (1000, 1003, 200),
    "q8_tile_kernel 128 256 1": (2003, 2000, 100), "q8_tile_kernel 128 256 0": (2003, 2000, 100),
    "q8_tile_kernel 256 512 1": (3600, 3601, 6150),
}


def kernel_of(x, ldx, sx, w, ldw, sw, M, N, K, y, code):
    names = kernels_of(lambda stream: P.q8_linear(x, ldx, sx, w, ldw, sw, None, 0, M, N, K, y, code, y.stride(0), stream))
    assert len(names) == 1
    return names[0]


def is_kernel(mangled, kernel):
    name, *numbers = kernel.split()
    want = "".join("Li%sE" % v for v in numbers[:3]) if name == "q8_stream_kernel" else "Li%sELi%sELb%sE" % tuple(numbers)
    return name + "I" in mangled and want in mangled


class Product:
    """The operands of one product; `ldx`, `ldw`, `ldy` pitches, `off` the bytes in front of the first row."""

    def __init__(self, M, N, K, kind="fp32", ldx=None, ldw=None, ldy=None, off=0, seed=0):
        self.M, self.N, self.K, (self.dt, self.code) = M, N, K, TYPES[kind]
        self.ldx, self.ldw, self.ldy = ldx or K, ldw or K, ldy or N
        g = gen(seed + 7919 * M + 104729 * N + K)
        buf = [torch.empty(r * ld + off + 64, dtype=torch.int8, device="cuda") for r, ld in ((M, self.ldx), (N, self.ldw))]
        self.x, self.w = (b[off:off + r * ld].view(r, ld) for b, r, ld in zip(buf, (M, N), (self.ldx, self.ldw)))
        self.x[:, :K], self.w[:, :K] = levels(g, M, K), levels(g, N, K)
        self.sx, self.sw = torch.rand(M, generator=g, device="cuda") * 0.02, torch.rand(N, generator=g, device="cuda") * 1e-3
        self.b = torch.randn(N, generator=g, device="cuda") * 0.1
        self.y = torch.full((M + 1, self.ldy), 3.0, dtype=self.dt, device="cuda")
        torch.cuda.synchronize()

    def enqueue(self, stream=None, relu=0):
        P.q8_linear(self.x, self.ldx, self.sx, self.w, self.ldw, self.sw, self.b, relu, self.M, self.N, self.K, self.y, self.code, self.ldy, stream)

    def reach(self, kernel):
        names = kernels_of(self.enqueue)
        assert len(names) == 1 and is_kernel(names[0], kernel), (kernel, names)
        return self

    def check(self, relu=False):
        torch.cuda.synchronize()
        assert torch.all(self.y[self.M] == 3.0) and torch.all(self.y[:, self.N:] == 3.0)   # what lies behind stays as it was
        check(self.y[:self.M, :self.N], wanted(self.x, self.K, self.sx, self.w, self.sw, self.b, relu), self.dt)


def pitches(kernel, K, extra=0):
    """A pitch for K levels that reaches the aligned or the unaligned kernel."""
    if kernel.endswith(" 1"):
        return (K + 15) // 16 * 16 + 16 * extra
    return K + (K % 16 == 0) + extra * 16


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("kernel", list(SIZES))
def test_lengths_of_k(kernel, kind):
    M, N, K0 = SIZES[kernel]
    if "stream" in kernel:
        Ks = (K0, K0 + 1, K0 + 64)
    elif " 256 512 " in kernel:   # every kind of rest behind whole pairs of steps
        Ks = (K0, 6144, 6145, 6159, 6160, 6161, 6207, 6208, 6209, 6271, 6272, 6273)
    else:
        Ks = (K0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 191, 193, 256, 320, 384, 449, 513, 640)
    for K in Ks:
        ld = pitches(kernel, K)
        p = Product(M, N, K, kind, ld, ld).reach(kernel)
        for relu in (0, 1):
            p.enqueue(relu=relu)
            p.check(bool(relu))


@pytest.mark.parametrize("kernel", list(SIZES))
def test_pitches_and_alignments(kernel):
    M, N, K = SIZES[kernel]
    a, b, c = (pitches(kernel, K, e) for e in (0, 1, 7))
    for ldx, ldw, off, ldy, kind in ((a, b, 0, N + 3, "bf16"), (c, a, 16, N + 1, "fp32"), (b, c, 32, N + 5, "fp16"), (a, a, 48, N, "bf16")):
        p = Product(M, N, K, kind, ldx, ldw, ldy, off).reach(kernel)
        p.enqueue()
        p.check()
    if kernel.endswith(" 0"):
        for off in (1, 4, 8, 13):   # one side's rows on 16-byte borders, or both but for where they begin
            p = Product(M, N, K, "bf16", (K + 15) // 16 * 16, K + 1, N, 16 * (off == 4), seed=off).reach(kernel)
            p.enqueue()
            p.check()
            p = Product(M, N, K, "bf16", (K + 15) // 16 * 16, (K + 15) // 16 * 16 + 16, N, off).reach(kernel)
            p.enqueue()
            p.check()


@pytest.mark.parametrize("kernel", [k for k in SIZES if k != "q8_stream_kernel 16 4 4"])   # (takes a short k only)
def test_longest_sums_stay_exact(kernel):
    """K at its limit with all levels -128: the sum is 2^31 - 2^14, the largest there is."""
    K = P.Q8_LINEAR_MAX_K
    M, N, _ = SIZES[kernel]
    ld = pitches(kernel, K)
    x, w = (torch.full((r, ld), -128, dtype=torch.int8, device="cuda") for r in (M, N))
    sx, sw = torch.ones(M, device="cuda"), torch.ones(N, device="cuda")
    y = torch.zeros(M, N, device="cuda")
    assert is_kernel(kernel_of(x, ld, sx, w, ld, sw, M, N, K, y, P.DQN_TYPE_FP32), kernel)
    P.q8_linear(x, ld, sx, w, ld, sw, None, 0, M, N, K, y, P.DQN_TYPE_FP32, N, None)
    torch.cuda.synchronize()
    assert torch.all(y.double() == float(np.float32(16384 * K)))


@pytest.mark.parametrize("kernel", list(SIZES))
def test_scales_at_the_ends_and_nan(kernel):
    M, N, K = SIZES[kernel]
    ld = pitches(kernel, K)
    p = Product(M, N, K, "fp32", ld, ld).reach(kernel)
    p.b.zero_()
    p.sx[0], p.sx[1], p.sx[2], p.sx[M - 1] = 1e-30, 1e30, float("nan"), 2e36
    p.sw[:] = 1e-30
    p.sw[1], p.sw[2], p.sw[N - 1] = float("nan"), 0.0, 1e-38
    for relu in (0, 1):
        p.enqueue(relu=relu)
        torch.cuda.synchronize()
        y, want = p.y[:M, :N].double(), wanted(p.x, K, p.sx, p.w, p.sw, p.b, bool(relu))
        assert torch.equal(torch.isnan(y), torch.isnan(want))
        fine = torch.isfinite(want)
        assert torch.all((y - want).abs()[fine] <= want.abs()[fine] * 2.0 ** -23 + 2.0 ** -150)


@pytest.mark.parametrize("kernel", list(SIZES))
def test_replayed_graphs(kernel):
    M, N, K = SIZES[kernel]
    ld, g, stream = pitches(kernel, K), gen(8), torch.cuda.Stream()
    p = Product(M, N, K, "bf16", ld, ld).reach(kernel)
    p.enqueue(stream)
    p.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        p.enqueue(stream)
    for _ in range(3):
        p.x[:, :K] = levels(g, M, K)
        p.y[:M, :N] = 1.0
        torch.cuda.synchronize()
        graph.replay()
        p.check()


@pytest.mark.parametrize("kernel", [k for k in SIZES if "tile" in k])
def test_offsets_at_the_ends_of_32_bits(kernel):
    """The widest pitch that the aligned tiles take (a lane's place within a tile is a 32-bit offset), and the first that they leave to the others, whose rows lie as far apart."""
    M, N, K = SIZES[kernel]
    wide = (1 << 23) - 16 if kernel.endswith(" 1") else 1 << 23
    narrow = (K + 15) // 16 * 16
    for ldx, ldw in ((wide, narrow), (narrow, wide)):
        p = Product(M, N, K, "fp32", ldx, ldw).reach(kernel)
        p.enqueue()
        p.check()
        del p
        torch.cuda.empty_cache()


def test_more_tiles_than_the_chip_holds():
    """Ragged rows and columns of many tiles: every piece of y is written, by its own tile."""
    for M, N, K, pad in ((20000, 3001, 64, 0), (129, 60001, 80, 0), (60001, 129, 48, 1)):
        run(M, N, K, "fp16", pad=(pad, pad, 1))
