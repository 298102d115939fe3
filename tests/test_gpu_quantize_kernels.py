"""q8_quantize_rows kernel by kernel (threads per row, vectors of 16 bytes per thread): every test asserts which kernel its sizes reach, so that a moved line cannot empty it."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2111_01264_amd as P
from tests.gpu_kernels import kernels_of
from tests.test_gpu_quantize_rows import TYPES, run

# rows, columns of two bytes: of four, half of them fill as many vectors
SIZES = {"64 2": [(700, 40), (5, 1023), (600, 1024)], "256 4": [(5, 1025), (3, 3072), (513, 3079), (600, 8192)], "256 8": [(600, 8193), (513, 16384)],
         "1024 8": [(512, 3080), (7, 8192), (33, 12000), (2, 16385), (600, 16391), (1, 65536)], "1024 0": [(2, 65537), (513, 65541)]}


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("kernel", list(SIZES))
def test_levels(kernel, kind):
    dt, code = TYPES[kind]
    for rows, cols in SIZES[kernel]:
        if kind == "fp32":
            cols = (cols + 1) // 2
        for pad in (0, 3):
            g = torch.Generator(device="cuda")
            g.manual_seed(rows + cols)
            x = (torch.randn(rows, cols + pad, generator=g, device="cuda") * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))).to(dt)
            if rows > 4:
                x[1] = 0.0
                x[2, cols - 1] = float("nan")
                x[3, 0] = float("-inf")
            scale, q = torch.empty(rows, device="cuda"), torch.empty(rows, cols, dtype=torch.int8, device="cuda")
            names = kernels_of(lambda stream: P.q8_quantize_rows(x, code, cols + pad, rows, cols, q, cols, scale, None, 0, stream))
            threads, vectors = kernel.split()
            assert len(names) == 1 and "quantize_rows_kernel" in names[0] and "Li%sELi%sE" % (threads, vectors) in names[0], (rows, cols, names)
            run(x, cols + pad, rows, cols, code, guard=pad)
            if rows * cols > 1 << 23:
                break
