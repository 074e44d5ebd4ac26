"""GPU parity of MXFP8 x MXFP4 products with K in several runs, fp16 output, on every tile that takes them: fp32 partial results and the launch that adds them up."""
import pytest
import torch

from oracle import mxfp8 as M8
from paper_2601_07475_amd import binding as B
from paper_2601_07475_amd import workloads as wk

from test_gpu_mx8 import assert_product, output, packed_weights
from test_gpu_parity import dev, say

pytestmark = pytest.mark.gpu

# M, N, K, S, rows and columns of the tile; K off its unit of 128
SHAPES = [(140, 56, 1696, 0, 64, 128), (194, 1831, 19360, 0, 64, 256), (1379, 258, 10528, 96, 128, 128), (791, 2433, 6816, 0, 128, 256),
          (1346, 1427, 10080, 0, 192, 256),
          # a prompt into a down projection, whose plan named a tile that there is no kernel of
          (1153, 3584, 18976, 0, 192, 256)]


@pytest.mark.parametrize("M,N,K,S,rows,cols", SHAPES)
def test_runs_of_k(M, N, K, S, rows, cols):
    kernel, tile_rows, tile_cols, runs = B.arcq_mx8_gemm_route(M, N, K, S, torch.float16, True)
    say(f"mx8_gemm M={M} N={N} K={K} S={S} on {tile_rows} x {tile_cols}, {runs} runs")
    assert (kernel, tile_rows, tile_cols) == (B.ROUTE_TILES, rows, cols) and runs > 1
    need = B.arcq_mx8_gemm_workspace_size(M, N, K)
    assert need >= runs * M * N * 4
    ac, asc = M8.quantize_act(wk.activations(wk.Workload("t", M, K, N, 0, max(1, K // 100), "loguniform20_100", 0.02, M)))
    wc, wsc = packed_weights(N, K, S, M + 1)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    raw, y = output(M, N, torch.float16, 1)
    B.arcq_mx8_gemm(dev(ac), dev(asc), dev(wc), dev(wsc), y=y, workspace=ws)
    assert_product(y, *M8.gemm(ac, asc, wc, wsc), K)
    y.fill_(12345.0)
    assert bool((raw == 12345.0).all())
