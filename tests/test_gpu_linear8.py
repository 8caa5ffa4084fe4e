"""Linear layers in 8-bit integers against the plain 64-bit form."""
import pytest
import torch

import paper_2501_09253_amd as ps
import prompt_oracle as po
from test_gpu_prompt_attention import DT, make
from test_gpu_kv8 import CODE

pytestmark = pytest.mark.gpu


def check(got, x, w, b, res):
    """Whole numbers are summed exactly; the sum as fp32, two scales and their two products: five roundings of the product; two
    additions of what stands beside it; one rounding of the result."""
    qx, sx = po.steps(x)
    qw, sw = po.steps(w.t().contiguous())
    main = (qx @ qw.t()) * (sx * sw.t())
    beside = [t.double() for t in (b, res) if t is not None]
    want = main + sum(beside)
    size = main.abs() + sum(t.abs() for t in beside)
    tol = 5 * po.U * main.abs() + 2 * po.U * size + po.HALF[x.dtype] * want.abs() + 1e-37
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    err = (got - want).abs()
    assert torch.all((err <= tol) | torch.isnan(want)), (err / tol).nan_to_num().max()


SHAPES = [(1, 64, 64), (1, 1, 1), (3, 77, 5), (12, 256, 512), (16, 4100, 130), (17, 128, 255), (33, 640, 1280), (64, 1000, 77), (130, 320, 264),
          (257, 129, 1000), (300, 2048, 640), (128, 128, 128), (129, 8200, 40), (700, 1536, 768)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K,N", SHAPES)
def test_against_64_bits(rows, K, N, dtype):
    x = make(1, (rows, K), DT[dtype]) * torch.logspace(-3, 3, rows)[:, None].to(DT[dtype])
    w, b, res = make(2, (K, N), DT[dtype], K ** -0.5), make(3, (N,), DT[dtype]), make(4, (rows, N), DT[dtype])
    for bias in (b, None):
        layer = ps.Linear8(w.cuda(), None if bias is None else bias.cuda(), CODE[dtype])
        for r in (res, None):
            check(layer.forward(x.cuda(), res=None if r is None else r.cuda()), x, w, bias, r)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [5, 200])
def test_rows_apart_and_in_place(rows, dtype):
    K, N = 96, 160
    wide, w, b = make(1, (rows, K + 24), DT[dtype]), make(2, (K, N), DT[dtype]), make(3, (N,), DT[dtype])
    layer = ps.Linear8(w.cuda(), b.cuda(), CODE[dtype])
    for off in (0, 8, 3):                                               # 3: rows off the 16-byte grid
        x = wide.cuda()[:, off:off + K]
        check(layer.forward(x), x.cpu(), w, b, None)
    y = make(4, (rows, N), DT[dtype])
    dev = y.cuda()
    layer.forward(x, res=dev, y=dev)
    check(dev, x.cpu(), w, b, y)
    odd = ps.Linear8(w[:, :77].contiguous().cuda(), None, CODE[dtype])
    buf = torch.zeros(rows * 77 + 1, dtype=DT[dtype], device="cuda")
    odd.forward(x, y=buf[1:].view(rows, 77))                            # an output off the 16-byte grid
    check(buf[1:].view(rows, 77), x.cpu(), w[:, :77], None, None)
    assert buf[0] == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_zeros_extremes_and_what_is_not_finite(dtype):
    x, w = make(1, (40, 64), DT[dtype]), make(2, (64, 48), DT[dtype])
    x[0], w[:, 3] = 0, 0
    x[1] *= 1e-30
    x[2, 5], x[3, 5], w[7, 9] = float("inf"), float("nan"), float("-inf")
    layer = ps.Linear8(w.cuda(), None, CODE[dtype])
    check(layer.forward(x.cuda()), x, w, None, None)


def test_the_largest_sums_are_exact():
    """All numbers +-127 at the largest K: sums of 2.1e9 in 32 bits."""
    K = 131072
    x = torch.ones((2, K), dtype=torch.float32)
    x[1] = -1
    w = torch.ones((K, 3), dtype=torch.float32)
    w[:, 1] = -1
    w[0, 2] = 0.5
    layer = ps.Linear8(w.cuda(), None, ps.F32)
    check(layer.forward(x.cuda()), x, w, None, None)


def test_graph_streams_and_workspace():
    x, w, res = make(1, (150, 320), torch.bfloat16).cuda(), make(2, (320, 192), torch.bfloat16).cuda(), make(3, (150, 192), torch.bfloat16).cuda()
    layer = ps.Linear8(w, None, ps.BF16)
    ws = torch.empty(layer.workspace_bytes(150), dtype=torch.uint8, device="cuda")
    y = torch.empty_like(res)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = layer.forward(x, res=res, workspace=ws)
    side.synchronize()
    assert torch.equal(layer.forward(x, res=res), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(x, res=res, y=y, workspace=ws)
    for i in range(3):
        x.copy_(make(20 + i, (150, 320), torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, layer.forward(x, res=res))
