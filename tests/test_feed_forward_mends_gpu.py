"""Feed-forward operators: refusals and promises beside the formulas (aliases, capture, gradients, types of blocks, bits of a row in a batch)."""
import pytest
import torch

from paper_1202_3173_b200 import StrassenError, binding

from .test_feed_forward_gpu import BF16, E4M3, EPS, F16, F32, check_rows, gen, norm64, rows, strided, weights

pytestmark = pytest.mark.gpu


def sw():
    import paper_1202_3173_b200 as m
    return m


def test_a_workspace_in_the_weights_or_an_argument_is_refused():
    """More than 16 rows in e4m3, which need a workspace: in the laid-out weights it would overwrite them for this and every later call."""
    m, n, k = 20, 1024, 512
    q, s, z = weights(n, k, 128, False, BF16, 1)
    matrix = sw().W4Matrix(q, s)
    x, xs = rows(m, k, E4M3, 2)
    out = torch.empty(m, n, device="cuda", dtype=BF16)
    need = binding.strassen_w4_workspace_bytes(matrix.handle, m, binding.STRASSEN_E4M3, x.data_ptr(), k)
    assert 0 < need < matrix.nbytes
    before = matrix._packed.clone()
    for at in (matrix._packed, x, xs, out):
        with pytest.raises(StrassenError) as e:
            binding.strassen_w4_matmul(matrix.handle, m, binding.STRASSEN_E4M3, x.data_ptr(), k, xs.data_ptr(), binding.STRASSEN_BF16, out.data_ptr(), n, at.data_ptr(),
                                       need, torch.cuda.current_stream().cuda_stream)
        assert e.value.status == -4, str(e.value)
    torch.cuda.synchronize()
    assert torch.equal(matrix._packed, before)


def test_a_matrix_collected_during_a_capture_leaves_it_whole():
    q, s, z = weights(300, 512, 64, True, BF16, 3)
    x, _ = rows(4, 512, BF16, 4)
    kept, dropped = (sw().W4Matrix(q, s, z, group=64) for _ in range(2))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        want = dropped(x)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        del dropped
        got = kept(x)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_the_memory_of_a_matrix_is_not_reused_under_products_on_other_streams():
    n, k = 1024, 4096
    q, s, z = weights(n, k, 128, False, BF16, 5)
    x, _ = rows(4, k, BF16, 6)
    want = sw().W4Matrix(q, s)(x)
    torch.cuda.synchronize()
    matrix = sw().W4Matrix(q, s)
    nbytes, side = matrix.nbytes, torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100000000)             # some 50 ms
        got = matrix(x)
    del matrix
    others = [torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    del others
