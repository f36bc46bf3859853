"""GPU: the product of 8-bit integers where only some of the capacity's rows are in use, at counts around the borders of its tiles."""
import pytest
import torch

import paper_2607_12121_b200 as fd
from test_gpu_matmul_int8 import _check, _operand, _run
import int8_ref as ref

pytestmark = pytest.mark.gpu

# K shared out to one CTA and to several, and CTA pairs
SHAPES = [(300, 384, 1536), (300, 384, 4608), (1001, 1152, 4608), (500, 1152, 4608), (300, 300, 250), (300, 4608, 640)]


@pytest.mark.parametrize("used", [0, 1, 127, 128, 129, 200, 255, 256, 257, 299])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_counts_at_tile_borders(m, n, k, used):
    _run(m, n, k, "bf16", used=used)
    _run(m, n, k, "f32", used=used, gelu=True, width=n + 4)


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_counts_from_replay_to_replay(m, n, k):
    """One graph, whose count goes up and down: tiles that rested work again, tiles that worked leave their outputs."""
    (a8, a_s), (w8, w_s) = _operand(m, k, 1), _operand(n, k, 2)
    out, used = torch.full((m, n), 5.0, device="cuda"), torch.tensor([m], dtype=torch.int32, device="cuda")
    want, err = ref.matmul(a8, a_s, w8, w_s)
    fd.fd_matmul_int8(a8, a_s, w8, w_s, out, rows_used=used)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fd.fd_matmul_int8(a8, a_s, w8, w_s, out, rows_used=used)
        fd.fd_matmul_int8(a8, a_s, w8, w_s, out, rows_used=used)
    for count in (m, 1, 0, 129, m - 1, 128, -4, m + 9):
        used.fill_(count)
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        count = max(0, min(m, count))
        _check(out[:count], want[:count], err[:count])
        assert bool((out[count:] == 5.0).all())


@pytest.mark.parametrize("used", [0, 5, 128, 300])
def test_waits_are_bounded_with_a_count(used):
    """Tiles behind the count wait for nothing; the others' waits run out."""
    m, n, k = 300, 384, 1536
    (a8, a_s), (w8, w_s) = _operand(m, k, 1), _operand(n, k, 2)
    out, status = torch.full((m, n), 5.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    count = torch.tensor([used], dtype=torch.int32, device="cuda")
    fd.fd_matmul_int8(a8, a_s, w8, w_s, out, rows_used=count, status_out=status, _call=fd.binding._call_matmul_int8_selftest)
    assert int(status) == fd.FD_ERR_TIMEOUT and bool((out[used:] == 5.0).all())
    fd.fd_matmul_int8(a8, a_s, w8, w_s, out, rows_used=count, status_out=status)
    assert int(status) == 0 and bool((out[used:] == 5.0).all())
    want, err = ref.matmul(a8, a_s, w8, w_s)
    _check(out[:used], want[:used], err[:used])
