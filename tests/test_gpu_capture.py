"""Calls that a captured stream refuses leave the capture as it was."""
import pytest

from paper_2608_14575_amd import hwr, routed

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def test_adamw_is_not_made_under_capture():
    s = torch.cuda.Stream()
    ops = routed.RoutedOps(stream=s.cuda_stream)
    p, g, m, v = (torch.ones(300, device="cuda") for _ in range(4))
    t = (hwr.hwr_adamw_tensor * 1)((300, p.data_ptr(), g.data_ptr(), None, m.data_ptr(), v.data_ptr(), None, None))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        p.add_(1)
        for make in (lambda: routed.AdamW(ops, [p], [g], lr=1e-3), lambda: routed.AdamW(ops, [p], [g], lr=1e-3, state={"m": [m], "v": [v]}),
                     lambda: hwr.hwr_adamw_init(ops.ctx, hwr.hwr_adamw_config(hwr.HWR_F32, 32, 1, t))):
            with pytest.raises(hwr.HwrError) as e:
                make()
            assert e.value.status == hwr.HWR_ERR_STATE
        p.mul_(2)
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
    assert (p == 22).all()                     # ((1 + 1) 2 + 1) 2 ...
    ops.close()
