"""Two captured graphs that share a workspace, replayed over outputs that hold something else: every output is written again by every replay."""
import pytest
import torch

from test_gpu_training_run import _buffers, _chain, _eager, _fill, _outputs

pytestmark = pytest.mark.gpu


def _poison(s):
    """All outputs; of dy_perm, whose rows behind the last kept one stay as they were, the rows that inv names."""
    named = s["inv"][s["inv"] >= 0].long()
    for t in _outputs(s):
        if t is s["back"]["dy_perm"]:
            t[named] = 7.0
        else:
            t.fill_(7)
    s["scan"][2].fill_(7.0)                                          # the states between the scan and its gradient


def test_replays_write_every_output():
    import paper_2605_11537_amd as moe
    a = _buffers(moe)
    b = _buffers(moe, ws=a["ws"])
    graphs = []
    for i, s in enumerate((a, b)):
        _fill(s, 60 + i)
        _eager(moe, s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _chain(moe, s)
        graphs.append(g)
    want = [_eager(moe, s) for s in (a, b)]
    for order in ((0, 1), (1, 0), (0, 0), (1, 1), (0, 1, 0)):
        a["ws"].random_(0, 256)
        for s in (a, b):
            _poison(s)
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        for i, s in enumerate((a, b)):
            same = [torch.equal(x, y) for x, y in zip(_outputs(s), want[i])]
            assert all(same) if i in order else not any(same), (order, i, same)
