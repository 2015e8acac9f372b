"""Several dropouts of one captured step: an offset each, and one counter in device memory that they share."""

import numpy as np
import pytest

from oracle.dropout import dropout_keep

pytestmark = pytest.mark.gpu


def _case(msg):
    print(f"\n[gpu case] {msg}", flush=True)


def test_offset_and_counter_add_up():
    import torch
    import paper_2605_22791_amd as g2
    x = torch.ones(1001, device="cuda")
    for offset, count in ((0, 0), (3, 5), (1 << 40, (1 << 24) + 1), ((1 << 64) - 1, 2), (-5, 3), (7, -8)):
        _case(f"offset {offset} and {count}")
        more = torch.tensor([count], device="cuda")
        want = dropout_keep(1001, 0.5, 11, offset + count)
        y = g2.gdr2_dropout_fwd(x, 0.5, 11, offset=offset, more=more)
        dx = g2.gdr2_dropout_bwd(x, 0.5, 11, offset=offset, more=more)
        assert np.array_equal((y != 0).cpu().numpy(), want) and np.array_equal((dx != 0).cpu().numpy(), want)


def test_two_dropouts_of_a_replayed_step_drop_different_elements():
    import torch
    import paper_2605_22791_amd as g2
    _case("two dropouts, one counter, replayed")
    n = 3001
    x, step = torch.ones(n, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")

    def run():
        a = g2.gdr2_dropout_fwd(x, 0.4, 6, offset=0, more=step)
        b = g2.gdr2_dropout_fwd(x, 0.4, 6, offset=1, more=step)
        return a, b, g2.gdr2_dropout_bwd(x, 0.4, 6, offset=1, more=step)

    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, b, db = run()
        step += 2
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        first, second = (dropout_keep(n, 0.4, 6, 2 * k + j) for j in (0, 1))
        assert np.array_equal((a != 0).cpu().numpy(), first) and not np.array_equal(first, second)
        assert np.array_equal((b != 0).cpu().numpy(), second) and np.array_equal((db != 0).cpu().numpy(), second)
        torch.zeros(1000, device="cuda").sum().item()  # eager work between the replays


def test_refusals():
    import torch
    import paper_2605_22791_amd as g2
    _case("refusals")
    x, one = torch.zeros(8, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    for more, offset in ((one, one), (one.cpu(), 0), (one.float(), 0), (torch.zeros(2, dtype=torch.int64, device="cuda"), 0)):
        for call in (g2.gdr2_dropout_fwd, g2.gdr2_dropout_bwd):
            with pytest.raises(ValueError):
                call(x, 0.1, 0, offset=offset, more=more)
