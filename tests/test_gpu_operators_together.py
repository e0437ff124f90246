"""Products, decaying states and group norms called by several host threads at a time, on streams of their own and on one stream: the same bits."""
import threading

import pytest
import torch

from test_gpu_decay import BF, F, Case
from test_gpu_group_norm import inputs as norm_inputs
from test_gpu_linear import inputs as linear_inputs

pytestmark = pytest.mark.gpu


def works():
    """Calls of several launches each: split and cut products, cut sequences, large samples; each returns its results."""
    from paper_2609_31938_b200 import tokens as tk
    calls = []
    for dtype, m, n, k in ((F, 300, 500, 2048), (BF, 90, 1100, 4096), (F, 5, 900, 4096)):
        x, w, b, r = linear_inputs(m, n, k, dtype, seed=m)
        calls.append(lambda x=x, w=w, b=b, r=r: (tk.linear(x, w, b, activation="silu", residual=r),))
    for dtype in (BF, F):
        c = Case([900, 3, 1], 2, 1, 64, 64, dtype, seed=2)
        batch = tk.StreamBatch(c.starts, c.slot, 900)

        def attend(c=c, batch=batch):
            memory = tk.DecayMemory(c.states.clone())
            out = memory.attend(c.q, c.k, c.v, c.g, batch)
            assert memory.status() == 0
            return out, memory.states
        calls.append(attend)
    x, w, b, _, _ = norm_inputs(3, 40_000, 128, F, seed=3)
    calls.append(lambda: (tk.group_norm(x, 8, w, b, activation="gelu_tanh"),))
    return calls


@pytest.mark.parametrize("own_streams", [True, False])
def test_threads(own_streams):
    from paper_2609_31938_b200 import tokens as tk
    calls = works()
    want = [[t.clone() for t in f()] for f in calls]
    torch.cuda.synchronize()
    wrong, device = [], torch.cuda.current_device()

    def run(i):
        try:
            torch.cuda.set_device(device)
            stream = torch.cuda.Stream() if own_streams else torch.cuda.default_stream()
            with torch.cuda.stream(stream):
                for turn in range(12):
                    at = (turn + i) % len(calls)
                    got = calls[at]()
                    stream.synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(got, want[at])):
                        wrong.append((i, turn, at))
        except Exception as e:                                            # (an assertion in a thread would go unseen)
            wrong.append((i, repr(e)))

    threads = [threading.Thread(target=run, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(240)
    assert not wrong and tk.status() == 0, wrong


def test_graphs_of_one_pool_replayed_in_turn():
    calls = works()
    want = [[t.clone() for t in f()] for f in calls[:3] + calls[5:]]
    graphs, outs, pool = [], [], torch.cuda.graph_pool_handle()
    for f in calls[:3] + calls[5:]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], pool=pool):
            outs.append(f())
    for order in ((0, 1, 2, 3), (3, 1, 0, 2), (2, 2, 3, 3)):
        for i in order:
            for o in outs[i]:
                o.zero_()
            graphs[i].replay()
            assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i])), (order, i)
