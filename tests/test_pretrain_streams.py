"""The worker's iteration and its callers' streams: it runs on a stream of its own where the chip is divided, or where it was made under another
stream than it is called under.  What the caller enqueued before (tokens, peers' buffers) comes first, and what the caller enqueues
afterwards (the next peers, a look at the loss) comes behind it, without any synchronisation of the device."""
import contextlib

import pytest
import torch

from paper_2502_11058_amd import pretrain as T


class _Stream:
    def __init__(self, name, log):
        self.name, self.log = name, log

    def wait_stream(self, other):
        self.log.append(f"{self.name} behind {other.name}")


class _Loss:
    def __init__(self, log):
        self.log = log

    def detach(self):
        return self

    def record_stream(self, s):
        self.log.append(f"loss used on {s.name}")


def test_the_order_of_an_iteration(monkeypatch):
    log = []
    caller, own = _Stream("caller", log), _Stream("own", log)
    current = [caller]

    @contextlib.contextmanager
    def under(s):
        current.append(s)
        yield
        current.pop()

    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[-1])
    monkeypatch.setattr(torch.cuda, "stream", under)
    worker = T.Pretraining.__new__(T.Pretraining)

    class Overlap:
        main_stream = own

        def begin(self, r, with_stats):
            log.append(f"begin on {current[-1].name}")

        def backward(self, loss):
            log.append(f"backward on {current[-1].name}")

        def end(self):
            log.append(f"end on {current[-1].name}")

    class Model:
        def loss(self, *args):
            log.append(f"forward on {current[-1].name}")
            return _Loss(log)

    worker.overlap, worker.model, worker.params, worker.table = Overlap(), Model(), {}, None
    worker.rep = type("Rep", (), {"dev": "cuda:0"})()
    worker.iteration(0, None, None)
    steps = ["begin on own", "forward on own", "backward on own", "end on own"]
    assert [x for x in log if x in steps] == steps
    assert log.index("own behind caller") < log.index("begin on own")
    assert log.index("caller behind own") > log.index("end on own")
    assert "loss used on caller" in log and current == [caller]


@pytest.mark.gpu
@pytest.mark.parametrize("side_cus", [0, 32])
def test_without_synchronisation_from_another_stream(side_cus):
    """Losses of iterations that follow each other without a wait, called under a stream of the test's, are those of iterations with the
    device synchronised between all steps.  Equal but for torch's products, which may sum in another order on other compute units: a unit
    of bf16 in the hidden states' sums, 2^-8 of the loss at most."""
    def run(stream, wait):
        worker = T.Pretraining(T.MODELS["small_llama"](), side_cus=side_cus)
        torch.cuda.synchronize()            # (made under the default stream)
        losses = []
        with torch.cuda.stream(stream):
            for r in range(6):
                tokens, targets = worker.batch(4, 128)
                worker.peers(r)
                if wait:
                    torch.cuda.synchronize()
                losses.append(worker.iteration(r, tokens, targets))
                if wait:
                    torch.cuda.synchronize()
            losses = torch.stack(losses).tolist()
        torch.cuda.synchronize()
        worker.close()
        return losses

    want = run(torch.cuda.current_stream(), True)
    got = run(torch.cuda.Stream(), False)
    assert all(abs(a - b) <= 2.0 ** -8 * a for a, b in zip(want, got)), (want, got)
