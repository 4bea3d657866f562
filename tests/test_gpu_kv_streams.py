"""Steps on several streams and from several threads, each with a plan of its own, give what they give alone."""
import threading

import pytest
import torch

from tests.test_gpu_kv_attend import BF, FH, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(dev):
    yield


def cases():
    return [Case([(3000, 1), (70, 1)], 8, 2, 128, BF, seed=30), Case([(900, 200), (40, 40)], 8, 2, 64, FH, seed=31),
            Case([(5000, 3)], 8, 4, 128, BF, True, seed=32), Case([(1500, 60)], 4, 1, 256, BF, seed=33)]


def step(c, plan, stream, times=8):
    outs = []
    q = c.q.cuda()
    stream.wait_stream(torch.cuda.default_stream())
    with torch.cuda.stream(stream):
        for _ in range(times):
            outs.append(c.run(plan=plan, q=q))
    stream.synchronize()
    return outs


def test_streams_with_plans_of_their_own():
    cs = cases()
    want = [c.check() for c in cs]
    streams, plans, qs = [torch.cuda.Stream() for _ in cs], [c.plan() for c in cs], [c.q.cuda() for c in cs]
    torch.cuda.synchronize()
    got = [[] for _ in cs]
    for _ in range(8):  # enqueued in turn, so that they overlap
        for i, c in enumerate(cs):
            with torch.cuda.stream(streams[i]):
                got[i].append(c.run(plan=plans[i], q=qs[i]))
    torch.cuda.synchronize()
    for mine, (out, lse) in zip(got, want):
        assert all(torch.equal(o, out) and torch.equal(x, lse) for o, x in mine)


def test_threads():
    cs = cases()
    want = [c.check() for c in cs]
    plans, streams, got, errors = [c.plan() for c in cs], [torch.cuda.Stream() for _ in cs], [None] * len(cs), []

    def work(i):
        try:
            torch.cuda.set_device(0)
            got[i] = step(cs[i], plans[i], streams[i])
        except Exception as e:  # reported below, in the test's own thread
            errors.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(cs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    torch.cuda.synchronize()
    assert not errors and all(not t.is_alive() for t in threads)
    for mine, (out, lse) in zip(got, want):
        assert all(torch.equal(o, out) and torch.equal(x, lse) for o, x in mine)
