"""The decoder step's operators called by several threads of a program."""
import threading
import time

import pytest
import torch

from test_gpu_cache import amq, filled, tables  # noqa: F401

pytestmark = pytest.mark.gpu


def calls(amq, seed):
    """Each operator with inputs of its own."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    table, pages = tables(gen, 3, [3000, 17, 450], 16)
    cache = filled(amq, gen, pages, 16, 2, 64, 3)
    n = torch.tensor([3000, 17, 450], dtype=torch.int32, device="cuda")
    q = torch.randn((3, 2, 4, 64), device="cuda", generator=gen)
    logits, scores = torch.randn((12, 5000), device="cuda", generator=gen), -torch.rand((3, 4), device="cuda", generator=gen)
    parents = torch.randint(4, (3, 4), device="cuda", generator=gen, dtype=torch.int32)
    states = [torch.randn((3, 4, 200), device="cuda", generator=gen)]
    out = [torch.empty_like(states[0])]
    W = amq.pack(torch.randn((300, 2, 256), device="cuda", generator=gen)), torch.rand((300, 2), device="cuda", generator=gen)
    x = amq.pack(torch.randn((5, 2, 256), device="cuda", generator=gen)), torch.rand((5, 2), device="cuda", generator=gen)
    rows = [t[0, :3].reshape(3, 1, *t.shape[2:]).contiguous() for t in cache]
    return [lambda: amq.binary_gemm_act(*W, *x, 256, activation=amq.ACT_GELU), lambda: amq.cache_attention(q, cache, table, n, 0.1),
            lambda: amq.beam_select(logits, scores)[2], lambda: amq.beam_reorder(states, parents, out)[0],
            lambda: amq.cache_append(*rows, cache, table, n, 64)]


def test_threads_with_streams_of_their_own(amq):  # noqa: F811
    """Four threads, each with a stream and inputs of its own, answer what one thread alone does."""
    alone = [[f() for f in calls(amq, seed)[:4]] for seed in range(4)]
    torch.cuda.synchronize()
    failed = []

    def work(seed):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                mine = calls(amq, seed)[:4]
                for _ in range(50):
                    got = [f() for f in mine]
                torch.cuda.current_stream().synchronize()
                assert all(torch.equal(g, w) for g, w in zip(got, alone[seed]))
        except BaseException as e:
            failed.append(e)

    threads = [threading.Thread(target=work, args=(seed,)) for seed in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed


@pytest.mark.parametrize("which", range(5))
def test_a_full_queue_holds_up_the_thread_that_fills_it(amq, which):  # noqa: F811
    """Behind two seconds of GPU work, more launches than the device's queue takes: the thread that makes them waits, the others run on."""
    f = calls(amq, 9)[which]
    f()
    torch.cuda.synchronize()
    torch.cuda._sleep(4 * 10 ** 9)
    started = time.monotonic()
    filler = threading.Thread(target=lambda: [f() for _ in range(3000)])
    filler.start()
    longest, last = 0.0, started
    while filler.is_alive():
        time.sleep(0.001)
        now = time.monotonic()
        longest, last = max(longest, now - last), now
    filler.join()
    torch.cuda.synchronize()
    assert last - started > 1.0                             # (the queue was full)
    assert longest < 0.7
