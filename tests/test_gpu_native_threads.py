"""The calls of the operators beside the filter leave Python's lock while the library works: a launch waits where its stream's queue is full,
and the other threads of the program go on."""
import threading
import time

import pytest
import torch

from paper_2609_21102_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("call", ["adamw_step", "grad_norm", "mx4_quantize", "mx4_dequantize", "mx4_gemm"])
def test_other_threads_run_while_a_launch_waits(call):
    """A stream that is busy for a good second takes some thousand launches; the next one waits. A thread that does nothing but wake up
    each millisecond meanwhile is never kept away for half as long as that."""
    ctx = binding.Context(0)
    t = [torch.ones(64, device="cuda") for _ in range(4)]
    group, step = binding.AdamWGroup(t[:1], t[1:2], t[2:3]), torch.zeros(1, dtype=torch.int64, device="cuda")
    out = torch.zeros(2, device="cuda")
    q = ctx.defl_mx4_quantize(torch.ones(1, 4, 64, device="cuda"))
    run = {"adamw_step": lambda: ctx.defl_adamw_step(group, t[3:], 1e-3, 1), "grad_norm": lambda: ctx.defl_grad_norm(t, out=out, step=step),
           "mx4_quantize": lambda: ctx.defl_mx4_quantize(t[0].view(1, 1, 64)), "mx4_dequantize": lambda: ctx.defl_mx4_dequantize(q),
           "mx4_gemm": lambda: ctx.defl_mx4_gemm(q, q)}[call]
    run()
    torch.cuda.synchronize()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    torch.cuda._sleep(10 ** 8)
    end.record()
    end.synchronize()
    cycles = int(1200.0 / start.elapsed_time(end) * 10 ** 8)
    worst, done = [0.0], threading.Event()

    def tick():
        last = time.perf_counter()
        while not done.is_set():
            time.sleep(0.001)
            now = time.perf_counter()
            worst[0] = max(worst[0], now - last)
            last = now

    ticker = threading.Thread(target=tick)
    ticker.start()
    began = time.perf_counter()
    torch.cuda._sleep(cycles)
    while not torch.cuda.current_stream().query() and time.perf_counter() - began < 10:
        run()
    took = time.perf_counter() - began
    done.set()
    ticker.join()
    torch.cuda.synchronize()
    ctx.close()
    # (the stream's time goes with the clock, which the first kernel may have met at another step; a thread is off its core for 0.1 s at most)
    assert took > 0.6
    assert worst[0] < 0.5 * took, (worst, took)


def test_one_context_on_two_threads_and_streams():
    """Calls on one context take turns, each on its own thread's stream: results are those of a thread alone."""
    ctx = binding.Context(0)
    xs = [torch.randn(1, 200 + 90 * i, 480, device="cuda") for i in range(2)]
    call = lambda x: ctx.defl_mx4_gemm(ctx.defl_mx4_quantize(x, "nvfp4"), ctx.defl_mx4_quantize(x, "nvfp4"))  # noqa: E731
    want = [call(x) for x in xs]
    torch.cuda.synchronize()
    same, errors = [None, None], []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                outs = [call(xs[i]) for _ in range(100)]
                torch.cuda.current_stream().synchronize()
                same[i] = all(torch.equal(o, want[i]) for o in outs)
        except Exception as e:
            errors.append(repr(e))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    assert same == [True, True]
    ctx.close()
