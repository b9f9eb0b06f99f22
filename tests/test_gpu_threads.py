"""The calls of the argument extension from several host threads."""
import threading
import time

import pytest
import torch

from tests.test_gpu_window import _gen, _i32, make, queries

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("what", ["rotate", "append", "decode", "chunk"])
def test_other_threads_run_while_a_call_waits_for_the_queue(what):
    """A stream is kept busy for about a second and more calls are made than the device's queue holds: the caller waits, the
    other Python thread does not."""
    from paper_2609_33184_b200 import binding as ssb
    g = _gen(0)
    cache = make(ssb, 16, 1, 1, 64, 16, 64, 1)
    ctx = ssb.Context(1, 1, 1, 64, 1, 1, 64, max_chunks=2)
    rope = ssb.Rope([1.0 / (i + 1) for i in range(32)])
    Q, K, V = (queries(g, 1, 1, 1, 64) for _ in range(3))
    O, n = torch.empty_like(Q), _i32([9])

    def call():
        if what == "rotate":
            ctx.ss_rope_rotate(rope, Q, None, O, None)
        elif what == "append":
            ctx.ss_kv_append(cache, K, V, rope, None, Q, O, n)
        elif what == "decode":
            ctx.ss_decode_window(Q, 0.125, cache, 5, 0, n, O)
        else:
            ctx.ss_verify_chunk_window(cache, 5, 0, n)

    if what == "chunk":
        ctx.ss_verify_begin(Q, 0.125)
    call()
    torch.cuda.synchronize()
    stop, gaps = threading.Event(), [0.0]

    def tick():
        last = time.perf_counter()
        while not stop.is_set():
            time.sleep(0.002)
            now = time.perf_counter()
            gaps[0] = max(gaps[0], now - last)
            last = now

    t = threading.Thread(target=tick)
    t.start()
    began = time.perf_counter()
    torch.cuda._sleep(2_000_000_000)
    for _ in range(6000):
        call()
    took = time.perf_counter() - began
    stop.set()
    t.join()
    torch.cuda.synchronize()
    if what == "chunk":
        ctx.ss_verify_abort()
    assert ctx.ss_poll_status() == (0, 0)
    ctx.close()
    assert took > 0.5, "the queue took all calls: nothing was waited for"
    assert gaps[0] < took / 2, (gaps[0], took)                # (as long as the wait, where it stands still)


def test_threads_with_a_context_each():
    """Steps and rounds of four threads at once, a context and a stream each: the bits of one after the other."""
    from paper_2609_33184_b200 import binding as ssb
    jobs = []
    for i in range(4):
        g, bits, T = _gen(i), 16 if i % 2 else 8, 1 + i
        cache = make(ssb, bits, 3, 2, 64, 16, 640, i)
        jobs.append((bits, cache, ssb.Context(3, 4, 2, 64, T, T, 640), torch.cuda.Stream(), queries(g, 3, 4, T, 64), queries(g, 3, 2, T, 64),
                     queries(g, 3, 2, T, 64), _i32([600 - i, 5, 200]), ssb.Rope([0.5 ** j for j in range(32)])))

    def run(job, out):
        bits, cache, ctx, stream, Q, K, V, n, rope = job
        append = ctx.ss_kv8_append if bits == 8 else ctx.ss_kv_append
        decode = ctx.ss_decode8_window if bits == 8 else ctx.ss_decode_window
        chunk = ctx.ss_verify_chunk8_window if bits == 8 else ctx.ss_verify_chunk_window
        with torch.cuda.stream(stream):
            for _ in range(50):
                Qr, O, O2, LSE = torch.empty_like(Q), torch.empty_like(Q), torch.empty_like(Q), torch.empty(Q.shape[:3], device=DEV)
                append(cache, K, V, rope, None, Q, Qr, n)
                decode(Qr, 0.125, cache, 90, 3, n, O, LSE)
                ctx.ss_verify_begin(Qr, 0.125)
                chunk(cache, 90, 3, n)
                ctx.ss_verify_local(K, V)
                ctx.ss_verify_finalize(O2, None)
                out.append((O, LSE, O2))
            stream.synchronize()
        assert ctx.ss_poll_status(stream) == (0, 0)

    torch.cuda.synchronize()
    alone, at_once = [[] for _ in jobs], [[] for _ in jobs]
    for job, out in zip(jobs, alone):
        run(job, out)
    threads = [threading.Thread(target=run, args=x) for x in zip(jobs, at_once)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for job, x, y in zip(jobs, alone, at_once):
        assert len(x) == len(y) == 50
        for a, b in zip(x, y):
            for u, v in zip(a, b):
                assert torch.equal(u, v)
        job[2].close()
