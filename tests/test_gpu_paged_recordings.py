"""GPU tests of attention calls in recorded graphs: the counters that save a launch are of a recording, not of each of its calls."""
import pytest
import torch

from test_gpu_paged import DEV, dev, make, paged  # noqa: F401  (paged: fixture)

pytestmark = pytest.mark.gpu


def call_of(paged, seed=1):
    gen = torch.Generator().manual_seed(seed)
    c, _, table = make(paged, gen, [3000, 2000], 64, 8, 4, 128, "fp8", "bf16", "f32")
    q = dev(torch.randn((2, 32, 128), generator=gen).to(torch.bfloat16))
    idx = dev(torch.randint(0, 2000, (2, 8, 700), generator=gen).int())
    table, lens = dev(table), torch.tensor([3000, 2000], dtype=torch.int32, device=DEV)
    return c, lambda: (c.attn(q, table, lens), c.gather_attn(q, idx, table, lens))


def test_calls_of_a_recording_share_their_counters(paged):
    c, step = call_of(paged)
    want = step()
    torch.cuda.synchronize()
    left = len(c._scratch.spare)
    assert left > 2
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            res = [step() for _ in range(40)]  # as many layers
        graphs.append((graph, res))
    assert len(c._scratch.spare) == left - 2
    for i in range(4):
        for graph, res in graphs:
            for r in res:
                for t in r:
                    t.zero_()
            graph.replay()
            again = step()
            torch.cuda.synchronize()
            for r in res + [again]:
                for a, b in zip(r, want):
                    assert torch.equal(a, b), i


def test_streams_of_one_recording_have_counters_of_their_own(paged):
    c, step = call_of(paged)
    want = step()
    torch.cuda.synchronize()
    left = len(c._scratch.spare)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream(device=DEV)
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        with torch.cuda.stream(side):
            b = [step() for _ in range(4)]
        a = [step() for _ in range(4)]
        main.wait_stream(side)
    assert len(c._scratch.spare) == left - 2
    for _ in range(4):
        for r in a + b:
            for t in r:
                t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for r in a + b:
            for x, y in zip(r, want):
                assert torch.equal(x, y)


def test_ordinary_calls_make_room_for_more_recordings(paged):
    from parity_utils import count_launches

    c, step = call_of(paged)
    step()
    torch.cuda.synchronize()
    kept, c._scratch.spare = c._scratch.spare, []
    step()  # finds none left and makes some
    assert len(c._scratch.spare) > 0 and not any(bool(t.any()) for t in c._scratch.spare)
    assert count_launches(lambda: step()) == 2
    held = {t.data_ptr() for t in kept + c._scratch.spare}
    assert len(held) == len(kept) + len(c._scratch.spare)


def test_a_first_call_may_be_recorded(paged):
    # a device that no cache was made on before: the counters are there with the cache, not with its first ordinary call
    known = paged._devices.pop(torch.cuda.current_device(), None)
    try:
        c, step = call_of(paged)
        left = len(c._scratch.spare)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            res = step()
        assert left > 0 and len(c._scratch.spare) == left - 1 and not c._scratch.streams
        for _ in range(3):
            graph.replay()
            want = step()
            torch.cuda.synchronize()
            for a, b in zip(res, want):
                assert torch.equal(a, b)
    finally:
        if known is not None:
            paged._devices[torch.cuda.current_device()] = known
