"""Which rows a reader whose layers mix takes for one request, and the table of turns that its runs share."""
import pytest

from gpu_util import require_gpu


def _small(device="cuda", layers=1):
    import torch
    from paper_2107_06960_amd import reader as R
    params = R.draw_params(64, 2, 32, layers, device=device, mix_heads=2, mix_dim=32)
    gen = torch.Generator().manual_seed(1)
    tokens, maps = torch.randn(6, 64, generator=gen).bfloat16().to(device), torch.randn(2, 3, 3, 64, generator=gen).bfloat16().to(device)
    positions = torch.tensor([0, 1, 2, 0, 1, 2], dtype=torch.int32, device=device)
    return lambda: R.Reader(params, 2, 1, 32, mix_heads=2, mix_dim=32), tokens, maps, positions


def test_requests_that_nothing_tells_are_refused():
    """Without offsets, slots and memory the rows of different requests would be taken for one."""
    import torch
    make, tokens, maps, positions = _small("cpu")
    with pytest.raises(ValueError, match="offsets"):
        make().run(tokens, maps, positions=positions)
    with pytest.raises(ValueError, match="offsets"):
        make().run(tokens, maps, positions=positions, q_offsets=torch.tensor([0, 3, 6], dtype=torch.int32))


def test_turns_are_there_before_the_first_run():
    from paper_2107_06960_amd import operators as O
    import torch
    make, *_ = _small("cpu")
    assert torch.equal(make().turns, O.rotary_turns(16, device="cpu"))


@pytest.mark.gpu
def test_requests_by_offsets_and_by_memory():
    require_gpu()
    import torch
    make, tokens, maps, positions = _small()
    reader = make()
    two = torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda")
    want = reader.run(tokens, maps, positions=positions, offsets=two)
    assert torch.equal(reader.run(tokens, maps, positions=positions, memory=reader.memory(2)), want)
    alone = torch.cat([reader.run(tokens[i:i + 3], maps[i // 3:i // 3 + 1], positions=positions[:3],
                                  offsets=torch.tensor([0, 3], dtype=torch.int32, device="cuda")) for i in (0, 3)])
    assert (alone.float() - want.float()).norm() <= 2 * 2.0 ** -8 * want.float().norm()


@pytest.mark.gpu
def test_a_first_run_inside_a_capture():
    """A reader that first runs while a graph records: its eager runs, before any replay, and the replays agree."""
    require_gpu()
    import torch
    make, tokens, maps, positions = _small()
    positions.mul_(1000)
    off = torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda")
    want = make().run(tokens, maps, positions=positions, offsets=off)
    reader = make()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = reader.run(tokens, maps, positions=positions, offsets=off)
    assert torch.equal(reader.run(tokens, maps, positions=positions, offsets=off), want)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        assert torch.equal(reader.run(tokens, maps, positions=positions, offsets=off), want)


@pytest.mark.gpu
def test_a_first_run_on_another_stream():
    require_gpu()
    import torch
    make, tokens, maps, positions = _small()
    off = torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda")
    want = make().run(tokens, maps, positions=positions, offsets=off)
    reader = make()
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    results = []
    for s in (one, two):  # neither waits for the other
        with torch.cuda.stream(s):
            results.append(reader.run(tokens, maps, positions=positions, offsets=off))
    torch.cuda.synchronize()
    assert all(torch.equal(r, want) for r in results)
