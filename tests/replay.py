"""A step captured into a graph and replayed on inputs that change between the replays, each against the eager step."""
import torch


def replayed(step, change, times=4):
    """step() enqueues on the current stream and returns its output tensors (the same ones each time, or tensors of the graph's
    own memory); change() alters its inputs in place."""
    step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            held = step()
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(times):
        change()
        want = [t.clone() for t in step()]
        for t in held:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a.nan_to_num(-7.0), b.nan_to_num(-7.0))
