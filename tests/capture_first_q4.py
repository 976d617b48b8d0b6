"""Run as a program in a fresh process (test_gpu_q4_step.py starts it): the first calls this process ever makes - a whole step over a cache held
in 4 bits - are recorded by a stream capture right after ctcspec_create, replayed, and compared bit for bit with eager calls made afterwards."""
import os
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path[:0] = [HERE, os.path.dirname(HERE)]


def main():
    import torch
    from test_gpu_q4_step import Run, make, same, upload_step
    m = make(10)
    stream = torch.cuda.Stream()
    run = Run(m, stream=stream)
    steps = [upload_step(s) for s in m["steps"]]
    live = {name: t.clone() for name, t in steps[0].items()}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        run.step(live)
    eager = Run(m)
    for r in (run, eager):
        r.append(m["prompt"])
    for d in steps:
        for name, t in d.items():
            live[name].copy_(t)
        torch.cuda.synchronize()
        graph.replay()
        eager.step(d)
        assert same(run.state(), eager.state())
    print("capture-first ok", flush=True)


if __name__ == "__main__":
    main()
