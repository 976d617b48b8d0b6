"""Steps of a verification pass over a cache held in 4 bits, the calls together as they are used: kv_append_q4 of the prompts, then in every
step q4_verify_attn per layer, verify_head_argmax, verify_sample_filtered, accept_longest and kv_commit_q4 per layer - one after the other,
in a captured graph, and on two streams at once."""
import contextlib
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import oracle
import paper_2412_00061_amd as pkg
from paper_2412_00061_amd import binding
from test_gpu_prefix_attn import mask_words
from workloads.device import dev_f32, dev_i32, dev_i64, to_device
from workloads.generate import round_to_storage

LAYERS, B, H, HKV, N, DH, V, T, CAP, STEPS = 2, 3, 6, 2, 14, 80, 9, 4, 230, 4
WINDOW, SINK, SCALE = 60, 5, DH ** -0.5
PROMPTS = [150, 1, 33]
NODES = [[14, 9, 1], [1, 14, 14], [14, 0, 5], [7, 14, 14]]  # of each step; 0: a place not in use, its root counts
SHAPES = {"q": (LAYERS, B, H, N, DH), "kt": (LAYERS, B, HKV, N, DH), "vt": (LAYERS, B, HKV, N, DH)}


def values(rng, *s):
    return round_to_storage(rng.standard_normal(s, dtype=np.float32), "bf16")


def make(seed):
    """Prompts, the head, and the steps' inputs: trees whose siblings have different tokens of few, so that some are drawn."""
    rng = np.random.default_rng(seed)
    m = dict(prompt=values(rng, 2, LAYERS, B, HKV, max(PROMPTS), DH), w=values(rng, V, H * DH), temperature=np.float32([0.7, 0.0, 1.3]),
             top_k=np.int32([5, 0, 0]), top_p=np.float32([0.9, 1.0, 0.95]), min_p=np.float32([0.0, 0.0, 0.02]), steps=[])
    for n in NODES:
        s = {name: values(rng, *shape) for name, shape in SHAPES.items()}
        token, parent, depth = (np.full((B, N), -1, np.int32) for _ in range(3))
        seen = np.zeros((B, N, N), bool)
        for b in range(B):
            used = {}
            for i in range(n[b]):
                at = int(rng.choice([j for j in range(i) if depth[b, j] < T])) if i else -1
                parent[b, i], depth[b, i] = at, depth[b, at] + 1 if i else 0
                seen[b, i] = seen[b, at] if i else False
                seen[b, i, i] = True
                token[b, i] = rng.choice([v for v in range(V) if v not in used.get(at, ())])
                used.setdefault(at, []).append(token[b, i])
        s.update(n=np.int32(n), token=token, parent=parent, depth=depth, seen=seen, u=rng.random((B, N), dtype=np.float32))
        m["steps"].append(s)
    return m


def upload_step(s):
    d = {name: to_device(s[name], "bf16") for name in SHAPES}
    d.update({name: dev_i32(s[name]) for name in ("n", "token", "parent", "depth")}, u=dev_f32(s["u"]),
             mask=dev_i64(mask_words(s["seen"], N).view(np.int64)))
    return d


class Run:
    """The buffers of a batch, and its calls."""

    def __init__(self, m, stream=None):
        self.ctx = pkg.Context(max_batch=B, max_slots=1, max_topk=1, max_vocab_rows=16, max_nodes=N, max_heads=H, max_head_dim=DH, stream=stream)
        self.w, self.off = to_device(m["w"], "bf16"), dev_i64(np.int64([2, 0, 1]) * HKV * CAP)
        self.filters = dict(top_k=dev_i32(m["top_k"]), top_p=dev_f32(m["top_p"]), min_p=dev_f32(m["min_p"]))
        self.temperature = dev_f32(m["temperature"])
        blocks = -(-DH // 32)
        self.cache = [[torch.full((B * HKV * CAP, blocks * 16 if i % 2 == 0 else blocks), 255, dtype=torch.uint8, device="cuda") for i in range(4)]
                      for _ in range(LAYERS)]
        self.length = dev_i32([0] * B)
        self.longer = torch.zeros_like(self.length)
        self.out = dict(attn=torch.zeros((LAYERS, B, H, N, DH), dtype=torch.bfloat16, device="cuda"),
                        hidden=torch.zeros((B, N, H * DH), dtype=torch.bfloat16, device="cuda"), lse=torch.zeros((LAYERS, B, H, N), device="cuda"),
                        logits=torch.zeros((B, N, V), device="cuda"), target_argmax=dev_i32(np.zeros((B, N))), target_sampled=dev_i32(np.zeros((B, N))),
                        n_kept=dev_i32(np.zeros((B, N))), logp=torch.zeros((B, N), device="cuda"), accept_len=dev_i32(np.zeros(B)),
                        accept_nodes=dev_i32(np.zeros((B, T + 1))), accept_tokens=dev_i32(np.zeros((B, T + 1))), next_token=dev_i32(np.zeros(B)))
        self.ws = torch.empty(pkg.q4_verify_attn_workspace_bytes(B, H, HKV, DH, N), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()

    def append(self, prompt):
        rows, longer = dev_i32(PROMPTS), dev_i32([0] * B)
        layers = [to_device(prompt[:, i], "bf16") for i in range(LAYERS)]
        torch.cuda.synchronize()
        for kv, cache in zip(layers, self.cache):
            pkg.kv_append_q4(self.ctx, kv[0], kv[1], rows, pkg.q4_cache(*cache), self.off, self.length, CAP, ctx_len_out=longer)
        torch.cuda.synchronize()
        self.length.copy_(longer)
        torch.cuda.synchronize()

    def step(self, d):
        o = self.out
        for i, cache in enumerate(self.cache):
            pkg.q4_verify_attn(self.ctx, d["q"][i], pkg.q4_cache(*cache), self.off, self.length, CAP, d["kt"][i], d["vt"][i], d["n"], d["mask"], SCALE,
                               node_depth=d["depth"], window=WINDOW, sink=SINK, out_dtype=torch.bfloat16, want_lse=True, workspace=self.ws,
                               out=dict(out=o["attn"][i], lse=o["lse"][i]))
        o["hidden"].view(B, N, H, DH).copy_(o["attn"][LAYERS - 1].transpose(1, 2))
        pkg.verify_head_argmax(self.ctx, o["hidden"], self.w, d["n"], want_logits=True, out=o)
        pkg.verify_sample_filtered(self.ctx, o["logits"], d["n"], d["u"], self.temperature, **self.filters, want_kept=True, want_logp=True, out=o)
        pkg.accept_longest(self.ctx, d["n"], d["token"], d["parent"], d["depth"], o["target_sampled"], T, out=o)
        for i, cache in enumerate(self.cache):
            pkg.kv_commit_q4(self.ctx, d["kt"][i], d["vt"][i], o["accept_len"], o["accept_nodes"], pkg.q4_cache(*cache), self.off, self.length, CAP,
                             ctx_len_out=self.longer)
        self.length.copy_(self.longer)

    def state(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (*self.out.values(), self.length, *(p for c in self.cache for p in c))]


def same(a, b):
    """Equal, NaN of the same bits too."""
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


@pytest.fixture(scope="module")
def eager():
    m = make(8)
    run, states = Run(m), []
    run.append(m["prompt"])
    for s in m["steps"]:
        run.step(upload_step(s))
        states.append(run.state())
    run.ctx.close()
    return m, states


@pytest.mark.gpu
def test_the_steps_against_the_oracle():
    from test_gpu_q4_attn import check
    m = make(8)
    run = Run(m)
    run.append(m["prompt"])
    place, length = [2, 0, 1], list(PROMPTS)
    stored = [[np.full(tuple(p.view(B, HKV, CAP, -1).shape), 255, np.uint8) for p in cache] for cache in run.cache]
    for i in range(LAYERS):
        for kv in range(2):
            codes, scales = oracle.q4_encode(m["prompt"][kv, i])
            for b, L in enumerate(length):
                stored[i][2 * kv][b, :, :L], stored[i][2 * kv + 1][b, :, :L] = codes[b, :, :L], scales[b, :, :L]

    def compare_cache():
        for i in range(LAYERS):
            for want, got in zip(stored[i], run.cache[i]):
                assert np.array_equal(want, got.view(B, HKV, CAP, -1).cpu().numpy()[place]), i
        assert run.length.tolist() == length

    compare_cache()
    accepted = 0
    for at, s in enumerate(m["steps"]):
        for t in run.out.values():
            t.zero_()
        torch.cuda.synchronize()
        run.step(upload_step(s))
        torch.cuda.synchronize()
        o = {name: t.cpu() for name, t in run.out.items()}
        for i in range(LAYERS):
            c = dict(B=B, H=H, Hkv=HKV, N=N, dh=DH, cap=CAP, ctx=list(length), n=list(s["n"]), scale=SCALE, window=WINDOW, sink=SINK, q=s["q"][i],
                     kt=s["kt"][i], vt=s["vt"][i], parts=stored[i], seen=s["seen"], depth=s["depth"])
            check(c, dict(out=o["attn"][i], lse=o["lse"][i]), sentinel=0.0)
        hidden, logits = o["hidden"].double().numpy(), o["logits"].double().numpy()
        for b in range(B):
            n = int(s["n"][b])
            # products of bf16 numbers are exact in float32, a sum of D of them is off by at most D 2^-24 of their magnitudes
            exact, size = hidden[b, :n] @ m["w"].T.astype(np.float64), np.abs(hidden[b, :n]) @ np.abs(m["w"].T.astype(np.float64))
            assert np.all(np.abs(logits[b, :n] - exact) <= H * DH * 2.0 ** -24 * size), (at, b)
            for node in range(n):
                want = oracle.sample_filtered(o["logits"][b, node].numpy(), float(s["u"][b, node]), float(m["temperature"][b]), int(m["top_k"][b]),
                                              float(m["top_p"][b]), float(m["min_p"][b]))
                assert (int(o["target_sampled"][b, node]), int(o["n_kept"][b, node])) == want[:2], (at, b, node)
            # (accept_longest counts the root as there, in a place not in use too, and the commit appends its row)
            count, nodes, tokens, following = oracle.accept_longest(s["token"][b], s["parent"][b], max(n, 1), o["target_sampled"][b].numpy(), T)
            assert int(o["accept_len"][b]) == count and o["accept_nodes"][b].tolist() == list(nodes), (at, b)
            assert o["accept_tokens"][b].tolist() == list(tokens) and int(o["next_token"][b]) == following
            accepted += count
            path = list(nodes[:count + 1])
            for i in range(LAYERS):
                for kv, rows in enumerate((s["kt"][i], s["vt"][i])):
                    codes, scales = oracle.q4_encode(rows[b][:, path])
                    L = length[b]
                    stored[i][2 * kv][b, :, L:L + count + 1], stored[i][2 * kv + 1][b, :, L:L + count + 1] = codes, scales
            length[b] += count + 1
        compare_cache()
    assert accepted >= 1  # (a path beyond a root was committed)
    run.ctx.close()


@pytest.mark.gpu
def test_the_steps_captured(eager):
    """One graph for every step of the batch, replayed with other trees, lengths and scratch; eager work in between."""
    m, states = eager
    stream = torch.cuda.Stream()
    run = Run(m, stream=stream)
    steps = [upload_step(s) for s in m["steps"]]
    live = {name: t.clone() for name, t in steps[0].items()}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        run.step(live)
    for again in range(2):
        run.length.zero_()
        for cache in run.cache:
            for p in cache:
                p.fill_(255)
        for t in run.out.values():
            t.zero_()
        torch.cuda.synchronize()
        run.append(m["prompt"])
        for d, want in zip(steps, states):
            for name, t in d.items():
                live[name].copy_(t)
            run.ws.fill_(255)
            torch.cuda.synchronize()
            graph.replay()
            assert same(run.state(), want), again
    run.ctx.close()


@pytest.mark.gpu
def test_the_steps_on_two_streams_at_once(eager):
    m, states = eager
    other = make(9)
    runs, inputs = [], []
    for x in (m, other):
        stream = torch.cuda.Stream()
        runs.append((Run(x, stream=stream), stream))
        runs[-1][0].append(x["prompt"])
        inputs.append([upload_step(s) for s in x["steps"]])
    torch.cuda.synchronize()
    for i in range(STEPS):
        for (run, stream), d in zip(runs, inputs):
            with torch.cuda.stream(stream):
                run.step(d[i])
    assert same(runs[0][0].state(), states[-1])
    alone = Run(other)
    alone.append(other["prompt"])
    for d in inputs[1]:
        alone.step(d)
    assert same(alone.state(), runs[1][0].state())
    for run in (alone, *(r for r, _ in runs)):
        run.ctx.close()


@pytest.mark.gpu
def test_the_first_calls_of_a_process_captured():
    program = os.path.join(os.path.dirname(os.path.abspath(__file__)), "capture_first_q4.py")
    r = subprocess.run([sys.executable, program], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "capture-first ok" in r.stdout, r.stdout + r.stderr


def test_scratch_comes_from_the_stream_of_the_context(monkeypatch):
    """(On the CPU: what is asked for, and on which stream.)"""
    class Context:
        stream, handle = "the context's", None

        class lib:
            q4_verify_attn = staticmethod(lambda *a: 0)

        @staticmethod
        def _check(rc, what):
            assert rc == 0

    now, asked, empty = ["current"], [], torch.empty

    @contextlib.contextmanager
    def stream(s):
        now.append(s)
        yield
        now.pop()

    def allocate(*a, **k):
        if k.get("dtype") == torch.uint8:
            asked.append(now[-1])
        return empty(*a, **k)

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch, "empty", allocate)
    monkeypatch.setattr(binding, "_ptr", lambda t, dtype=None: None)
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    i = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    pkg.q4_verify_attn(Context, z(2, 4, 5, 64), binding._Q4Cache(), i(0, 8).long(), i(8, 3), 8, z(2, 2, 5, 64), z(2, 2, 5, 64), i(5, 5),
                       torch.ones((2, 5, 1), dtype=torch.int64), 0.125)
    assert asked == ["the context's"] and now == ["current"]
