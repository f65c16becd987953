"""Products with run-time scales and the 4-bit cache together: captured as a process's
first calls, and on two streams at once."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ip():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_30846_gb300 as ip
    ip.load()
    return ip


class Step:
    """Products in every form (a few tokens, K shared by CTAs, one CTA a tile, pairs), rows
    into a cache, the attention over it (with and without a second launch), rows back."""

    def __init__(self, ip, seed):
        self.ip = ip
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.ws = torch.zeros(ip.kv4_attention_workspace_bytes(2, 5, 4, 2, 1000), dtype=torch.uint8, device="cuda")
        self.cache, self.table = ip.kv4_cache(64, 2, 32), torch.randperm(64, generator=g, device="cuda").int().view(2, 32)
        self.start = torch.zeros(2, dtype=torch.int32, device="cuda")
        self.lens = torch.full((2,), 900, dtype=torch.int32, device="cuda")
        self.k, self.q = rand(2, 900, 2, 128).bfloat16(), rand(2, 5, 4, 128).bfloat16()
        sizes = ((1, 64, 48, torch.bfloat16), (200, 1500, 700, torch.float16), (2000, 1024, 4096, torch.float32),
                 (500, 5000, 4096, torch.bfloat16))
        self.x = [rand(m, k).to(t) for m, k, n, t in sizes]
        self.w = [ip_rows(torch.randint(-127, 128, (n, k), generator=g, device="cuda")) for m, k, n, t in sizes]
        self.sw = [rand(n).abs() for m, k, n, t in sizes]
        torch.cuda.synchronize()

    def __call__(self):
        ip, out = self.ip, []
        for x, w, sw in zip(self.x, self.w, self.sw):
            q, s = ip.quantize_rows_i8(x)
            out += [q, s, ip.linear_scaled_i8(q, s, w, sw, act=ip.ACT_SWISH, dtype=x.dtype, workspace=self.ws)]
        ip.kv4_append(self.k, self.k, self.start, self.table, self.cache, workspace=self.ws)
        for n in (1000, 600):
            out.append(ip.kv4_attention(self.q, self.lens.clamp(max=n), self.table, self.cache, max_len=n,
                                        workspace=self.ws))
        return out + list(ip.kv4_read(self.cache, self.start, self.table, 900, dtype=torch.bfloat16, workspace=self.ws))


def ip_rows(w):
    """int8 rows that start on 16 bytes."""
    base = torch.zeros(w.shape[0], -(-w.shape[1] // 16) * 16, dtype=torch.int8, device="cuda")
    base[:, :w.shape[1]] = w
    return base[:, :w.shape[1]]


FIRST = """
import torch, paper_2609_30846_gb300 as ip
from test_decode_capture_gpu import Step
ip.load()
step, graph = Step(ip, 1), torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = step()
graph.replay()
torch.cuda.synchronize()
want = step()
assert ip.status(step.ws) == 0 and all(torch.equal(a, b) for a, b in zip(got, want))
"""


def test_a_process_may_begin_with_a_capture(ip):
    here = os.path.dirname(os.path.abspath(__file__))
    env = dict(os.environ, PYTHONPATH=os.pathsep.join([os.path.dirname(here), here]))
    r = subprocess.run([sys.executable, "-c", FIRST], env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


def test_two_streams_at_once(ip):
    steps = [Step(ip, 1), Step(ip, 2)]
    want = [s() for s in steps]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(8):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                got[i].append(steps[i]())
    torch.cuda.synchronize()
    for i in (0, 1):
        assert ip.status(steps[i].ws) == 0
        for out in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(out, want[i]))
