"""A captured decoding loop of several tokens that advances its own positions and lengths between the calls: what a
kernel of the graph writes, the next one's position, page and length loads read."""
import numpy as np
import pytest
import torch

from kv_cases import cos_sin, dev, host_bits
from paper_2506_03781_amd import uniquan as uq
from paper_2506_03781_amd.cache import KVCache

pytestmark = pytest.mark.gpu
F32 = np.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    uq.lib()
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


STEPS = 5


class Loop:
    """n sequences at positions of their own; every step appends a token, advances and attends."""

    def __init__(self, fmt, seed):
        rs = np.random.default_rng(seed)
        n, n_kv, H, d = 4, 2, 8, 64
        self.c = KVCache(48, n_kv, n, 12, d=d, page_len=16, fmt=fmt, group=32 if fmt == "u4" else None)
        self.pages = torch.from_numpy(rs.permutation(48).reshape(n, 12).astype(np.int32)).cuda()
        self.c.table.copy_(self.pages)
        self.start = np.array([140, 0, 15, 63], np.int32)
        rows = int(self.start.sum())
        x = dev(rs.standard_normal((rows, 2 * n_kv * d)).astype(F32))
        self.c.append(x[:, :n_kv * d], x[:, n_kv * d:],
                      dev(np.concatenate([np.arange(v) for v in self.start]).astype(np.int32)),
                      seq=dev(np.repeat(np.arange(n), self.start).astype(np.int32)))
        self.pos, self.lens = dev(self.start.copy()), dev(self.start.copy())
        self.cs = dev(cos_sin(192, d))
        self.x = dev(rs.standard_normal((STEPS, n, (H + 2 * n_kv) * d)).astype(F32))
        self.Q = torch.empty(n, H * d, device="cuda", dtype=torch.bfloat16)
        self.O = torch.empty(STEPS, n, H * d, device="cuda", dtype=torch.bfloat16)
        self.lse = torch.empty(STEPS, n, H, device="cuda")
        self.K, self.V = (torch.empty(n_kv, n, 192, d, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        self.H, self.w, self.ws = H * d, n_kv * d, self.c.workspace(H)

    def run(self):
        """STEPS tokens; the page of the first sequence's oldest positions goes in the middle."""
        for i in range(STEPS):
            x = self.x[i]
            self.c.append(x[:, self.H:self.H + self.w], x[:, self.H + self.w:], self.pos, q=x[:, :self.H], q_out=self.Q,
                          cs=self.cs)
            self.lens += 1
            if i == 2:
                self.c.table[0, :1].fill_(-1)
            self.c.attend(self.Q, self.lens, self.O[i], self.lse[i], ws=self.ws)
            self.pos += 1
        self.c.read(self.lens, 192, self.K, self.V)

    def rewind(self):
        self.pos.copy_(dev(self.start))
        self.lens.copy_(dev(self.start))
        self.c.table.copy_(self.pages)
        for t in (self.O, self.lse, self.K, self.V):
            t.fill_(float("nan"))
        torch.cuda.synchronize()

    def outputs(self):
        torch.cuda.synchronize()
        out = [self.O, self.lse, self.K, self.V, self.c.k, self.c.v, self.pos, self.lens]
        return [host_bits(t).copy() for t in out + ([self.c.k_stat, self.c.v_stat] if self.c.group else [])]


@pytest.mark.parametrize("fmt", ["bf16", "u8", "u4"])
def test_loop_that_advances_itself(fmt):
    a, b, other = Loop(fmt, 1), Loop(fmt, 1), Loop(fmt, 2)
    a.run()
    want = a.outputs()
    assert np.isfinite(want[1]).all() and len({w.tobytes() for w in want[1]}) == STEPS
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.run()
    for replay in range(4):
        b.rewind()
        g.replay()
        other.rewind()
        other.run()
        for got, w in zip(b.outputs(), want):
            assert np.array_equal(got, w), (fmt, replay)


@pytest.mark.parametrize("shared", [False, True])
def test_two_graphs_and_their_workspaces(shared):
    """Two captured loops replayed in turn: each with the workspace that attend takes for itself while it is captured,
    or both with one, which may be used again once a replay is done."""
    loops, graphs, wants = [], [], []
    for seed, fmt in ((3, "bf16"), (4, "u4")):
        eager = Loop(fmt, seed)
        eager.run()
        wants.append(eager.outputs())
        s = Loop(fmt, seed)
        s.ws = loops[0].ws if shared and loops else s.ws if shared else None
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.run()
        loops.append(s)
        graphs.append(g)
    for _ in range(3):
        for s in loops:
            s.rewind()
        for g in graphs:
            g.replay()
        for s, want in zip(loops, wants):
            assert all(np.array_equal(x, y) for x, y in zip(s.outputs(), want))


def test_current_stream_other_than_the_default():
    """Under a stream that torch makes current, attend takes its workspace there."""
    a, b = Loop("u8", 5), Loop("u8", 5)
    a.ws = b.ws = None
    side = torch.cuda.Stream()
    a.run()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        b.run()
    for x, y in zip(a.outputs(), b.outputs()):
        assert np.array_equal(x, y)
