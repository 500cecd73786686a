"""Rotation, append and read back on a stream of their own and captured in a
graph; the counts, positions and slots they are given are read anew by every
call."""
import numpy as np
import pytest
import torch

from cache_harness import DEV, Cache

pytestmark = pytest.mark.gpu
B, C, HQ, H, D, PAGE, ROOM = 3, 2, 8, 2, 64, 4, 64


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_26472_amd import epikv
    epikv.lib()
    return epikv


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Calls:
    """Buffers and argument structs of one loop over a cache, built once."""

    def __init__(self, E, fmt):
        self.E = E
        self.c = Cache(E, np.random.default_rng(5), fmt, B, H, D, PAGE, ROOM, fill=0)
        self.rope = E.default_rope(rotary_dim=D, n_pos=256)
        self.table = torch.empty(256, D // 2, 2, device=DEV)
        E.epikv_rope_table(self.rope, self.table)

        def rows(heads):
            return torch.zeros(B, C, heads, D, dtype=torch.bfloat16, device=DEV)
        self.q, self.q_out, self.x = rows(HQ), rows(HQ), rows(HQ)
        self.k, self.v, self.k_held, self.v_held = rows(H), rows(H), rows(H), rows(H)
        self.n, self.nn, self.first, self.positions = (ints([0] * B) for _ in range(4))
        self.ids = torch.full((B, ROOM), -1, dtype=torch.int32, device=DEV)
        self.status = ints([0] * B)
        c = self.c
        self.append = E.make_append_io(C, c.pool, 0, c.table, c.ld_pt, self.n, self.k, self.v, n_new=self.nn,
                                       rope=self.rope, table=self.table, positions=self.positions, q=self.q,
                                       q_out=self.q_out, pos=self.ids, ld_s=ROOM, seq_status=self.status)
        self.read = E.make_read_io(C, c.pool, 0, c.table, c.ld_pt, self.first, self.k_held, self.v_held,
                                   seq_status=self.status)

    def load(self, step):
        """Another step's inputs, in place."""
        g = torch.Generator(device=DEV).manual_seed(step)
        for t in (self.q, self.k, self.v):
            t.copy_(torch.randn(t.shape, generator=g, device=DEV))
        self.n.copy_(ints([C + 3 * step, C * (step + 1), 1 + step]))
        self.nn.copy_(ints([C, C, step % 2]))
        self.first.copy_(self.n - C)
        self.first.clamp_(min=0)
        self.positions.copy_(ints([40 * step, 7, 100 - step]))

    def run(self, stream=None):
        E = self.E
        E.epikv_rope(self.rope, self.table, E.DTYPE_BF16, B, C, HQ, D, self.q, self.x, self.positions,
                     transpose=True, seq_status=self.status, stream=stream)
        E.epikv_append(self.c.cfg, self.append, stream=stream)
        E.epikv_read(self.c.cfg, self.read, stream=stream)

    def differs(self, other):
        """Which outputs' bytes are not the other's."""
        a, b = ((s.x, s.q_out, s.k_held, s.v_held, s.ids, s.c.bytes, s.status) for s in (self, other))
        names = ("x", "q_out", "k_held", "v_held", "ids", "pool", "status")
        return [m for m, s, t in zip(names, a, b) if not torch.equal(s.view(torch.uint8), t.view(torch.uint8))]


@pytest.mark.parametrize("fmt", [0, 1])
def test_inputs_are_read_anew(E, fmt):
    """One set of structs whose tensors change in place, against fresh ones."""
    one = Calls(E, fmt)
    for step in range(4):
        one.load(step)
        fresh = Calls(E, fmt)
        fresh.load(step)
        fresh.c.bytes.copy_(one.c.bytes)
        fresh.ids.copy_(one.ids)
        fresh.q_out.copy_(one.q_out)  # (padding tokens' queries are not written)
        one.run()
        fresh.run()
        assert one.differs(fresh) == []
        if fmt == 0:  # the new values, where a sequence has a whole chunk of them
            assert torch.equal(one.v_held[:2], one.v[:2])


@pytest.mark.parametrize("fmt", [0, 1])
def test_another_stream(E, fmt):
    one, two = Calls(E, fmt), Calls(E, fmt)
    side = torch.cuda.Stream()
    for step in range(3):
        one.load(step)
        one.run()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            two.load(step)
        two.run(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert one.differs(two) == []


@pytest.mark.parametrize("fmt", [0, 1])
def test_replays_of_a_graph(E, fmt):
    """Captured once; every replay, with other inputs and eager work between,
    gives the eager call's bytes."""
    one, two = Calls(E, fmt), Calls(E, fmt)
    two.load(0)
    two.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        two.run()
    two.c.bytes.zero_()
    two.ids.fill_(-1)
    two.status.zero_()
    for step in range(5):
        one.load(step)
        one.run()
        two.load(step)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert one.differs(two) == [], step
