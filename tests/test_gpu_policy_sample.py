"""policy_sample against the oracle in 64 bits, through the C boundary.

An index has to be the oracle's, except where u lies within `slack` of a border between two indices: each weight is a whole multiple
of 2^-40 of the largest, so it is off by at most 2^-41 of a mass of at least 1, and n of them by n 2^-41; fp64's own roundings add
2^-45 at most at these lengths.  logp: that, and half a step of fp32."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2111_01264_amd as P
from oracle import actor

TYPES = {"fp32": (torch.float32, P.DQN_TYPE_FP32), "bf16": (torch.bfloat16, P.DQN_TYPE_BF16), "fp16": (torch.float16, P.DQN_TYPE_FP16)}
INF, NAN = float("inf"), float("nan")


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


class Call:
    """One call's buffers, guarded behind the last row."""

    def __init__(self, scores, n, u, t=None, k=None, p=None, m=None, want_logp=True):
        dev = lambda v, dt: None if v is None else torch.as_tensor(v, dtype=dt).cuda().contiguous()  # noqa: E731
        f, i = torch.float32, torch.int32
        assert scores.shape[1] == n
        self.x, self.n, self.rows = scores, n, scores.shape[0]
        self.t, self.k, self.p, self.m, self.u = dev(t, f), dev(k, i), dev(p, f), dev(m, f), dev(u, f)
        self.index = torch.full((self.rows + 1,), -7, dtype=i, device="cuda")
        self.logp = torch.full((self.rows + 1,), 9.0, device="cuda") if want_logp else None
        self.work = torch.empty(max(16, P.policy_sample_workspace(self.rows, n)), dtype=torch.uint8, device="cuda").fill_(0xA5)
        torch.cuda.synchronize()

    def enqueue(self, stream=None):
        ld = self.x.stride(0) if self.rows > 1 else max(self.n, 1)
        P.policy_sample(self.x, TYPES_BY[self.x.dtype], ld, self.rows, self.n, self.t, self.k, self.p, self.m, self.u, self.index, self.logp, self.work, self.work.numel(), stream)

    def check(self):
        torch.cuda.synchronize()
        rows = self.rows
        assert self.index[rows].item() == -7 and (self.logp is None or self.logp[rows].item() == 9.0)
        got = self.index[:rows].cpu().numpy()
        logp = None if self.logp is None else self.logp[:rows].cpu().numpy().astype(np.float64)
        x = self.x.float().cpu().numpy()
        host = lambda v, default: np.full(rows, default) if v is None else v.cpu().numpy()  # noqa: E731
        t, k, p, m, u = host(self.t, 1.0), host(self.k, 0), host(self.p, 1.0), host(self.m, 0.0), host(self.u, 0.0)
        slack = self.n * 2.0 ** -41 + 2.0 ** -45
        near = 0
        for r in range(rows):
            d = actor.draw(x[r, :self.n], u[r], t[r], int(k[r]), float(p[r]), float(m[r]), slack)
            if d.filter_margin <= slack:   # top-p's border: one entry more or less may be kept
                near += 1
                assert 0 <= got[r] < self.n and x[r, got[r]] > -INF
                continue
            assert d.low <= got[r] <= d.high, (r, got[r], d, t[r], k[r], p[r], m[r], u[r])
            if logp is not None and got[r] == d.index:
                assert (np.isnan(logp[r]) and np.isnan(d.logp)) or abs(logp[r] - d.logp) <= 2.0 ** -24 * abs(d.logp) * 1.001 + slack, (r, logp[r], d)
        return near

    def run(self, stream=None):
        self.enqueue(stream)
        return self.check()


TYPES_BY = {dt: code for dt, code in TYPES.values()}

FILTERS = [dict(), dict(t=0.7), dict(k=1), dict(k=5), dict(k=50), dict(k=1000), dict(p=0.9), dict(p=0.2, t=2.0), dict(k=40, p=0.95), dict(k=3000, p=0.5), dict(m=0.05), dict(m=1.0),
           dict(t=1.5, k=100, p=0.99, m=0.01), dict(t=0.0), dict(t=0.05, p=0.999), dict(t=50.0, p=0.9)]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n", [1, 2, 3, 17, 18, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000, 1023, 1024, 1025, 4097, 8192, 20000, 50021, 131072])
def test_lengths_and_filters(kind, n):
    dt, _ = TYPES[kind]
    g = gen(n)
    rows = len(FILTERS)
    x = (3 * torch.randn(rows, n, generator=g, device="cuda")).to(dt)
    of = lambda key, off: [f.get(key, off) for f in FILTERS]  # noqa: E731
    u = torch.rand(rows, generator=g, device="cuda")
    assert Call(x, n, u, of("t", 1.0), of("k", 0), of("p", 1.0), of("m", 0.0)).run() <= 2
    # each filter alone, the others' arrays absent; a different number of rows
    half = x[:3]
    Call(half, n, u[:3], t=[0.5, 1.0, 2.0]).run()
    Call(half, n, u[:3], k=[2, 20, n]).run()
    Call(half, n, u[:3], p=[0.3, 0.9, 1.0]).run()
    Call(half, n, u[:3], m=[0.0, 0.1, 2.0], want_logp=False).run()


@pytest.mark.parametrize("rows,n", [(1, 18), (5, 18), (512, 18), (4096, 4), (1000, 32), (300, 100), (64, 3001), (100, 9000), (600, 2000)])
def test_many_rows(rows, n):
    g = gen(rows + n)
    x = 2 * torch.randn(rows, n, generator=g, device="cuda")
    pick = lambda v: torch.tensor(v, device="cuda")[torch.randint(len(v), (rows,), generator=g, device="cuda")]  # noqa: E731
    Call(x, n, torch.rand(rows, generator=g, device="cuda"), pick([0.0, 0.5, 1.0, 3.0]), pick([0, 1, 2, 7, n]), pick([0.5, 0.9, 1.0]), pick([0.0, 0.1])).run()


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,n", [(9, 49151), (9, 49152), (70, 50000), (128, 49999), (130, 49999), (2, 300000)])
def test_rows_shared_out_and_not(kind, rows, n):
    """Both sides of the lines between one workgroup per row and several, filters mixed."""
    g = gen(rows * n)
    x = (2 * torch.randn(rows, n, generator=g, device="cuda")).to(TYPES[kind][0])
    x[1::3, ::7] = -INF
    pick = lambda v: torch.tensor(v, device="cuda")[torch.randint(len(v), (rows,), generator=g, device="cuda")]  # noqa: E731
    u = torch.rand(rows, generator=g, device="cuda")
    Call(x, n, u, pick([0.0, 0.7, 1.0, 1.0, 4.0]), pick([0, 0, 30, 192, 193, 5000, n // 2]), pick([0.3, 0.9, 0.99, 1.0]), pick([0.0, 0.0, 0.01])).run()
    Call(x, n, u, p=pick([0.5, 0.95])).run()
    Call(x, n, u, t=pick([0.5, 2.0])).run()


@pytest.mark.parametrize("n", [17000, 60000])
def test_bf16_values_of_every_size(n):
    """Zeros, tiny, ordinary and large values, of few and of many kinds: those that have a place in the table of values and those that have none."""
    g = gen(n)
    rows = 140
    x = 2 * torch.randn(rows, n, generator=g, device="cuda")
    x[0::7, ::3] = 0.0
    x[1::7, ::2] *= 1e-9
    x[2::7, ::5] = -400.0
    x[3::7] = torch.round(x[3::7])
    x[4::7] *= 2.0 ** -30
    x[5::7, 5] = 3e4
    x = x.bfloat16()
    u = torch.rand(rows, generator=g, device="cuda")
    rep = lambda v: torch.tensor([v[(r // 7) % len(v)] for r in range(rows)])  # noqa: E731
    Call(x, n, u, rep([1.0, 0.5, 30.0, 1.0]), rep([0, 300, 0, 2000, 40]), rep([0.9, 1.0, 0.5, 0.99])).run()
    Call(x, n, u, rep([1.0, 200.0]), None, None, rep([0.0, 0.001])).run()


@pytest.mark.parametrize("n", [6, 40, 700, 5000, 40000])
def test_equal_scores_go_by_index(n):
    """Weights of exactly 1: kept sets and borders are whole numbers, with no rounding anywhere."""
    x = torch.zeros(6, n, device="cuda")
    x[:, 1::2] = -0.0   # the same score
    x[3, ::3] = -INF
    x[4] = torch.finfo(torch.float32).min
    x[5] = INF
    for k in (0, 2, n // 2, n - 1):
        for p in (1.0, 0.5, 0.25):
            for u in (0.0, 0.25, 0.5, 1 - 2.0 ** -24):
                c = Call(x, n, [u] * 6, k=[k] * 6, p=[p] * 6)
                c.enqueue()
                torch.cuda.synchronize()
                got = c.index[:6].tolist()
                for r in (0, 1, 2, 4, 5):
                    size = k if k else n
                    kept = size if p == 1.0 else int(np.ceil(p * size))
                    assert got[r] == int(np.floor(u * kept)), (r, k, p, u)
                live = [i for i in range(n) if i % 3]
                size = min(k, len(live)) if k else len(live)
                kept = size if p == 1.0 else int(np.ceil(p * size))
                assert got[3] == live[int(np.floor(u * kept))], (k, p, u)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n", [5, 50, 900, 30000])
def test_masks_infinities_and_nan(kind, n):
    dt, _ = TYPES[kind]
    low = torch.finfo(dt).min
    g = gen(n)
    x = torch.randn(10, n, generator=g, device="cuda")
    x[0] = -INF                                    # nothing left
    x[1, :] = -INF; x[1, n - 1] = -3.0             # one left, the last
    x[2, : n - 2] = low                            # masked with the type's lowest value
    x[3] = low                                     # all of it: a row of equals
    x[4, n // 2] = NAN
    x[5, 1] = INF; x[5, n - 1] = INF               # share the mass
    x[6, n - 1] = NAN; x[6, 0] = INF
    x[7, 0] = torch.finfo(dt).max; x[7, 1] = low
    x[8, : n - 1] = -INF; x[8, 0] = NAN
    x = x.to(dt)
    for t in (1.0, 0.0, 1e-30, 1e30):
        for k, p in ((0, 1.0), (3, 1.0), (0, 0.9), (2, 0.5)):
            c = Call(x, n, torch.rand(10, generator=g, device="cuda"), [t] * 10, [k] * 10, [p] * 10)
            c.run()
            assert c.index[[0, 4, 6, 8]].tolist() == [-1] * 4 and torch.isnan(c.logp[[0, 4, 6, 8]]).all()


def test_refused_settings_and_the_ends_of_u():
    g = gen(1)
    for n in (18, 3000, 40000):
        x = torch.randn(9, n, generator=g, device="cuda")
        c = Call(x, n, [0.5] * 9, t=[-1.0, NAN, INF, 1.0, 1.0, 1.0, -0.0, 1.0, 1.0], p=[1.0, 1.0, 1.0, NAN, 1.0, 1.0, 1.0, -0.5, 2.0], m=[0.0, 0.0, 0.0, 0.0, NAN, 0.0, 0.0, 0.0, -1.0])
        c.u[5] = NAN
        c.run()
        assert c.index[:6].tolist() == [-1] * 6 and (c.index[6:9] >= 0).all()
        for u in (-3.0, 0.0, 1.0 - 2.0 ** -24, 1.0, 1e30, INF, -INF):
            c = Call(x, n, [u] * 9, k=[0, 7, 0, 1, n, -5, 2, n + 9, 3])
            c.run()


def test_no_scores():
    c = Call(torch.zeros(3, 0, device="cuda"), 0, [0.1, 0.2, 0.3])
    c.x = torch.zeros(3, 1, device="cuda")
    c.run()
    assert c.index.tolist() == [-1, -1, -1, -7]


@pytest.mark.parametrize("kind", list(TYPES))
def test_pitches_and_alignments(kind):
    dt, _ = TYPES[kind]
    g = gen(2)
    for n, ld in ((18, 25), (1001, 1006), (30001, 30006)):
        big = (2 * torch.randn(5, ld, generator=g, device="cuda")).to(dt)
        for off in (0, 1, 2, 3, 5):
            Call(big[:, off:off + n], n, torch.rand(5, generator=g, device="cuda"), k=[0, 0, 20, 0, 9], p=[1.0, 0.9, 1.0, 0.5, 0.7]).run()


@pytest.mark.parametrize("order", ["up", "down", "far"])
def test_ordered_rows(order):
    """Rows whose large scores all lie together: no part of the row is like another."""
    for n in (1000, 30000, 131072):
        for dt in (torch.float32, torch.bfloat16):
            x = torch.linspace(-8, 8, n, device="cuda").to(dt).repeat(6, 1)
            if order == "down":
                x = x.flip(1).contiguous()
            if order == "far":
                x[:] = -20.0
                x[:, n - 300:] = torch.linspace(0, 1, 300, device="cuda").to(dt)
            Call(x, n, [0.03, 0.5, 0.97, 0.2, 0.8, 0.6], k=[0, 100, 2000, 0, 0, 64], p=[1.0, 1.0, 0.9, 0.95, 0.5, 0.8]).run()


def test_longest_row():
    n = P.POLICY_SAMPLE_MAX_N
    x = torch.randn(1, n, generator=gen(3), device="cuda").bfloat16()
    for f in (dict(), dict(k=[50]), dict(p=[0.9]), dict(k=[100000], p=[0.8])):
        Call(x, n, [0.71], **f).run()


def test_rows_past_four_gigabytes():
    """Offsets that pass 32 bits."""
    rows, n, ld = 70, 20, 1 << 25
    big = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld)
    big[:, :n] = torch.randn(rows, n, generator=gen(4), device="cuda").bfloat16()
    Call(big[:, :n], n, torch.rand(rows, generator=gen(5), device="cuda")).run()


def test_another_stream_and_replayed_graphs_with_a_workspace_each():
    stream = torch.cuda.Stream()
    g = gen(7)
    calls = [Call(3 * torch.randn(rows, n, generator=g, device="cuda"), n, torch.rand(rows, generator=g, device="cuda"), k=[kk] * rows, p=[pp] * rows)
             for rows, n, kk, pp in ((2, 40000, 50, 0.9), (2, 40000, 0, 0.9), (3, 40000, 0, 1.0), (30, 18, 0, 1.0))]
    graphs = []
    for c in calls:
        c.run(stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            c.enqueue(stream)
        graphs.append(graph)
    for _ in range(3):
        for c in calls:
            c.x.copy_(3 * torch.randn(c.rows, c.n, generator=g, device="cuda"))
            c.u.copy_(torch.rand(c.rows, generator=g, device="cuda"))
            c.index[:c.rows] = -3
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        for c in calls:
            c.check()


def test_the_same_result_on_every_run():
    x = torch.randn(4, 131072, generator=gen(8), device="cuda")
    c = Call(x, 131072, [0.1, 0.4, 0.6, 0.9], p=[0.9, 0.95, 1.0, 0.5])
    c.run()
    first = (c.index.clone(), c.logp.clone())
    for _ in range(3):
        c.enqueue()
        torch.cuda.synchronize()
        assert torch.equal(first[0], c.index) and torch.equal(first[1], c.logp)
