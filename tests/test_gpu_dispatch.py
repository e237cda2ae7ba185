"""Routes, KV placement and release on the GPU against the plain versions (oracle/draws.py): whole numbers throughout,
every output equal, and what a call must not touch left as it was."""
import sys

import numpy as np
import pytest

from oracle import draws as O
from paper_2502_07903_amd import hx

pytestmark = pytest.mark.gpu


def say(msg: str) -> None:
    print(f"[gpu] {msg}", flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def torch():
    import torch as T
    if not T.cuda.is_available():
        pytest.fail("GPU tests need a ROCm GPU (torch.cuda.is_available() is False)")
    hx.lib()
    return T


def bits(rng, n):
    d = rng.integers(0, 1 << 64, n, dtype=np.uint64)
    d[:1] = 0
    d[-1:] = (1 << 64) - 1
    return d


def dev(torch, a, dt=np.int32):
    return torch.as_tensor(np.ascontiguousarray(np.asarray(a, dt))).to("cuda")


# ------------------------------------------------------------------ routes

def network(torch, dims, n_p, n_d):
    """A network batch of which only the counts matter."""
    net = hx.FlowNetBuffers.empty(dims, len(n_p))
    net.n_p.copy_(torch.as_tensor(np.asarray(n_p, np.int32)))
    net.n_d.copy_(torch.as_tensor(np.asarray(n_d, np.int32)))
    return net


def check_route(torch, dims, n_p, n_d, flow, draws, cand, lists=True):
    net = network(torch, dims, n_p, n_d)
    out = hx.RouteBuffers.empty(dims, len(draws))
    for t in (out.prefill, out.decode, out.p_order, out.p_base, out.d_order, out.d_base, out.workspace):
        t.fill_(0x55)
    if not lists:
        out.p_order = out.p_base = out.d_order = out.d_base = None
    hx.route_requests(net, dev(torch, flow), dev(torch, draws.view(np.int64), np.int64), out, cand=cand)
    torch.cuda.synchronize()
    want = O.route(n_p[cand], n_d[cand], *dims, flow[:, cand], draws)
    for k in ("prefill", "decode") + (("p_order", "p_base", "d_order", "d_base") if lists else ()):
        assert np.array_equal(getattr(out, k).cpu().numpy(), want[k]), k
    return out


@pytest.mark.parametrize("P,D", [(1, 1), (1, 7), (5, 1), (4, 4), (16, 16), (3, 200), (64, 64), (127, 128), (255, 255)])
@pytest.mark.parametrize("n", [1, 2, 63, 64, 1000, 1024, 1025, 2049, 5000])
def test_route_sizes(torch, P, D, n):
    rng = np.random.default_rng([31, P, D, n])
    dims, N = (P, D, P * D), 3
    flow = np.where(rng.random((P * D, N)) < 0.5, 0, rng.integers(0, 5000, (P * D, N))).astype(np.int32)
    flow[rng.integers(0, P * D), 1] += 1
    say(f"route {n} over {P} x {D}")
    check_route(torch, dims, [P] * N, [D] * N, flow, bits(rng, n), 1)


def test_route_many(torch):
    rng = np.random.default_rng(32)
    P, D = 60, 64
    flow = rng.integers(-2000, 3000, (P * D + 50, 2)).astype(np.int32)
    say("route 70001")
    check_route(torch, (70, 64, P * D + 50), [P, P], [D, D], flow, bits(rng, 70001), 0)
    check_route(torch, (70, 64, P * D + 50), [P, P], [D, D], flow, bits(rng, 4097), 1, lists=False)


@pytest.mark.parametrize("P,D", [(3, 4), (100, 90)])
def test_route_more_than_the_chunks(torch, P, D):
    """More requests than 128 chunks of 1,024: a chunk is several of them."""
    rng = np.random.default_rng([36, P])
    flow = rng.integers(0, 9, (P * D, 1)).astype(np.int32)
    say(f"route 150001 over {P} x {D}")
    check_route(torch, (P, D, P * D), [P], [D], flow, bits(rng, 150001), 0)


@pytest.mark.parametrize("n", [10, 3000])
def test_route_nothing(torch, n):
    """No flow at all, no nodes on a side, counts past the arrays or negative: no routes, every list whole."""
    rng = np.random.default_rng([33, n])
    dims = (4, 5, 20)
    flow = rng.integers(1, 100, (20, 8)).astype(np.int32)
    flow[:, 0] = 0
    flow[:, 1] = -7
    n_p = [4, 4, 0, 4, 5, -1, 4, 2]
    n_d = [5, 5, 5, 0, 4, 3, 6, -3]
    for cand in range(8):
        say(f"route without flow {cand}")
        out = check_route(torch, dims, n_p, n_d, flow, bits(rng, n), cand)
        assert (out.decode == -1).all()


def test_route_large_flows(torch):
    """Capacities at their limit: the running sums pass 32 bits."""
    rng = np.random.default_rng(34)
    flow = np.full((120 * 100, 1), hx.CAP_MAX, np.int32)
    say("route large flows")
    check_route(torch, (120, 100, 12000), [120], [100], flow, bits(rng, 3000), 0)
    flow = np.full((300, 1), (1 << 31) - 1, np.int32)
    check_route(torch, (20, 15, 300), [20], [15], flow, bits(rng, 3000), 0)


def test_route_frequencies(torch):
    """40,000 draws follow the flows within five standard deviations."""
    rng = np.random.default_rng(35)
    flow = np.array([[1], [0], [3], [4]], np.int32)
    out = check_route(torch, (2, 2, 4), [2], [2], flow, bits(rng, 40000), 0)
    got = np.bincount((out.prefill * 2 + out.decode).cpu().numpy(), minlength=4) / 40000
    want = flow[:, 0] / 8
    assert (np.abs(got - want) <= 5 * np.sqrt(want * (1 - want) / 40000)).all()


# ------------------------------------------------------------------ KV memory

class Memory:
    """A pool and rows on the device beside their plain copies on the host; every call is made on both."""

    def __init__(self, torch, blocks, bs, rows, max_blocks, pad=0):
        self.torch, self.bs, self.n, self.max_blocks = torch, bs, rows, max_blocks
        self.pool = hx.KvPool.create(blocks, bs)
        full = torch.full((rows + 2, max_blocks + pad), -9, dtype=torch.int32, device="cuda")
        self.full = full
        self.rows = hx.KvRows(full[:rows, :max_blocks], torch.full((rows,), -1, dtype=torch.int32, device="cuda"),
                              torch.zeros(rows, dtype=torch.int32, device="cuda"))
        self.ws = hx.kv_workspace(rows, len(blocks))
        self.ws.fill_(0x55)
        self.h = dict(base=self.pool.base.cpu().numpy(), free_list=self.pool.free_list.cpu().numpy(),
                      free=self.pool.free_count.cpu().numpy(), table=full.cpu().numpy().copy(),
                      replica=np.full(rows, -1, np.int32), held=np.zeros(rows, np.int32))

    def set(self, **kw):
        for k, v in kw.items():
            self.h[k] = np.asarray(v, np.int32).copy()
            t = {"replica": self.rows.replica, "held": self.rows.held, "free": self.pool.free_count,
                 "free_list": self.pool.free_list, "table": self.full}[k]
            t.copy_(self.torch.as_tensor(self.h[k]))

    def same(self, tag):
        self.torch.cuda.synchronize()
        for k, t in (("table", self.full), ("held", self.rows.held), ("free", self.pool.free_count),
                     ("free_list", self.pool.free_list), ("replica", self.rows.replica)):
            assert np.array_equal(t.cpu().numpy(), self.h[k]), f"{tag}: {k}"

    def place(self, new, max_slots=None, tag="place"):
        torch, h, n = self.torch, self.h, self.n
        new = np.asarray(new, np.int32)
        total = int(np.maximum(new.astype(np.int64), 0).sum())
        max_slots = total + 3 if max_slots is None else max_slots
        slots = torch.full((max_slots + 2,), -7, dtype=torch.int64, device="cuda")
        tok = torch.full((n + 1,), 5, dtype=torch.int64, device="cuda")
        placed = torch.full((n,), 9, dtype=torch.uint8, device="cuda")
        hx.kv_place(self.pool, self.rows, dev(torch, new), tok, slots[:max_slots], placed, self.ws)
        want = np.full(max_slots + 2, -7, np.int64)
        w_tok, w_placed, h["held"], h["free"] = O.place(self.bs, h["base"], h["free_list"], h["free"],
                                                        h["table"][:n], self.max_blocks, h["replica"], h["held"], new,
                                                        want[:max_slots])
        self.same(tag)
        assert np.array_equal(tok.cpu().numpy(), w_tok), tag
        assert np.array_equal(placed.cpu().numpy(), w_placed), tag
        assert np.array_equal(slots.cpu().numpy(), want), tag
        return w_placed

    def release(self, done, tag="release"):
        h, n = self.h, self.n
        hx.kv_release(self.pool, self.rows, dev(self.torch, done, np.uint8), self.ws)
        h["held"], h["free"] = O.release(self.bs, h["base"], h["free_list"], h["free"], h["table"][:n],
                                         self.max_blocks, h["replica"], h["held"], done)
        self.same(tag)


@pytest.mark.parametrize("rows,R,bs", [(1, 1, 1), (1, 1, 16), (5, 2, 3), (63, 1, 16), (64, 4, 16), (200, 255, 8),
                                       (1000, 7, 32), (1024, 16, 16), (1025, 16, 16), (2500, 128, 24), (5000, 3, 16),
                                       (9000, 64, 65536)])
def test_serving_steps(torch, rows, R, bs):
    """Prompts, then decode steps of single tokens, chunks and releases, on pools that run out."""
    rng = np.random.default_rng([41, rows, R, bs])
    width = max(2, 1500 // bs)
    blocks = rng.integers(0, 2 * max(1, rows // R) * max(2, 200 // bs) + 2, R)
    m = Memory(torch, blocks, bs, rows, width, pad=int(rng.integers(0, 4)))
    m.set(replica=rng.integers(-1, R, rows))
    say(f"kv steps: {rows} rows, {R} replicas, blocks of {bs}")
    m.place(np.where(rng.random(rows) < 0.1, 0, rng.integers(1, 400, rows)), tag="prompts")
    for step in range(3):
        m.place(np.ones(rows), tag=f"step {step}")
    m.release((rng.random(rows) < 0.3) * rng.integers(0, 3, rows), tag="some")
    m.place(rng.integers(0, 60, rows), tag="chunks")
    m.place(np.zeros(rows), tag="nothing")
    m.release(np.ones(rows), tag="all")
    assert np.array_equal(m.h["free"], np.diff(m.h["base"]))


def test_more_rows_than_the_chunks(torch):
    rows, R = 140001, 3
    rng = np.random.default_rng(46)
    m = Memory(torch, [60000, 50000, 1], 16, rows, 4)
    m.set(replica=rng.integers(-1, R, rows))
    say("kv 140001 rows")
    m.place(rng.integers(0, 30, rows), tag="prompts")
    m.place(np.ones(rows), tag="tokens")
    m.release(rng.random(rows) < 0.7)


@pytest.mark.parametrize("rows", [3, 700, 4000])
def test_place_then_release_restores(torch, rows):
    rng = np.random.default_rng([42, rows])
    R = 5
    m = Memory(torch, [rows * 4] * R, 16, rows, 100)
    m.set(replica=rng.integers(0, R, rows))
    start = m.h["free_list"].copy()
    m.place(rng.integers(1, 200, rows))
    m.release(np.ones(rows))
    assert np.array_equal(m.h["free_list"], start)


@pytest.mark.parametrize("rows", [40, 1300])
def test_rows_not_served(torch, rows):
    """Rows on no replica, negative lengths, tables and slots that are too short, lengths past 2^31: refused, counted
    and marked, and the rest served as if they were not there."""
    rng = np.random.default_rng([43, rows])
    m = Memory(torch, [rows] * 3, 16, rows, 12, pad=1)
    rep = rng.integers(0, 3, rows)
    rep[::7] = rng.choice([-1, 3, 255, 256, -(1 << 31), (1 << 31) - 1], len(rep[::7]))
    held = np.zeros(rows)
    held[3::11] = -5
    held[5::13] = (1 << 31) - 1
    m.set(replica=rep, held=held)
    new = rng.integers(0, 30, rows)
    new[1::9] = -3
    new[2::9] = 16 * 12 + 1     # one block past the table
    new[4::9] = 16 * 12
    say(f"kv rows not served: {rows}")
    m.place(new, tag="all slots")
    m.place(rng.integers(0, 9, rows), max_slots=int(rows * 2), tag="few slots")
    m.place(rng.integers(0, 9, rows), max_slots=0, tag="no slots")
    m.release(np.ones(rows))


@pytest.mark.parametrize("rows", [12, 2000])
def test_pool_counts_out_of_range(torch, rows):
    """Free counts below zero or past the replica's range are clamped, and blocks that would not fit stay."""
    m = Memory(torch, [40, 0, 30, 50], 4, rows, 8)
    m.set(replica=np.arange(rows) % 4, free=[500, 9, -3, 50])
    say("kv counts out of range")
    m.place(np.full(rows, 9))
    m.set(free=[38, 0, 0, 49])
    m.release(np.ones(rows), tag="more than fits")


def test_slots_past_32_bits(torch):
    m = Memory(torch, [64], 65536, 20, 4)
    m.set(free_list=np.arange((1 << 31) - 64, 1 << 31)[::-1], replica=np.zeros(20))
    say("kv slots past 32 bits")
    m.place(np.full(20, 70000))


@pytest.mark.parametrize("lens", [[100000, 1, 0, 250000], [0, 0, 0], [1], [4096] * 300])
def test_long_prompts(torch, lens):
    m = Memory(torch, [40000], 16, len(lens), 250000 // 16 + 1)
    m.set(replica=np.zeros(len(lens)))
    say(f"kv long prompts {lens[:4]}")
    m.place(lens)
    m.place(np.ones(len(lens)))
    m.release(np.ones(len(lens)))


def test_separate_outputs(torch):
    """free_out and held_out apart from the inputs: the inputs stay, and the call can be made again."""
    rows = 600
    rng = np.random.default_rng(44)
    m = Memory(torch, [900] * 4, 16, rows, 20)
    m.set(replica=rng.integers(0, 4, rows))
    new = dev(torch, rng.integers(1, 90, rows))
    free, held = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
    tok = torch.zeros(rows + 1, dtype=torch.int64, device="cuda")
    placed = torch.zeros(rows, dtype=torch.uint8, device="cuda")
    seen = []
    for _ in range(2):
        slots = torch.full((90 * rows,), -7, dtype=torch.int64, device="cuda")
        hx.kv_place(m.pool, m.rows, new, tok, slots, placed, m.ws, free_out=free, held_out=held)
        seen.append([t.clone() for t in (slots, free, held, tok, placed, m.full)])
    assert all(torch.equal(a, b) for a, b in zip(*seen))
    assert (m.rows.held == 0).all() and (m.pool.free_count == 900).all()
    assert torch.equal(held, torch.where(placed != 0, new, 0))


@pytest.mark.parametrize("rows", [200, 3000])
def test_captured_and_replayed(torch, rows):
    """Route, place, two token steps and release captured together; every replay on new draws and lengths equal to the
    eager calls on a copy of the same memory."""
    rng = np.random.default_rng([45, rows])
    P, D = 5, 6
    flow = dev(torch, rng.integers(1, 50, (P * D, 1)))
    net = network(torch, (P, D, P * D), [P], [D])
    draws = torch.zeros(rows, dtype=torch.int64, device="cuda")
    new = torch.zeros(rows, dtype=torch.int32, device="cuda")
    one = torch.ones(rows, dtype=torch.int32, device="cuda")
    done = torch.ones(rows, dtype=torch.uint8, device="cuda")

    def side():
        s = dict(out=hx.RouteBuffers.empty((P, D, P * D), rows), pool=hx.KvPool.create([rows * 2] * D, 16),
                 ws=hx.kv_workspace(rows, D), tok=torch.zeros(rows + 1, dtype=torch.int64, device="cuda"),
                 slots=torch.zeros(100 * rows, dtype=torch.int64, device="cuda"),
                 placed=torch.zeros(rows, dtype=torch.uint8, device="cuda"), rows=hx.KvRows.empty(rows, 12))
        s["rows"].replica = s["out"].decode
        return s

    def steps(s):
        hx.route_requests(net, flow, draws, s["out"])
        for k in (new, one, one):
            hx.kv_place(s["pool"], s["rows"], k, s["tok"], s["slots"], s["placed"], s["ws"])
        hx.kv_release(s["pool"], s["rows"], done, s["ws"])

    a, b = side(), side()
    say(f"dispatch captured, {rows} rows")
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        steps(a)
        steps(b)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        steps(a)
    for i in range(4):
        draws.copy_(torch.as_tensor(bits(rng, rows).view(np.int64)))
        new.copy_(torch.as_tensor(rng.integers(1, 90, rows).astype(np.int32)))
        done.copy_(torch.as_tensor((rng.random(rows) < 0.8).astype(np.uint8)))
        g.replay()
        steps(b)
        torch.cuda.synchronize()
        for x, y in ((a["out"].decode, b["out"].decode), (a["out"].d_order, b["out"].d_order),
                     (a["slots"], b["slots"]), (a["rows"].table, b["rows"].table), (a["rows"].held, b["rows"].held),
                     (a["pool"].free_list, b["pool"].free_list), (a["pool"].free_count, b["pool"].free_count)):
            assert torch.equal(x, y), f"replay {i}"


def test_refuses(torch):
    m = Memory(torch, [10, 10], 16, 4, 5)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
    tok, slots = torch.zeros(5, dtype=torch.int64, device="cuda"), torch.zeros(9, dtype=torch.int64, device="cuda")
    placed = torch.zeros(4, dtype=torch.uint8, device="cuda")
    good = dict(pool=m.pool, rows=m.rows, n_new=i32(4), tok_base=tok, slots=slots, placed=placed, workspace=m.ws)
    hx.kv_place(**good)
    for k, v in (("n_new", i32(5)), ("n_new", i32(4).long()), ("n_new", i32(4).cpu()), ("tok_base", tok[:4]),
                 ("slots", slots.int()), ("placed", placed[:3]), ("free_out", i32(3)), ("held_out", i32(4).cpu()),
                 ("rows", hx.KvRows(m.rows.table.t(), m.rows.replica, m.rows.held)),
                 ("rows", hx.KvRows(m.rows.table, m.rows.replica[:3], m.rows.held)),
                 ("pool", hx.KvPool(16, m.pool.base[:2], m.pool.free_list, m.pool.free_count))):
        with pytest.raises(ValueError):
            hx.kv_place(**dict(good, **{k: v}))
    with pytest.raises(hx.HxError):
        hx.kv_place(**dict(good, workspace=m.ws[:0]))
    with pytest.raises(hx.HxError):
        hx.kv_place(**dict(good, pool=hx.KvPool(0, m.pool.base, m.pool.free_list, m.pool.free_count)))
    with pytest.raises(ValueError):
        hx.kv_release(m.pool, m.rows, i32(4), m.ws)
    net = network(torch, (2, 2, 4), [2], [2])
    out = hx.RouteBuffers.empty((2, 2, 4), 3)
    flow, d = dev(torch, np.ones((4, 1))), torch.zeros(3, dtype=torch.int64, device="cuda")
    for f in (lambda: hx.route_requests(net, flow[:3], d, out), lambda: hx.route_requests(net, flow, d[:2], out),
              lambda: hx.route_requests(net, flow.long(), d, out), lambda: hx.route_requests(net, flow, d.cpu(), out)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(hx.HxError):
        hx.route_requests(net, flow, d, out, cand=1)


@pytest.mark.parametrize("rows", [5, 1500])
def test_release_stops_at_the_first_that_does_not_fit(torch, rows):
    """A large row that does not fit among small ones that would, before and after it, on two replicas."""
    m = Memory(torch, [3 * rows, 3 * rows], 2, rows, 4)
    m.set(replica=np.arange(rows) % 2)
    m.place(np.full(rows, 2))
    held = np.full(rows, 2)
    held[rows // 2] = 8
    m.set(held=held, table=np.arange((rows + 2) * 4).reshape(rows + 2, 4),
          free=[3 * rows - rows // 4 - 2, 3 * rows - 1])
    say(f"kv release of a row that does not fit: {rows}")
    m.release(np.ones(rows), tag="one does not fit")
    assert 0 < (m.h["held"] > 0).sum() < rows and m.h["held"][rows // 2] == 8
