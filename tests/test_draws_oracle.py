"""CPU checks of the draw and dispatch calls: the plain versions (oracle/draws.py) on values worked by hand, and the
library's refusals, which come before any device access (the pointers below are never dereferenced)."""
import ctypes as C

import numpy as np
import pytest

from oracle import draws as O
from paper_2502_07903_amd import hx

FULL = (1 << 64) - 1


def u(x):
    """The draw whose upper 53 bits are floor(x * 2^53)."""
    return int(x * 2.0 ** 53) << 11


# ------------------------------------------------------------------ the plain draw

LOG = np.log(np.array([1.0, 2.0, 4.0, 1.0]))  # weights 1/8, 2/8, 4/8, 1/8


@pytest.mark.parametrize("at,pick", [(0.0, 0), (0.12, 0), (0.13, 1), (0.37, 1), (0.38, 2), (0.87, 2), (0.88, 3)])
def test_plain_draw_by_weight(at, pick):
    got = O.sample_row(LOG, u(at))
    assert got[0] == pick and got[2] == 4
    assert got[1] == pytest.approx(np.log([0.125, 0.25, 0.5, 0.125][pick]), abs=1e-12)


def test_plain_draw_filters():
    assert O.sample_row(LOG, u(0.99), k=2) == (2, pytest.approx(np.log(2 / 3)), 2)
    assert O.sample_row(LOG, u(0.99), k=3)[0] == 2 and O.sample_row(LOG, u(0.0), k=3)[0] == 0  # the tie's lower index
    assert O.sample_row(LOG, u(0.0), p=0.5)[2] == 1 and O.sample_row(LOG, u(0.0), p=0.51)[2] == 2
    assert O.sample_row(LOG, u(0.0), k=2, p=0.6)[2] == 1  # 4 of the first two's 6
    assert O.sample_row(LOG, u(0.0), q=0.3)[2] == 2 and O.sample_row(LOG, u(0.0), q=2.0)[2] == 1
    assert O.sample_row(LOG, u(0.5), p=0.0) == (2, 0.0, 1)


def test_plain_draw_masks_and_parameters():
    inf = np.inf
    assert O.sample_row(np.array([-inf, np.nan]), 0) == (-1, -inf, 0)
    assert O.sample_row(np.array([O.I32_MIN, O.I32_MIN], np.int32), 0) == (-1, -inf, 0)
    assert O.sample_row(np.array([1.0, inf, -inf, inf]), FULL)[0] == 3
    assert O.sample_row(np.array([1.0, inf, -inf, inf]), 0)[0] == 1
    assert O.sample_row(np.array([3.0, 5.0, 5.0]), FULL, T=0.0) == (1, 0.0, 1)
    low = np.full(4, np.finfo(np.float32).min, np.float32)
    assert O.sample_row(low, u(0.6)) == (2, pytest.approx(np.log(0.25)), 4)
    for bad in (dict(T=-1.0), dict(T=inf), dict(T=np.nan), dict(p=np.nan), dict(q=np.nan)):
        assert O.sample_row(LOG, 0, **bad) == (-1, -inf, 0)


# ------------------------------------------------------------------ the plain dispatch

def test_plain_routes():
    flow = [0, 3, -5, 1, 0, 4]  # 2 prefill nodes x 3 decode nodes, total 8
    draws = [0, (FULL >> 3) * 3, ((3 << 64) // 8) + 1, FULL, FULL // 2 + 1]
    r = O.route(2, 3, 2, 4, 6, flow, draws)
    assert r["prefill"].tolist() == [0, 0, 1, 1, 1]
    assert r["decode"].tolist() == [1, 1, 0, 2, 2]
    assert r["p_order"].tolist() == [0, 1, 2, 3, 4] and r["p_base"].tolist() == [0, 2, 5]
    assert r["d_order"].tolist() == [2, 0, 1, 3, 4] and r["d_base"].tolist() == [0, 1, 3, 5, 5]
    none = O.route(2, 3, 2, 4, 6, [0] * 6, draws)
    assert (none["decode"] == -1).all() and none["d_base"].tolist() == [0] * 5
    assert none["d_order"].tolist() == [0, 1, 2, 3, 4]
    assert (O.route(3, 3, 2, 4, 6, flow, draws)["decode"] == -1).all()


def test_plain_place_and_release():
    base, free_list, free = np.array([0, 4, 6]), np.array([3, 2, 1, 0, 1, 0]), np.array([4, 2])
    table = np.full((4, 3), -1, np.int32)
    slots = np.full(12, -7, np.int64)
    tok, placed, held, left = O.place(2, base, free_list, free, table, 3, [0, 1, 0, 0], [0, 0, 0, 0], [3, 1, 5, 2], slots)
    # row 2 needs three blocks of the two that replica 0 has left, and closes it for row 3
    assert tok.tolist() == [0, 3, 4, 9, 11] and placed.tolist() == [1, 1, 0, 0] and left.tolist() == [2, 1]
    assert table.tolist() == [[0, 1, -1], [0, -1, -1], [-1] * 3, [-1] * 3]
    assert slots.tolist() == [0, 1, 2, 0] + [-1] * 7 + [-7]
    tok, placed, held, left = O.place(2, base, free_list, left, table, 3, [0, 1, 0, 0], held, [1, 1, 0, 1], slots)
    assert placed.all() and slots[:3].tolist() == [3, 1, 4] and held.tolist() == [4, 2, 0, 1] and left.tolist() == [1, 1]
    again = free_list.copy()
    held, left = O.release(2, base, again, left, table, 3, [0, 1, 0, 0], held, [1, 1, 1, 1])
    assert held.tolist() == [0] * 4 and left.tolist() == [4, 2] and again.tolist() == free_list.tolist()


# ------------------------------------------------------------------ refusals

FAKE = 0x1000


def _sample(mutate=None):
    a = dict(scores=hx.hx_scores(4, 100, 1, 100, FAKE), params=hx.hx_sampling(FAKE, FAKE, FAKE, FAKE), rnd=FAKE, pick=FAKE,
             logp=None, kept=None, ws=FAKE, bytes=1 << 30)
    if mutate:
        mutate(a)
    by = lambda s: None if s is None else C.byref(s)
    return hx.lib().hx_sample(by(a["scores"]), by(a["params"]), a["rnd"], a["pick"], a["logp"], a["kept"], a["ws"],
                              C.c_size_t(a["bytes"]), None)


@pytest.mark.parametrize("mutate", [
    lambda a: a.update(scores=None), lambda a: a.update(params=None), lambda a: a.update(rnd=None),
    lambda a: a.update(pick=None), lambda a: a.update(ws=None), lambda a: a.update(ws=FAKE + 16),
    lambda a: a.update(bytes=0), lambda a: setattr(a["scores"], "n_rows", 0),
    lambda a: setattr(a["scores"], "n_cols", 0), lambda a: setattr(a["scores"], "n_cols", -5),
    lambda a: setattr(a["scores"], "type", 4), lambda a: setattr(a["scores"], "type", -1),
    lambda a: setattr(a["scores"], "row_stride", -1), lambda a: setattr(a["scores"], "data", None),
    lambda a: setattr(a["scores"], "data", FAKE + 2),   # float32 at two bytes
    lambda a: (setattr(a["scores"], "type", 2), setattr(a["scores"], "data", FAKE + 1)),
], ids=lambda f: "")
def test_sample_refuses(mutate):
    assert _sample(mutate) == hx.HX_EINVAL


def _net():
    return hx.hx_flownet(8, 16, 16, 64, *([FAKE] * 9))


def _route(mutate=None):
    a = dict(net=_net(), cand=3, kv=FAKE, rnd=FAKE, out=hx.hx_routes(10, *([FAKE] * 6)), ws=FAKE, bytes=1 << 30)
    if mutate:
        mutate(a)
    by = lambda s: None if s is None else C.byref(s)
    return hx.lib().hx_route_requests(by(a["net"]), a["cand"], a["kv"], a["rnd"], by(a["out"]), a["ws"],
                                      C.c_size_t(a["bytes"]), None)


@pytest.mark.parametrize("mutate", [
    lambda a: a.update(net=None), lambda a: a.update(cand=-1), lambda a: a.update(cand=8), lambda a: a.update(kv=None),
    lambda a: a.update(rnd=None), lambda a: a.update(out=None), lambda a: a.update(ws=None),
    lambda a: a.update(ws=FAKE + 1), lambda a: a.update(bytes=1), lambda a: setattr(a["net"], "n_p", None),
    lambda a: setattr(a["net"], "max_p", 256), lambda a: setattr(a["net"], "max_d", 0),
    lambda a: setattr(a["net"], "max_pd", 0), lambda a: setattr(a["out"], "n_req", 0),
    lambda a: setattr(a["out"], "prefill", None), lambda a: setattr(a["out"], "decode", None),
    lambda a: setattr(a["out"], "p_order", None), lambda a: setattr(a["out"], "d_base", None),  # half a pair
], ids=lambda f: "")
def test_route_refuses(mutate):
    assert _route(mutate) == hx.HX_EINVAL


def _kv(release, mutate=None):
    a = dict(pool=hx.hx_kv_pool(4, 16, FAKE, FAKE, FAKE, FAKE), rows=hx.hx_kv_rows(8, 10, 12, FAKE, FAKE, FAKE, FAKE),
             new=FAKE, tok=FAKE, slots=FAKE, max_slots=100, placed=FAKE, ws=FAKE, bytes=1 << 30)
    if mutate:
        mutate(a)
    by = lambda s: None if s is None else C.byref(s)
    if release:
        return hx.lib().hx_kv_release(by(a["pool"]), by(a["rows"]), a["new"], a["ws"], C.c_size_t(a["bytes"]), None)
    return hx.lib().hx_kv_place(by(a["pool"]), by(a["rows"]), a["new"], a["tok"], a["slots"], a["max_slots"],
                                a["placed"], a["ws"], C.c_size_t(a["bytes"]), None)


BOTH = [
    lambda a: a.update(pool=None), lambda a: a.update(rows=None), lambda a: a.update(new=None),
    lambda a: a.update(ws=None), lambda a: a.update(ws=FAKE + 128), lambda a: a.update(bytes=3),
    lambda a: setattr(a["pool"], "n_replicas", 0), lambda a: setattr(a["pool"], "n_replicas", 256),
    lambda a: setattr(a["pool"], "block_size", 0), lambda a: setattr(a["pool"], "block_size", 65537),
    lambda a: setattr(a["pool"], "base", None), lambda a: setattr(a["pool"], "free_list", None),
    lambda a: setattr(a["pool"], "free_count", None), lambda a: setattr(a["pool"], "free_out", None),
    lambda a: setattr(a["rows"], "n_rows", 0), lambda a: setattr(a["rows"], "max_blocks", 0),
    lambda a: setattr(a["rows"], "table_stride", 9), lambda a: setattr(a["rows"], "block_table", None),
    lambda a: setattr(a["rows"], "replica", None), lambda a: setattr(a["rows"], "held", None),
    lambda a: setattr(a["rows"], "held_out", None),
]


@pytest.mark.parametrize("mutate", BOTH, ids=lambda f: "")
def test_kv_refuses(mutate):
    assert _kv(False, mutate) == hx.HX_EINVAL
    assert _kv(True, mutate) == hx.HX_EINVAL


@pytest.mark.parametrize("mutate", [
    lambda a: a.update(tok=None), lambda a: a.update(placed=None), lambda a: a.update(slots=None),
    lambda a: a.update(max_slots=-1),
], ids=lambda f: "")
def test_place_refuses(mutate):
    assert _kv(False, mutate) == hx.HX_EINVAL


def test_workspace_sizes():
    L = hx.lib()
    assert L.hx_sample_workspace_bytes(0, 5) == 0 and L.hx_sample_workspace_bytes(5, 0) == 0
    assert L.hx_route_workspace_bytes(256, 1, 1, 1) == 0 and L.hx_route_workspace_bytes(1, 1, 1, 0) == 0
    assert L.hx_kv_workspace_bytes(1, 256) == 0 and L.hx_kv_workspace_bytes(0, 1) == 0
    for n in (L.hx_sample_workspace_bytes(3, 7), L.hx_route_workspace_bytes(255, 255, 65025, 1 << 20),
              L.hx_kv_workspace_bytes(1 << 20, 255)):
        assert n > 0 and n % 256 == 0


def test_pool_refuses():
    with pytest.raises(ValueError):
        hx.KvPool.create([], 16, device="cpu")
    with pytest.raises(ValueError):
        hx.KvPool.create([3, -1], 16, device="cpu")


def test_plain_release_stops_at_the_first_that_does_not_fit():
    # replica 0 has room for two blocks, replica 1 for two: from the last row down, row 3 takes one of replica 0's,
    # row 2 needs two and closes it, row 0 would fit but comes after it; row 4's blocks go to replica 1
    base, free_list = np.array([0, 4, 6]), np.array([0, 1, -1, -1, -1, -1])
    table = np.array([[5, -1], [-1, -1], [6, 7], [8, -1], [3, 4]])
    held, left = O.release(2, base, free_list, np.array([2, 0]), table, 2, [0, 0, 0, 0, 1], [2, 0, 3, 1, 4], [1] * 5)
    assert held.tolist() == [2, 0, 3, 0, 0] and left.tolist() == [3, 2]
    assert free_list.tolist() == [0, 1, 8, -1, 4, 3]


@pytest.mark.parametrize("slots", [(1 << 35) - 2047, 1 << 43, (1 << 43) + 2048, (1 << 63) - 1])
def test_place_refuses_more_slots_than_a_grid_has(slots):
    """Before anything is launched: no row is served, and no block taken."""
    assert _kv(False, lambda a: a.update(max_slots=slots)) == hx.HX_EINVAL
