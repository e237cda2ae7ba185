"""Performance cases of the operators that follow a scored batch: one entry drawn from each row of scores
(temperature, top-k, top-p, min-p), requests routed along the edges of a maximum flow, and the blocks and
slots of the routed requests' KV caches.

Each case is a dict of plain values; `kind` names the operator:

  sample   hx.sample on rows of scores: flow values of candidate placements (i32) or a decode replica's logits
  route    hx.route_requests on one network's flow assignment
  place    hx.kv_place: blocks and token slots for every row's new tokens (prompts, chunks, single tokens)
  release  hx.kv_release: the blocks of finished rows back to their replicas' free lists

With `own` false a pass computes the same from elementary torch operations, with `own` true it is the library's
call.  Random draws are inputs (64 random bits each).  Lengths follow the request lengths of
paper_2502_07903_amd/inputs.py (lognormal, prompts up to 4,096 tokens, outputs up to 2,048).
"""
import math

import numpy as np
import torch

own = False

I32_MIN = -(1 << 31)
TYPES = {"i32": torch.int32, "f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _sample(name, rows, cols, dtype, top_k=0, top_p=0, min_p=0, pad=0, shared=0):
    c = dict(kind="sample", rows=rows, cols=cols, dtype=dtype, top_k=top_k, top_p=top_p, min_p=min_p, pad=pad,
             shared=shared)
    return dict(c, name=name) if name else c


def _route(name, prefill, decode, requests, nets):
    c = dict(kind="route", prefill=prefill, decode=decode, requests=requests, nets=nets)
    return dict(c, name=name) if name else c


def _kv(name, kind, rows, replicas, block, mean_held, mean_new, room):
    c = dict(kind=kind, rows=rows, replicas=replicas, block=block, mean_held=mean_held, mean_new=mean_new, room=room)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The next parent of a small search (256 scored placements): latency and launches are all there is.
        _sample("sample 1 x 256 i32", 1, 256, "i32"),
        # The next parent of the headline search batch, among its 64 best placements.
        _sample("sample 1 x 65536 i32 top-k", 1, 65536, "i32", top_k=64),
        # Sixteen refinement chains advanced together, each over its own 131,072 children.
        _sample("sample 16 x 131072 i32 top-p", 16, 131072, "i32", top_p=1),
        # Tokens of a small decode batch from rows of logits, every filter on.
        _sample("sample 32 x 32000 f32 all", 32, 32000, "f32", top_k=50, top_p=1, min_p=1),
        # Tokens of a large decode batch over a vocabulary of no round size, rows padded.
        _sample("sample 256 x 50257 f16 top-p min-p", 256, 50257, "f16", top_p=1, min_p=1, pad=7),
        # The largest: 1,024 rows of 131,072 logits, temperature only (every entry has weight).
        _sample("sample 1024 x 131072 bf16", 1024, 131072, "bf16"),
        # A burst of requests over the four replicas a side of a small cluster.
        _route("route 256 over 4 x 4", 4, 4, 256, 1),
        # A long queue of requests over per-GPU flow nodes of a 128-GPU cluster, the network one
        # column of a batch.
        _route("route 65536 over 64 x 64", 64, 64, 65536, 8),
        # One decode step of a serving batch: every row one more token, few need a block.
        _kv("place 256 rows x 1 token", "place", 256, 4, 16, 700, 1, 1.5),
        # A queue of prompts entering a cluster's decode replicas, more than their memory takes.
        _kv("place 4096 prompts", "place", 4096, 16, 16, 0, 1024, 0.9),
        # A few finished requests of a decode step.
        _kv("release 256 rows", "release", 256, 4, 16, 1000, 0, 1.0),
        # A drained cluster: every row's blocks go back.
        _kv("release 8192 rows", "release", 8192, 64, 16, 1500, 0, 1.0),
    ]


def _log_int(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["sample"] * 6 + ["route"] * 2 + ["place"] * 3 + ["release"] * 2)
    if kind == "sample":
        cols = _log_int(rng, 64, 262144)
        rows = _log_int(rng, 1, max(1, min(1024, (1 << 27) // cols)))
        dtype = rng.choice(["i32", "i32", "f32", "f16", "bf16"])
        filters = rng.choice(["", "k", "p", "m", "kp", "kpm", "pm"])
        return _sample("", rows, cols, dtype, _log_int(rng, 1, 2000) if "k" in filters else 0, int("p" in filters),
                       int("m" in filters), rng.choice([0, 0, 1, 8, 13]), int(dtype == "i32" and rng.random() < 0.3))
    if kind == "route":
        return _route("", _log_int(rng, 1, 64), _log_int(rng, 1, 64), _log_int(rng, 1, 65536), _log_int(rng, 1, 64))
    rows = _log_int(rng, 1, 8192)
    replicas = _log_int(rng, 1, 128)
    block = rng.choice([1, 8, 16, 16, 24, 32, 64, 256])
    if kind == "release":
        return _kv("", "release", rows, replicas, block, _log_int(rng, 1, 1500), 0, 1.0)
    if rng.random() < 0.4:
        return _kv("", "place", rows, replicas, block, _log_int(rng, 1, 1500), 1, rng.choice([0.5, 1.0, 1.5]))
    return _kv("", "place", rows, replicas, block, rng.choice([0, 0, 300]), _log_int(rng, 2, 1500),
               rng.choice([0.7, 1.0, 1.5]))


# ------------------------------------------------------------------ inputs

def _bits(n, gen):
    """n draws of 64 random bits, as int64 bit patterns."""
    d = gen.device
    hi = torch.randint(-(1 << 31), 1 << 31, (n,), generator=gen, device=d, dtype=torch.int64)
    lo = torch.randint(0, 1 << 32, (n,), generator=gen, device=d, dtype=torch.int64)
    return (hi << 32) | lo


def _prepare_sample(c, gen):
    d, R, N = gen.device, c["rows"], c["cols"]
    held = 1 if c["shared"] else R
    row = lambda lo, hi, n=R: lo + (hi - lo) * torch.rand(n, generator=gen, device=d)
    if c["dtype"] == "i32":
        # candidates' flow values in milli-requests a second, some placements infeasible
        x = 18000.0 + 2000.0 * torch.randn((held, N + c["pad"]), generator=gen, device=d)
        x = torch.where(torch.rand(x.shape, generator=gen, device=d) < 0.1, 0.0, x).clamp_(min=0).to(torch.int32)
        t = row(100.0, 1000.0)
    else:
        # logits with an exponential tail, peaked in some rows and flat in others, a few tokens banned
        x = torch.rand((held, N + c["pad"]), generator=gen, device=d).clamp_(min=1e-7).log_()
        x = x * -row(0.4, 1.3, held)[:, None] - 4.0
        x = x.masked_fill_(torch.rand(x.shape, generator=gen, device=d) < 0.01, -math.inf).to(TYPES[c["dtype"]])
        t = row(0.6, 1.4)
        t = torch.where(torch.rand(R, generator=gen, device=d) < 0.1, 0.0, t)
    x = x[:, :N].expand(R, N) if c["shared"] else x[:, :N]
    s = dict(case=c, x=x, temperature=t, draws=_bits(R, gen), top_k=None, top_p=None, min_p=None)
    if c["top_k"]:
        k = torch.randint(max(1, c["top_k"] // 2), 2 * c["top_k"] + 1, (R,), generator=gen, device=d)
        s["top_k"] = torch.where(torch.rand(R, generator=gen, device=d) < 0.1, 0, k).to(torch.int32)
    if c["top_p"]:
        s["top_p"] = row(0.6, 1.05).clamp_(max=1.0)
    if c["min_p"]:
        s["min_p"] = row(-0.02, 0.15).clamp_(min=0.0)
    if own:
        from paper_2502_07903_amd import hx
        s["params"] = hx.Sampling(s["temperature"], s["top_k"], s["top_p"], s["min_p"])
        s["out"] = hx.SampleBuffers.empty(R, N, device=d)
    return s


def _prepare_route(c, gen):
    d, P, D, M = gen.device, c["prefill"], c["decode"], c["nets"]
    flow = torch.randint(0, 4000, (P * D, M), generator=gen, device=d)
    flow = torch.where(torch.rand((P * D, M), generator=gen, device=d) < 0.6, 0, flow).to(torch.int32)
    s = dict(case=c, kv_flow=flow, draws=_bits(c["requests"], gen), cand=M // 2)
    if own:
        from paper_2502_07903_amd import hx
        s["net"] = hx.FlowNetBuffers.empty((P, D, P * D), M, device=d)
        s["net"].n_p.fill_(P)
        s["net"].n_d.fill_(D)
        s["out"] = hx.RouteBuffers.empty((P, D, P * D), c["requests"], device=d)
    return s


def _lengths(mean, n, gen, most):
    """n lognormal lengths in a random order: the distribution's quantiles, their sum the same for every seed."""
    q = (torch.arange(n, device=gen.device, dtype=torch.float64) + 0.5) / n
    x = torch.exp(math.log(max(mean, 1)) - 0.3 + 0.8 * math.sqrt(2.0) * torch.erfinv(2.0 * q - 1.0))
    return x.round().clamp(1, most).to(torch.int64)[torch.randperm(n, generator=gen, device=gen.device)]


def _before(replica, count, R):
    """Sum of count over the earlier rows of the same replica, and each replica's total (int64)."""
    one = torch.zeros((replica.numel(), R), dtype=torch.int64, device=replica.device)
    has = replica >= 0
    one[has, replica[has]] = count[has]
    cum = one.cumsum(0)
    mine = cum.gather(1, replica.clamp(min=0)[:, None])[:, 0] - count
    return mine, cum[-1]


def _prepare_kv(c, gen):
    d, n, R, bs = gen.device, c["rows"], c["replicas"], c["block"]
    most = 6144
    held = _lengths(c["mean_held"], n, gen, most) if c["mean_held"] else torch.zeros(n, dtype=torch.int64, device=d)
    if c["kind"] == "place":
        new = _lengths(c["mean_new"], n, gen, 4096) if c["mean_new"] > 1 else torch.ones(n, dtype=torch.int64, device=d)
        if c["mean_new"] == 1:
            new[torch.randperm(n, generator=gen, device=d)[:n // 50]] = 0  # rows that wait in this step
    else:
        new = torch.zeros(n, dtype=torch.int64, device=d)
    replica = torch.randint(0, R, (n,), generator=gen, device=d)
    replica = torch.where(torch.rand(n, generator=gen, device=d) < 0.02, -1, replica)
    has = replica >= 0
    everyone, held = held, torch.where(has, held, 0)
    b0 = (held + bs - 1) // bs
    need = torch.where(has, (held + new + bs - 1) // bs - b0, 0)
    at, used = _before(replica, torch.where(has, b0, 0), R)
    room = (c["room"] * _before(replica, need, R)[1].double()).long()
    cap = used + room + (1 if c["kind"] == "place" else 0)
    base = torch.zeros(R + 1, dtype=torch.int64, device=d)
    base[1:] = cap.cumsum(0)
    total = int(base[-1])
    longest = int(((everyone + bs - 1) // bs).sum() + c["room"] * (new // bs + 2).sum()) + R  # of any seed's lists
    # every replica's blocks in a random order: the rows' own first, the free ones after them
    owner = torch.repeat_interleave(torch.arange(R, device=d), cap)
    key = owner.double() + torch.rand(total, generator=gen, device=d, dtype=torch.float64)
    blocks = torch.argsort(key) - base[owner]
    width = (most + 4096) // bs + 3
    table = torch.full((n, width), -1, dtype=torch.int32, device=d)
    r = torch.repeat_interleave(torch.arange(n, device=d), b0)
    col = torch.arange(r.numel(), device=d) - (b0.cumsum(0) - b0)[r]
    table[r, col] = blocks[base[replica[r].clamp(min=0)] + at[r] + col].to(torch.int32)
    free_list = torch.full((longest,), -1, dtype=torch.int32, device=d)
    q = torch.arange(total, device=d) - base[owner]
    spare = q >= used[owner]
    free_list[(base[owner] + q - used[owner])[spare]] = blocks[spare].to(torch.int32)
    s = dict(case=c, replica=replica.to(torch.int32), held=held.to(torch.int32), table=table, base=base.to(torch.int32),
             free_list=free_list, free_count=(cap - used).to(torch.int32),
             free_out=torch.zeros(R, dtype=torch.int32, device=d), held_out=torch.zeros(n, dtype=torch.int32, device=d))
    if c["kind"] == "place":
        s["new"] = new.to(torch.int32)
        tokens = int(new.sum()) + 5
        s["slots"] = torch.full((tokens,), -7, dtype=torch.int64, device=d)
        s["tok_base"] = torch.zeros(n + 1, dtype=torch.int64, device=d)
        s["placed"] = torch.zeros(n, dtype=torch.uint8, device=d)
    else:
        s["done"] = (torch.rand(n, generator=gen, device=d) < 0.9).to(torch.uint8)
    if own:
        from paper_2502_07903_amd import hx
        s["pool"] = hx.KvPool(bs, s["base"], s["free_list"], s["free_count"])
        s["rows"] = hx.KvRows(s["table"], s["replica"], s["held"])
        s["workspace"] = hx.kv_workspace(n, R, device=d)
    return s


def prepare(case, seed):
    gen = torch.Generator(torch.device("cuda")).manual_seed(int(seed))
    if case["kind"] == "sample":
        return _prepare_sample(case, gen)
    if case["kind"] == "route":
        return _prepare_route(case, gen)
    return _prepare_kv(case, gen)


# ------------------------------------------------------------------ plain forms

def _plain_sample(s):
    # in 64 bits throughout: a pick is a comparison with a running sum, and a border is never far away
    x = s["x"]
    gone = x == I32_MIN if x.dtype == torch.int32 else torch.isnan(x) | (x == -math.inf)
    x = torch.where(gone, -math.inf, x.double())
    R, N = x.shape
    t = s["temperature"].double()[:, None]
    m = x.max(1, keepdim=True).values
    some = m[:, 0] > -math.inf
    z = torch.where(x == m, 0.0, (x - m) / t)
    z = torch.where(gone, -math.inf, z)
    w = z.exp()
    eligible = N - gone.sum(1)
    kept = eligible
    if s["top_k"] is not None or s["top_p"] is not None or s["min_p"] is not None:
        order = torch.sort(x, dim=1, descending=True, stable=True).indices
        ws = w.gather(1, order)
        rank = torch.arange(N, device=x.device)[None, :]
        if s["top_k"] is not None:
            k = s["top_k"].long()
            kept = torch.where(k > 0, torch.minimum(k, eligible), eligible)
        if s["top_p"] is not None:
            p = s["top_p"].double()
            cum = torch.where(rank < kept[:, None], ws, 0.0).cumsum(1)
            enough = (cum < p[:, None] * cum[:, -1:]).sum(1) + 1
            kept = torch.where(p < 1, torch.minimum(enough, kept), kept)
        if s["min_p"] is not None:
            kept = torch.minimum(kept, (ws >= s["min_p"].double()[:, None]).sum(1)).clamp(min=1)
        keep = torch.zeros_like(gone).scatter_(1, order, rank < kept[:, None])
        w = torch.where(keep, w, 0.0)
    cum = w.cumsum(1)
    u = ((s["draws"] >> 11) & ((1 << 53) - 1)).double() * 2.0 ** -53
    last = N - 1 - (w.flip(1) > 0).long().argmax(1)
    pick = torch.minimum((cum <= (u[:, None] * cum[:, -1:])).sum(1), last)
    logp = z.gather(1, pick[:, None])[:, 0] - cum[:, -1].log()
    greedy = t[:, 0] == 0
    pick = torch.where(greedy, (x == m).long().argmax(1), pick)
    logp = torch.where(greedy, 0.0, logp)
    kept = torch.where(greedy, 1, kept)
    pick = torch.where(some, pick, -1)
    return dict(pick=pick.to(torch.int32), logp=torch.where(some, logp, -math.inf).float(),
                kept=torch.where(some, kept, 0).to(torch.int32))


def _plain_group(node, nodes):
    """Requests in a stable order of their node (those without one last), and where each node's run starts."""
    key = torch.where(node < 0, nodes, node)
    order = torch.sort(key, stable=True).indices
    count = (key[:, None] == torch.arange(nodes, device=key.device)).sum(0)
    base = torch.zeros(nodes + 1, dtype=torch.int64, device=key.device)
    base[1:] = count.cumsum(0)
    return order.to(torch.int32), base.to(torch.int32)


def _plain_route(s):
    P, D = s["case"]["prefill"], s["case"]["decode"]
    cum = s["kv_flow"][:, s["cand"]].clamp(min=0).long().cumsum(0)
    total = cum[-1]
    hi, lo = (s["draws"] >> 32) & 0xFFFFFFFF, s["draws"] & 0xFFFFFFFF
    t = (hi * total + ((lo * total) >> 32)) >> 32  # floor(draw * total / 2^64), exact: total < 2^31
    edge = torch.searchsorted(cum, t, right=True)
    ok = total > 0
    prefill = torch.where(ok, edge // D, -1)
    decode = torch.where(ok, edge % D, -1)
    po, pb = _plain_group(prefill, P)
    do, db = _plain_group(decode, D)
    return dict(prefill=prefill.to(torch.int32), decode=decode.to(torch.int32), p_order=po, p_base=pb, d_order=do,
                d_base=db)


def _plain_place(s):
    c, bs, R = s["case"], s["case"]["block"], s["case"]["replicas"]
    n, replica, held, new = c["rows"], s["replica"].long(), s["held"].long(), s["new"].long()
    dev, has = replica.device, replica >= 0
    b0 = (held + bs - 1) // bs
    need = torch.where(has, (held + new + bs - 1) // bs - b0, 0)
    at, _ = _before(replica, need, R)
    free = s["free_count"].long()[replica.clamp(min=0)]
    placed = has & ((need == 0) | (at + need <= free))
    tok = torch.zeros(n + 1, dtype=torch.int64, device=dev)
    tok[1:] = new.cumsum(0)
    r = torch.repeat_interleave(torch.arange(n, device=dev), torch.where(placed, need, 0))
    col = torch.arange(r.numel(), device=dev) - torch.repeat_interleave(
        torch.where(placed, need, 0).cumsum(0) - torch.where(placed, need, 0), torch.where(placed, need, 0)) + b0[r]
    src = s["base"].long()[replica[r]] + free[r] - 1 - (at[r] + col - b0[r])
    s["table"][r, col] = s["free_list"][src]
    r = torch.repeat_interleave(torch.arange(n, device=dev), new)
    pos = held[r] + torch.arange(r.numel(), device=dev) - tok[r]
    block = s["table"][r, torch.where(placed[r], pos // bs, 0)].long()
    s["slots"][:r.numel()] = torch.where(placed[r], block * bs + pos % bs, -1)
    taken = torch.zeros(R, dtype=torch.int64, device=dev)
    taken.index_add_(0, replica.clamp(min=0), torch.where(placed, need, 0))
    s["placed"].copy_(placed)
    s["tok_base"].copy_(tok)
    s["held_out"].copy_(torch.where(placed, held + new, held))
    s["free_out"].copy_(s["free_count"] - taken)
    return {k: s[k] for k in ("table", "slots", "tok_base", "placed", "held_out", "free_out")}


def _plain_release(s):
    bs, R, replica, held = s["case"]["block"], s["case"]["replicas"], s["replica"].long(), s["held"].long()
    done = (s["done"] != 0) & (replica >= 0)
    blocks = torch.where(done, (held + bs - 1) // bs, 0)
    at, total = _before(replica, blocks, R)
    r = torch.repeat_interleave(torch.arange(replica.numel(), device=replica.device), blocks)
    col = torch.arange(r.numel(), device=replica.device) - (blocks.cumsum(0) - blocks)[r]
    # the last row's last block lands lowest, so that releasing what was just placed restores the list
    q = replica[r]
    dst = s["base"].long()[q] + s["free_count"].long()[q] + total[q] - 1 - (at[r] + col)
    s["free_list"][dst] = s["table"][r, col]
    s["held_out"].copy_(torch.where(done, 0, held))
    s["free_out"].copy_(s["free_count"] + total)
    return {k: s[k] for k in ("free_list", "held_out", "free_out")}


def run(state):
    kind = state["case"]["kind"]
    if not own:
        return {"sample": _plain_sample, "route": _plain_route, "place": _plain_place, "release": _plain_release}[kind](
            state)
    from paper_2502_07903_amd import hx
    if kind == "sample":
        o = hx.sample(state["x"], state["draws"], state["out"], state["params"])
        return dict(pick=o.pick, logp=o.logp, kept=o.kept)
    if kind == "route":
        o = hx.route_requests(state["net"], state["kv_flow"], state["draws"], state["out"], cand=state["cand"])
        return dict(prefill=o.prefill, decode=o.decode, p_order=o.p_order, p_base=o.p_base, d_order=o.d_order,
                    d_base=o.d_base)
    if kind == "place":
        hx.kv_place(state["pool"], state["rows"], state["new"], state["tok_base"], state["slots"], state["placed"],
                    state["workspace"], free_out=state["free_out"], held_out=state["held_out"])
        return {k: state[k] for k in ("table", "slots", "tok_base", "placed", "held_out", "free_out")}
    hx.kv_release(state["pool"], state["rows"], state["done"], state["workspace"], free_out=state["free_out"],
                  held_out=state["held_out"])
    return {k: state[k] for k in ("free_list", "held_out", "free_out")}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    if case["kind"] == "sample":
        n = case["rows"] * case["cols"]
        read = (case["cols"] if case["shared"] else n) * (4 if case["dtype"] in ("i32", "f32") else 2)
        # per entry: the difference from the maximum, its scaling, the exponential, the running sum
        return {"bytes": read + 36 * case["rows"], "flops": 4 * n}
    if case["kind"] == "route":
        edges = case["prefill"] * case["decode"]
        return {"bytes": 4 * edges + 24 * case["requests"] + 4 * (case["prefill"] + case["decode"] + 2),
                "flops": case["requests"] * max(1, math.ceil(math.log2(edges + 1)))}
    rows, bs = case["rows"], case["block"]
    if case["kind"] == "release":
        blocks = 0.9 * rows * math.ceil(max(case["mean_held"], 1) / bs)
        return {"bytes": int(8 * blocks) + 13 * rows + 12 * case["replicas"], "flops": 4 * rows}
    tokens = rows * case["mean_new"]
    return {"bytes": int(8 * tokens + 8 * tokens / bs) + 25 * rows + 12 * case["replicas"], "flops": 4 * rows}


# ------------------------------------------------------------------ from the definitions, on the host

def _exact_sample(s):
    x = s["x"].cpu()
    host = x.float().numpy() if x.dtype != torch.int32 else x.numpy()
    R, N = host.shape
    u64 = s["draws"].cpu().numpy().view(np.uint64)
    par = {k: None if s[k] is None else s[k].cpu().numpy() for k in ("temperature", "top_k", "top_p", "min_p")}
    pick, logp, kept = np.full(R, -1, np.int32), np.full(R, -np.inf), np.zeros(R, np.int32)
    for r in range(R):
        row = host[r].astype(np.float64)
        at = np.flatnonzero(~np.isnan(row) & (row > -np.inf) & (row != I32_MIN))
        if at.size == 0:
            continue
        v, t = row[at], float(par["temperature"][r])
        top = v.max()
        if t == 0:
            pick[r], logp[r], kept[r] = at[v == top][0], 0.0, 1
            continue
        z = np.where(v == top, 0.0, (v - top) / t)
        w = np.exp(z)
        k = at.size
        by = np.arange(k)
        if any(par[q] is not None for q in ("top_k", "top_p", "min_p")):
            by = np.argsort(-v, kind="stable")
        if par["top_k"] is not None and par["top_k"][r] > 0:
            k = min(k, int(par["top_k"][r]))
        n = k
        if par["top_p"] is not None and par["top_p"][r] < 1:
            run_sum = np.cumsum(w[by[:k]], dtype=np.longdouble)
            n = min(n, 1 + int((run_sum < float(par["top_p"][r]) * run_sum[-1]).sum()))
        if par["min_p"] is not None:
            n = max(1, min(n, int((w >= float(par["min_p"][r])).sum())))
        mine = np.sort(by[:n]) if n < at.size else np.arange(n)
        run_sum = np.cumsum(w[mine], dtype=np.longdouble)
        goal = np.longdouble(int(u64[r]) >> 11) * np.longdouble(2.0) ** -53 * run_sum[-1]
        j = mine[int(np.searchsorted(run_sum, goal, side="right"))]
        pick[r], logp[r], kept[r] = at[j], float(z[j] - np.log(run_sum[-1])), n
    return dict(pick=pick, logp=logp, kept=kept)


def _exact_route(s):
    P, D = s["case"]["prefill"], s["case"]["decode"]
    flow = [max(0, int(v)) for v in s["kv_flow"][:, s["cand"]].cpu().tolist()]
    total = sum(flow)
    ends = np.cumsum(np.array(flow, np.int64))
    n = s["case"]["requests"]
    edges = [int(np.searchsorted(ends, ((d & ((1 << 64) - 1)) * total) >> 64, side="right")) if total else -1
             for d in s["draws"].cpu().tolist()]
    lists = {"p": [[] for _ in range(P)], "d": [[] for _ in range(D)]}
    out = dict(prefill=np.full(n, -1, np.int32), decode=np.full(n, -1, np.int32))
    rest = []
    for i, e in enumerate(edges):
        if e < 0:
            rest.append(i)
            continue
        out["prefill"][i], out["decode"][i] = e // D, e % D
        lists["p"][e // D].append(i)
        lists["d"][e % D].append(i)
    for side in "pd":
        out[side + "_order"] = np.array(sum(lists[side], []) + rest, np.int32)
        out[side + "_base"] = np.concatenate([[0], np.cumsum([len(q) for q in lists[side]])]).astype(np.int32)
    return out


def _exact_kv(s):
    c = s["case"]
    bs, n = c["block"], c["rows"]
    h = {k: v.cpu().numpy().copy() for k, v in s.items() if isinstance(v, torch.Tensor)}
    base, free_list, table = h["base"], h["free_list"], h["table"]
    free, held = h["free_count"].astype(np.int64), h["held"].astype(np.int64)
    left, out_held = free.copy(), held.copy()
    if c["kind"] == "release":
        for i in reversed(range(n)):
            r = h["replica"][i]
            if h["done"][i] and r >= 0:
                b = -(-int(held[i]) // bs)
                to = base[r] + left[r]
                free_list[to:to + b] = table[i, :b][::-1]
                left[r] += b
                out_held[i] = 0
        return dict(free_list=free_list, held_out=out_held.astype(np.int32), free_out=left.astype(np.int32))
    tok, slots, placed = np.zeros(n + 1, np.int64), h["slots"], np.zeros(n, np.uint8)
    closed = np.zeros(len(left), bool)  # a replica that has refused a row takes no later row that needs a block
    for i in range(n):
        r, new = h["replica"][i], int(h["new"][i])
        tok[i + 1] = tok[i] + new
        b0, b1 = -(-int(held[i]) // bs), -(-(int(held[i]) + new) // bs)
        if r >= 0 and b1 > b0 and (closed[r] or b1 - b0 > left[r]):
            closed[r] = True
        elif r >= 0:
            top = base[r] + left[r]
            table[i, b0:b1] = free_list[top - (b1 - b0):top][::-1]
            left[r] -= b1 - b0
            placed[i] = 1
            out_held[i] = held[i] + new
            pos = np.arange(held[i], held[i] + new)
            slots[tok[i]:tok[i + 1]] = table[i, pos // bs].astype(np.int64) * bs + pos % bs
            continue
        slots[tok[i]:tok[i + 1]] = -1
    return dict(table=table, slots=slots, tok_base=tok, placed=placed, held_out=out_held.astype(np.int32),
                free_out=left.astype(np.int32))


def exact(case, seed):
    if case["kind"] == "sample" and case["rows"] * case["cols"] > 1 << 26 and (
            case["top_k"] or case["top_p"] or case["min_p"]):
        return None  # a host sort of so many entries takes too long
    s = prepare(case, seed)
    return {"sample": _exact_sample, "route": _exact_route, "place": _exact_kv, "release": _exact_kv}[case["kind"]](s)
