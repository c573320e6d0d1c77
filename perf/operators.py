"""Speculative decoding and a bounded cache over the paged KV cache: what a serving loop pays for them.

Four operators over the cache that the decode step keeps (64-token pages, bf16, grouped-query heads):

  tree      attention of a tree of drafted tokens over the cache (tree_attn): every node attends to the committed
            context and to the drafted nodes that its mask names
  turn      the bookkeeping of one speculative step: ancestor masks and depths of the new trees (tree_build), the path
            that the model's own tokens accept (tree_accept), its keys and values moved to the end of the committed
            context in every layer (tree_commit)
  weighted  dense decode attention that also adds up the attention weight each cached token receives
            (weighted_decode_attn)
  evict     the tokens of least accumulated weight leave the cache, the rest move together in order, keys rotated to
            their new positions (kv_evict)

Shapes are those of perf/cases.py (the repository's workloads) and a generic one with eight query heads per kv-head;
caches and queries are N(0, 1), pages in shuffled order, contexts uniform or lognormal.  `own` false: plain torch forms in
32 bits; true: the calls a program makes through the public binding.
"""
import math
import random
import statistics

import numpy as np
import torch

own = False

DEV = "cuda"
PAGE = 64
VOCAB = 128256
EPS = 1e-5

SHAPES = {
    "tiny": dict(d=256, hq=4, hkv=2, hd=64, ff=1024, theta=0.0),
    "generic": dict(d=768, hq=12, hkv=4, hd=64, ff=2080, theta=10000.0),
    "group8": dict(d=4096, hq=32, hkv=4, hd=128, ff=11008, theta=10000.0),
    "llama1b": dict(d=2048, hq=32, hkv=8, hd=64, ff=8192, theta=500000.0),
    "llama8b": dict(d=4096, hq=32, hkv=8, hd=128, ff=14336, theta=500000.0),
}


def _case(kind, shape="llama1b", batch=1, context=0, sigma=0.0, nodes=0, ragged=0, layers=1, decay=1000, keep=0, sinks=0,
          window=1, name=None):
    c = dict(kind=kind, shape=shape, batch=batch, context=context, sigma=sigma, nodes=nodes, ragged=ragged, layers=layers,
             decay=decay, keep=keep, sinks=sinks, window=window)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one short chat on the smallest model: a chain of launches, nothing to stream
        _case("tree", "tiny", 1, 500, nodes=8, name="tree_tiny"),
        # one user, a long document, a small tree: the cache of one sequence has to be spread over the chip
        _case("tree", "llama8b", 1, 30001, nodes=25, name="tree_single_long"),
        # a small server with a draft head of a few candidates
        _case("tree", "llama1b", 16, 4096, nodes=16, name="tree_batch16"),
        # contexts that differ by two orders of magnitude, trees cut to what each draft was sure of
        _case("tree", "llama1b", 48, 4096, sigma=1.0, nodes=33, ragged=1, name="tree_ragged_batch48"),
        # the largest trees over long contexts, 128-wide heads: a matrix product's worth of rows per cache byte
        _case("tree", "llama8b", 16, 16384, nodes=64, name="tree_8b_batch16"),
        # one user's step: a tree of a few dozen nodes through a 16-layer model
        _case("turn", "llama1b", 1, 1999, nodes=26, layers=16, name="turn_single"),
        # a full server's step, trees of every size
        _case("turn", "llama1b", 64, 700, sigma=0.7, nodes=64, ragged=1, layers=16, name="turn_batch64"),
        # one user's decode step with the weights kept
        _case("weighted", "llama1b", 1, 8191, name="weighted_single"),
        # a full server batch, weights that fade
        _case("weighted", "llama1b", 128, 4096, sigma=1.0, decay=990, name="weighted_ragged_batch128"),
        # the larger model at long contexts
        _case("weighted", "llama8b", 64, 16384, name="weighted_8b_batch64"),
        # a quarter of the cache stays: a few sinks, the last 128 tokens and the heavy ones
        _case("evict", "llama1b", 16, 4096, keep=250, sinks=4, window=128, name="evict_quarter_batch16"),
        # long ragged contexts of the larger model, half of each stays
        _case("evict", "llama8b", 24, 9000, sigma=0.8, keep=500, sinks=4, window=2, name="evict_half_8b_ragged"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tree", "tree", "tree", "turn", "weighted", "weighted", "evict", "evict"])
    shape = rng.choice(["tiny", "generic", "group8", "llama1b", "llama1b", "llama8b", "llama8b"])
    S = SHAPES[shape]
    if kind == "turn":
        return _case(kind, shape, _log(rng, 1, 128), _log(rng, 1, 900), rng.choice([0.0, 0.7]), _log(rng, 1, 64),
                     rng.randint(0, 1), rng.randint(1, 16 if S["hd"] == 64 else 8))
    sigma = rng.choice([0.0, 0.5, 1.0])
    batch = _log(rng, 1, 128)
    room = 1e9 / (batch * S["hkv"] * S["hd"] * 4 * math.exp(sigma * sigma / 2))  # at most 1 GB of cache
    context = max(33, min(_log(rng, 33, 24000), int(room)))
    c = _case(kind, shape, batch, context, sigma)
    if kind == "tree":
        c.update(nodes=_log(rng, 1, 64), ragged=rng.randint(0, 1))
    if kind == "weighted":
        c.update(decay=rng.choice([1000, 1000, 990, 900]))
    if kind == "evict":
        c.update(keep=rng.randint(20, 980), sinks=rng.choice([0, 4, 16]), window=rng.choice([1, 2, 32, 128]))
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
_NAMES = ("k", "v", "q", "weights", "pages", "trees")


def _generator(seed, name):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + _NAMES.index(name))
    return g


def _normal(seed, name, shape):
    return torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=_generator(seed, name))


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).to(DEV)


def _lengths(c):
    """Committed context lengths: the middles of B equal shares of the distribution, shortest first."""
    B, T = c["batch"], c["context"]
    if not c["sigma"]:
        return [T] * B
    z = [statistics.NormalDist().inv_cdf((i + 0.5) / B) for i in range(B)]
    return [max(min(T, 256), min(32768, int(round(T * math.exp(c["sigma"] * x))))) for x in z]


def _node_counts(c):
    """Drafted nodes of each sequence: all alike, or one to all of them in an order that no length follows."""
    B, N = c["batch"], c["nodes"]
    return [1 + (11 * i + 5) % N for i in range(B)] if c["ragged"] else [N] * B


def _accepted(c):
    """Nodes of each sequence that get accepted, the root among them: about a fifth of a tree, eight at most."""
    return [1 + (5 * i + 3) % max(1, min(8, -(-n // 4))) for i, n in enumerate(_node_counts(c))]


def _kept(c):
    """Tokens of each sequence that stay: the budget, the sinks and the window at least."""
    budget = [max(1, n * c["keep"] // 1000) for n in _lengths(c)]
    forced = [min(c["sinks"], n) + min(c["window"], n - min(c["sinks"], n)) for n in _lengths(c)]
    return budget, [min(n, max(b, f)) for n, b, f in zip(_lengths(c), budget, forced)]


def _trees(c, seed):
    """Parents, drafted tokens and the model's own tokens: random trees in which a random chain from the root is right."""
    rng = random.Random(int(seed) * 7 + 3)
    N = c["nodes"]
    parents, draft, target = (np.full((c["batch"], N), -1, np.int32) for _ in range(3))
    for b, (n, a) in enumerate(zip(_node_counts(c), _accepted(c))):
        chain = [0] + sorted(rng.sample(range(1, n), a - 1))
        tokens = rng.sample(range(VOCAB), n + 1)
        place = {node: j for j, node in enumerate(chain)}
        for i in range(n):
            parents[b, i] = -1 if i == 0 else chain[place[i] - 1] if i in place else rng.randrange(max(0, i - 12), i)
            draft[b, i] = tokens[i]
            target[b, i] = rng.randrange(VOCAB)
        for j, node in enumerate(chain):
            target[b, node] = tokens[chain[j + 1]] if j + 1 < a else tokens[n]
    return parents, draft, target


def _masks(parents):
    """The ancestors of each node, itself among them, as 64-bit masks."""
    out = np.zeros(parents.shape, np.uint64)
    for b, row in enumerate(parents):
        for i, p in enumerate(row):
            if i == 0 or p >= 0:
                out[b, i] = (out[b, p] if p >= 0 else np.uint64(0)) | (np.uint64(1) << np.uint64(i))
    return out.view(np.int64)


def prepare(case, seed):
    c, S = case, SHAPES[case["shape"]]
    B, N = c["batch"], c["nodes"]
    lens = _lengths(c)
    full = [n + m for n, m in zip(lens, _node_counts(c))] if N else lens
    need = [-(-n // PAGE) for n in full]
    max_pages, used = max(need), sum(need)
    spare = [-(-n // PAGE) for n in _kept(c)[1]] if c["kind"] == "evict" else [0] * B
    order = torch.randperm(used + sum(spare), generator=_generator(seed, "pages"), device=DEV).int().cpu().numpy()
    table, dst_table = np.full((B, max_pages), -1, np.int32), np.full((B, max_pages), -1, np.int32)
    at = 0
    for t, counts in ((table, need), (dst_table, spare)):
        for b, n in enumerate(counts):
            t[b, :n] = order[at:at + n]
            at += n
    pages = used + sum(spare)
    pool = (c["layers"], pages, S["hkv"], PAGE, S["hd"])
    s = dict(case=dict(c), B=B, N=N, max_pages=max_pages, pages=pages, table=_i32(table), lens=_i32(full),
             k=_normal(seed, "k", pool), v=_normal(seed, "v", pool))
    if N:
        parents, draft, target = _trees(c, seed)
        s["n_nodes"] = _i32(_node_counts(c))
    if c["kind"] == "tree":
        s["mask"] = torch.from_numpy(_masks(parents)).to(DEV)
        s["q"] = _normal(seed, "q", (B, N, S["hq"], S["hd"]))
        s["out"] = torch.zeros_like(s["q"])
    if c["kind"] == "turn":
        s.update(parents=_i32(parents), draft=_i32(draft), target=_i32(target))
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=DEV)  # noqa: E731
        s.update(mask=torch.zeros((B, N), dtype=torch.int64, device=DEV), depth=i32(B, N), path=i32(B, N), path_len=i32(B),
                 next_token=i32(B), new_lens=i32(B))
    if c["kind"] == "weighted":
        s["q"] = _normal(seed, "q", (B, S["hq"], S["hd"]))
        s["out"] = torch.zeros_like(s["q"])
    if c["kind"] in ("weighted", "evict"):  # what a few hundred steps leave: a heavy tail, tokens that nobody looked at
        x = torch.empty((B, S["hkv"], max_pages * PAGE), device=DEV).normal_(0.0, 1.0, generator=_generator(seed, "weights"))
        s["weights"] = torch.where(x < -1.3, 0.0, torch.exp(1.5 * x))
    if c["kind"] == "evict":
        s.update(budgets=_i32(_kept(c)[0]), dst_table=_i32(dst_table), dst_weights=torch.zeros_like(s["weights"]),
                 dst_lens=torch.zeros(B, dtype=torch.int32, device=DEV),
                 kept_idx=torch.full((B, S["hkv"], max_pages * PAGE), -1, dtype=torch.int32, device=DEV))
    if own:
        _handle(s)
    return s


# ---------------------------------------------------------------------------
# the framework's operators
# ---------------------------------------------------------------------------
def _handle(s):
    """What a serving program keeps beside its cache: the shape, the descriptors and a workspace."""
    from paper_2605_10875_b200 import binding as sol

    c, S = s["case"], SHAPES[s["case"]["shape"]]
    s["shape"] = sol.make_shape(S["d"], S["hq"], S["hkv"], S["hd"], S["ff"], PAGE, EPS, S["theta"], c["sinks"], c["window"])
    s["kvs"] = [sol.make_kv(s["k"][x], s["v"][x], s["table"], s["lens"], s["max_pages"], s["pages"]) for x in range(c["layers"])]
    if s["N"]:
        s["tree"] = sol.make_tree(s["N"], s["n_nodes"], s["mask"])
    if c["kind"] == "tree":
        s["ws_bytes"] = sol.tree_workspace_bytes(s["shape"], s["B"], s["max_pages"], s["N"])
    else:
        s["ws_bytes"] = 256 if c["kind"] == "turn" else sol.workspace_bytes(s["shape"], s["B"], s["max_pages"])
    s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device=DEV)
    sol.workspace_init(s["ws"], s["ws_bytes"], torch.cuda.current_stream())
    s["sol"] = sol


def _run_own(s):
    sol, c, B, st = s["sol"], s["case"], s["B"], torch.cuda.current_stream()
    if c["kind"] == "tree":
        sol.tree_attn(s["shape"], s["q"], s["kvs"][0], s["tree"], B, s["out"], s["ws"], s["ws_bytes"], st)
        return {"out": s["out"]}
    if c["kind"] == "turn":
        sol.tree_build(B, s["N"], s["n_nodes"], s["parents"], s["mask"], s["depth"], st)
        sol.tree_accept(B, s["N"], s["n_nodes"], s["parents"], s["draft"], s["target"], s["path"], s["path_len"],
                        s["next_token"], st)
        sol.tree_commit(s["shape"], s["kvs"], s["tree"], B, s["path"], s["path_len"], s["new_lens"], s["ws"], st)
        return {n: s[n] for n in ("mask", "depth", "path", "path_len", "next_token", "new_lens", "k", "v")}
    if c["kind"] == "weighted":
        sol.weighted_decode_attn(s["shape"], s["q"], s["kvs"][0], B, c["decay"] / 1000.0, s["weights"], s["out"], s["ws"],
                                 s["ws_bytes"], st)
        return {"out": s["out"], "weights": s["weights"]}
    sol.kv_evict(s["shape"], s["kvs"][0], B, s["budgets"], s["weights"], s["dst_table"], s["dst_weights"], s["dst_lens"],
                 s["kept_idx"], s["ws"], s["ws_bytes"], st)
    return {n: s[n] for n in ("kept_idx", "dst_lens", "dst_weights", "k", "v")}


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _cached(pool, table):
    """[B][heads][T][hd] float32: the sequences' rows in order, T slots of pages each."""
    x = pool[table.clamp(min=0).long()]  # [B][pages][heads][PAGE][hd]
    return x.transpose(1, 2).flatten(2, 3).float()


def _softmax_parts(scores, seen):
    """exp(score - row maximum) where seen, else 0, and the row sums."""
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    return p, p.sum(-1, keepdim=True)


def _attend(s, q, seen):
    """q [B][heads][group][rows][hd] float32, seen [B][1][1][rows][T]: outputs and weights."""
    K, V = _cached(s["k"][0], s["table"]), _cached(s["v"][0], s["table"])
    there = torch.arange(K.shape[2], device=DEV) < s["lens"][:, None]
    V = V.masked_fill(~there[:, None, :, None], 0.0)  # slots behind a sequence hold anything
    B, H, G, R, hd = q.shape
    scores = (q.reshape(B, H, G * R, hd) @ K.transpose(2, 3)).view(B, H, G, R, -1) / math.sqrt(hd)
    p, total = _softmax_parts(scores, seen)
    p = torch.where(total > 0, p / total, 0.0)
    return (p.view(B, H, G * R, -1) @ V).view(B, H, G, R, hd), p


def _plain_tree(s):
    S = SHAPES[s["case"]["shape"]]
    B, N, H, hd = s["B"], s["N"], S["hkv"], S["hd"]
    G = S["hq"] // H
    t = torch.arange(s["max_pages"] * PAGE, device=DEV)
    first = (s["lens"] - s["n_nodes"])[:, None]  # slot of node 0
    node = (t - first).clamp(0, 63)  # [B][T]
    named = ((s["mask"][:, :, None] >> node[:, None, :]) & 1).bool() & (t < s["lens"][:, None])[:, None, :]
    seen = (t < first)[:, None, :] | named  # [B][N][T]
    q = s["q"].float().view(B, N, H, G, hd).permute(0, 2, 3, 1, 4)
    o, _ = _attend(s, q, seen[:, None, None])
    o = o.permute(0, 3, 1, 2, 4).reshape(B, N, S["hq"], hd).to(torch.bfloat16)
    real = (torch.arange(N, device=DEV) < s["n_nodes"][:, None])[:, :, None, None]
    s["out"].copy_(torch.where(real, o, s["out"]))
    return {"out": s["out"]}


def _plain_turn(s):
    B, N, L = s["B"], s["N"], s["case"]["layers"]
    i = torch.arange(N, device=DEV)
    real = i < s["n_nodes"][:, None]
    up = s["parents"].clamp(min=0).long()
    child = (s["parents"][:, :, None] == i) & real[:, :, None]  # [B][node][its parent]
    anc = (child | (torch.eye(N, device=DEV, dtype=torch.bool) & real[:, :, None])).float()
    for _ in range(6):  # ancestors up to 2, 4, ... 64 steps away
        anc = (anc @ anc > 0).float()
    anc = anc > 0
    s["mask"].copy_(torch.where(real, (anc.long() << i).sum(-1), s["mask"]))
    s["depth"].copy_(torch.where(real, anc.sum(-1).int() - 1, s["depth"]))
    # a node is right if its token is the one that the model puts after its parent, and no earlier sibling is
    right = (s["draft"] == s["target"].gather(1, up)) & (s["parents"] >= 0) & real
    rank = (child & right[:, :, None]).long().cumsum(1).gather(2, up[:, :, None]).squeeze(2)
    good = (right & (rank == 1)) | ((i == 0) & real)
    on_path = (~anc | good[:, None, :]).all(-1) & real
    count = on_path.sum(-1).int()
    place = torch.where(on_path, i, N).sort(-1).values
    s["path"].copy_(torch.where(i < count[:, None], place.int(), s["path"]))
    s["path_len"].copy_(count)
    last = torch.where(on_path, i, 0).amax(-1, keepdim=True)
    s["next_token"].copy_(s["target"].gather(1, last).squeeze(1))
    first = s["lens"] - s["n_nodes"]
    s["new_lens"].copy_(first + count)
    moved = i < count[:, None]
    src = (first[:, None] + torch.where(moved, s["path"], 0)).long()
    dst = (first[:, None] + torch.where(moved, i, 0)).long()  # rows past the path: the root onto itself
    page = lambda slot: s["table"].gather(1, slot // PAGE).long()  # noqa: E731
    at = torch.arange(L, device=DEV)[:, None, None]
    for pool in (s["k"], s["v"]):
        rows = pool.transpose(2, 3)  # [layers][pages][PAGE][heads][hd]
        rows[at, page(dst), dst % PAGE] = rows[at, page(src), src % PAGE]
    return {n: s[n] for n in ("mask", "depth", "path", "path_len", "next_token", "new_lens", "k", "v")}


def _plain_weighted(s):
    c, S = s["case"], SHAPES[s["case"]["shape"]]
    B, H, hd = s["B"], S["hkv"], S["hd"]
    t = torch.arange(s["max_pages"] * PAGE, device=DEV)
    last = s["lens"][:, None] - 1
    q = s["q"].float().view(B, H, S["hq"] // H, 1, hd)
    o, p = _attend(s, q, (t <= last)[:, None, None, None])
    s["out"].copy_(o.reshape(B, S["hq"], hd))
    got = p.sum((2, 3))  # [B][heads][T]
    new = torch.where((t == last)[:, None], got, s["weights"] * (c["decay"] / 1000.0) + got)
    s["weights"].copy_(torch.where((t <= last)[:, None], new, s["weights"]))
    return {"out": s["out"], "weights": s["weights"]}


def _plain_evict(s):
    c, S = s["case"], SHAPES[s["case"]["shape"]]
    H, hd = S["hkv"], S["hd"]
    T = s["max_pages"] * PAGE
    t = torch.arange(T, device=DEV)
    lens = s["lens"][:, None]
    sinks = lens.clamp(max=c["sinks"])
    window = (lens - sinks).clamp(max=c["window"])
    forced = (t < sinks) | ((t >= lens - window) & (t < lens))
    count = torch.minimum(torch.maximum(s["budgets"][:, None], sinks + window), lens)[:, :, None]  # [B][1][1]
    score = torch.where(forced[:, None], math.inf, s["weights"]).masked_fill((t >= lens)[:, None], -math.inf)
    order = score.sort(dim=-1, descending=True, stable=True).indices
    keep = torch.zeros_like(score, dtype=torch.bool).scatter_(2, order, (t < count).expand_as(score))
    kept = torch.where(keep, t, T).sort(-1).values  # [B][H][T]: kept tokens in order, then T
    live = t < count
    s["kept_idx"].copy_(torch.where(live, kept.int(), s["kept_idx"]))
    s["dst_lens"].copy_(count.flatten())
    old = torch.where(live, kept, 0)
    s["dst_weights"].copy_(torch.where(live, s["weights"].gather(2, old), s["dst_weights"]))
    new = torch.where(live, t, 0)
    old = torch.where(live, old, old[:, :, :1])  # rows past the last: the first one again
    page = lambda table, slot: table[:, None].expand(-1, H, -1).gather(2, slot // PAGE).long()  # noqa: E731
    h = torch.arange(H, device=DEV)[:, None]
    src, dst = (page(s["table"], old), h, old % PAGE), (page(s["dst_table"], new), h, new % PAGE)
    K, V = s["k"][0], s["v"][0]
    V[dst] = V[src]
    if not S["theta"]:
        K[dst] = K[src]
    else:
        x = K[src].float()
        half = hd // 2
        speed = S["theta"] ** (-2.0 * torch.arange(half, device=DEV, dtype=torch.float64) / hd)
        angle = torch.remainder((new - old)[..., None].double() * speed, 2 * math.pi)
        cos, sin = angle.cos().float(), angle.sin().float()
        lo, hi = x[..., :half], x[..., half:]
        K[dst] = torch.cat((lo * cos - hi * sin, hi * cos + lo * sin), -1).to(torch.bfloat16)
    return {n: s[n] for n in ("kept_idx", "dst_lens", "dst_weights", "k", "v")}


_PLAIN = {"tree": _plain_tree, "turn": _plain_turn, "weighted": _plain_weighted, "evict": _plain_evict}


def run(state):
    if own:
        return _run_own(state)
    return _PLAIN[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------
# the least a pass has to move and compute
# ---------------------------------------------------------------------------
def work(case):
    c, S = case, SHAPES[case["shape"]]
    row, lens = S["hd"] * 2, _lengths(c)
    G = S["hq"] // S["hkv"]
    if c["kind"] == "turn":
        moves = sum(a - 1 for a in _accepted(c)) * c["layers"] * S["hkv"]
        nodes = sum(_node_counts(c))
        return {"bytes": moves * row * 4 + nodes * (3 * 4 + 8 + 4) + sum(_accepted(c)) * 4 + c["batch"] * 20, "flops": 0}
    if c["kind"] == "evict":
        kept = sum(_kept(c)[1]) * S["hkv"]
        return {"bytes": kept * (row * 4 + 12) + sum(lens) * S["hkv"] * 4, "flops": kept * S["hd"] * 3}
    rows = [G * n for n in _node_counts(c)] if c["kind"] == "tree" else [G] * c["batch"]
    full = [n + m for n, m in zip(lens, _node_counts(c))] if c["kind"] == "tree" else lens
    cells = sum(full) * S["hkv"]
    got = {"bytes": cells * row * 2 + sum(rows) * S["hkv"] * row * 2,
           "flops": sum(r * n for r, n in zip(rows, full)) * S["hkv"] * S["hd"] * 4}
    if c["kind"] == "weighted":
        got["bytes"] += cells * 8
    return got


# ---------------------------------------------------------------------------
# the definitions, in 64 bits, a sequence at a time
# ---------------------------------------------------------------------------
def _rows(pool, pages, n):
    """[heads][n][hd] float64: the first n tokens of a sequence."""
    x = pool[pages[: -(-n // PAGE)].long()]
    return x.permute(1, 0, 2, 3).reshape(pool.shape[1], -1, pool.shape[3])[:, :n].double()


def _exact_tree(s):
    S = SHAPES[s["case"]["shape"]]
    H, G, hd, N = S["hkv"], S["hq"] // S["hkv"], S["hd"], s["N"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    for b, (T, n) in enumerate(zip(s["lens"].tolist(), s["n_nodes"].tolist())):
        K, V = _rows(s["k"][0], s["table"][b], T), _rows(s["v"][0], s["table"][b], T)
        named = torch.tensor([[(m >> j) & 1 for j in range(n)] for m in s["mask"][b, :n].tolist()], device=DEV).bool()
        q = s["q"][b, :n].double().view(n, H, G, hd)
        scores = torch.einsum("nhgd,htd->hgnt", q, K) * hd ** -0.5
        scores[..., T - n:] = torch.where(named, scores[..., T - n:], -math.inf)
        out[b, :n] = torch.einsum("hgnt,htd->nhgd", scores.softmax(-1), V).reshape(n, S["hq"], hd)
    return {"out": out}


def _exact_weighted(s):
    c, S = s["case"], SHAPES[s["case"]["shape"]]
    H, G, hd = S["hkv"], S["hq"] // S["hkv"], S["hd"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    weights = s["weights"].double()
    for b, T in enumerate(s["lens"].tolist()):
        q = s["q"][b].double().view(H, G, hd)
        p = (torch.einsum("hgd,htd->hgt", q, _rows(s["k"][0], s["table"][b], T)) / math.sqrt(hd)).softmax(-1)
        out[b] = torch.einsum("hgt,htd->hgd", p, _rows(s["v"][0], s["table"][b], T)).reshape(S["hq"], hd)
        weights[b, :, : T - 1] *= c["decay"] / 1000.0
        weights[b, :, T - 1] = 0.0
        weights[b, :, :T] += p.sum(1)
    return {"out": out, "weights": weights}


def _exact_evict(s):
    c, S = s["case"], SHAPES[s["case"]["shape"]]
    H, hd, half = S["hkv"], S["hd"], S["hd"] // 2
    k, v, dst_weights = s["k"].double(), s["v"].double(), s["dst_weights"].double()
    for b, (T, count) in enumerate(zip(_lengths(c), _kept(c)[1])):
        w = s["weights"][b, :, :T].double()
        first = min(c["sinks"], T)
        w[:, :first] = w[:, max(first, T - c["window"]):] = math.inf
        # rank by weight, then by index: argsort of the negated weights keeps the order of equal ones
        kept = torch.argsort(-w, dim=1, stable=True)[:, :count].sort(1).values  # [H][count]
        t = torch.arange(count, device=DEV)
        dst_weights[b, :, :count] = s["weights"][b].double().gather(1, kept)
        K, V = _rows(s["k"][0], s["table"][b], T), _rows(s["v"][0], s["table"][b], T)
        take = kept[:, :, None].expand(-1, -1, hd)
        K, V = K.gather(1, take), V.gather(1, take)
        if S["theta"]:
            turns = torch.exp(torch.arange(half, device=DEV).double() * (-2.0 / hd) * math.log(S["theta"]))
            z = torch.complex(K[..., :half], K[..., half:])
            a = (t - kept)[..., None].double() * turns
            z = z * torch.complex(torch.cos(a), torch.sin(a))
            K = torch.cat((z.real, z.imag), -1)
        pages = s["dst_table"][b].long()[t // PAGE]
        k[0, pages, :, t % PAGE] = K.transpose(0, 1)
        v[0, pages, :, t % PAGE] = V.transpose(0, 1)
    return {"kept_idx": None, "dst_lens": None, "dst_weights": dst_weights, "k": k, "v": v}


def _exact_turn(s):
    """The walk from the root, node by node; only the moved rows are numbers to compare."""
    k, v = s["k"].double(), s["v"].double()
    lens, table = s["lens"].tolist(), s["table"].cpu()
    parents, draft, target = (s[n].cpu().numpy() for n in ("parents", "draft", "target"))
    for b, n in enumerate(s["n_nodes"].tolist()):
        path = [0]
        while True:
            hits = [i for i in range(n) if parents[b, i] == path[-1] and draft[b, i] == target[b, path[-1]]]
            if not hits:
                break
            path.append(hits[0])
        src, dst = (torch.tensor([lens[b] - n + j for j in js]) for js in (path, range(len(path))))
        for pool in (k, v):
            rows = pool[:, table[b][src // PAGE].long(), :, src % PAGE]
            pool[:, table[b][dst // PAGE].long(), :, dst % PAGE] = rows
    return {"k": k, "v": v}


def exact(case, seed):
    s = prepare(case, seed)
    return {"tree": _exact_tree, "turn": _exact_turn, "weighted": _exact_weighted, "evict": _exact_evict}[case["kind"]](s)
