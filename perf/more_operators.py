"""Performance cases of drafted trees over a fork's K/V cache: each branch has a tree of drafted tokens
checked in one pass over the shared prefix, instead of one token a pass.

A case is one of four kinds of work:

* ``layout``: from each node's parent, which nodes it sees and its position (``tree_layout``).
* ``attend``: attention of every node over the shared prefix, its branch's suffix and the nodes it sees
  (``Plan.tree_attend``, ``Plan.tree_attend_paged``).
* ``sample``: the token that temperature, top-k, top-p and min-p leave for a given random number
  (``sample``).
* ``accept``: the drafted nodes that the chosen tokens confirm, their K/V rows moved behind the suffix
  (``tree_accept``, ``tree_accept_paged``).

``run`` computes the plain form in elementary torch operations, or, where ``own`` is true, calls the
library.  Lengths and tree shapes come from the case (``len_seed``), values from the seed: N(0, 1) queries,
keys and values, keys scaled per (KV head, channel) by a LogNormal(0, 0.5) factor, in bf16.
"""
import math
import random

import torch

own = False

PAGE = 16
UNIT = 2.0 ** 44  # the largest weight of a row: weights are whole numbers of its 2^-44


def _case(name, kind, **more):
    c = dict(kind=kind, **more)
    if name:
        c["name"] = name
    return c


def _attend(name, hq, hkv, d, branches, nodes, prefix, suffix, *, paged=False, len_seed=1):
    return _case(name, "attend", hq=hq, hkv=hkv, d=d, branches=branches, nodes=nodes, prefix=prefix, suffix_lo=suffix[0],
                 suffix_hi=suffix[1], paged=paged, len_seed=len_seed)


def _accept(name, hkv, d, branches, nodes, suffix, *, paged=False, len_seed=1):
    return _case(name, "accept", hkv=hkv, d=d, branches=branches, nodes=nodes, suffix_lo=suffix[0], suffix_hi=suffix[1],
                 paged=paged, len_seed=len_seed)


def listed():
    return [
        # the trees of one step of a fork: latency
        _case("layout-step", "layout", branches=5, nodes=16, len_seed=1),
        # a server's batch of trees, the largest trees
        _case("layout-batch", "layout", branches=512, nodes=64, len_seed=2),
        # the smallest fork: head dim 64, a short context; launches and latency
        _attend("tree-tiny", 8, 2, 64, 5, 8, 512, (0, 64)),
        # nothing drafted: one token a branch at the 32k context
        _attend("tree-single", 40, 8, 128, 5, 1, 32768, (512, 2048)),
        # the usual draft: 16 nodes a branch at the 32k context
        _attend("tree-long", 40, 8, 128, 5, 16, 32768, (512, 2048)),
        # an odd tree over a page pool, a context that ends inside a page
        _attend("tree-paged", 32, 8, 128, 4, 13, 23017, (0, 700), paged=True),
        # the largest trees: 64 nodes a branch
        _attend("tree-wide", 40, 8, 128, 5, 64, 32768, (512, 2048)),
        # one token for each branch: latency
        _case("sample-step", "sample", rows=5, vocab=32000, bf16=True, filters="mixed"),
        # a token for every node of the largest trees
        _case("sample-nodes", "sample", rows=320, vocab=128000, bf16=False, filters="mixed"),
        # a batch's rows over a large odd vocabulary, nothing filtered
        _case("sample-plain", "sample", rows=80, vocab=200003, bf16=True, filters="none"),
        # the accepted nodes of one step, contiguous suffixes
        _accept("accept-step", 8, 128, 5, 16, (512, 2048)),
        # a server's batch on a page pool
        _accept("accept-paged", 8, 128, 80, 64, (0, 700), paged=True, len_seed=2),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["layout", "attend", "attend", "attend", "sample", "sample", "accept"])
    seed = rng.randrange(1 << 20)
    if kind == "layout":
        return _case(None, kind, branches=_log_uniform(rng, 1, 512), nodes=rng.randint(1, 64), len_seed=seed)
    if kind == "sample":
        rows = _log_uniform(rng, 1, 320)
        return _case(None, kind, rows=rows, vocab=_log_uniform(rng, 1000, min(262144, 320 * 128000 // rows)), bf16=rng.random() < 0.5,
                     filters=rng.choice(["mixed", "mixed", "none"]))
    d, hkv = rng.choice([64, 128, 128]), rng.choice([2, 4, 8, 8])
    paged, low = rng.random() < 0.5, rng.randint(0, 256)
    suffix = low, low + _log_uniform(rng, 1, 1700)
    if kind == "accept":
        return _accept(None, hkv, d, _log_uniform(rng, 1, 80), rng.randint(1, 64), suffix, paged=paged, len_seed=seed)
    group = rng.choice([1, 4, 5, 5, 7, 8])
    branches = rng.randint(1, 8)
    nodes = _log_uniform(rng, 1, 64)
    prefix = _log_uniform(rng, 100, min(65536, 320 * 5 * 32768 // (branches * nodes * group)))
    return _attend(None, hkv * group, hkv, d, branches, nodes, prefix, suffix, paged=paged, len_seed=seed)


def _suffixes(c):
    """Committed suffix length of each branch."""
    r = random.Random(c["len_seed"])
    return [r.randint(c["suffix_lo"], c["suffix_hi"]) for _ in range(c["branches"])]


def _trees(c):
    """Each branch's parents: node 0 the root, the others behind one of the eight nodes before them, some places unused."""
    r = random.Random(c["len_seed"] + 1)
    trees = []
    for _ in range(c["branches"]):
        used = [0]
        parents = [-1]
        for i in range(1, c["nodes"]):
            if r.random() < 0.05:
                parents.append(-1)
            else:
                parents.append(r.choice(used[-8:]))
                used.append(i)
        trees.append(parents)
    return trees


def _masks(trees):
    """The nodes that each node sees, itself among them, as the bits of an int64 [branches, nodes]."""
    rows = []
    for parents in trees:
        m = []
        for i, a in enumerate(parents):
            m.append(1 << i | (m[a] if a >= 0 else 0))
        rows.append([x - (1 << 64) if x >> 63 else x for x in m])
    return torch.tensor(rows, dtype=torch.int64)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731

    def whole(high, *shape):
        return torch.randint(high, shape, generator=gen, device="cuda", dtype=torch.int32)

    s = {"case": c}
    if c["kind"] == "layout":
        b, n = c["branches"], c["nodes"]
        # other inputs for another seed: the trees in another order, other positions
        s["parents"] = i32(_trees(c))[torch.randperm(b, generator=gen, device="cuda")].contiguous()
        s["base"] = whole(130000, b)
        s["masks"] = torch.empty(b, n, dtype=torch.int64, device="cuda")
        s["positions"] = torch.empty(b, n, dtype=torch.int32, device="cuda")
        return s
    if c["kind"] == "sample":
        r, v = c["rows"], c["vocab"]
        # a few likely tokens over a wide bulk, as a model's last layer gives them
        x = torch.randn(r, v, generator=gen, device="cuda") * 2.5
        for likely in (3, 12, 50):
            at = torch.randint(v, (r, likely), generator=gen, device="cuda")
            x.scatter_add_(1, at, 8 + 3 * torch.randn(r, likely, generator=gen, device="cuda"))
        s["logits"] = x.bfloat16() if c["bf16"] else x
        s["u"] = torch.rand(r, generator=gen, device="cuda")
        s["temperature"] = 0.3 + 1.2 * torch.rand(r, generator=gen, device="cuda")
        s["top_k"] = s["top_p"] = s["min_p"] = None
        if c["filters"] == "mixed":
            pick = lambda of: torch.tensor(of, device="cuda")[whole(len(of), r).long()]  # noqa: E731
            s["temperature"] = torch.where(torch.rand(r, generator=gen, device="cuda") < 0.1, 0.0, s["temperature"])
            s["top_k"] = pick([0, 0, 1, 20, 50, 1000]).int()
            s["top_p"] = pick([1.0, 0.5, 0.9, 0.95])
            s["min_p"] = pick([0.0, 0.0, 0.02, 0.1])
        s["tokens"] = torch.empty(r, dtype=torch.int32, device="cuda")
        s["logprob"] = torch.empty(r, device="cuda")
        s["workspace"] = None
        if own:
            from paper_2608_13667_amd import forkattn as fa
            s["workspace"] = fa.sample_workspace(r, v)
        return s

    hkv, d, b, n = c["hkv"], c["d"], c["branches"], c["nodes"]
    scale = torch.exp(0.5 * torch.randn(hkv, 1, d, generator=gen, device="cuda")).bfloat16()

    def values(*shape):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16)

    def keys(*shape):
        return values(*shape).mul_(scale)

    prefix, suffix, trees = c.get("prefix", 0), _suffixes(c), _trees(c)
    cap = max(suffix) + n
    s["lens"], s["masks"] = i32(suffix), _masks(trees).cuda()
    if c["paged"]:
        shared, each = -(-prefix // PAGE), -(-cap // PAGE)
        ids = torch.randperm(shared + b * each + 3, generator=gen, device="cuda").to(torch.int32)
        s["table"] = torch.cat([ids[:shared].expand(b, shared), ids[shared: shared + b * each].view(b, each)], 1).contiguous()
        s["k_pool"], s["v_pool"] = keys(len(ids), hkv, PAGE, d), values(len(ids), hkv, PAGE, d)
        s["prefix_len"] = i32([prefix] * b)
    else:
        s["prefix_k"], s["prefix_v"] = keys(hkv, prefix, d), values(hkv, prefix, d)
        s["suffix_k"], s["suffix_v"] = keys(b, hkv, cap, d), values(b, hkv, cap, d)
    if c["kind"] == "accept":
        s["parents"] = i32(trees)
        s["targets"] = whole(32000, b, n)
        # a drafted token is often the one chosen behind its parent
        chosen = torch.gather(s["targets"], 1, s["parents"].long().clamp(min=0))
        s["tokens"] = torch.where(torch.rand(b, n, generator=gen, device="cuda") < 0.5, chosen, whole(32000, b, n))
        s["path"] = torch.empty(b, n, dtype=torch.int32, device="cuda")
        s["count"], s["next"] = (torch.empty(b, dtype=torch.int32, device="cuda") for _ in "cn")
        return s
    s["q"] = values(b, n, c["hq"], d)
    s["out"] = torch.empty(b, n, c["hq"], d, device="cuda")
    s["lse"] = torch.empty(b, n, c["hq"], device="cuda")
    s["plan"] = None
    if own:
        from paper_2608_13667_amd import forkattn as fa
        if c["paged"]:
            s["plan"] = fa.Plan.tree_paged_plan(c["hq"], hkv, d, b, n, prefix, s["table"].shape[1], s["k_pool"].shape[0], cap)
        else:
            s["plan"] = fa.Plan.tree_plan(c["hq"], hkv, d, b, n, prefix, cap, cap)
    return s


# ------------------------------------------------------------------------------------------- plain forms

def _bits(masks, n):
    """[branches, nodes] int64 -> truth values [branches, nodes, n]."""
    return (masks[..., None] >> torch.arange(n, device="cuda") & 1).bool()


def _run_layout(s):
    if own:
        from paper_2608_13667_amd import forkattn as fa
        fa.tree_layout(s["parents"], s["base"], s["masks"], s["positions"])
        return {"masks": s["masks"], "positions": s["positions"]}
    a = s["parents"].long()
    n = a.shape[1]
    at = torch.arange(n, device="cuda")
    step = (a[..., None] == at) & (a < at)[..., None]
    reach = (step | torch.eye(n, dtype=torch.bool, device="cuda")).float()
    # six squarings: behind one node are at most 63 others
    reach = ((reach @ reach) > 0).float()
    reach = ((reach @ reach) > 0).float()
    reach = ((reach @ reach) > 0).float()
    reach = ((reach @ reach) > 0).float()
    reach = ((reach @ reach) > 0).float()
    reach = (reach @ reach) > 0
    s["masks"].copy_((reach.long() << at).sum(-1))
    s["positions"].copy_(s["base"][:, None] + reach.sum(-1) - 1)
    return {"masks": s["masks"], "positions": s["positions"]}


def _cache(s):
    """Prefix [hkv, prefix, d] and suffixes [b, hkv, cap, d] of K and of V."""
    if not s["case"]["paged"]:
        return (s["prefix_k"], s["prefix_v"]), (s["suffix_k"], s["suffix_v"])
    prefix = s["case"].get("prefix", 0)
    shared = -(-prefix // PAGE)
    table = s["table"].long()
    head = [p[table[0, :shared]].transpose(0, 1).flatten(1, 2)[:, :prefix] for p in (s["k_pool"], s["v_pool"])]
    return head, [p[table[:, shared:]].transpose(1, 2).flatten(2, 3) for p in (s["k_pool"], s["v_pool"])]


def _run_attend(s):
    c = s["case"]
    if own:
        if c["paged"]:
            s["plan"].tree_attend_paged(s["q"], s["k_pool"], s["v_pool"], s["table"], s["lens"], s["masks"], s["out"], s["lse"])
        else:
            s["plan"].tree_attend(s["q"], s["prefix_k"], s["prefix_v"], s["suffix_k"], s["suffix_v"], s["lens"], s["masks"], s["out"],
                                  s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    (pk, pv), (sk, sv) = _cache(s)
    b, n, hkv, d = c["branches"], c["nodes"], c["hkv"], c["d"]
    group, cap = c["hq"] // hkv, sk.shape[2]
    q = s["q"].float().view(b, n, hkv, group, d) * (1 / math.sqrt(d))
    # the prefix against all rows of a KV head, each suffix against its branch's
    x = q.permute(2, 0, 1, 3, 4).reshape(hkv, b * n * group, d) @ pk.float().transpose(1, 2)
    y = q.permute(0, 2, 1, 3, 4).reshape(b, hkv, n * group, d) @ sk.float().transpose(2, 3)
    u = torch.arange(cap, device="cuda") - s["lens"][:, None]  # a suffix row's node, negative where it is committed
    seen = torch.gather(_bits(s["masks"], n), 2, u.clamp(0, n - 1).long()[:, None].expand(b, n, cap))
    seen = (u < 0)[:, None] | (seen & (u < n)[:, None])
    y = y.view(b, hkv, n, group, cap).masked_fill_(~seen[:, None, :, None], -math.inf)
    rows = lambda z: z.view(hkv, b, n, group, -1).permute(1, 0, 2, 3, 4)  # noqa: E731
    m = torch.maximum(y.amax(-1, keepdim=True), rows(x.amax(-1)))
    p = torch.exp(x.sub_(m.permute(1, 0, 2, 3, 4).reshape(hkv, b * n * group, 1)))
    py = torch.exp(y.sub_(m))
    total = py.sum(-1, keepdim=True) + rows(p.sum(-1))
    o = (py.view(b, hkv, n * group, cap) @ sv.float()).view(b, hkv, n, group, d) + rows(p @ pv.float())
    s["out"].copy_((o / total).permute(0, 2, 1, 3, 4).reshape(b, n, c["hq"], d))
    s["lse"].copy_((m + torch.log(total)).permute(0, 2, 1, 3, 4).reshape(b, n, c["hq"]))
    return {"out": s["out"], "lse": s["lse"]}


def _run_sample(s):
    if own:
        from paper_2608_13667_amd import forkattn as fa
        fa.sample(s["logits"], s["u"], s["tokens"], s["logprob"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                  min_p=s["min_p"], workspace=s["workspace"])
        return {"tokens": s["tokens"], "logprob": s["logprob"]}
    x = s["logits"].float()
    r, v = x.shape
    place = torch.arange(v, device="cuda")
    top, first = x.max(1, keepdim=True)
    t = s["temperature"][:, None].double()
    w = torch.round(torch.exp((x.double() - top) / t) * UNIT).long()
    w = torch.where(t > 0, w, ((x == top) & (place >= first)).long() * int(UNIT))
    if s["top_k"] is not None:
        ws, order = torch.sort(x, dim=1, descending=True, stable=True)
        ws = torch.gather(w, 1, order)
        k = s["top_k"][:, None]
        ws = torch.where((k <= 0) | (place < k), ws, 0)
        before = ws.cumsum(1) - ws
        keep = before.double() < s["top_p"][:, None].double() * ws.sum(1, keepdim=True).double()
        keep = (keep | (s["top_p"][:, None] >= 1) | (place == 0)) & (ws.double() >= s["min_p"][:, None].double() * UNIT)
        # of equal logits at temperature 0 the first in order is the lowest place: it alone is kept
        keep &= (t > 0) | (place == 0)
        w = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ws, 0))
    else:
        w = torch.where((t > 0) | (place == x.argmax(1, keepdim=True)), w, 0)
    run_sum = w.cumsum(1)
    total = run_sum[:, -1:]
    mark = torch.floor(s["u"][:, None].double() * total.double()).long()
    at = (run_sum > torch.minimum(mark, total - 1)).int().argmax(1, keepdim=True)
    s["tokens"].copy_(at[:, 0])
    s["logprob"].copy_(torch.log(torch.gather(w, 1, at).double() / total.double())[:, 0])
    return {"tokens": s["tokens"], "logprob": s["logprob"]}


def _run_accept(s):
    c = s["case"]
    done = {"path": s["path"], "count": s["count"], "next": s["next"]}
    done.update({"k": s["k_pool"], "v": s["v_pool"]} if c["paged"] else {"k": s["suffix_k"], "v": s["suffix_v"]})
    tree = (s["parents"], s["masks"], s["tokens"], s["targets"])
    if own:
        from paper_2608_13667_amd import forkattn as fa
        if c["paged"]:
            fa.tree_accept_paged(*tree, s["k_pool"], s["v_pool"], s["table"], s["prefix_len"], s["lens"], s["path"], s["count"], s["next"],
                                 advance=False)
        else:
            fa.tree_accept(*tree, s["suffix_k"], s["suffix_v"], s["lens"], s["path"], s["count"], s["next"], advance=False)
        return done
    parents, masks, tokens, targets = tree
    b, n = parents.shape
    place = torch.arange(n, device="cuda")
    behind = parents.long().clamp(min=0)
    right = (parents >= 0) & (tokens == torch.gather(targets, 1, behind))
    twin = (parents[:, :, None] == parents[:, None]) & (tokens[:, :, None] == tokens[:, None]) & (place[:, None] > place)
    right &= ~twin.any(2)
    right[:, 0] = True
    seen = _bits(masks, n)
    accepted = (~seen | right[:, None]).all(2) & right
    count = accepted.sum(1)
    order = torch.argsort((~accepted).int(), dim=1, stable=True)  # the accepted nodes in order, then the others
    s["path"].copy_(torch.where(place < count[:, None], order, -1))
    s["count"].copy_(count)
    s["next"].copy_(torch.gather(targets, 1, torch.gather(order, 1, count[:, None] - 1))[:, 0])
    # row place j from node path[j]; the rows behind the accepted ones stay as they are
    source = s["lens"][:, None].long() + torch.where(place < count[:, None], order, place)
    target = s["lens"][:, None].long() + place
    branch = torch.arange(b, device="cuda")[:, None]
    if c["paged"]:
        page, slot = s["table"].long(), source % PAGE
        s["k_pool"][page[branch, target // PAGE], :, target % PAGE] = s["k_pool"][page[branch, source // PAGE], :, slot]
        s["v_pool"][page[branch, target // PAGE], :, target % PAGE] = s["v_pool"][page[branch, source // PAGE], :, slot]
    else:
        s["suffix_k"][branch, :, target] = s["suffix_k"][branch, :, source]
        s["suffix_v"][branch, :, target] = s["suffix_v"][branch, :, source]
    return done


_RUN = {"layout": _run_layout, "attend": _run_attend, "sample": _run_sample, "accept": _run_accept}


def run(state):
    return _RUN[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------- what it takes

def work(case):
    c = case
    if c["kind"] == "layout":
        nodes = c["branches"] * c["nodes"]
        return {"bytes": 4 * nodes + 4 * c["branches"] + 12 * nodes, "flops": 0}
    if c["kind"] == "sample":
        return {"bytes": c["rows"] * (c["vocab"] * (2 if c["bf16"] else 4) + 28), "flops": 0}
    b, n, hkv, d, suffix = c["branches"], c["nodes"], c["hkv"], c["d"], _suffixes(c)
    if c["kind"] == "accept":
        # the trees, and on average about one accepted node a branch besides the root, read and written
        return {"bytes": b * n * 24 + b * 12 + b * 2 * 2 * hkv * d * 2, "flops": 0}
    masks = _masks(_trees(c))
    seen = [sum(bin(x & (1 << 64) - 1).count("1") for x in row) for row in masks.tolist()]
    pairs = sum(n * (c["prefix"] + u) + k for u, k in zip(suffix, seen))
    keys = c["prefix"] + sum(suffix) + b * n
    rows = b * n * c["hq"]
    return {"bytes": 4 * hkv * keys * d + rows * (2 * d + 4 * d + 4) + 8 * b * n, "flops": 4 * d * c["hq"] * pairs}


# ------------------------------------------------------------------------------------------- in 64 bits

def _exact_sample(s):
    """Probabilities in 64 bits, the filters one after the other on each row's sorted list."""
    r, v = s["logits"].shape
    tokens, logprob = [], []
    for i in range(r):
        x, t, u = s["logits"][i].double(), float(s["temperature"][i]), float(s["u"][i])
        if t <= 0:
            tokens.append(int((x == x.max()).nonzero()[0]))
            logprob.append(0.0)
            continue
        order = torch.argsort(-x, stable=True)
        p = torch.softmax(x[order] / t, 0)
        if s["top_k"] is not None:
            k, top_p, min_p = int(s["top_k"][i]), float(s["top_p"][i]), float(s["min_p"][i])
            if k > 0:
                p[k:] = 0
            if top_p < 1:
                past = torch.cumsum(p, 0) - p >= top_p * p.sum()
                past[0] = False
                p[past] = 0
            p[p < min_p * p[0]] = 0
        kept = torch.zeros_like(p)
        kept[order] = p
        c = torch.cumsum(kept, 0)
        at = min(int(torch.searchsorted(c, u * c[-1], right=True)), v - 1)
        tokens.append(at)
        logprob.append(float(torch.log(kept[at] / c[-1])))
    return {"tokens": torch.tensor(tokens, dtype=torch.int32), "logprob": torch.tensor(logprob, dtype=torch.float64)}


def _exact_attend(s):
    c = s["case"]
    hkv, d, b, n = c["hkv"], c["d"], c["branches"], c["nodes"]
    group, suffix = c["hq"] // hkv, _suffixes(c)
    out = torch.empty(b, n, c["hq"], d, dtype=torch.float64, device="cuda")
    lse = torch.empty(b, n, c["hq"], dtype=torch.float64, device="cuda")
    prefix, ends = _cache(s)
    for i, length in enumerate(suffix):
        hidden = torch.zeros(n, 1, c["prefix"] + length + n, dtype=torch.bool, device="cuda")
        for j in range(n):
            hidden[:, 0, c["prefix"] + length + j] = (s["masks"][i] >> j & 1) == 0
        for g in range(hkv):
            k, v = (torch.cat([p[g], e[i, g, : length + n]]).double() for p, e in zip(prefix, ends))
            heads = slice(g * group, (g + 1) * group)
            x = (s["q"][i, :, heads].double() @ k.T / math.sqrt(d)).masked_fill(hidden, -math.inf)
            lse[i, :, heads] = torch.logsumexp(x, -1)
            out[i, :, heads] = torch.softmax(x, -1) @ v
    return {"out": out, "lse": lse}


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "sample":
        return _exact_sample(s)
    if case["kind"] == "attend":
        return _exact_attend(s)
    return None  # whole numbers and copies: equal or wrong
