"""What the speculative-decoding and cache-budget operators are measured on.

Five operators next to the decode step: attention for a tree of drafted tokens over the K-cache, verification of the
drafted tokens, commit of the accepted ones into the cache, accumulation of attention weights per cache row, and eviction
of the rows with little weight.  `run` computes them either in a plain form (elementary torch operations, float32, float64
where 32 bits lose what matters) or through the library's entry points, as `own` says.

The cache layout, the rotation (pair (j, j + d_k/2) turned by -t theta^(-2j/d_k)) and the weights W_KV are the ones of
include/slim.h."""
import math
import random

import torch

own = False
DEV = "cuda:0"
_weights = {}        # W_KV by shape: a program's weights, the same for all inputs
_contexts = {}       # library contexts by shape, which a program makes once


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # a small model's float32 cache, one user, eight drafts: latency
        dict(name="tree_f32_1500", op="tree", dtype="f32", d=384, H=6, theta=1.0e4, B=1, lo=1500, hi=1500, n=8, page=0),
        # one user of a mid-sized model, head width 96, an odd number of drafts, keys in pages of 64 rows
        dict(name="tree_bf16_4k_paged", op="tree", dtype="bf16", d=1536, H=16, theta=1.0e4, B=1, lo=4093, hi=4093, n=5, page=64),
        # a serving batch of ragged contexts on the 4096-wide shape, sixteen drafts each
        dict(name="tree_bf16_batch16", op="tree", dtype="bf16", d=4096, H=32, theta=1.0e6, B=16, lo=8192, hi=16384, n=16, page=0),
        # one very long context with the widest tree
        dict(name="tree_bf16_128k", op="tree", dtype="bf16", d=4096, H=32, theta=1.0e6, B=1, lo=131001, hi=131001, n=64, page=0),
        # verification for one user: a handful of drafts
        dict(name="verify_1", op="verify", B=1, n=5, V=32000, kids=2),
        # verification for a serving batch with wide trees and a large vocabulary
        dict(name="verify_64", op="verify", B=64, n=16, V=131072, kids=3),
        # accepted rows of one user into a paged cache
        dict(name="commit_1", op="commit", dtype="bf16", d=1536, H=16, theta=1.0e4, B=1, lo=4093, hi=4093, n=5, page=64),
        # accepted rows of a large batch with the widest trees
        dict(name="commit_64", op="commit", dtype="bf16", d=4096, H=32, theta=1.0e6, B=64, lo=100, hi=960, n=64, page=0),
        # attention weights of one step on the small float32 cache
        dict(name="weights_f32_1500", op="weights", dtype="f32", d=384, H=6, theta=1.0e4, B=1, lo=1500, hi=1500, page=0),
        # attention weights of one step of the ragged serving batch
        dict(name="weights_bf16_batch16", op="weights", dtype="bf16", d=4096, H=32, theta=1.0e6, B=16, lo=8192, hi=16384, page=0),
        # a small float32 cache brought down to a third
        dict(name="evict_f32_1500", op="evict", dtype="f32", d=384, H=6, theta=1.0e4, B=1, lo=1500, hi=1500, page=0, budget=500, recent=64),
        # the ragged serving batch brought down to 4096 rows a sequence
        dict(name="evict_bf16_batch16", op="evict", dtype="bf16", d=4096, H=32, theta=1.0e6, B=16, lo=8192, hi=16384, page=0, budget=4096, recent=512),
    ]


def _log(rng, a, b):
    return max(a, min(b, int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))))


def draw(rng):
    op = rng.choice(["tree", "tree", "tree", "verify", "commit", "weights", "evict"])
    if op == "verify":
        V = _log(rng, 1000, 131072)
        B = _log(rng, 1, 64)
        n = _log(rng, 1, max(1, min(64, 64 * 16 * 131072 // (B * V))))
        return dict(op=op, B=B, n=n, V=V, kids=rng.randint(1, 4))
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if dtype == "f32":
        H, d_k = rng.choice([(6, 64), (4, 96), (8, 64), (5, 40)])
    else:
        H, d_k = rng.choice([(32, 128), (32, 128), (16, 96), (20, 64), (8, 128), (12, 64), (10, 100)])
    # the shapes that run without tensor cores are held to smaller contexts
    slow = dtype == "f32" or d_k == 100
    d = H * d_k
    B = _log(rng, 1, 32)
    most = 16 * 12288 * 4096 // (64 if slow else 1)
    hi = _log(rng, 1, max(1, min(131072, most // (B * d))))
    lo = max(1, int(hi * rng.uniform(0.3, 1.0)))
    theta = rng.choice([0.0, 1.0e4, 1.0e6])
    page = rng.choice([0, 0, 16, 64, 256])
    c = dict(op=op, dtype=dtype, d=d, H=H, theta=theta, B=B, lo=lo, hi=hi, page=page)
    if op == "tree":
        # no more products than the longest listed case
        c["n"] = _log(rng, 1, max(1, min(64, int(1.0e12 // (2 * B * hi * d * H)))))
    elif op == "commit":
        c["n"] = _log(rng, 1, 64)
    elif op == "evict":
        if dtype == "bf16" and rng.random() < 0.3:
            c["dtype"], c["page"] = "fp8", 0
        c["budget"] = max(1, int(hi * rng.uniform(0.2, 0.9)))
        c["recent"] = int(c["budget"] * rng.uniform(0.0, 0.5))
    return c


def _lengths(c):
    """Ragged context lengths of a case, the first the longest."""
    return [c["hi"] if b == 0 else c["lo"] + int((c["hi"] - c["lo"]) * ((0.6180339887 * b) % 1.0)) for b in range(c["B"])]


def _t_cap(c):
    t = c["hi"] + 64
    g = c.get("page") or 16
    return (t + g - 1) // g * g


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _tdtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _wkv(c):
    """W_KV [d][d] in the cache's type."""
    key = (c["d"], c["dtype"])
    if key not in _weights:
        g = _gen(c["d"])
        _weights[key] = (torch.randn(c["d"], c["d"], device=DEV, generator=g) / math.sqrt(c["d"])).to(_tdtype(c))
    return _weights[key]


def _context(c):
    from paper_2503_05840_b200 import binding as B
    key = (c["d"], c["H"], c["theta"], c["dtype"])
    if key not in _contexts:
        kind = {"f32": B.SLIM_F32, "bf16": B.SLIM_BF16, "fp8": B.SLIM_FP8}[c["dtype"]]
        ctx = B.slim_create(c["d"], c["H"], c["d"] // c["H"], c["theta"], kind)
        if c["op"] == "tree" or c["dtype"] != "fp8":
            B.slim_set_wkv(ctx, _wkv(c).float().cpu().numpy())
        _contexts[key] = ctx
    return _contexts[key]


class _Cache:
    """The library's view of the state's key storage."""

    def __init__(self, c, s):
        from paper_2503_05840_b200 import binding as B
        self.B, self.ctx = B, _context(c)
        if c["page"]:
            num_pages, rows = s["K"].shape[0], s["K"].shape[1]
            self.cache = B.slim_cache_create_paged(self.ctx, s["K"], num_pages, rows, s["table"], c["B"], s["table"].shape[1])
        else:
            self.cache = B.slim_cache_create(self.ctx, s["K"], c["B"], _t_cap(c))

    def __del__(self):
        self.B.slim_cache_destroy(self.cache)


def _parents(gen, B, n, kids):
    """Random trees of n nodes with at most `kids` children a node, node 0 the root; the last few nodes of some are padding."""
    out = []
    for b in range(B):
        live = n if b % 3 == 0 else max(1, n - gen.randrange(0, max(1, n // 3) + 1))
        free, par = {0: 0}, [-1]
        for i in range(1, live):
            p = gen.choice([u for u in free if free[u] < kids][-4:])     # deep rather than bushy
            free[p] += 1
            free[i] = 0
            par.append(p)
        out.append(par + [-2] * (n - live))
    return torch.tensor(out, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    c, s = case, {"case": case}
    g, r = _gen(seed), random.Random(seed)
    B = c["B"]
    if c["op"] == "verify":
        n, V = c["n"], c["V"]
        s["parents"] = _parents(r, B, n, c["kids"])
        s["p"], s["q"] = (torch.empty(B, n, V, device=DEV) for _ in range(2))
        s["tokens"] = torch.zeros(B, n, dtype=torch.int32, device=DEV)
        step = max(1, (1 << 27) // (n * V))
        for b in range(0, B, step):
            logits = 3.0 * torch.randn(min(step, B - b), n, V, device=DEV, generator=g)
            s["p"][b:b + step] = torch.softmax(logits, -1)
            # a draft that knows the target roughly
            s["q"][b:b + step] = torch.softmax(logits + 0.7 * torch.randn(logits.shape, device=DEV, generator=g), -1)
        up = s["parents"].long().clamp(min=0)
        rows = (torch.arange(B, device=DEV)[:, None] * n + up).reshape(-1)
        for a in range(0, B * n, 256):
            s["tokens"].view(-1)[a:a + 256] = torch.multinomial(s["q"].view(B * n, V)[rows[a:a + 256]], 1, generator=g)[:, 0].int()
        s["r"] = torch.rand(B, n, device=DEV, generator=g)
        s["path"] = torch.empty(B, n, dtype=torch.int32, device=DEV)
        s["count"] = torch.empty(B, dtype=torch.int32, device=DEV)
        s["next"] = torch.empty(B, dtype=torch.int32, device=DEV)
        if own:
            s["ctx"] = _context(dict(d=384, H=6, theta=0.0, dtype="f32", op="verify"))
        return s
    d, t_cap, td = c["d"], _t_cap(c), _tdtype(c)
    lens = _lengths(c)
    s["lengths"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    rows_of = (B * t_cap // c["page"], c["page"]) if c["page"] else (B, t_cap)
    if c["dtype"] == "fp8":     # codes, then one exponent for each row and head; finite codes only
        codes = (B * t_cap * d + 15) // 16 * 16
        K = torch.randint(0, 126, (codes + B * t_cap * c["H"],), device=DEV, generator=g, dtype=torch.uint8)
        s["K"] = K
    else:
        # keys with directions of unequal strength, and queries that share a direction with some of them
        scale = 0.5 + 1.5 * torch.rand(d, device=DEV, generator=g)
        common = torch.randn(d, device=DEV, generator=g)
        K = torch.empty(*rows_of, d, dtype=td, device=DEV)
        flat = K.view(-1, d)
        for a in range(0, flat.shape[0], 1 << 15):
            x = torch.randn(min(1 << 15, flat.shape[0] - a), d, device=DEV, generator=g)
            x += 0.5 * common * (torch.rand(x.shape[0], 1, device=DEV, generator=g) < 0.02)
            flat[a:a + (1 << 15)] = x * scale
        s["K"] = K
    if c["page"]:               # pages in any order
        s["table"] = torch.randperm(rows_of[0], device=DEV, generator=g).int().view(B, t_cap // c["page"]).contiguous()
    if c["op"] == "tree" or c["op"] == "commit":
        n = c["n"]
        s["k_tree"] = (torch.randn(B, n, d, device=DEV, generator=g) * scale).to(td)
    if c["op"] == "tree":
        s["q"] = (torch.randn(B, n, d, device=DEV, generator=g) + 0.3 * common).to(td)
        s["parents"] = _parents(r, B, n, 3)
        s["W_KV"] = _wkv(c)
        s["o"] = torch.empty(B, n, d, dtype=td, device=DEV)
    elif c["op"] == "commit":
        paths = [sorted(r.sample(range(n), r.randint(1, n))) for _ in range(B)]
        s["path"] = torch.tensor([p + [-1] * (n - len(p)) for p in paths], dtype=torch.int32, device=DEV)
        s["count"] = torch.tensor([len(p) for p in paths], dtype=torch.int32, device=DEV)
    elif c["op"] == "weights":
        s["q"] = (torch.randn(B, d, device=DEV, generator=g) + 0.3 * common).to(td)
        s["acc"] = (2.0 * c["H"] / c["hi"]) * torch.rand(B, t_cap, device=DEV, generator=g)      # a few earlier steps' worth
    elif c["op"] == "evict":
        # a few rows hold most of the weight, as heavy hitters do; equal values occur
        s["acc"] = (torch.rand(B, t_cap, device=DEV, generator=g).pow(6) * 64).mul(1024).round().div(1024)
        s["kept"] = torch.empty(B, c["budget"], dtype=torch.int32, device=DEV)
    if own:
        s["h"] = h = _Cache(c, s)
        need = 0
        if c["op"] == "tree":
            need = h.B.slim_tree_workspace_bytes(h.ctx, B, t_cap, c["n"])
        elif c["op"] == "weights":
            need = h.B.slim_weights_workspace_bytes(h.ctx, B, t_cap)
        elif c["op"] == "evict":
            need = h.B.slim_evict_workspace_bytes(h.ctx, B, t_cap)
        s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    c = s["case"]
    if own:
        return _own(s, c)
    return {"tree": _plain_tree, "verify": _plain_verify, "commit": _plain_commit, "weights": _plain_weights, "evict": _plain_evict}[c["op"]](s, c)


def _own(s, c):
    from paper_2503_05840_b200 import binding as B
    st = torch.cuda.current_stream().cuda_stream
    op = c["op"]
    if op == "verify":
        B.slim_tree_verify(s["ctx"], s["p"], s["q"], s["tokens"], s["parents"], s["r"], c["B"], c["n"], c["V"],
                           s["path"], s["count"], s["next"], st)
        return {"path": s["path"], "count": s["count"], "next": s["next"]}
    h = s["h"]
    if op == "tree":
        B.slim_tree_decode(h.ctx, s["q"], s["k_tree"], h.cache, s["lengths"], s["parents"], c["n"], s["o"], s["ws"], st)
        return s["o"]
    if op == "commit":
        B.slim_tree_commit(h.ctx, h.cache, s["k_tree"], s["lengths"], s["path"], s["count"], c["n"], st)
        return s["K"]
    acc = s["acc"].clone()      # the statistics of the program's next step
    if op == "weights":
        B.slim_accumulate_weights(h.ctx, s["q"], h.cache, s["lengths"], acc, s["ws"], st)
        return acc
    B.slim_evict(h.ctx, h.cache, s["lengths"], acc, c["budget"], c["recent"], s["kept"], s["ws"], st)
    return {"K": s["K"], "acc": acc, "kept": s["kept"]}


def _rows(s, c, T):
    """The first T cache rows of every sequence, [B, T, d], as they are stored."""
    if not c["page"]:
        return s["K"][:, :T]
    t = torch.arange(T, device=DEV)
    return s["K"].view(-1, c["d"])[s["table"][:, t // c["page"]].long() * c["page"] + t % c["page"]]


def _rotate(x, pos, c):
    """x [B, T, H, d_k] float32 at positions pos [B, T]; the angles in 64 bits."""
    if not c["theta"]:
        return x
    half = x.shape[-1] // 2
    freq = c["theta"] ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
    a = pos.double()[..., None] * freq
    cos, sin = a.cos().float()[:, :, None], a.sin().float()[:, :, None]
    x1, x2 = x[..., :half], x[..., half:]
    return torch.cat([x1 * cos + x2 * sin, x2 * cos - x1 * sin], -1)


def _ancestors(parents):
    """[B, n, n]: whether token j is token i or one of its ancestors; padding has none."""
    B, n = parents.shape
    live = parents >= -1
    up = torch.nn.functional.one_hot(parents.long().clamp(min=-1) + 1, n + 1)[..., 1:].double()
    reach = torch.linalg.matrix_power(torch.eye(n, dtype=torch.float64, device=DEV) + up, max(n, 1)) > 0.5
    return reach & live[:, :, None]


def _plain_tree(s, c):
    B, n, d, H = c["B"], c["n"], c["d"], c["H"]
    T, dk = c["hi"], c["d"] // c["H"]
    L = s["lengths"].long()
    see = _ancestors(s["parents"])
    depth = (see.sum(-1) - 1).clamp(min=0)
    live = torch.arange(T, device=DEV) < L[:, None]
    K = torch.cat([_rows(s, c, T).float().masked_fill(~live[..., None], 0.0),
                   s["k_tree"].float().masked_fill((s["parents"] < -1)[..., None], 0.0)], 1)        # [B, T + n, d]
    pos = torch.cat([torch.arange(T, device=DEV).expand(B, T), L[:, None] + depth], 1)
    mask = torch.cat([(live[:, None] & (s["parents"] >= -1)[..., None]).expand(B, n, T), see], 2)   # [B, n, T + n]
    q = _rotate(s["q"].float().view(B, n, H, dk), L[:, None] + depth, c).transpose(1, 2)
    k = _rotate(K.view(B, T + n, H, dk), pos, c).permute(0, 2, 3, 1)
    a = (q @ k) / math.sqrt(dk)
    a = a.masked_fill(~mask[:, None], -math.inf)
    a = torch.exp(a - a.amax(-1, keepdim=True).clamp(min=-1e30))
    total = a.sum(-1, keepdim=True)
    u = (a.view(B, H * n, T + n) @ K).view(B, H, n, d) / total.clamp(min=1e-30)
    o = u @ s["W_KV"].float().view(d, H, dk).transpose(0, 1)
    return o.transpose(1, 2).reshape(B, n, d).to(s["q"].dtype)


def _plain_verify(s, c):
    B, n = c["B"], c["n"]
    par, tok, r = s["parents"].long(), s["tokens"].long(), s["r"].double()
    node = torch.arange(n, device=DEV)
    same = (par[:, :, None] == par[:, None, :]) & (node[:, None] > node)
    rank = same.sum(-1)
    W, q = s["p"].double(), s["q"].double()
    S = torch.ones(B, n, 1, dtype=torch.float64, device=DEV)
    chosen = torch.full((B, n), -1, dtype=torch.long, device=DEV)
    for j in range(c["kids"]):      # the j-th child of every node, each test on what the earlier ones left
        is_j = (par >= 0) & (rank == j)
        child = torch.full((B, n + 1), -1, dtype=torch.long, device=DEV)
        child.scatter_(1, torch.where(is_j, par, n), node.expand(B, n))
        child = child[:, :n]
        x = tok.gather(1, child.clamp(min=0))[..., None]
        take = (r.gather(1, child.clamp(min=0))[..., None] * S * q.gather(2, x) < W.gather(2, x))[..., 0]
        open_ = (child >= 0) & (chosen < 0)
        chosen = torch.where(open_ & take, child, chosen)
        rest = (W - S * q).clamp(min=0)
        mass = rest.sum(-1, keepdim=True)
        left = (open_ & ~take)[..., None] & (mass > 0)
        W, S = torch.where(left, rest, W), torch.where(left, mass, S)
    see = _ancestors(s["parents"])
    picked = (par >= 0) & (chosen.gather(1, par.clamp(min=0)) == node)
    picked[:, 0] = True
    on = ~(see & ~picked[:, None]).any(-1) & see[:, :, 0]
    path = torch.where(on, node, n).sort(-1).values
    cum = W.cumsum(-1)
    total = cum[..., -1:]
    token = (cum <= r[:, :1, None] * total).sum(-1).clamp(max=c["V"] - 1)
    last = torch.where(on, node, -1).amax(-1)
    nxt = torch.where(total[..., 0] > 0, token, -1).gather(1, last[:, None])[:, 0]
    s["path"].copy_(torch.where(path < n, path, -1))
    s["count"].copy_(on.sum(-1))
    s["next"].copy_(nxt)
    return {"path": s["path"], "count": s["count"], "next": s["next"]}


def _plain_commit(s, c):
    n = c["n"]
    j = torch.arange(n, device=DEV)
    b, j = torch.nonzero(j < s["count"][:, None], as_tuple=True)
    rows = s["k_tree"][b, s["path"][b, j].long()]
    t = s["lengths"][b].long() + j
    if c["page"]:
        s["K"][s["table"][b, t // c["page"]].long(), t % c["page"]] = rows
    else:
        s["K"][b, t] = rows
    return s["K"]


def _plain_weights(s, c):
    B, H, T = c["B"], c["H"], c["hi"]
    dk = c["d"] // H
    L = s["lengths"].long()
    live = torch.arange(T, device=DEV) < L[:, None]
    k = _rotate(_rows(s, c, T).float().view(B, T, H, dk), torch.arange(T, device=DEV).expand(B, T), c)
    q = _rotate(s["q"].float().view(B, 1, H, dk), (L - 1)[:, None], c)
    a = (k.transpose(1, 2) @ q.permute(0, 2, 3, 1))[..., 0] / math.sqrt(dk)                          # [B, H, T]
    a = torch.softmax(a.masked_fill(~live[:, None], -math.inf), -1)
    acc = s["acc"].clone()
    acc[:, :T] += a.sum(1)
    return acc


def _plain_evict(s, c):
    B, n, rec, T = c["B"], c["budget"], c["recent"], c["hi"]
    L = s["lengths"].long()[:, None]
    t = torch.arange(T, device=DEV)
    acc = s["acc"].clone()
    over = L > n
    key = torch.where(t >= L - rec, math.inf, acc[:, :T])
    key = torch.where(over, key, -t.float())                          # a short sequence keeps its first rows
    key = torch.where(t < L, key, -math.inf)
    order = torch.sort(key, descending=True, stable=True).indices[:, :n]
    if order.shape[1] < n:
        order = torch.nn.functional.pad(order, (0, n - order.shape[1]))
    j = torch.arange(n, device=DEV)
    order = torch.where(j < L, order, T).sort(-1).values
    s["kept"].copy_(torch.where(order < T, order, -1))
    b, j = torch.nonzero((order < T) & over, as_tuple=True)
    old = order[b, j]
    acc[:, :T] = torch.where(over & (t < L), 0.0, acc[:, :T])
    acc[b, j] = s["acc"][b, old]
    if c["dtype"] == "fp8":
        d, H, t_cap = c["d"], c["H"], _t_cap(c)
        at = (B * t_cap * d + 15) // 16 * 16
        codes, exps = s["K"][:B * t_cap * d].view(B, t_cap, d), s["K"][at:].view(B, t_cap, H)
        codes[b, j] = codes[b, old]
        exps[b, j] = exps[b, old]
    elif c["page"]:
        g, K, tab = c["page"], s["K"], s["table"].long()
        K[tab[b, j // g], j % g] = K[tab[b, old // g], old % g]
    else:
        s["K"][b, j] = s["K"][b, old]
    return {"K": s["K"], "acc": acc, "kept": s["kept"]}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["op"] == "verify":     # one row of p and of q for each sequence: where the walk ends, and the final draw
        return {"bytes": 8.0 * c["B"] * c["V"] + 24.0 * c["B"] * c["n"], "flops": 4.0 * c["B"] * c["V"]}
    es = {"f32": 4, "bf16": 2, "fp8": 1}[c["dtype"]]
    B, d, H, L = c["B"], c["d"], c["H"], sum(_lengths(c))
    if c["op"] == "tree":
        n = c["n"]
        return {"bytes": es * (L * d + 3.0 * B * n * d + d * d), "flops": 2.0 * (L + B * n) * n * d * (H + 1) + 2.0 * B * n * d * d}
    if c["op"] == "commit":
        return {"bytes": 2.0 * es * B * (c["n"] + 1) / 2 * d + 4.0 * B * c["n"], "flops": 0}
    if c["op"] == "weights":
        return {"bytes": es * (L * d + B * d) + 8.0 * L, "flops": 2.0 * L * d}
    moved = sum(min(c["budget"], x) for x in _lengths(c) if x > c["budget"])
    return {"bytes": 2.0 * moved * d * es + 4.0 * L + 8.0 * moved, "flops": 0}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _stored(s, c, b):
    """Sequence b's live rows, [L, d]."""
    L = int(s["lengths"][b])
    if not c["page"]:
        return s["K"][b, :L]
    return torch.cat([s["K"][int(x)] for x in s["table"][b].tolist()])[:L]


def _turned(x, pos, c):
    """Complex rows [T, H, d_k / 2]: the pair (x_j, x_{j + d_k/2}) as one number, turned by -pos theta_j."""
    T = x.shape[0]
    x = x.double().view(T, c["H"], 2, -1)
    z = torch.complex(x[:, :, 0].contiguous(), x[:, :, 1].contiguous())
    if c["theta"]:
        half = z.shape[-1]
        w = torch.tensor([c["theta"] ** (-j / half) for j in range(half)], dtype=torch.float64, device=DEV)
        z = z * torch.polar(torch.ones_like(w), -pos.double()[:, None] * w)[:, None]
    return z


def exact(case, seed):
    c = case
    if c["op"] == "verify":
        return None             # whole numbers only
    s = prepare(case, seed)
    B, H, d = c["B"], c["H"], c["d"]
    if c["op"] == "commit":
        for b in range(B):
            for j in range(int(s["count"][b])):
                t = int(s["lengths"][b]) + j
                row = s["k_tree"][b, int(s["path"][b, j])]
                if c["page"]:
                    s["K"][int(s["table"][b, t // c["page"]]), t % c["page"]] = row
                else:
                    s["K"][b, t] = row
        return s["K"]
    if c["op"] == "evict":
        acc = s["acc"].clone()
        for b in range(B):
            L, n = int(s["lengths"][b]), c["budget"]
            if L <= n:
                continue
            a = s["acc"][b, :L - c["recent"]].tolist()
            keep = sorted(sorted(range(len(a)), key=lambda t: (-a[t], t))[:n - c["recent"]]) + list(range(L - c["recent"], L))
            acc[b, :L] = 0
            acc[b, :n] = s["acc"][b, keep]
            if c["dtype"] == "fp8":
                continue
            rows = _stored(s, c, b)[keep].clone()
            if c["page"]:
                for a0 in range(0, n, c["page"]):
                    part = rows[a0:a0 + c["page"]]
                    s["K"][int(s["table"][b, a0 // c["page"]]), :len(part)] = part
            else:
                s["K"][b, :n] = rows
        return {"K": None if c["dtype"] == "fp8" else s["K"], "acc": acc, "kept": None}
    scale = 1.0 / math.sqrt(d // H)
    if c["op"] == "weights":
        acc = s["acc"].double()
        for b in range(B):
            L = int(s["lengths"][b])
            k = _turned(_stored(s, c, b), torch.arange(L, device=DEV), c)
            q = _turned(s["q"][b:b + 1], torch.tensor([L - 1], device=DEV), c)
            a = (k * q.conj()).real.sum(-1) * scale                   # [L, H]
            acc[b, :L] += torch.softmax(a, 0).sum(1)
        return acc
    n, dk = c["n"], d // H
    out = torch.zeros(B, n, d, dtype=torch.float64, device=DEV)
    W = s["W_KV"].double()
    for b in range(B):
        par = s["parents"][b].tolist()
        chain = [[] for _ in range(n)]
        for i, p in enumerate(par):
            chain[i] = [] if p < -1 else (chain[p] if p >= 0 else []) + [i]
        L = int(s["lengths"][b])
        depth = torch.tensor([max(len(x) - 1, 0) for x in chain], device=DEV)
        hide = torch.ones(n, n, dtype=torch.bool, device=DEV)
        for i, x in enumerate(chain):
            hide[i, x] = False
        rows, own_rows = _stored(s, c, b), s["k_tree"][b]
        zk = _turned(rows, torch.arange(L, device=DEV), c)
        zt, zq = _turned(own_rows, L + depth, c), _turned(s["q"][b], L + depth, c)
        rows, own_rows = rows.double(), own_rows.double()
        for h in range(H):
            far = lambda z: torch.cat([z[:, h].real, z[:, h].imag], -1)
            a = torch.cat([far(zq) @ far(zk).T, (far(zq) @ far(zt).T).masked_fill(hide, -math.inf)], 1) * scale
            w = torch.softmax(a, -1)
            u = w[:, :L] @ rows + w[:, L:] @ own_rows
            out[b, :, h * dk:(h + 1) * dk] = u @ W[:, h * dk:(h + 1) * dk]
        for i, x in enumerate(chain):
            if not x:
                out[b, i] = 0
    return out
