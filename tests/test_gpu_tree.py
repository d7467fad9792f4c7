"""Drafted tokens through the C ABI: attention for a tree over the cache, verification, commit -- against the float64
definitions.  Cache rows behind the lengths, unused pages and padding tokens hold NaN.

Tolerances are worst-case bounds worked out from the roundings (u = half a step of the type):
  arguments     a sum of d_k products with relative errors e_s each is off by at most
                arg e_s, arg = sum |q_j k_j| / sqrt(d_k); e_s = 2^-9 + (d_k + 16) 2^-24 on the tensor cores (operands rounded
                to 11 bits, 2^-11 each time: keys once, queries once or twice), (d_k + 16) 2^-24 else
  probabilities relative error 2 arg e_s + (T + 16) 2^-24 (numerator and denominator), + 2^-8 where they are rounded
                to bf16, times mass = (sum p |k|) |W_KV|
  u, o          2^-8 each of mass and |o| where rounded to bf16; sums of d products (d + 16) 2^-24 of mass."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as do
from paper_2503_05840_b200 import binding as B
from paper_2503_05840_b200 import synth
from paper_2503_05840_b200.layer import SlimLayer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def tolerance(o, mass, arg, T, d, d_k, dtype, tensor_cores):
    f = 2.0 ** -24
    es = (d_k + 16) * f + (2.0 ** -9 if tensor_cores else 0.0)
    ep = 2 * arg[:, None] * es + (T + 16) * f + (2.0 ** -8 if tensor_cores else 0.0)
    ep = np.expm1(ep)
    tol = mass * (ep + (d + 16) * f + (2.0 ** -8 if tensor_cores else 0.0))
    return tol + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * (np.abs(o) + tol) + 1e-30


def random_parents(g, n, pad=True):
    par = [-1]
    for i in range(1, n):
        p = int(g.integers(-1, i)) if g.random() < 0.9 else -1
        par.append(-2 if pad and g.random() < 0.15 else p)
    for i in range(n):          # a child of padding is padding too (otherwise the tree is refused)
        if par[i] >= 0 and par[par[i]] < -1:
            par[i] = -2
    return par


def to_dev(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(DEV, torch.float32 if dtype == "f32" else torch.bfloat16)


class Case:
    """Inputs of one batch, the library's objects over them, and the definition's answer."""

    def __init__(self, d, H, theta, dtype, lengths, parents, page=0, seed=0, spread=1.0, t_cap=None):
        g = np.random.default_rng(seed)
        self.d, self.H, self.theta, self.dtype = d, H, theta, dtype
        self.lengths, self.parents = np.array(lengths, np.int32), np.array(parents, np.int32)
        self.batch, self.n = self.parents.shape
        rnd = lambda *s: synth.round_to_dtype(spread * g.standard_normal(s), dtype)
        self.q, self.kt = rnd(self.batch, self.n, d), rnd(self.batch, self.n, d)
        self.K = [rnd(int(L), d) for L in lengths]
        self.W = synth.round_to_dtype(g.standard_normal((d, d)) / np.sqrt(d), dtype).astype(np.float64)
        for b, chains in enumerate(map(do.tree_chains, parents)):
            for i, c in enumerate(chains):
                if not c:
                    self.q[b, i] = self.kt[b, i] = np.nan
        t_cap = t_cap or max(max(lengths), 1) + 7
        if page:
            t_cap = -(-t_cap // page) * page
        self.t_cap, self.page = t_cap, page
        self.ctx = B.slim_create(d, H, d // H, theta, B.SLIM_F32 if dtype == "f32" else B.SLIM_BF16)
        B.slim_set_wkv(self.ctx, self.W)
        td = torch.float32 if dtype == "f32" else torch.bfloat16
        if page:
            mp = t_cap // page
            pages = self.batch * mp + 3
            tab = g.permutation(pages)[:self.batch * mp].astype(np.int32).reshape(self.batch, mp)
            self.store = torch.full((pages, page, d), float("nan"), dtype=td, device=DEV)
            self.table = torch.from_numpy(tab).to(DEV)
            self.cache = B.slim_cache_create_paged(self.ctx, self.store, pages, page, self.table, self.batch, mp)
            self.where = lambda b, t: (int(tab[b, t // page]), t % page)
        else:
            self.store = torch.full((self.batch, t_cap, d), float("nan"), dtype=td, device=DEV)
            self.cache = B.slim_cache_create(self.ctx, self.store, self.batch, t_cap)
            self.where = lambda b, t: (b, t)
        for b in range(self.batch):
            rows = to_dev(self.K[b], dtype)
            if page:
                for a in range(0, len(rows), page):
                    self.store[self.where(b, a)[0], :len(rows[a:a + page])] = rows[a:a + page]
            else:
                self.store[b, :len(rows)] = rows
        self.dq, self.dkt = to_dev(self.q, dtype), to_dev(self.kt, dtype)
        self.dlen, self.dpar = torch.from_numpy(self.lengths).to(DEV), torch.from_numpy(self.parents).to(DEV)
        self.o = torch.full((self.batch, self.n, d), float("nan"), dtype=td, device=DEV)
        self.ws = torch.empty(B.slim_tree_workspace_bytes(self.ctx, self.batch, t_cap, self.n), dtype=torch.uint8, device=DEV)
        self.ws.fill_(255)      # NaN in every scratch word

    def call(self, stream=None):
        st = (stream or torch.cuda.current_stream()).cuda_stream
        B.slim_tree_decode(self.ctx, self.dq, self.dkt, self.cache, self.dlen, self.dpar, self.n, self.o, self.ws, st)

    def status(self):
        return B.slim_device_status(self.ctx, torch.cuda.current_stream().cuda_stream)

    def check(self, got=None):
        got = (self.o if got is None else got).float().cpu().numpy().astype(np.float64)
        d_k = self.d // self.H
        tc = self.dtype == "bf16" and self.d % 64 == 0 and d_k in (64, 96, 128)
        worst = 0.0
        for b in range(self.batch):
            o, mass, arg = do.tree_attention(self.q[b], self.kt[b], self.K[b], list(self.parents[b]), self.W, self.H, self.theta)
            tol = tolerance(o, mass, arg, len(self.K[b]) + self.n, self.d, d_k, self.dtype, tc)
            err = np.abs(got[b] - o)
            assert np.all(err <= tol), f"sequence {b}: {np.max(err / tol):.2f} of the bound"
            for i, c in enumerate(do.tree_chains(list(self.parents[b]))):
                if not c:
                    assert np.all(got[b, i] == 0)
            norm = np.linalg.norm(o)
            if norm > 0:
                worst = max(worst, np.linalg.norm(got[b] - o) / norm)
        return worst

    def close(self):
        B.slim_cache_destroy(self.cache)
        B.slim_destroy(self.ctx)

    def __enter__(self):
        return self

    def __exit__(self, *a):
        torch.cuda.synchronize()
        self.close()


LENGTHS = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300]


@pytest.mark.parametrize("d,H,theta,dtype,page,n", [
    (384, 6, 1.0e4, "f32", 0, 8), (384, 6, 0.0, "f32", 16, 5), (200, 5, 1.0e4, "f32", 0, 3), (24, 3, 1.0e4, "f32", 0, 64),
    (512, 4, 1.0e6, "bf16", 0, 16), (512, 4, 0.0, "bf16", 0, 64), (512, 8, 1.0e4, "bf16", 16, 7), (384, 4, 1.0e4, "bf16", 64, 33),
    (576, 6, 1.0e4, "bf16", 48, 2), (1280, 20, 0.0, "bf16", 0, 5), (192, 2, 1.0e4, "bf16", 0, 1), (64, 1, 1.0e4, "bf16", 0, 64),
    (128, 1, 1.0e4, "bf16", 32, 17), (1000, 10, 1.0e4, "bf16", 0, 6), (80, 2, 1.0e4, "bf16", 16, 9)])
def test_tree_against_the_definition(d, H, theta, dtype, page, n):
    g = np.random.default_rng(d + n)
    parents = [random_parents(g, n) for _ in LENGTHS]
    parents[3] = [-2] * n                                    # a sequence that drafted nothing
    with Case(d, H, theta, dtype, LENGTHS, parents, page, seed=n) as c:
        c.call()
        assert c.status() == B.SLIM_OK
        worst = c.check()
        print(f"worst relative error of a sequence {worst:.2e}")


@pytest.mark.parametrize("spread", [0.05, 4.0, 12.0])
def test_flat_and_peaked_softmax(spread):
    g = np.random.default_rng(5)
    with Case(512, 4, 1.0e4, "bf16", [700, 257], [random_parents(g, 12) for _ in range(2)], seed=7, spread=spread) as c:
        c.call()
        assert c.status() == B.SLIM_OK
        c.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_arguments_that_jump_between_blocks_of_rows(dtype):
    """Every block of 128 rows lies at another level of softmax arguments, hundreds apart both ways: the reference exponent
    changes from block to block and blocks far below the top must vanish, not overflow."""
    d, H, L = 256, 2, 128 * 7 + 40
    with Case(d, H, 0.0, dtype, [L], [[-1, 0, 1, -1]], seed=3) as c:
        level = np.array([0, 40, -300, 35, 300, 299, -20, 290], np.float32)[np.arange(L) // 128]
        c.q[:] = 0; c.q[..., ::32] = 8.0                      # every head's argument is 8 * sum of its columns' strides / sqrt(d_k)
        c.K[0][:, ::32] = 0.01 * c.K[0][:, ::32] + level[:, None] * np.float32(np.sqrt(d // H) / 32.0)
        c.K[0] = synth.round_to_dtype(c.K[0], dtype)
        c.kt[0, :, ::32] = 30.0
        c.kt = synth.round_to_dtype(c.kt, dtype)
        c.store[0, :L] = to_dev(c.K[0], dtype)
        c.dq, c.dkt = to_dev(c.q, dtype), to_dev(c.kt, dtype)
        c.call()
        assert c.status() == B.SLIM_OK
        c.check()


@pytest.mark.parametrize("key,query", [(3.0e5, 2.0e-6), (1.0e9, 1.0e-9), (1.0e-7, 1.0e7), (2.0e-5, 3.0e4), (1.0e-30, 1.0e3)])
def test_keys_and_queries_of_any_magnitude(key, query):
    """Keys beyond the range of the 16-bit products, and far below it, against queries that make up for it."""
    with Case(256, 2, 1.0e4, "bf16", [200, 17], [[-1, 0, 1, 0], [-1, -1, 0, 2]], seed=6) as c:
        c.K = [synth.round_to_dtype(k * np.float32(key), "bf16") for k in c.K]
        c.kt = synth.round_to_dtype(c.kt * np.float32(key), "bf16")
        c.q = synth.round_to_dtype(c.q * np.float32(query), "bf16")
        for b, k in enumerate(c.K):
            c.store[b, :len(k)] = to_dev(k, "bf16")
        c.dq, c.dkt = to_dev(c.q, "bf16"), to_dev(c.kt, "bf16")
        c.call()
        assert c.status() == B.SLIM_OK
        c.check()


@pytest.mark.parametrize("d,H,dtype,lengths,n", [(384, 6, "f32", [1500], 8), (384, 6, "f32", [5003], 3), (1000, 10, "bf16", [2100, 40], 1), (200, 5, "f32", [900] * 3, 64)])
def test_long_rows_in_parts_on_the_cuda_cores(d, H, dtype, lengths, n):
    """The keys cut into up to 32 parts, whose sums the projection adds."""
    g = np.random.default_rng(n)
    with Case(d, H, 1.0e4, dtype, lengths, [random_parents(g, n) for _ in lengths], seed=6) as c:
        c.call()
        assert c.status() == B.SLIM_OK
        c.check()


@pytest.mark.parametrize("d,H,dtype,n", [(128, 2, "bf16", 2), (64, 1, "bf16", 1), (24, 3, "f32", 2)])
def test_the_largest_batch(d, H, dtype, n):
    g = np.random.default_rng(15)
    lengths = [int(x) for x in g.integers(0, 41, 2048)]
    with Case(d, H, 1.0e4, dtype, lengths, [random_parents(g, n) for _ in lengths], page=16, seed=9) as c:
        c.call()
        assert c.status() == B.SLIM_OK
        c.check()


def test_many_sequences_and_the_cuda_core_kernels_agree():
    g = np.random.default_rng(13)
    lengths = [int(x) for x in g.integers(0, 70, 150)]
    with Case(128, 2, 1.0e4, "bf16", lengths, [random_parents(g, 3) for _ in lengths], page=16, seed=8) as c:
        c.call()
        assert c.status() == B.SLIM_OK
        c.check()
        fast = c.o.clone()
        B.slim_set_path(c.ctx, B.SLIM_PATH_GENERIC)
        c.o.fill_(float("nan"))
        c.call()
        assert c.status() == B.SLIM_OK
        c.check()
        assert torch.equal(fast == 0, c.o == 0)


def test_a_layer_keeps_the_scratch_that_a_graph_uses():
    lay = SlimLayer(128, 2, 64, 1.0e4, "bf16", 1, 64, DEV)
    try:
        lay.set_wkv(np.eye(128))
        lay.k.normal_()
        q, kt = (torch.randn(1, 4, 128, device=DEV).bfloat16() for _ in range(2))
        lens, par = torch.tensor([50], dtype=torch.int32, device=DEV), torch.tensor([[-1, 0, 1, 1]], dtype=torch.int32, device=DEV)
        graph, o = torch.cuda.CUDAGraph(), torch.empty_like(q)
        with pytest.raises(RuntimeError):
            with torch.cuda.graph(torch.cuda.CUDAGraph()):
                lay.tree_decode(q, kt, lens, par, o)
        want = lay.tree_decode(q, kt, lens, par).clone()
        with torch.cuda.graph(graph):
            lay.tree_decode(q, kt, lens, par, o)
        big = [torch.randn(1, 64, 128, device=DEV).bfloat16() for _ in range(2)]
        lay.tree_decode(*big, lens, torch.arange(-1, 63, dtype=torch.int32, device=DEV)[None].contiguous())      # a larger scratch
        other = [torch.full((1 << 20,), 255, dtype=torch.uint8, device=DEV) for _ in range(64)]
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want) and all(bool((x == 255).all()) for x in other)
    finally:
        lay.close()


def test_layers_on_streams_at_once_and_eviction_in_a_graph():
    torch.manual_seed(0)
    layers, calls = [], []
    try:
        for d, H, dtype, batch, t_cap in [(1024, 8, "bf16", 3, 700), (768, 8, "bf16", 2, 900), (640, 10, "bf16", 4, 500), (384, 6, "f32", 2, 900)]:
            lay = SlimLayer(d, H, d // H, 1.0e4, dtype, batch, t_cap, DEV)
            layers.append(lay)
            lay.set_wkv(np.random.default_rng(d).standard_normal((d, d)) / np.sqrt(d))
            lay.k.normal_()
            q, kt = (torch.randn(batch, 7, d, device=DEV).to(lay.tdtype) for _ in range(2))
            lens = torch.randint(300, t_cap - 64, (batch,), dtype=torch.int32, device=DEV)
            par = torch.tensor([[-1, 0, 0, 1, 2, 3, 3]] * batch, dtype=torch.int32, device=DEV)
            calls.append((lay, q, kt, lens, par, q[:, 0].contiguous()))
        run = lambda lay, q, kt, lens, par, q1: (lay.tree_decode(q, kt, lens, par),
                                                 lay.accumulate_weights(q1, lens, torch.zeros(lay.batch, lay.t_cap, device=DEV)))
        want = [tuple(x.clone() for x in run(*c)) for c in calls]
        torch.cuda.synchronize()
        streams, got = [torch.cuda.Stream() for _ in calls], [[] for _ in calls]
        for _ in range(20):
            for k, c in enumerate(calls):
                with torch.cuda.stream(streams[k]):
                    got[k].append(run(*c))
        torch.cuda.synchronize()
        for k in range(len(calls)):
            assert all(torch.equal(x, y) for g in got[k] for x, y in zip(g, want[k])), k
            assert layers[k].device_status() == B.SLIM_OK
        # one layer's scratch in a graph that evicts and attends, eager calls of the same layer between the replays
        lay, q, kt, lens, par, _ = calls[0]
        K0, acc0 = lay.k.clone(), torch.rand(lay.batch, lay.t_cap, device=DEV)
        acc = acc0.clone()

        def shorten():
            return lay.evict(lens, acc, 200, 30), lay.tree_decode(q, kt, torch.clamp(lens, max=200), par)

        first = [x.clone() for x in shorten()]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            later = shorten()
        for _ in range(3):
            lay.k.copy_(K0)
            acc.copy_(acc0)
            graph.replay()
            assert all(torch.equal(x, y) for x, y in zip(first, later))
            lay.tree_decode(q, kt, lens, par)
    finally:
        torch.cuda.synchronize()
        for lay in layers:
            lay.close()


def test_broken_trees_and_lengths_are_reported():
    with Case(128, 2, 1.0e4, "bf16", [20, 20], [[-1, 0, 1], [-1, 0, 1]], seed=1) as c:
        c.dpar = torch.tensor([[-1, 1, 0], [-1, -2, 1]], dtype=torch.int32, device=DEV)     # its own parent; a child of padding
        c.call()
        assert c.status() == B.SLIM_ERR_TREE
        c.parents = np.array([[-1, -2, 0], [-1, -2, -2]], np.int32)
        c.check()
        c.dlen = torch.tensor([-5, 10 ** 9], dtype=torch.int32, device=DEV)                 # nothing cached; clamped to the capacity
        c.store[1] = 0
        c.call()
        assert c.status() == B.SLIM_ERR_TREE                 # the tree is still broken: of two reports the higher code stays
        c.dpar = torch.tensor([[-1, -2, 0], [-1, -2, -2]], dtype=torch.int32, device=DEV)
        c.call()
        assert c.status() == B.SLIM_ERR_CAPACITY
        assert torch.isfinite(c.o.float()).all()
    with Case(128, 2, 1.0e4, "bf16", [20, 40], [[-1], [-1]], page=16, seed=1) as c:
        c.store[0] = 0                                       # what a page id outside the pool is replaced by
        c.table[1, 1] = 10 ** 6
        c.call()
        assert c.status() == B.SLIM_ERR_CAPACITY
        assert torch.isfinite(c.o.float()).all()


def test_refusals():
    with Case(128, 2, 1.0e4, "bf16", [20], [[-1, 0]], seed=1) as c:
        L, st = B.lib(), torch.cuda.current_stream().cuda_stream
        p = lambda x: x.data_ptr() if torch.is_tensor(x) else x
        call = lambda **k: L.slim_tree_decode(*[p(k.get(name, v)) for name, v in (
            ("ctx", c.ctx), ("q", c.dq), ("k_tree", c.dkt), ("cache", c.cache), ("lengths", c.dlen), ("parents", c.dpar), ("n", c.n),
            ("o", c.o), ("ws", c.ws), ("st", st))])
        assert call() == B.SLIM_OK
        for k in ("q", "k_tree", "cache", "lengths", "parents", "o", "ws"):
            assert call(**{k: None}) == B.SLIM_ERR_INVALID_ARG, k
        for k, x in (("q", c.dq), ("k_tree", c.dkt), ("o", c.o), ("ws", c.ws)):
            assert call(**{k: x.data_ptr() + 8}) == B.SLIM_ERR_INVALID_ARG, k
        for n in (0, -1, 65):
            assert call(n=n) == B.SLIM_ERR_INVALID_ARG
            assert L.slim_tree_workspace_bytes(c.ctx, 1, 16, n) == 0
        other = B.slim_create(128, 2, 64, 1.0e4, B.SLIM_BF16)
        assert call(ctx=other) == B.SLIM_ERR_INVALID_ARG       # a cache of another context
        cache = B.slim_cache_create(other, c.store, 1, c.t_cap)
        assert call(ctx=other, cache=cache) == B.SLIM_ERR_NO_WEIGHTS
        B.slim_cache_destroy(cache); B.slim_destroy(other)
        fp8 = SlimLayer(128, 2, 64, 0.0, "fp8", 1, 32, DEV)
        fp8.set_wkv(np.eye(128))
        with pytest.raises(B.SlimError) as e:
            fp8.tree_decode(c.dq, c.dkt, c.dlen, c.dpar)
        assert e.value.status == B.SLIM_ERR_UNSUPPORTED
        with pytest.raises(B.SlimError) as e:
            fp8.tree_commit(c.dkt, c.dlen, c.dpar, c.dlen)
        assert e.value.status == B.SLIM_ERR_UNSUPPORTED
        fp8.close()
        lay = SlimLayer(128, 2, 64, 1.0e4, "bf16", 1, 32, DEV)
        lay.set_wkv(np.eye(128))
        for bad in (dict(q=c.dq.float()), dict(k_tree=c.dkt[:, :1]), dict(lengths=c.dlen.long()), dict(parents=c.dpar.cpu()),
                    dict(q=c.dq.transpose(1, 2).contiguous().transpose(1, 2)), dict(o=c.o[:, :1])):
            with pytest.raises(ValueError):
                lay.tree_decode(**{**dict(q=c.dq, k_tree=c.dkt, lengths=c.dlen, parents=c.dpar), **bad})
        lay.close()


def test_repeatable_on_streams_and_in_graphs():
    g = np.random.default_rng(11)
    with Case(512, 4, 1.0e4, "bf16", [900, 130], [random_parents(g, 9) for _ in range(2)], seed=2) as c:
        c.call()
        torch.cuda.synchronize()
        want = c.o.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        c.o.fill_(float("nan"))
        side.wait_stream(torch.cuda.current_stream())
        c.call(side)
        side.synchronize()
        assert torch.equal(c.o, want)
        graphs = []
        for _ in range(2):                                   # two graphs that share the workspace, replayed in turn
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                c.call()
            graphs.append(graph)
        for graph in graphs + graphs:
            c.o.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(c.o, want)
        c.lengths[:] = [500, 77]                             # a replay reads the lengths that are there then
        c.dlen.copy_(torch.from_numpy(c.lengths))
        c.K = [c.K[0][:500], c.K[1][:77]]
        graphs[0].replay()
        assert c.status() == B.SLIM_OK
        c.check()


@pytest.mark.parametrize("d,H,n,lengths", [(512, 4, 40, [130, 5]), (4096, 32, 17, [3000, 64, 0]), (1280, 20, 64, [700])])
def test_two_hundred_calls_give_the_same_bits(d, H, n, lengths):
    """Calls back to back, with CTAs that have no block of their own among them."""
    g = np.random.default_rng(n)
    with Case(d, H, 1.0e4, "bf16", lengths, [random_parents(g, n) for _ in lengths], seed=4) as c:
        c.call()
        want = c.o.clone()
        differ = torch.zeros((), dtype=torch.int64, device=DEV)
        for _ in range(200):
            c.call()
            differ += (c.o != want).sum()
        assert c.status() == B.SLIM_OK
        assert differ.item() == 0


def test_tree_pages_behind_four_billion_elements():
    """A pool whose last pages lie beyond 2^32 elements from its start."""
    d, H, page, L = 4096, 32, 64, 200
    pages = (1 << 32) // (page * d) + 8
    with Case(d, H, 1.0e4, "bf16", [L], [[-1, 0, 0, 1]], page=page, seed=9) as small:
        small.call()
        torch.cuda.synchronize()
        pool = torch.empty((pages, page, d), dtype=torch.bfloat16, device=DEV)
        mp = small.table.shape[1]
        pool[-mp:] = small.store[small.table[0].long()]
        table = torch.arange(pages - mp, pages, dtype=torch.int32, device=DEV)[None].contiguous()
        cache = B.slim_cache_create_paged(small.ctx, pool, pages, page, table, 1, mp)
        st = torch.cuda.current_stream().cuda_stream
        o = torch.empty_like(small.o)
        B.slim_tree_decode(small.ctx, small.dq, small.dkt, cache, small.dlen, small.dpar, 4, o, small.ws, st)
        assert small.status() == B.SLIM_OK
        assert torch.equal(o, small.o)
        path, count = torch.tensor([[0, 1, 3, -1]], dtype=torch.int32, device=DEV), torch.tensor([3], dtype=torch.int32, device=DEV)
        B.slim_tree_commit(small.ctx, cache, small.dkt, small.dlen, path, count, 4, st)
        assert small.status() == B.SLIM_OK
        rows = pool[-mp:].view(-1, d)
        assert torch.equal(rows[L:L + 3], small.dkt[0, [0, 1, 3]]) and rows[L + 3:small.t_cap].isnan().all()
        B.slim_cache_destroy(cache)


# ------------------------------------------------------------------------------------------------ verification
def run_verify(ctx, p, q, tokens, parents, r):
    Bn, n, V = p.shape
    dev = lambda x, t: torch.from_numpy(np.ascontiguousarray(x)).to(DEV, t)
    path = torch.full((Bn, n), 77, dtype=torch.int32, device=DEV)
    count, nxt = (torch.full((Bn,), 77, dtype=torch.int32, device=DEV) for _ in range(2))
    args = [dev(p, torch.float32), dev(q, torch.float32), dev(tokens, torch.int32), dev(parents, torch.int32), dev(r, torch.float32)]
    B.slim_tree_verify(ctx, *args, Bn, n, V, path, count, nxt, torch.cuda.current_stream().cuda_stream)
    return path.cpu().numpy(), count.cpu().numpy(), nxt.cpu().numpy(), B.slim_device_status(ctx, torch.cuda.current_stream().cuda_stream)


@pytest.fixture()
def ctx():
    c = B.slim_create(64, 1, 64, 0.0, B.SLIM_F32)
    yield c
    B.slim_destroy(c)


def draws(g, Bn, n, V, kids, sharp=2.0, close=1.0):
    lp = sharp * g.standard_normal((Bn, n, V))
    lq = lp + close * g.standard_normal((Bn, n, V))
    p, q = (np.exp(x - x.max(-1, keepdims=True)) for x in (lp, lq))
    p, q = ((x / x.sum(-1, keepdims=True)).astype(np.float32) for x in (p, q))
    parents, tokens = np.full((Bn, n), -2, np.int32), np.zeros((Bn, n), np.int32)
    for b in range(Bn):
        used = {0: 0}
        parents[b, 0] = -1
        for i in range(1, n if b % 4 else max(1, n - 2)):
            u = int(g.choice([x for x in used if used[x] < kids][-3:]))
            used[u] += 1
            used[i] = 0
            parents[b, i] = u
            tokens[b, i] = g.choice(V, p=q[b, u].astype(np.float64) / q[b, u].astype(np.float64).sum())
    return p, q, tokens, parents, g.random((Bn, n)).astype(np.float32)


@pytest.mark.parametrize("Bn,n,V,kids", [(1, 1, 1, 1), (3, 4, 2, 2), (40, 8, 5, 4), (16, 12, 131, 3), (9, 64, 1000, 5), (5, 6, 32003, 2), (2, 5, 131072, 3)])
def test_verification_against_the_definition(ctx, Bn, n, V, kids):
    g = np.random.default_rng(V)
    p, q, tokens, parents, r = draws(g, Bn, n, V, kids)
    path, count, nxt, status = run_verify(ctx, p, q, tokens, parents, r)
    assert status == B.SLIM_OK
    for b in range(Bn):
        want, t = do.verify(p[b], q[b], tokens[b], parents[b], r[b])
        assert list(path[b]) == want + [-1] * (n - len(want)) and count[b] == len(want)
        assert nxt[b] == t


def test_verification_edges(ctx):
    V = 700
    one = np.zeros((1, 3, V), np.float32)
    one[0, 0, 5] = 1.0; one[0, 1, 9] = 1.0; one[0, 2, 11] = 1.0
    tok, par = np.array([[0, 5, 9]], np.int32), np.array([[-1, 0, 1]], np.int32)
    # the draft is the target: everything is accepted, whatever the numbers; the draw is the only token there is
    path, count, nxt, st = run_verify(ctx, one, one, tok, par, np.array([[0.999, 0.999, 0.0]], np.float32))
    assert st == B.SLIM_OK and count[0] == 3 and nxt[0] == 11
    # a token that the target gives no probability is never accepted, not even for r = 0
    path, count, nxt, st = run_verify(ctx, one, one, np.array([[0, 6, 9]], np.int32), par, np.zeros((1, 3), np.float32))
    assert count[0] == 1 and nxt[0] == 5 and list(path[0]) == [0, -1, -1]
    # nothing left of the residual (p = q and a token outside both): the distribution stays; no positive value at all: -1
    path, count, nxt, st = run_verify(ctx, 0 * one, one, tok, par, np.full((1, 3), 0.5, np.float32))
    assert count[0] == 1 and nxt[0] == -1 and st == B.SLIM_OK
    # tokens outside the vocabulary and parents that are not earlier nodes are padding, and reported
    path, count, nxt, st = run_verify(ctx, one, one, np.array([[0, V, 9]], np.int32), par, np.zeros((1, 3), np.float32))
    assert st == B.SLIM_ERR_TREE and count[0] == 1
    path, count, nxt, st = run_verify(ctx, one, one, tok, np.array([[-1, 2, 1]], np.int32), np.zeros((1, 3), np.float32))
    assert st == B.SLIM_ERR_TREE and count[0] == 1
    # draws at the ends of the range
    flat = np.full((1, 1, V), 1.0 / V, np.float32)
    for r0, want in ((0.0, 0), (np.float32(1 - 2.0 ** -24), V - 1)):
        _, _, nxt, _ = run_verify(ctx, flat, flat, np.zeros((1, 1), np.int32), np.array([[-1]], np.int32), np.array([[r0]], np.float32))
        assert nxt[0] == want
    # NaN where a row of probabilities should be: no token, and the call comes back
    path, count, nxt, st = run_verify(ctx, one * np.nan, one, tok, par, np.full((1, 3), 0.5, np.float32))
    assert count[0] == 1 and nxt[0] == -1


def test_verify_refusals(ctx):
    x = torch.zeros(64, device=DEV)
    i = torch.zeros(64, dtype=torch.int32, device=DEV)
    for n, V, b in ((0, 4, 1), (65, 4, 1), (1, 0, 1), (1, 4, 0), (1, 4, 4096)):
        with pytest.raises(B.SlimError) as e:
            B.slim_tree_verify(ctx, x, x, i, i, x, b, n, V, i, i, i)
        assert e.value.status == B.SLIM_ERR_INVALID_ARG


# ------------------------------------------------------------------------------------------------ commit, and the whole loop
@pytest.mark.parametrize("d,H,dtype,page", [(128, 2, "bf16", 0), (128, 2, "bf16", 16), (10, 5, "bf16", 0), (6, 3, "f32", 0), (384, 6, "f32", 32)])
def test_commit_writes_accepted_rows_only(d, H, dtype, page):
    n = 6
    with Case(d, H, 0.0, dtype, [30, 17, 0, 40, 12], [[-1] * n] * 5, page=page, seed=4, t_cap=48) as c:
        path = torch.tensor([[0, 2, 5, -1, -1, -1], [0, 1, 2, 3, 4, 5], [3, -1, -1, -1, -1, -1], [0, 6, -1, -1, -1, -1], [-1] * 6],
                            dtype=torch.int32, device=DEV)
        count = torch.tensor([3, 6, 1, 2, 0], dtype=torch.int32, device=DEV)
        before = c.store.clone()
        st = torch.cuda.current_stream().cuda_stream
        B.slim_tree_commit(c.ctx, c.cache, c.dkt, c.dlen, path, count, n, st)
        assert c.status() == B.SLIM_ERR_TREE                 # sequence 3 names token 6 of 6: left as it was
        want = before.clone()
        for b, rows in ((0, [0, 2, 5]), (1, range(6)), (2, [3])):
            for j, i in enumerate(rows):
                want[c.where(b, int(c.lengths[b]) + j)] = c.dkt[b, i]
        assert torch.equal(torch.nan_to_num(c.store.float(), nan=1e9), torch.nan_to_num(want.float(), nan=1e9))
        over = torch.tensor([c.t_cap - 2] * 5, dtype=torch.int32, device=DEV)
        B.slim_tree_commit(c.ctx, c.cache, c.dkt, over, path, torch.tensor([3] * 5, dtype=torch.int32, device=DEV), n, st)
        assert c.status() in (B.SLIM_ERR_CAPACITY, B.SLIM_ERR_TREE)
        B.slim_tree_commit(c.ctx, c.cache, c.dkt, c.dlen, path, torch.tensor([-1, 7, 0, 0, 0], dtype=torch.int32, device=DEV), n, st)
        assert c.status() == B.SLIM_ERR_TREE
        assert torch.equal(torch.nan_to_num(c.store.float(), nan=1e9), torch.nan_to_num(want.float(), nan=1e9))


@pytest.mark.parametrize("dtype,tol", [("f32", 1e-4), ("bf16", 2e-2)])
def test_draft_verify_commit_and_decode_go_together(dtype, tol):
    """Two rounds of drafting on one layer: the accepted path's outputs are what decode steps over the committed cache give."""
    d, H, n, V, Bn = 512, 4, 6, 50, 3
    g = np.random.default_rng(21)
    lay = SlimLayer(d, H, d // H, 1.0e4, dtype, Bn, 128, DEV)
    try:
        lay.set_wkv(synth.round_to_dtype(g.standard_normal((d, d)) / np.sqrt(d), dtype).astype(np.float64))
        rnd = lambda *s: to_dev(synth.round_to_dtype(g.standard_normal(s), dtype), dtype)
        lengths = torch.tensor([40, 0, 63], dtype=torch.int32, device=DEV)
        lay.append_k(rnd(Bn, 64, d), torch.zeros(Bn, dtype=torch.int32, device=DEV))
        for _ in range(2):
            p, q, tokens, parents, r = draws(g, Bn, n, V, 2, close=0.3)
            dev = lambda x, t: torch.from_numpy(np.ascontiguousarray(x)).to(DEV, t)
            parents_d = dev(parents, torch.int32)
            tq, tk = rnd(Bn, n, d), rnd(Bn, n, d)
            o = lay.tree_decode(tq, tk, lengths, parents_d)
            path, count, nxt = lay.tree_verify(dev(p, torch.float32), dev(q, torch.float32), dev(tokens, torch.int32), parents_d, dev(r, torch.float32))
            lay.tree_commit(tk, lengths, path, count)
            assert lay.device_status() == B.SLIM_OK
            hp, hc = path.cpu().numpy(), count.cpu().numpy()
            for j in range(int(hc.max())):
                at = [hp[b, j] if j < hc[b] else hp[b, 0] for b in range(Bn)]
                steps = torch.stack([tq[b, at[b]] for b in range(Bn)])
                upto = (lengths + torch.tensor([j + 1 if j < hc[b] else 1 for b in range(Bn)], device=DEV)).int()
                one = lay.decode(steps.contiguous(), upto).clone()
                for b in range(Bn):
                    rms = one[b].pow(2).mean().sqrt()
                    assert ((o[b, at[b]].float() - one[b]).abs() / torch.maximum(one[b].abs(), rms)).max().item() <= tol
            lengths += count
            assert int(nxt.min()) >= 0
    finally:
        lay.close()


# ------------------------------------------------------------------------------------------------ rows that are not attended, numbers that are not finite
@pytest.mark.parametrize("value", [1.0e5, -1.0e10, 1.0e30, 3.0e38, float("inf")])
@pytest.mark.parametrize("d,H,theta,dtype,page,n", [
    (512, 4, 1.0e4, "bf16", 0, 16), (512, 8, 1.0e4, "bf16", 16, 9), (384, 4, 0.0, "bf16", 64, 33), (384, 6, 1.0e4, "f32", 0, 5)])
def test_rows_that_are_not_attended_hold_large_numbers(d, H, theta, dtype, page, n, value):
    """Rows behind the lengths, unused pages and padding drafts hold numbers beyond the range of the 16-bit products."""
    g = np.random.default_rng(n)
    lengths = [1, 15, 17, 100, 130, 0, 250]
    parents = [random_parents(g, n) for _ in lengths]
    parents[1] = [-1, 0] + [-2] * (n - 2)
    with Case(d, H, theta, dtype, lengths, parents, page, seed=n + 1) as c:
        was = [(x, x.isnan()) for x in (c.store, c.dq, c.dkt)]
        for x, dead in was:
            x[dead] = 0
        c.call()
        want = c.o.clone()
        for x, dead in was:
            x[dead] = value
        c.call()
        assert c.status() == B.SLIM_OK
        c.check()
        assert torch.equal(c.o, want)


@pytest.mark.parametrize("key", [1.0e6, 1.0e12, 1.0e30])
def test_neighbouring_sequences_and_drafts_hold_large_numbers(key):
    """A tile of 16 rows reaches into the next sequence's rows and drafts, which lie `key` times higher (and its queries as
    much lower); a capacity and a number of drafts that are no multiples of 16."""
    g = np.random.default_rng(3)
    with Case(512, 4, 1.0e4, "bf16", [107, 107, 50, 107], [random_parents(g, 5, pad=False) for _ in range(4)], seed=8, t_cap=107) as c:
        for b in (1, 3):
            c.K[b] = synth.round_to_dtype(c.K[b] * np.float32(key), "bf16")
            c.kt[b] = synth.round_to_dtype(c.kt[b] * np.float32(key), "bf16")
            c.q[b] = synth.round_to_dtype(c.q[b] / np.float32(key), "bf16")
            c.store[b, :107] = to_dev(c.K[b], "bf16")
        c.dq, c.dkt = to_dev(c.q, "bf16"), to_dev(c.kt, "bf16")
        c.call()
        assert c.status() == B.SLIM_OK
        c.check()


@pytest.mark.parametrize("dtype,key", [("bf16", 1.0e6), ("bf16", 1.0e10), ("bf16", 1.0e30), ("f32", 1.0e10)])
def test_a_key_far_above_its_neighbours(dtype, key):
    """Rows that are `key` in one element, against which the queries are positive: their argument is so low that their
    probability is 0, so the others' results are those without them (no rotation, so the positions do not matter)."""
    d, H, n = 256, 2, 9
    out = np.array([3, 40, 41, 77, 199, 255])
    with Case(d, H, 0.0, dtype, [260, 140], [[-1, 0, 1, -1, 0, 4, 5, 6, -1], [-1] * 9], seed=5) as c:
        c.q[..., ::128] = 1.0 + np.abs(c.q[..., ::128])
        for b in range(2):
            rows = out[out < len(c.K[b])]
            c.K[b][rows, ::128] = -key
            c.K[b] = synth.round_to_dtype(c.K[b], dtype)
            c.store[b, :len(c.K[b])] = to_dev(c.K[b], dtype)
            c.K[b] = np.delete(c.K[b], rows, axis=0)
        c.q = synth.round_to_dtype(c.q, dtype)
        c.dq = to_dev(c.q, dtype)
        c.call()
        assert c.status() == B.SLIM_OK
        c.check()


@pytest.mark.parametrize("d,H,dtype,L", [(512, 4, "bf16", 40), (512, 8, "bf16", 300), (384, 6, "f32", 40), (384, 6, "f32", 1500), (200, 2, "bf16", 100)])
def test_padding_gets_zeros_beside_keys_that_are_not_finite(d, H, dtype, L):
    """0 x infinity is no number: a padding token's row is 0 all the same, whatever the cached rows and live drafts hold."""
    with Case(d, H, 1.0e4, dtype, [L, L], [[-1, 0, -2, 0, -7], [-2] * 5], seed=2) as c:
        c.dkt[0, 3, 3] = float("inf")
        c.store[0, 11, 5:9] = float("nan")
        c.store[1, 7, d - 1] = float("-inf")
        c.call()
        assert c.status() == B.SLIM_OK
        assert (c.o[0, [2, 4]] == 0).all() and (c.o[1] == 0).all()
        assert not torch.isfinite(c.o[0, [0, 1, 3]].float()).any()


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("d,H,dtype,n", [(512, 4, "bf16", 12), (512, 8, "bf16", 3), (384, 4, "bf16", 40), (384, 6, "f32", 5), (200, 2, "bf16", 5)])
def test_a_query_that_is_not_finite_gives_no_numbers(d, H, dtype, n, value):
    """One token's query, and one head of another's: NaN in what they determine, nothing else changes."""
    g = np.random.default_rng(n)
    lengths = [0, 40, 300]
    d_k = d // H
    with Case(d, H, 1.0e4, dtype, lengths, [random_parents(g, n, pad=False) for _ in lengths], seed=n) as c:
        c.call()
        torch.cuda.synchronize()
        want = c.o.clone()
        c.check(want)
        c.dq[:, 1] = value
        c.dq[:, 2, d_k] = value                              # an element of head 1
        c.call()
        assert c.status() == B.SLIM_OK
        bad = torch.zeros_like(c.o, dtype=torch.bool)
        bad[:, 1] = True
        bad[:, 2, d_k:2 * d_k] = True
        assert c.o[bad].isnan().all()
        c.check(torch.where(bad, want, c.o))


@pytest.mark.parametrize("d,H,dtype", [(512, 4, "bf16"), (512, 8, "bf16"), (384, 6, "f32"), (200, 2, "bf16")])
def test_a_key_that_is_not_finite_reaches_every_token(d, H, dtype):
    """... of its sequence, also the first token of an empty context; padding still gets a zero row."""
    n = 5
    parents = [[-1, 0, -2, 0, 3]] * 5
    with Case(d, H, 1.0e4, dtype, [0, 40, 40, 150, 40], parents, seed=2) as c:
        c.dkt[0, 0, 7] = float("nan")                        # nothing cached: the tokens' own keys are all there is
        c.dkt[1, 4, 3] = float("inf")                        # a leaf, which the others do not attend
        c.store[2, 11] = float("nan")
        c.store[3, 5, d - 1] = float("-inf")
        c.call()
        assert c.status() == B.SLIM_OK
        live = torch.tensor([0, 1, 3, 4], device=DEV)
        assert not torch.isfinite(c.o[:4, live].float()).any()
        assert (c.o[:, 2] == 0).all()
        got = c.o.clone()
        got[:4] = 0
        c.lengths, c.K = c.lengths[4:], c.K[4:]
        c.q, c.kt, c.parents, c.batch = c.q[4:], c.kt[4:], c.parents[4:], 1
        c.check(got[4:])


def test_verification_reports_children_of_padding(ctx):
    V = 40
    one = np.zeros((2, 4, V), np.float32)
    one[..., 5] = 1.0
    tok = np.full((2, 4), 5, np.int32)
    par = np.array([[-1, -2, 1, 0], [-1, 0, 1, 2]], np.int32)          # token 2 of the first hangs on padding
    path, count, nxt, st = run_verify(ctx, one, one, tok, par, np.zeros((2, 4), np.float32))
    assert st == B.SLIM_ERR_TREE
    assert list(path[0]) == [0, 3, -1, -1] and list(path[1]) == [0, 1, 2, 3] and list(count) == [2, 4] and list(nxt) == [5, 5]
    par[0] = [-5, -2, -2, 0]                                           # node 0 is the root whatever stands there
    path, count, nxt, st = run_verify(ctx, one, one, tok, par, np.zeros((2, 4), np.float32))
    assert st == B.SLIM_OK and list(path[0]) == [0, 3, -1, -1]


@pytest.mark.parametrize("V", [700, 701])
@pytest.mark.parametrize("rejections", [1, 2, 3, 5])
def test_a_nan_among_the_probabilities_is_not_lost_by_a_rejection(ctx, V, rejections):
    """W = max(W - S q, 0) of a NaN is a NaN, in p or in q: no token is drawn from such a row."""
    n = rejections + 1
    g = np.random.default_rng(V)
    p = np.full((3, n, V), 1.0 / V, np.float32)
    q = p.copy()
    tok = np.tile(np.arange(n, dtype=np.int32), (3, 1))
    p[:, 0, :n] = 0.0                                                  # none of the drafted tokens is accepted
    p[0, 0, V - 2] = np.nan
    q[1, 0, 300] = np.nan
    par = np.tile(np.array([-1] + [0] * rejections, np.int32), (3, 1))
    path, count, nxt, st = run_verify(ctx, p, q, tok, par, g.random((3, n)).astype(np.float32))
    assert st == B.SLIM_OK and list(count) == [1, 1, 1]
    assert list(nxt[:2]) == [-1, -1] and nxt[2] >= n


def test_scratch_is_given_back_and_shared():
    """A layer holds one scratch however its calls grow, captured ones aside; layers may share one."""
    d, H, batch, t_cap = 512, 4, 2, 600
    lens, W = torch.tensor([500, 77], dtype=torch.int32, device=DEV), np.eye(d)
    par = lambda n: torch.arange(-1, n - 1, dtype=torch.int32, device=DEV).repeat(batch, 1)
    rnd = lambda n: torch.randn(batch, n, d, device=DEV).bfloat16()
    lay = SlimLayer(d, H, d // H, 1.0e4, "bf16", batch, t_cap, DEV)
    other = None
    try:
        lay.set_wkv(W)
        lay.k.normal_()
        most = max(B.slim_tree_workspace_bytes(lay.ctx, batch, t_cap, n) for n in range(1, 65))
        q, kt, o = rnd(64), rnd(64), torch.empty(batch, 64, d, dtype=torch.bfloat16, device=DEV)
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        for n in range(1, 65):
            lay.tree_decode(q[:, :n].contiguous(), kt[:, :n].contiguous(), lens, par(n), o.view(-1)[:batch * n * d].view(batch, n, d))
        held = torch.cuda.memory_allocated() - before
        assert held <= most + (4 << 20), (held, most)
        want = lay.tree_decode(q, kt, lens, par(64)).clone()
        other = SlimLayer(d, H, d // H, 1.0e4, "bf16", batch, t_cap, DEV, scratch=lay.scratch)
        other.set_wkv(W)
        other.k.copy_(lay.k)
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        assert torch.equal(other.tree_decode(q, kt, lens, par(64), o), want)
        assert torch.cuda.memory_allocated() == before
        # sized ahead: a capture may be the first call
        third = SlimLayer(d, H, d // H, 1.0e4, "bf16", batch, t_cap, DEV)
        third.set_wkv(W)
        third.k.copy_(lay.k)
        third.reserve_scratch(64)
        graph, o3 = torch.cuda.CUDAGraph(), torch.empty_like(o)
        p64 = par(64)
        with torch.cuda.graph(graph):
            third.tree_decode(q, kt, lens, p64, o3)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o3, want)
        third.close()
        for n in (-1, 65):
            with pytest.raises(ValueError):
                lay.reserve_scratch(n)
        with pytest.raises(ValueError):
            SlimLayer(d, H, d // H, 1.0e4, "bf16", batch, t_cap, DEV, scratch=torch.empty(5, device=DEV))
    finally:
        lay.close()
        if other is not None:
            other.close()


def test_scratch_that_grows_on_another_stream():
    """Calls on a stream that the scratch was not made on; when it grows there, the smaller one must not be handed to the
    first stream while calls still use it."""
    d, H, batch, t_cap = 1024, 8, 4, 4000
    lay = SlimLayer(d, H, d // H, 1.0e4, "bf16", batch, t_cap, DEV)
    try:
        lay.set_wkv(np.eye(d))
        lay.k.normal_()
        lens = torch.full((batch,), 3900, dtype=torch.int32, device=DEV)
        args = [[torch.randn(batch, n, d, device=DEV).bfloat16() for _ in range(2)] +
                [lens, torch.arange(-1, n - 1, dtype=torch.int32, device=DEV).repeat(batch, 1)] for n in (8, 64)]
        want = lay.tree_decode(*args[0]).clone()
        size, side = lay._extra[-1].numel(), torch.cuda.Stream()
        outs = [torch.empty_like(want) for _ in range(40)]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for o in outs:
                lay.tree_decode(*args[0], o)
            lay.tree_decode(*args[1])
        junk = [torch.full((size,), 255, dtype=torch.uint8, device=DEV) for _ in range(3)]
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o in outs) and len(junk) == 3
        assert lay.device_status() == B.SLIM_OK
    finally:
        lay.close()


def test_a_layer_on_the_current_device():
    """A device without an index is the current one."""
    lay = SlimLayer(128, 2, 64, 1.0e4, "bf16", 1, 64, "cuda")
    try:
        lay.set_wkv(np.eye(128))
        lay.k.normal_()
        q, kt = (torch.randn(1, 4, 128, device=DEV).bfloat16() for _ in range(2))
        i = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
        o = lay.tree_decode(q, kt, i(50), i([-1, 0, 1, 1]))
        assert torch.isfinite(o.float()).all() and lay.device_status() == B.SLIM_OK
        acc = lay.accumulate_weights(q[:, 0].contiguous(), i(50), torch.zeros(1, 64, device=DEV))
        assert abs(acc.sum().item() - 2) < 100 * 2.0 ** -23     # two heads, 50 rows: a hundred roundings
    finally:
        lay.close()


def test_commit_refuses_other_numbers_of_dimensions():
    lay = SlimLayer(128, 2, 64, 1.0e4, "bf16", 1, 64, DEV)
    try:
        kt = torch.randn(1, 4, 128, device=DEV).bfloat16()
        i = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
        for bad in (kt[0], kt[0, 0], kt[None]):
            with pytest.raises(ValueError):
                lay.tree_commit(bad, i(50), i([0, 1, -1, -1]), i(2))
        lay.tree_commit(kt, i(50), i([0, 1, -1, -1]), i(2))
        assert lay.device_status() == B.SLIM_OK
    finally:
        lay.close()


def test_a_graph_outlives_longer_position_tables():
    """A larger cache of the context, or more reserved positions, make longer position tables; a graph captured before goes on
    with those that it was captured with."""
    with Case(512, 4, 1.0e4, "bf16", [900, 130], [[-1, 0, 1, 0]] * 2, seed=2) as c:
        c.call()
        torch.cuda.synchronize()
        want = c.o.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.call()
        for rows in (5000, 100_000, 1_000_000):
            B.slim_reserve_positions(c.ctx, rows)
            other = [torch.full((1 << 20,), 255, dtype=torch.uint8, device=DEV) for _ in range(32)]
            c.o.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(c.o, want) and all(bool((x == 255).all()) for x in other)
        c.o.zero_()
        c.call()
        assert c.status() == B.SLIM_OK and torch.equal(c.o, want)


def attention_in_64_bits(c, b):
    """(o, mass, arg) of oracle.draft_oracle.tree_attention for sequence b, by plain torch operations on the device."""
    n, d, H, L = c.n, c.d, c.H, len(c.K[b])
    d_k, half = d // H, d // H // 2
    chains = do.tree_chains(list(c.parents[b]))
    see = torch.zeros(n, L + n, dtype=torch.bool, device=DEV)
    depth = torch.zeros(n, dtype=torch.float64, device=DEV)
    for i, chain in enumerate(chains):
        if chain:
            see[i, :L] = True
            see[i, [L + j for j in chain]] = True
            depth[i] = len(chain) - 1
    rows = torch.cat([to_dev(c.K[b], c.dtype), to_dev(np.nan_to_num(c.kt[b]), c.dtype)]).double()
    q = to_dev(np.nan_to_num(c.q[b]), c.dtype).double()
    W = torch.from_numpy(c.W).to(DEV)
    pos = torch.cat([torch.arange(L, device=DEV, dtype=torch.float64), L + depth])
    freq = c.theta ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half) if c.theta else torch.zeros(half, dtype=torch.float64, device=DEV)

    def turned(x, at):
        a = at[:, None] * freq
        x1, x2 = x[:, :half], x[:, half:]
        return torch.cat([x1 * a.cos() + x2 * a.sin(), x2 * a.cos() - x1 * a.sin()], 1)

    o, mass = (torch.zeros(n, d, dtype=torch.float64, device=DEV) for _ in range(2))
    arg = torch.zeros(n, dtype=torch.float64, device=DEV)
    for h in range(H):
        cols = slice(h * d_k, (h + 1) * d_k)
        qh, kh = turned(q[:, cols], L + depth), turned(rows[:, cols], pos)
        p = torch.softmax((qh @ kh.T / d_k ** 0.5).masked_fill(~see, -torch.inf), 1).nan_to_num()
        o[:, cols] = (p @ rows) @ W[:, cols]
        mass[:, cols] = (p @ rows.abs()) @ W[:, cols].abs()
        arg = torch.maximum(arg, (qh.abs() @ kh.abs().T / d_k ** 0.5).masked_fill(~see, 0).amax(1))
    return o.cpu().numpy(), mass.cpu().numpy(), arg.cpu().numpy()


@pytest.mark.parametrize("d,H,n,lengths,page", [
    (512, 8, 32, [200_003], 0),                              # the keys of every tile in parts, each taken as a whole by a pair
    (1024, 8, 64, [120_017], 0),                             # ... and two accumulators, a rest that is cut once more
    (1024, 16, 40, [70_001, 30_000], 64),                    # ragged, paged: all of it cut where the pairs' shares end
    (4096, 32, 17, [3000, 64, 0, 1], 0), (1280, 20, 64, [700, 2047], 16)])
def test_long_contexts_and_wide_models_on_the_tensor_cores(d, H, n, lengths, page):
    g = np.random.default_rng(n + d)
    with Case(d, H, 1.0e4, "bf16", lengths, [random_parents(g, n) for _ in lengths], page, seed=n) as c:
        c.call()
        assert c.status() == B.SLIM_OK
        got = c.o.float().cpu().numpy().astype(np.float64)
        for b in range(c.batch):
            o, mass, arg = attention_in_64_bits(c, b)
            tol = tolerance(o, mass, arg, len(c.K[b]) + n, d, d // H, "bf16", True)
            err = np.abs(got[b] - o)
            assert np.all(err <= tol), f"sequence {b}: {np.max(err / tol):.2f} of the bound"
            # In norm: the keys are random and know nothing of the roundings, so a weight's relative error moves the sum by no
            # more than its size.  P's half step 2^-8 and the output's, 2^-8; the arguments' (2 x 2^-11 of each of d_k products
            # of random signs, whose sum has variance 1) are a tenth of that, and half steps are half as large on average
            assert np.linalg.norm(err) <= 2.0 ** -7 * np.linalg.norm(o)
            for i, chain in enumerate(do.tree_chains(list(c.parents[b]))):
                if not chain:
                    assert np.all(got[b, i] == 0)


@pytest.mark.parametrize("dtype", [B.SLIM_F32, B.SLIM_BF16])
def test_a_cache_of_x_rows_is_refused(dtype):
    """An X-cache with square projections: its rows are no keys, so products of the query with them are no scores."""
    d, H, td = 128, 2, torch.float32 if dtype == B.SLIM_F32 else torch.bfloat16
    c = B.slim_xcache_create(d, H, 64, dtype)
    try:
        g = np.random.default_rng(0)
        B.slim_xcache_set_weights(c, g.standard_normal((d, d)), g.standard_normal((d, d)))
        store, x = torch.zeros(1, 32, d, dtype=td, device=DEV), torch.zeros(1, 2, d, dtype=td, device=DEV)
        cache = B.slim_cache_create(c, store, 1, 32)
        i = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
        need = max(B.slim_tree_workspace_bytes(c, 1, 32, 2), B.slim_weights_workspace_bytes(c, 1, 32))
        ws, acc = torch.empty(need, dtype=torch.uint8, device=DEV), torch.zeros(1, 32, device=DEV)
        for call in (lambda: B.slim_tree_decode(c, x, x, cache, i(9), i([-1, 0]), 2, torch.empty_like(x), ws),
                     lambda: B.slim_accumulate_weights(c, x, cache, i(9), acc, ws)):
            with pytest.raises(B.SlimError) as e:
                call()
            assert e.value.status == B.SLIM_ERR_UNSUPPORTED
        B.slim_cache_destroy(cache)
    finally:
        B.slim_destroy(c)


@pytest.mark.parametrize("page", [0, 16])
def test_keys_of_the_kernel_before_are_read(page):
    """Commit, weights, eviction and attention right behind one another, a hundred times on a stream without a pause: each
    reads by bulk copies what the one before has just stored.  The same calls with a pause between them give the same."""
    d, H, n, L0 = 512, 4, 16, 64
    with Case(d, H, 1.0e4, "bf16", [L0] * 4, [[-1] * n] * 4, page, seed=3, t_cap=160) as c:
        i = lambda v: torch.full((4,), v, dtype=torch.int32, device=DEV)
        acc, kept = torch.zeros(4, c.t_cap, device=DEV), torch.empty(4, L0, dtype=torch.int32, device=DEV)
        path = torch.arange(n, dtype=torch.int32, device=DEV).repeat(4, 1)
        ws = torch.empty(B.slim_weights_workspace_bytes(c.ctx, 4, c.t_cap), dtype=torch.uint8, device=DEV)
        ev = torch.empty(B.slim_evict_workspace_bytes(c.ctx, 4, c.t_cap), dtype=torch.uint8, device=DEV)
        lens0, lens1, counts = i(L0), i(L0 + n), i(n)
        torch.manual_seed(5)
        drafts, q1 = torch.randn(100, 4, n, d, device=DEV).bfloat16(), torch.randn(4, d, device=DEV).bfloat16()
        start, st = c.store.clone(), torch.cuda.current_stream().cuda_stream

        def loop(pause):
            c.store.copy_(start)
            acc.zero_()
            outs = torch.empty(100, 4, n, d, dtype=torch.bfloat16, device=DEV)
            torch.cuda.synchronize()
            for k in range(100):
                for call in (lambda: B.slim_tree_commit(c.ctx, c.cache, drafts[k], lens0, path, counts, n, st),
                             lambda: B.slim_accumulate_weights(c.ctx, q1, c.cache, lens1, acc, ws, st),
                             lambda: B.slim_evict(c.ctx, c.cache, lens1, acc, L0, 8, kept, ev, st),
                             lambda: B.slim_tree_decode(c.ctx, c.dq, drafts[k], c.cache, lens0, c.dpar, n, outs[k], c.ws, st)):
                    call()
                    if pause:
                        torch.cuda.synchronize()
            assert c.status() == B.SLIM_OK
            return outs, acc.clone(), kept.clone(), c.store.clone().nan_to_num(7.0)

        for x, y in zip(loop(True), loop(False)):
            assert torch.equal(x, y)


@pytest.mark.parametrize("key,query", [(1.0e36, 1.0e-36), (3.0e37, 1.0e-32), (1.0e-33, 1.0e36), (1.0e-36, 1.0e30), (1.0e30, 1.0e-30)])
def test_keys_and_queries_at_the_ends_of_the_range(key, query):
    """... of bfloat16, one against the other; each third token's query is 1e-6 of the others', each fifth key 1e-8."""
    with Case(256, 2, 1.0e4, "bf16", [200, 17, 0], [[-1, 0, 1, 0, 3, -2], [-1, -1, 0, 2, 3, 3], [-1, 0, 0, -2, 2, 2]], seed=6) as c:
        c.K = [k * np.float32(key) for k in c.K]
        for k in c.K:
            k[::5] *= np.float32(1.0e-8 if key > 1 else 1.0)
        c.K = [synth.round_to_dtype(k, "bf16") for k in c.K]
        c.q[:, ::3] *= np.float32(1.0e-6 if query > 1 else 1.0)
        c.kt = synth.round_to_dtype(c.kt * np.float32(key), "bf16")
        c.q = synth.round_to_dtype(c.q * np.float32(query), "bf16")
        for b, k in enumerate(c.K):
            c.store[b, :len(k)] = to_dev(k, "bf16")
        c.dq, c.dkt = to_dev(c.q, "bf16"), to_dev(c.kt, "bf16")
        c.call()
        assert c.status() == B.SLIM_OK
        c.check()


def test_a_drafting_round_in_a_graph():
    """Attention, verification and commit captured once and replayed on new inputs give what eager calls give."""
    d, H, n, V, Bn = 512, 4, 7, 131, 3
    g = np.random.default_rng(8)
    lay = SlimLayer(d, H, d // H, 1.0e4, "bf16", Bn, 128, DEV)
    try:
        lay.set_wkv(np.eye(d))
        lay.k.normal_()
        lay.reserve_scratch(n)
        lens = torch.zeros(Bn, dtype=torch.int32, device=DEV)
        dev = lambda x, t: torch.from_numpy(np.ascontiguousarray(x)).to(DEV, t)
        rounds = []
        for _ in range(3):
            p, q, tok, par, r = draws(g, Bn, n, V, 2, close=0.3)
            rounds.append((dev(p, torch.float32), dev(q, torch.float32), dev(tok, torch.int32), dev(par, torch.int32), dev(r, torch.float32),
                           *(torch.randn(Bn, n, d, device=DEV).bfloat16() for _ in range(2)), dev(g.integers(0, 100, Bn), torch.int32)))
        held = [x.clone() for x in rounds[0]]

        def one(p, q, tok, par, r, tq, tk, at):
            lens.copy_(at)
            o = lay.tree_decode(tq, tk, lens, par)
            path, count, nxt = lay.tree_verify(p, q, tok, par, r)
            lay.tree_commit(tk, lens, path, count)
            lens.add_(count)
            return o, path, count, nxt

        K0 = lay.k.clone()
        side = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            later = one(*held)
        for k in (0, 1, 2, 1):
            lay.k.copy_(K0)
            want = [x.clone() for x in one(*rounds[k])] + [lay.k.clone(), lens.clone()]
            lay.k.copy_(K0)
            for x, y in zip(held, rounds[k]):
                x.copy_(y)
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                graph.replay()
            torch.cuda.current_stream().wait_stream(side)
            for x, y in zip(want, list(later) + [lay.k, lens]):
                assert torch.equal(x, y)
        assert lay.device_status() == B.SLIM_OK
    finally:
        torch.cuda.synchronize()
        lay.close()


@pytest.mark.parametrize("key,query", [(3.2e38, 1.0e-38), (1.0e-38, 3.2e38)])
def test_the_largest_numbers_of_bfloat16(key, query):
    """Every element of the keys, or of the queries, within a tenth of the largest finite number."""
    with Case(256, 2, 1.0e4, "bf16", [200, 17, 0], [[-1, 0, 1, 0], [-1, -1, 0, 2], [-1, 0, -2, 1]], seed=6) as c:
        c.W *= 2.0 ** -10                                    # the outputs stay in range
        B.slim_set_wkv(c.ctx, c.W)
        size = lambda x, f: synth.round_to_dtype((np.sign(x) if f > 1 else x) * np.float32(f), "bf16")
        c.K, c.kt, c.q = [size(k, key) for k in c.K], size(c.kt, key), size(c.q, query)
        for b, k in enumerate(c.K):
            c.store[b, :len(k)] = to_dev(k, "bf16")
        c.dq, c.dkt = to_dev(c.q, "bf16"), to_dev(c.kt, "bf16")
        c.call()
        assert c.status() == B.SLIM_OK
        c.check()
