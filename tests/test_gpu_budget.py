"""Accumulated attention weights and eviction through the C ABI, against the float64 definitions."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as do
from oracle import slim_oracle as so
from paper_2503_05840_b200 import binding as B
from paper_2503_05840_b200 import synth
from paper_2503_05840_b200.layer import SlimLayer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LENGTHS = [0, 1, 15, 16, 17, 63, 64, 65, 255, 256, 257, 700]


def to_dev(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(DEV, torch.float32 if dtype == "f32" else torch.bfloat16)


def fresh_acc(g, batch, t_cap):
    return torch.from_numpy(g.random((batch, t_cap)).astype(np.float32)).to(DEV)


@pytest.mark.parametrize("d,H,theta,dtype,page", [
    (384, 6, 1.0e4, "f32", 0), (384, 6, 0.0, "f32", 16), (200, 5, 1.0e4, "f32", 0), (6, 3, 1.0e4, "f32", 0), (512, 4, 1.0e6, "bf16", 0),
    (512, 8, 0.0, "bf16", 64), (384, 4, 1.0e4, "bf16", 48), (1280, 20, 0.0, "bf16", 0), (1000, 10, 1.0e4, "bf16", 0), (80, 2, 1.0e4, "bf16", 16),
    (4096, 32, 1.0e6, "bf16", 0), (2048, 64, 1.0e4, "bf16", 0), (256, 1, 1.0e4, "bf16", 32)])
def test_weights_against_the_definition(d, H, theta, dtype, page):
    g = np.random.default_rng(d + H)
    d_k, batch = d // H, len(LENGTHS)
    t_cap = max(LENGTHS) + 5
    if page:
        t_cap = -(-t_cap // page) * page
    ctx = B.slim_create(d, H, d_k, theta, B.SLIM_F32 if dtype == "f32" else B.SLIM_BF16)
    td = torch.float32 if dtype == "f32" else torch.bfloat16
    K = [synth.round_to_dtype(1.5 * g.standard_normal((L, d)), dtype) for L in LENGTHS]
    q = synth.round_to_dtype(g.standard_normal((batch, d)), dtype)
    if page:
        mp = t_cap // page
        store = torch.full((batch * mp + 2, page, d), float("nan"), dtype=td, device=DEV)
        tab = g.permutation(batch * mp + 2)[:batch * mp].astype(np.int32).reshape(batch, mp)
        for b, L in enumerate(LENGTHS):
            for a in range(0, L, page):
                rows = to_dev(K[b][a:a + page], dtype)
                store[int(tab[b, a // page]), :len(rows)] = rows
        table = torch.from_numpy(tab).to(DEV)
        cache = B.slim_cache_create_paged(ctx, store, batch * mp + 2, page, table, batch, mp)
    else:
        store = torch.full((batch, t_cap, d), float("nan"), dtype=td, device=DEV)
        for b, L in enumerate(LENGTHS):
            store[b, :L] = to_dev(K[b], dtype)
        cache = B.slim_cache_create(ctx, store, batch, t_cap)
    try:
        ws = torch.full((B.slim_weights_workspace_bytes(ctx, batch, t_cap),), 255, dtype=torch.uint8, device=DEV)
        acc = fresh_acc(g, batch, t_cap)
        base = acc.cpu().numpy().astype(np.float64)
        dq, dl = to_dev(q, dtype), torch.tensor(LENGTHS, dtype=torch.int32, device=DEV)
        st = torch.cuda.current_stream().cuda_stream
        for _ in range(2):
            B.slim_accumulate_weights(ctx, dq, cache, dl, acc, ws, st)
        assert B.slim_device_status(ctx, st) == B.SLIM_OK
        got = acc.cpu().numpy().astype(np.float64)
        f = 2.0 ** -24
        for b, L in enumerate(LENGTHS):
            assert np.array_equal(got[b, L:], base[b, L:])
            if L == 0:
                continue
            w, arg = do.weights(q[b], K[b], H, theta)
            # arguments: d_k products and the steps of the rotation (at most 16 of them), each off by half a step of the
            # running value; the probability: numerator and denominator; the sums over rows and heads; two additions to acc
            ep = np.expm1(2 * arg * (d_k + 80) * f + (L + H + 32) * f)
            want = base[b, :L] + 2 * w
            assert np.all(np.abs(got[b, :L] - want) <= 2 * w * ep + 4 * f * want), b
    finally:
        torch.cuda.synchronize()
        B.slim_cache_destroy(cache)
        B.slim_destroy(ctx)


def test_weights_of_an_8_bit_cache_and_far_positions():
    g = np.random.default_rng(8)
    d, H = 512, 4
    lay = SlimLayer(d, H, 128, 1.0e4, "fp8", 2, 300, DEV)
    try:
        K = synth.round_to_dtype(g.standard_normal((2, 260, d)), "bf16")
        lay.append_k(to_dev(K, "bf16"), torch.zeros(2, dtype=torch.int32, device=DEV))
        stored = so.quantize_keys_e4m3(K.astype(np.float64).reshape(-1, d), H)
        codes, exps = stored[0], stored[1]
        val = so.e4m3_decode_table()[np.asarray(codes).astype(np.int64)].reshape(2, 260, H, 128) * np.exp2(np.asarray(exps, np.float64).reshape(2, 260, H, 1))
        acc = torch.zeros((2, 300), device=DEV)
        q = synth.round_to_dtype(g.standard_normal((2, d)), "bf16")
        lens = torch.tensor([260, 99], dtype=torch.int32, device=DEV)
        lay.accumulate_weights(to_dev(q, "bf16"), lens, acc)
        assert lay.device_status() == B.SLIM_OK
        for b, L in enumerate((260, 99)):
            w, arg = do.weights(q[b], val[b].reshape(260, d)[:L], H, 1.0e4)
            ep = np.expm1(2 * arg * (128 + 80) * 2.0 ** -24 + (L + H + 32) * 2.0 ** -24)
            assert np.all(np.abs(acc[b, :L].cpu().numpy() - w) <= w * ep + 4 * 2.0 ** -24 * w)
            assert torch.all(acc[b, L:] == 0)
    finally:
        lay.close()
    d, H, L = 128, 1, 150_001                                 # far positions: angles of 1.5e5 radians
    lay = SlimLayer(d, H, 128, 1.0e6, "bf16", 1, L + 3, DEV)
    try:
        K = synth.round_to_dtype(g.standard_normal((L, d)), "bf16")
        q = synth.round_to_dtype(g.standard_normal((1, d)), "bf16")
        lay.k[0, :L] = to_dev(K, "bf16")
        acc = torch.zeros((1, L + 3), device=DEV)
        lay.accumulate_weights(to_dev(q, "bf16"), torch.tensor([L], dtype=torch.int32, device=DEV), acc)
        assert lay.device_status() == B.SLIM_OK
        w, arg = do.weights(q[0], K, H, 1.0e6)
        ep = np.expm1(2 * arg * (128 + 80) * 2.0 ** -24 + (np.sqrt(L) + 4096) * 2.0 ** -24)   # sums run over at most 4096 terms in a row
        assert np.all(np.abs(acc[0, :L].cpu().numpy() - w) <= w * ep)
    finally:
        lay.close()


@pytest.mark.parametrize("d,H,dtype,page,budget,recent", [
    (128, 2, "bf16", 0, 64, 16), (128, 2, "bf16", 16, 100, 0), (384, 6, "f32", 0, 255, 255), (6, 3, "f32", 0, 1, 0), (10, 5, "bf16", 0, 17, 3),
    (64, 1, "fp8", 0, 90, 11), (24, 3, "fp8", 0, 90, 11), (4096, 32, "bf16", 64, 300, 32), (128, 2, "bf16", 0, 5000, 9), (256, 2, "f32", 0, 1, 1)])
def test_evict_against_the_definition(d, H, dtype, page, budget, recent):
    g = np.random.default_rng(budget + d)
    batch = len(LENGTHS)
    t_cap = -(-(max(LENGTHS) + 5) // 64) * 64 if page else max(LENGTHS) + 5
    kind = {"f32": B.SLIM_F32, "bf16": B.SLIM_BF16, "fp8": B.SLIM_FP8}[dtype]
    ctx = B.slim_create(d, H, d // H, 0.0, kind)
    try:
        if dtype == "fp8":
            store = torch.from_numpy(g.integers(0, 126, B.slim_cache_bytes(ctx, batch, t_cap)).astype(np.uint8)).to(DEV)
        else:
            rows = (batch * t_cap // page + 2, page) if page else (batch, t_cap)
            store = to_dev(g.standard_normal(rows + (d,)), dtype)
        if page:
            mp = t_cap // page
            tab = g.permutation(rows[0])[:batch * mp].astype(np.int32).reshape(batch, mp)
            table = torch.from_numpy(tab).to(DEV)
            cache = B.slim_cache_create_paged(ctx, store, rows[0], page, table, batch, mp)
        else:
            cache = B.slim_cache_create(ctx, store, batch, t_cap)
        # many equal values, both zeros, infinities, NaN, negative numbers
        a = np.round(g.standard_normal((batch, t_cap)) * 4).astype(np.float32) / 4
        a[:, 3::17] = 0.0; a[:, 5::19] = -0.0; a[:, 7::23] = np.inf; a[:, 11::29] = np.nan; a[:, 2::31] = -np.inf; a[:, 13::37] = 3e-42
        acc = torch.from_numpy(a).to(DEV)
        before = store.cpu().clone()
        kept = torch.full((batch, budget), 77, dtype=torch.int32, device=DEV)
        ws = torch.empty(B.slim_evict_workspace_bytes(ctx, batch, t_cap), dtype=torch.uint8, device=DEV)
        st = torch.cuda.current_stream().cuda_stream
        B.slim_evict(ctx, cache, torch.tensor(LENGTHS, dtype=torch.int32, device=DEV), acc, budget, recent, kept, ws, st)
        assert B.slim_device_status(ctx, st) == B.SLIM_OK
        want, want_acc = before.clone(), a.copy()
        for b, L in enumerate(LENGTHS):
            keep = do.evict(a[b], L, budget, recent)
            assert kept[b].tolist() == keep + [-1] * (budget - len(keep)), b
            if L <= budget:
                continue
            want_acc[b, :L] = 0
            want_acc[b, :budget] = a[b, keep]
            if dtype == "fp8":
                at = (batch * t_cap * d + 15) // 16 * 16
                for lo, w in ((0, d), (at, H)):
                    rows_w, rows_b = (x[lo:lo + batch * t_cap * w].view(batch, t_cap, w) for x in (want, before))
                    rows_w[b, :budget] = rows_b[b, keep]
            elif page:
                for j, t in enumerate(keep):
                    want[int(tab[b, j // page]), j % page] = before[int(tab[b, t // page]), t % page]
            else:
                want[b, :budget] = before[b, keep]
        assert torch.equal(store.cpu(), want)
        assert np.array_equal(acc.cpu().numpy(), want_acc, equal_nan=True)
    finally:
        torch.cuda.synchronize()
        B.slim_cache_destroy(cache)
        B.slim_destroy(ctx)


def test_evict_refusals_and_reports():
    lay = SlimLayer(64, 1, 64, 0.0, "bf16", 2, 32, DEV)
    try:
        acc, lens = torch.zeros((2, 32), device=DEV), torch.tensor([20, 20], dtype=torch.int32, device=DEV)
        for budget, recent in ((0, 0), (-1, 0), (8, 9), (8, -1)):
            with pytest.raises(B.SlimError) as e:
                lay.evict(lens, acc, budget, recent)
            assert e.value.status == B.SLIM_ERR_INVALID_ARG
        with pytest.raises(ValueError):
            lay.evict(lens, acc[:, :16], 8, 0)
        with pytest.raises(ValueError):
            lay.accumulate_weights(torch.zeros((2, 64), device=DEV), lens, acc)
        lay.evict(torch.tensor([20, 33], dtype=torch.int32, device=DEV), acc, 8, 2)      # clamped to the capacity, reported
        assert lay.device_status() == B.SLIM_ERR_CAPACITY
        with torch.cuda.device(DEV):
            kept = torch.empty((2, 8), dtype=torch.int32, device=DEV)
            for args in ((None, acc, kept, lay._extra[-1]), (lens, None, kept, lay._extra[-1]), (lens, acc, None, lay._extra[-1]), (lens, acc, kept, None)):
                with pytest.raises(B.SlimError):
                    B.slim_evict(lay.ctx, lay.cache, args[0], args[1], 8, 2, args[2], args[3])
    finally:
        lay.close()
    # an X-cache context of another projection width has no key scores
    ctx = B.slim_xcache_create(64, 2, 64, B.SLIM_BF16)
    assert B.slim_weights_workspace_bytes(ctx, 1, 16) == 0 and B.slim_tree_workspace_bytes(ctx, 1, 16, 4) == 0
    B.slim_destroy(ctx)


def test_decode_with_weights_and_eviction_go_together():
    """A few generate-phase steps under a budget: after an eviction the next step attends the kept rows, in order."""
    d, H, cap, budget, recent = 512, 4, 96, 48, 8
    g = np.random.default_rng(31)
    lay = SlimLayer(d, H, 128, 1.0e4, "bf16", 2, cap, DEV)
    try:
        W = synth.round_to_dtype(g.standard_normal((d, d)) / np.sqrt(d), "bf16").astype(np.float64)
        lay.set_wkv(W)
        host = [synth.round_to_dtype(g.standard_normal((60, d)), "bf16"), synth.round_to_dtype(g.standard_normal((30, d)), "bf16")]
        for b in range(2):
            lay.k[b, :len(host[b])] = to_dev(host[b], "bf16")
        acc = torch.zeros((2, cap), device=DEV)
        lens = torch.tensor([60, 30], dtype=torch.int32, device=DEV)
        for step in range(4):
            q, k = (synth.round_to_dtype(g.standard_normal((2, d)), "bf16") for _ in range(2))
            lens += 1
            host = [np.concatenate([host[b], k[b:b + 1]]) for b in range(2)]
            o = lay.decode_step(to_dev(q, "bf16"), to_dev(k, "bf16"), lens)
            for b in range(2):
                assert so.err_rms_norm(o[b].cpu().numpy().astype(np.float64), so.oracle_slim(q[b], host[b], W, H, 1.0e4)) <= 2e-2
            lay.accumulate_weights(to_dev(q, "bf16"), lens, acc)
            kept = lay.evict(lens, acc, budget, recent).cpu().numpy()
            for b in range(2):
                host[b] = host[b][[t for t in kept[b] if t >= 0]]
            lens.clamp_(max=budget)
            assert lay.device_status() == B.SLIM_OK
        assert [len(h) for h in host] == [48, 34]
    finally:
        lay.close()


@pytest.mark.parametrize("d,H,lengths,budget,recent", [(16, 1, [20000, 8191, 700, 0, 12345], 5000, 100), (16, 1, [9000, 8999], 8998, 0),
                                                       (2, 1, [450_001], 100_000, 7), (16, 1, [8192], 1, 0), (16, 1, [30000], 29999, 29999)])
def test_evict_of_long_contexts(d, H, lengths, budget, recent):
    g = np.random.default_rng(budget)
    t_cap, batch = max(max(lengths) + 3, 8192), len(lengths)
    lay = SlimLayer(d, H, d // H, 0.0, "f32", batch, t_cap, DEV)
    try:
        a = np.where(g.random((batch, t_cap)) < 0.4, 0.25, g.random((batch, t_cap))).astype(np.float32)
        k = g.standard_normal((batch, t_cap, d)).astype(np.float32)
        lay.k.copy_(torch.from_numpy(k))
        acc = torch.from_numpy(a).to(DEV)
        kept = lay.evict(torch.tensor(lengths, dtype=torch.int32, device=DEV), acc, budget, recent).cpu().numpy()
        assert lay.device_status() == B.SLIM_OK
        got, got_acc = lay.k.cpu().numpy(), acc.cpu().numpy()
        for b, L in enumerate(lengths):
            keep = do.evict(a[b], L, budget, recent)
            assert list(kept[b]) == keep + [-1] * (budget - len(keep)), b
            want, want_acc = k[b].copy(), a[b].copy()
            if L > budget:
                want[:budget] = k[b][keep]
                want_acc[:L] = 0
                want_acc[:budget] = a[b][keep]
            assert np.array_equal(got[b], want) and np.array_equal(got_acc[b], want_acc)
    finally:
        lay.close()


def test_evict_and_weights_behind_four_billion_elements():
    """A pool whose pages in use lie beyond 2^32 elements from its start, against the same rows near its start."""
    d, H, page, L = 4096, 32, 64, 320
    pages, mp = (1 << 32) // (page * d) + 8, L // page
    ctx = B.slim_create(d, H, 128, 1.0e4, B.SLIM_BF16)
    pool = torch.empty((pages, page, d), dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(3)
    rows = torch.randn(mp, page, d, device=DEV, generator=g).bfloat16()
    pool[:mp] = rows
    pool[-mp:] = rows
    q = torch.randn(1, d, device=DEV, generator=g).bfloat16()
    lens = torch.tensor([L - 5], dtype=torch.int32, device=DEV)
    st = torch.cuda.current_stream().cuda_stream
    got = []
    for first in (0, pages - mp):
        table = torch.arange(first, first + mp, dtype=torch.int32, device=DEV)[None].contiguous()
        cache = B.slim_cache_create_paged(ctx, pool, pages, page, table, 1, mp)
        acc = torch.zeros((1, L), device=DEV)
        ws = torch.empty(max(B.slim_weights_workspace_bytes(ctx, 1, L), B.slim_evict_workspace_bytes(ctx, 1, L)), dtype=torch.uint8, device=DEV)
        kept = torch.empty((1, 100), dtype=torch.int32, device=DEV)
        B.slim_accumulate_weights(ctx, q, cache, lens, acc, ws, st)
        total = acc.sum().item()
        B.slim_evict(ctx, cache, lens, acc, 100, 10, kept, ws, st)
        assert B.slim_device_status(ctx, st) == B.SLIM_OK
        got.append((acc.clone(), kept.clone(), pool[first:first + mp].clone(), total))
        B.slim_cache_destroy(cache)
    assert abs(got[0][3] - H) < 1e-3
    for x, y in zip(got[0][:3], got[1][:3]):
        assert torch.equal(x, y)
    B.slim_destroy(ctx)


@pytest.mark.parametrize("d,H,dtype", [(512, 4, "bf16"), (384, 6, "f32"), (1000, 10, "bf16"), (512, 8, "fp8")])
def test_a_weight_that_is_no_number_reaches_its_whole_sequence(d, H, dtype):
    """A row of keys, or one head of it, that is NaN: every softmax over it is, wherever the row stands and however the
    context is cut."""
    lay = SlimLayer(d, H, d // H, 1.0e4, dtype, 4, 520, DEV)
    try:
        torch.manual_seed(1)
        lens = torch.tensor([500, 500, 37, 300], dtype=torch.int32, device=DEV)
        if dtype == "fp8":
            lay.append_k(torch.randn(4, 520, d, device=DEV).bfloat16(), torch.zeros(4, dtype=torch.int32, device=DEV))
            codes = lay.k[:4 * 520 * d].view(4, 520, d)
            codes[0, 0], codes[1, 333, :d // H], codes[2, 36] = 0x7f, 0x7f, 0x7f
        else:
            lay.k.normal_()
            lay.k[0, 0], lay.k[1, 333, :d // H], lay.k[2, 36] = float("nan"), float("nan"), float("nan")
        q = torch.randn(4, d, device=DEV).to(lay.tdtype)
        acc = torch.ones(4, 520, device=DEV)
        lay.accumulate_weights(q, lens, acc)
        assert lay.device_status() == B.SLIM_OK
        for b, L in enumerate(lens.tolist()):
            assert acc[b, :L].isnan().all() if b < 3 else torch.isfinite(acc[b, :L]).all(), b
            assert (acc[b, L:] == 1).all()
        q[3, 0] = float("nan")                               # the query of the one that was left
        lay.accumulate_weights(q, lens, acc)
        assert acc[3, :300].isnan().all() and (acc[3, 300:] == 1).all()
    finally:
        lay.close()


def test_sizes_next_to_two_to_the_31_are_refused():
    """Row counts are walked in 32-bit steps: capacities and budgets above 2^30 are refused by the calls that would."""
    c = B.slim_create(2, 1, 2, 0.0, B.SLIM_F32)
    try:
        for t_cap in ((1 << 30) + 1, (1 << 31) - 1):
            assert B.slim_tree_workspace_bytes(c, 1, t_cap, 1) == 0
            assert B.slim_weights_workspace_bytes(c, 1, t_cap) == 0
            assert B.slim_evict_workspace_bytes(c, 1, t_cap) == 0
        assert B.slim_evict_workspace_bytes(c, 1, 1 << 30) > 0
        k, x, i = torch.zeros(64, 2, device=DEV), torch.zeros(64, device=DEV), torch.zeros(64, dtype=torch.int32, device=DEV)
        cache = B.slim_cache_create(c, k, 1, 64)
        ws = torch.empty(1 << 16, dtype=torch.uint8, device=DEV)
        with pytest.raises(B.SlimError) as e:
            B.slim_evict(c, cache, i, x, (1 << 30) + 1, 0, i, ws)
        assert e.value.status == B.SLIM_ERR_INVALID_ARG
        B.slim_cache_destroy(cache)
        B.slim_set_wkv(c, np.eye(2))
        far = B.slim_cache_create(c, k, 1, (1 << 30) + 1)   # (only the address is taken here; every call on it is refused)
        for call in (lambda: B.slim_tree_decode(c, x, x, far, i, i, 1, x, ws), lambda: B.slim_tree_commit(c, far, x, i, i, i, 1),
                     lambda: B.slim_accumulate_weights(c, x, far, i, x, ws), lambda: B.slim_evict(c, far, i, x, 4, 0, i, ws)):
            with pytest.raises(B.SlimError) as e:
                call()
            assert e.value.status == B.SLIM_ERR_UNSUPPORTED
        B.slim_cache_destroy(far)
    finally:
        B.slim_destroy(c)
