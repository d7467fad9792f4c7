"""The 4-bit K-cache: rows written, read back and attended over, against the float64 definitions."""
import numpy as np
import pytest
import torch

from oracle import prompt_oracle as po
from oracle import slim_oracle as so
from paper_2503_05840_b200 import binding as B
from paper_2503_05840_b200.layer import SlimLayer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _starts(n, first=0):
    return [first] + [first + sum(n[:i + 1]) for i in range(len(n))]


def _keys(n, d, seed, wide=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, d, generator=g)
    if wide:
        x = x * 10.0 ** torch.randint(-3, 3, (n, 1), generator=g).float()
    return x.bfloat16()


class Paged:
    """A paged cache of a layer's context, pages in random order."""

    def __init__(self, ctx, batch, max_pages, page_rows, seed=0, dtype=torch.uint8, d=0):
        self.ctx, self.t_cap = ctx, max_pages * page_rows
        n = batch * max_pages + 3
        self.pool = torch.zeros(B.slim_cache_bytes(ctx, n, page_rows), dtype=torch.uint8, device=DEV)
        perm = torch.randperm(n, generator=torch.Generator().manual_seed(seed))[:batch * max_pages]
        self.table = perm.int().view(batch, max_pages).contiguous().to(DEV)
        self.cache = B.slim_cache_create_paged(ctx, self.pool, n, page_rows, self.table, batch, max_pages)

    def close(self):
        B.slim_cache_destroy(self.cache)


@pytest.mark.parametrize("d,H,d_k", [(256, 2, 128), (1280, 20, 64), (1000, 10, 100), (36, 6, 6), (4096, 32, 128), (22, 1, 22)])
def test_codes_and_scales_are_the_definition(d, H, d_k):
    rows = [5, 0, 17, 1]
    layer = SlimLayer(d, H, d_k, 0.0, "fp4", 4, 32, DEV)
    x = _keys(sum(rows), d, d)
    x[3] = 0
    x[4, :] = torch.randint(-12, 13, (d,)).float() / 2          # on the borders between codes
    x[6, :5] = torch.tensor([70000.0, -1e30, 3.0, 61440.0, -0.0])
    x[7] = x[7] * 1e-7
    layer.append_rows(x.to(DEV), _i32([3, 0, 15, 31]), _i32(_starts(rows)))
    assert layer.device_status() == B.SLIM_OK
    codes, scales = np.zeros((4 * 32, d), dtype=np.uint8), np.zeros((4 * 32, (d + 31) // 32), dtype=np.uint8)
    at = [0 * 32 + 3 + i for i in range(5)] + [2 * 32 + 15 + i for i in range(17)] + [3 * 32 + 31]
    codes[at], scales[at] = po.fp4_quantise(x.double().numpy())
    assert np.array_equal(layer.k.cpu().numpy(), po.fp4_storage(codes, scales))
    back = layer.read_rows(_i32([3, 0, 15, 31]), _i32(_starts(rows)), sum(rows))
    assert np.array_equal(back.double().cpu().numpy(), po.fp4_values(codes[at], scales[at]))
    layer.close()


def test_groups_that_are_not_finite_read_back_as_nan():
    layer = SlimLayer(128, 2, 64, 0.0, "fp4", 1, 16, DEV)
    x = _keys(3, 128, 0)
    x[0, 40] = float("nan")
    x[1, 127] = float("inf")
    layer.append_rows(x.to(DEV), _i32([0]), _i32([0, 3]))
    got = layer.read_rows(_i32([0]), _i32([0, 3]), 3).cpu()
    bad = torch.zeros(3, 128, dtype=torch.bool)
    bad[0, 32:64] = bad[1, 96:] = True
    assert torch.equal(got.isnan(), bad)
    layer.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp4"])
@pytest.mark.parametrize("d,H", [(384, 6), (250, 5)])
def test_rows_written_and_read_in_pages(dtype, d, H):
    kind = {"f32": B.SLIM_F32, "bf16": B.SLIM_BF16, "fp4": B.SLIM_FP4}[dtype]
    ctx = B.slim_create(d, H, d // H, 1e4, kind)
    c = Paged(ctx, 3, 4, 16)
    rows, pos = [20, 64, 3], _i32([7, 0, 61])
    lead = 2
    x = _keys(sum(rows) + 2 * lead, d, 1)
    x = (x.float() if dtype == "f32" else x).to(DEV)
    cu = _i32(_starts(rows, lead))
    B.slim_append_rows(ctx, c.cache, x, pos, cu, x.shape[0])
    out = torch.full_like(x, 5.0)
    B.slim_read_rows(ctx, c.cache, pos, cu, x.shape[0], out)
    assert B.slim_device_status(ctx) == B.SLIM_OK
    want = x.clone()
    if dtype == "fp4":
        want = torch.from_numpy(po.fp4_values(*po.fp4_quantise(x.double().cpu().numpy()))).to(DEV, torch.bfloat16)
    want[:lead] = want[-lead:] = 5.0
    assert torch.equal(out, want)
    # by way of the block table: row 7 + 9 of sequence 0 is row 0 of its second page
    if dtype != "fp4":
        page = int(c.table[0, 1])
        assert torch.equal(c.pool.view(x.dtype).view(-1, 16, d)[page, 0], x[lead + 9])
    c.close()
    B.slim_destroy(ctx)


def test_rows_that_do_not_fit_are_left_alone():
    layer = SlimLayer(64, 1, 64, 0.0, "fp4", 2, 16, DEV)
    x = _keys(6, 64, 3).to(DEV)
    for pos, cu, kept in (([14, 0], [0, 3, 6], 1), ([-1, 0], [0, 3, 6], 1), ([0, 0], [3, 0, 6], None), ([0, 0], [0, 3, 7], None), ([2147483647, 0], [0, 3, 6], 1)):
        layer.k.zero_()
        layer.append_rows(x, _i32(pos), _i32(cu))
        assert layer.device_status() == B.SLIM_ERR_CAPACITY
        out = torch.full_like(x, 5.0)
        B.slim_read_rows(layer.ctx, layer.cache, _i32(pos), _i32(cu), 6, out)
        assert layer.device_status() == B.SLIM_ERR_CAPACITY
        if kept is not None:
            assert (out[:3] == 5).all() and not (out[3:] == 5).all()
            assert not layer.k[:16 * 32].any()
    ctx = layer.ctx
    c = Paged(ctx, 1, 2, 16)
    c.table[0, 1] = 99
    B.slim_append_rows(ctx, c.cache, x, _i32([13]), _i32([0, 6]), 6)
    assert layer.device_status() == B.SLIM_ERR_CAPACITY
    c.close()
    layer.close()


def _decode_case(d, H, d_k, theta, lengths, t_cap, seed, scale=1.0):
    """(layer, queries, keys as stored, W_KV) with the cache filled through append_rows."""
    B_ = len(lengths)
    g = torch.Generator().manual_seed(seed)
    layer = SlimLayer(d, H, d_k, theta, "fp4", B_, t_cap, DEV)
    W = (torch.randn(d, d, generator=g) / d ** 0.5).bfloat16().float().numpy().astype(np.float64)
    layer.set_wkv(W)
    q = torch.randn(B_, d, generator=g).bfloat16()
    n = [min(max(x, 0), t_cap) for x in lengths]
    x = (_keys(max(sum(n), 1), d, seed, wide=False).float() * scale).bfloat16()
    if sum(n):
        layer.append_rows(x.to(DEV), _i32([0] * B_), _i32(_starts(n) if sum(n) == x.shape[0] else [0] * (B_ + 1)))
    K = po.fp4_values(*po.fp4_quantise(x.double().numpy())) if sum(n) * d <= 400000 else None
    if K is None:
        K = layer.read_rows(_i32([0] * B_), _i32(_starts(n)), sum(n)).double().cpu().numpy()
    return layer, q, [K[a:b] for a, b in zip(_starts(n)[:-1], _starts(n)[1:])], W


def _reference(q, K, W, H, theta):
    """(o, allowed difference without the output's rounding) for one sequence."""
    L, d = K.shape
    dk = d // H
    o, tol = np.zeros(d), np.zeros(d)
    if L == 0:
        return o, tol
    qr = po.turned(q.reshape(1, H, dk), [L - 1], theta)[0]
    kr = po.turned(K.reshape(L, H, dk), np.arange(L), theta)
    for h in range(H):
        s = kr[:, h] @ qr[h] / np.sqrt(dk)
        mag = (np.abs(kr[:, h]) @ np.abs(qr[h])).max() / np.sqrt(dk)
        p = np.exp(s - s.max())
        p /= p.sum()
        u, ua = p @ K, p @ np.abs(K)
        w = W[:, h * dk:(h + 1) * dk]
        # Scores: rotated keys and queries rounded to 11 bits, the rotation's three roundings among them (four half steps of
        # 2^-11 and the tables'), times sqrt 2 for the two terms of a rotation; sums in float32.  Probabilities in 11 bits, in the sum
        # and beside it.  The weighted sums enter the projection as two terms of 11 bits; float32 sums of d terms.
        ds = 1.5 * 5 * 2.0 ** -11 * mag + 2.0 ** -18
        du = 2 * (ds + 2 * 2.0 ** -11) * ua
        o[h * dk:(h + 1) * dk] = u @ w
        tol[h * dk:(h + 1) * dk] = (du + (2.0 ** -18 + d * 2.0 ** -24) * ua) @ np.abs(w)
    return o, tol


def _check(layer, q, Ks, W, H, theta, lengths, o_dtype=torch.bfloat16):
    o = torch.full((len(lengths), layer.d), 3.0, dtype=o_dtype, device=DEV)
    layer.decode_typed(q.to(DEV), _i32(lengths), o=o)
    assert layer.device_status() == B.SLIM_OK
    got = o.double().cpu().numpy()
    for b, K in enumerate(Ks):
        want, tol = _reference(q[b].double().numpy(), K, W, H, theta)
        tol = tol + (2.0 ** -8 if o_dtype == torch.bfloat16 else 2.0 ** -23) * (np.abs(want) + tol)
        bad = ~(np.abs(got[b] - want) <= tol)
        assert not bad.any(), (b, np.argwhere(bad)[:4], got[b][bad][:4], want[bad][:4], tol[bad][:4])
    return got


SHAPES = [(512, 4, 128, 1e6), (256, 4, 64, 0.0), (1280, 20, 64, 0.0), (1536, 16, 96, 1e4), (768, 8, 96, 0.0), (1024, 8, 128, 0.0), (4096, 32, 128, 1e6),
          (384, 6, 64, 1e4), (500, 5, 100, 1e4), (36, 6, 6, 1e4), (512, 2, 256, 1e4), (192, 3, 64, 1e4), (4096, 64, 64, 0.0)]


@pytest.mark.parametrize("d,H,d_k,theta", SHAPES)
@pytest.mark.parametrize("o_dtype", [torch.bfloat16, torch.float32])
def test_decode(d, H, d_k, theta, o_dtype):
    lengths = [1, 0, 15, 16, 17, 130, 33, 300]
    layer, q, Ks, W = _decode_case(d, H, d_k, theta, lengths, 304, d + H)
    got = _check(layer, q, Ks, W, H, theta, lengths, o_dtype)
    assert not got[1].any()
    layer.close()


@pytest.mark.parametrize("d,H,d_k,theta,L", [(512, 4, 128, 1e6, 20001), (256, 4, 64, 0.0, 40000), (4096, 32, 128, 1e6, 5003), (500, 5, 100, 1e4, 3000)])
def test_decode_long_contexts(d, H, d_k, theta, L):
    layer, q, Ks, W = _decode_case(d, H, d_k, theta, [L, 7, L // 3], L, 5)
    _check(layer, q, Ks, W, H, theta, [L, 7, L // 3])
    layer.close()


@pytest.mark.parametrize("scale", [1e-4, 1e4, 3e-5])
def test_decode_small_and_large_keys(scale):
    layer, q, Ks, W = _decode_case(512, 4, 128, 1e4, [100, 333], 336, 3, scale)
    q = (q.float() / max(scale, 1e-3)).bfloat16()
    _check(layer, q, Ks, W, 4, 1e4, [100, 333])
    layer.close()


def test_decode_scores_that_run_away():
    """Later keys whose score exceeds every earlier one by hundreds: their rows get all the weight."""
    layer, q, Ks, W = _decode_case(512, 4, 128, 0.0, [400, 50], 400, 3)
    x = _keys(400, 512, 8, wide=False)
    x[250:] = (q[0].float() * torch.linspace(0.5, 40, 150)[:, None]).bfloat16()
    layer.append_rows(x.to(DEV), _i32([0, 0]), _i32([0, 400, 400]))
    Ks[0] = po.fp4_values(*po.fp4_quantise(x.double().numpy()))
    _check(layer, q, Ks, W, 4, 0.0, [400, 50])
    layer.close()


@pytest.mark.parametrize("page_rows,d,H,d_k,theta", [(16, 512, 4, 128, 1e4), (64, 1536, 16, 96, 1e4), (48, 250, 5, 50, 0.0)])
def test_decode_in_pages_is_decode_in_one_piece(page_rows, d, H, d_k, theta):
    lengths = [200, 0, 77, 192]
    t_cap = (200 + page_rows - 1) // page_rows * page_rows
    layer, q, Ks, W = _decode_case(d, H, d_k, theta, lengths, t_cap, 11)
    c = Paged(layer.ctx, 4, t_cap // page_rows, page_rows)
    rows = layer.read_rows(_i32([0] * 4), _i32(_starts(lengths)), sum(lengths))
    B.slim_append_rows(layer.ctx, c.cache, rows, _i32([0] * 4), _i32(_starts(lengths)), sum(lengths))
    want = layer.decode_typed(q.to(DEV), _i32(lengths))
    o = torch.empty_like(want)
    B.slim_decode_typed(layer.ctx, q.to(DEV), None, c.cache, _i32(lengths), o, B.SLIM_BF16, layer.workspace)
    assert layer.device_status() == B.SLIM_OK
    assert torch.equal(o, want)
    _check(layer, q, Ks, W, H, theta, lengths)
    c.table[0, 1] = -5                          # a page outside the pool is reported, and read as page 0
    B.slim_decode_typed(layer.ctx, q.to(DEV), None, c.cache, _i32(lengths), o, B.SLIM_BF16, layer.workspace)
    assert layer.device_status() == B.SLIM_ERR_CAPACITY
    c.close()
    layer.close()


@pytest.mark.parametrize("d,H,d_k", [(512, 4, 128), (250, 5, 50)])
def test_steps_append_then_attend(d, H, d_k):
    lengths = [16, 1, 40]
    layer, q, Ks, W = _decode_case(d, H, d_k, 1e4, [15, 0, 39], 48, 2)
    new = _keys(3, d, 77, wide=False)
    o = layer.decode_typed(q.to(DEV), _i32(lengths), k_new=new.to(DEV))
    assert layer.device_status() == B.SLIM_OK
    row = po.fp4_values(*po.fp4_quantise(new.double().numpy()))
    Ks = [np.concatenate([K, row[b:b + 1]]) for b, K in enumerate(Ks)]
    got = _check(layer, q, Ks, W, H, 1e4, lengths)
    assert np.array_equal(got, o.double().cpu().numpy())
    f = layer.decode_step(q.to(DEV), new.to(DEV), _i32(lengths))
    assert torch.equal(f.bfloat16(), o)         # the same float32 sums, rounded here
    layer.append_k(new.to(DEV), _i32([15, 0, 39]))
    assert torch.equal(layer.decode(q.to(DEV), _i32(lengths)), f)
    B.slim_decode_static_ws(layer.ctx, q.to(DEV), layer.cache, _i32(lengths), f)
    assert torch.equal(f.bfloat16(), o)
    layer.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
def test_typed_output_of_other_caches(dtype):
    g = torch.Generator().manual_seed(3)
    layer = SlimLayer(512, 4, 128, 1e4, dtype, 3, 64, DEV)
    layer.set_wkv((torch.randn(512, 512, generator=g) / 22).numpy())
    td = torch.float32 if dtype == "f32" else torch.bfloat16
    layer.append_k(torch.randn(3, 64, 512, generator=g).to(DEV, td), _i32([0, 0, 0]))
    q = torch.randn(3, 512, generator=g).to(DEV, td)
    f = layer.decode(q, _i32([64, 0, 30])).clone()
    assert torch.equal(layer.decode_typed(q, _i32([64, 0, 30]), o=torch.empty(3, 512, device=DEV, dtype=torch.bfloat16)), f.bfloat16())
    assert torch.equal(layer.decode_typed(q, _i32([64, 0, 30]), o=torch.empty(3, 512, device=DEV)), f)
    layer.close()


def test_not_finite_rows():
    layer, q, Ks, W = _decode_case(512, 4, 128, 1e4, [60, 60], 64, 2)
    want = layer.decode_typed(q.to(DEV), _i32([50, 60])).clone()
    bad = torch.full((1, 512), float("nan")).bfloat16().to(DEV)
    layer.append_rows(bad, _i32([55, 0]), _i32([0, 1, 1]))         # behind the first sequence's 50 rows
    assert torch.equal(layer.decode_typed(q.to(DEV), _i32([50, 60])), want)
    got = layer.decode_typed(q.to(DEV), _i32([56, 60]))
    assert got[0].isnan().all() and torch.equal(got[1], want[1])
    layer.k[:64 * 256].fill_(0xff)                                  # codes and scales of nothing in particular
    layer.k[2 * 64 * 256:].fill_(0xff)
    assert not layer.decode_typed(q.to(DEV), _i32([0, 0])).any()
    layer.close()


def test_prefill_fills_the_cache():
    layer, q, Ks, W = _decode_case(512, 4, 128, 1e4, [0, 0], 64, 2)
    x = _keys(2 * 40, 512, 4, wide=False).view(2, 40, 512)
    V = torch.empty(2, 40, 512, device=DEV)
    B.slim_prefill(layer.ctx, layer.cache, x.to(DEV), _i32([3, 0]), 40, V)
    got = layer.read_rows(_i32([3, 0]), _i32([0, 40, 80]), 80)
    assert layer.device_status() == B.SLIM_OK
    assert np.array_equal(got.double().cpu().numpy(), po.fp4_values(*po.fp4_quantise(x.view(80, 512).double().numpy())))
    W2 = torch.empty(2, 40, 512, device=DEV)
    B.slim_values_from_keys(layer.ctx, x.to(DEV), 80, W2)
    assert torch.equal(V, W2)
    layer.close()


def test_refusals():
    layer = SlimLayer(512, 4, 128, 1e4, "fp4", 1, 64, DEV)
    x = torch.zeros(1, 2, 512, device=DEV, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        layer.append_rows(x[0].float(), _i32([0]), _i32([0, 2]))
    with pytest.raises(ValueError):
        layer.read_rows(_i32([0, 0]), _i32([0, 2]), 2)
    with pytest.raises(B.SlimError) as e:
        layer.decode_typed(x[0, :1].contiguous(), _i32([1]))
    assert e.value.status == B.SLIM_ERR_NO_WEIGHTS
    layer.set_wkv(np.eye(512))
    calls = [lambda: layer.tree_decode(x, x, _i32([1]), _i32([[-1, 0]])), lambda: layer.tree_commit(x, _i32([1]), _i32([[0, -1]]), _i32([1])),
             lambda: layer.accumulate_weights(x[0, :1].contiguous(), _i32([1]), torch.zeros(1, 64, device=DEV)),
             lambda: layer.evict(_i32([1]), torch.zeros(1, 64, device=DEV), 1, 0),
             lambda: B.slim_decode_partial(layer.ctx, x, layer.cache, _i32([1]), _i32([0]), _i32([0]), x, x, layer.workspace),
             lambda: B.slim_xcache_create(512, 4, 128, B.SLIM_FP4),
             lambda: B.slim_xcache_set_weights(layer.ctx, np.eye(512), np.eye(512))]
    for call in calls:
        with pytest.raises(B.SlimError) as e:
            call()
        assert e.value.status == B.SLIM_ERR_UNSUPPORTED
    for bad in (B.SLIM_FP4, B.SLIM_FP8, 9):
        with pytest.raises(B.SlimError) as e:
            B.slim_decode_typed(layer.ctx, x, None, layer.cache, _i32([1]), x, bad, layer.workspace)
        assert e.value.status == B.SLIM_ERR_INVALID_ARG
    for call in (lambda: B.slim_append_rows(layer.ctx, layer.cache, x, _i32([0]), _i32([0, 2]), 0),
                 lambda: B.slim_read_rows(layer.ctx, layer.cache, _i32([0]), _i32([0, 2]), 2, x.data_ptr() + 1)):
        with pytest.raises(B.SlimError) as e:
            call()
        assert e.value.status == B.SLIM_ERR_INVALID_ARG
    layer.close()
    f = SlimLayer(512, 4, 128, 1e4, "fp8", 1, 64, DEV)
    with pytest.raises(B.SlimError) as e:
        f.append_rows(x[0], _i32([0]), _i32([0, 2]))
    assert e.value.status == B.SLIM_ERR_UNSUPPORTED
    f.close()


def test_chunked_prompt_then_decode():
    """A prompt in two chunks through the 4-bit cache, then a step: the run that the calls are for."""
    d, H, d_k, theta, n, m = 512, 4, 128, 1e4, 96, 70
    g = torch.Generator().manual_seed(1)
    layer, _, _, W = _decode_case(d, H, d_k, theta, [0, 0], 192, 2)
    k, q = _keys(2 * (n + m) + 2, d, 6, wide=False).to(DEV), torch.randn(2 * (n + m) + 2, d, generator=g).bfloat16().to(DEV)
    first, second, cu1, cu2 = k[:2 * n], k[2 * n:2 * (n + m)], _i32([0, n, 2 * n]), _i32([0, m, 2 * m])
    both = _i32([0, n + m, 2 * (n + m)])

    def values(keys):
        out = torch.empty(keys.shape, device=DEV)
        B.slim_values_from_keys(layer.ctx, keys, keys.shape[0], out, torch.cuda.current_stream().cuda_stream)
        return out

    layer.append_rows(first, _i32([0, 0]), cu1)
    o1 = layer.prompt_attention(q[:2 * n], first, values(first), cu1, cu1, n)
    layer.append_rows(second, _i32([n, n]), cu2)
    keys = layer.read_rows(_i32([0, 0]), both, 2 * (n + m))
    o2 = layer.prompt_attention(q[2 * n:2 * (n + m)], keys, values(keys), cu2, both, n + m)
    lens = _i32([n + m + 1] * 2)
    o3 = layer.decode_typed(q[-2:].contiguous(), lens, k_new=k[-2:].contiguous())
    assert layer.device_status() == B.SLIM_OK
    got = [x.double().cpu().numpy() for x in (o1, o2, o3)]
    stored, Q = keys.double().cpu().numpy().reshape(2, n + m, d), q.double().cpu().numpy()
    last = po.fp4_values(*po.fp4_quantise(k[-2:].double().cpu().numpy()))
    for b in range(2):
        raw = first[b * n:(b + 1) * n].double().cpu().numpy()
        for i, (K, rows, take) in enumerate(((raw, Q[b * n:(b + 1) * n], slice(b * n, (b + 1) * n)),
                                             (stored[b], Q[2 * n + b * m:2 * n + (b + 1) * m], slice(b * m, (b + 1) * m)),
                                             (np.concatenate([stored[b], last[b:b + 1]]), Q[-2 + b][None], slice(b, b + 1)))):
            V = K @ W
            want, pv, qk = po.attention(rows.reshape(-1, H, d_k), K.reshape(-1, H, d_k), V.reshape(-1, H, d_k), theta, True)
            # roundings as in the tests of the single calls; the values' own error (float32 sums, operands of 16 bits) 2^-8 of sum |K||W|
            tol = (2 * (8 * 2.0 ** -11 * qk[..., None] + 2.0 ** -18) + 3 * 2.0 ** -8) * pv + 2.0 ** -8 * np.abs(want) + 2.0 ** -8 * (np.abs(K) @ np.abs(W)).max()
            assert (np.abs(got[i][take].reshape(want.shape) - want) <= tol).all()
    layer.close()


def test_captured_steps():
    layer, q, Ks, W = _decode_case(512, 4, 128, 1e4, [60, 33], 128, 2)
    qd, new, lens, o = q.to(DEV), _keys(2, 512, 9, wide=False).to(DEV), _i32([61, 34]), torch.empty(2, 512, dtype=torch.bfloat16, device=DEV)
    layer.decode_typed(qd, lens, k_new=new, o=o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.decode_typed(qd, lens, k_new=new, o=o)
    for step in range(3):
        lens += 1
        new.copy_(_keys(2, 512, 20 + step, wide=False))
        graph.replay()
        want = layer.decode_typed(qd, lens)
        assert torch.equal(o, want)
    del graph
    layer.close()


def test_rows_on_two_streams():
    layer = SlimLayer(1024, 8, 128, 1e4, "fp4", 2, 512, DEV)
    x = _keys(1000, 1024, 1).to(DEV)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        layer.append_rows(x[:500], _i32([0, 0]), _i32([0, 500, 500]))
    layer.append_rows(x[500:], _i32([0, 0]), _i32([0, 0, 500]))
    torch.cuda.synchronize()
    got = layer.read_rows(_i32([0, 0]), _i32([0, 500, 1000]), 1000)
    want = torch.from_numpy(po.fp4_values(*po.fp4_quantise(x[::50].double().cpu().numpy())))
    assert torch.equal(got[::50].double().cpu(), want)
    layer.close()


# one to sixteen heads a CTA: one or two a warp, one or two sets of warps
HEADS = [(256, 2, 128, 0.0), (1280, 10, 128, 1e4), (2304, 18, 128, 1e6), (2560, 20, 128, 1e4), (2816, 22, 128, 1e4), (2304, 24, 96, 1e4),
         (3584, 28, 128, 1e4), (3840, 30, 128, 0.0), (1792, 28, 64, 1e4), (2048, 32, 64, 0.0)]


@pytest.mark.parametrize("d,H,d_k,theta", HEADS)
def test_decode_head_counts(d, H, d_k, theta):
    lengths = [1, 200, 16, 95, 0, 31]
    layer, q, Ks, W = _decode_case(d, H, d_k, theta, lengths, 203, H)
    _check(layer, q, Ks, W, H, theta, lengths)
    layer.close()


@pytest.mark.parametrize("d,H,d_k,theta", HEADS[::2] + [(4096, 32, 128, 1e6)])
def test_scores_run_away_in_some_units(d, H, d_k, theta):
    """Keys that repeat the query late in a sequence: the units that hold them are walked twice, their neighbours once."""
    lengths = [300, 40, 700, 3]
    layer, q, _, W = _decode_case(d, H, d_k, theta, lengths, 704, 5)
    x = _keys(700, d, 8, wide=False).float()
    at = [150, 151, 290, 420, 699]
    for i, t in enumerate(at):
        qt = po.turned(q[2].double().numpy().reshape(1, H, d_k), [lengths[2] - 1 - t], theta)[0]      # meets the query turned by its distance
        x[t] = torch.from_numpy(qt.reshape(-1)).float() * (1 + i)
    layer.append_rows(x.bfloat16().to(DEV), _i32([0] * 4), _i32([0, 0, 0, 700, 700]))
    K = layer.read_rows(_i32([0] * 4), _i32(_starts(lengths)), sum(lengths)).double().cpu().numpy()
    s = _starts(lengths)
    _check(layer, q, [K[a:b] for a, b in zip(s[:-1], s[1:])], W, H, theta, lengths)
    layer.close()


def test_more_sequences_than_workers():
    lengths = [(7 * i) % 50 for i in range(400)]
    layer, q, Ks, W = _decode_case(512, 4, 128, 1e4, lengths, 50, 1)
    _check(layer, q, Ks, W, 4, 1e4, lengths)
    layer.close()


@pytest.mark.parametrize("d,H,d_k", [(512, 4, 128), (250, 5, 50)])
def test_lengths_beyond_the_cache_are_clamped(d, H, d_k):
    layer, q, Ks, W = _decode_case(d, H, d_k, 1e4, [40, 40], 40, 4)
    want = layer.decode_typed(q.to(DEV), _i32([40, 0]))
    kept = layer.k.clone()
    got = layer.decode_typed(q.to(DEV), _i32([41, -7]), k_new=_keys(2, d, 1).to(DEV))
    assert layer.device_status() == B.SLIM_ERR_CAPACITY
    assert torch.equal(got, want) and torch.equal(layer.k, kept) and not got[1].any()
    layer.close()


def test_two_steps_at_once():
    """Two caches of one context on two streams, each with its own workspace."""
    layer, q, Ks, W = _decode_case(1024, 8, 128, 1e4, [900, 33], 1000, 6)
    other = torch.empty_like(layer.k).copy_(layer.k)
    cache = B.slim_cache_create(layer.ctx, other, 2, 1000)
    ws, o = torch.empty_like(layer.workspace), torch.empty(2, 1024, dtype=torch.bfloat16, device=DEV)
    qd, lens, l2 = q.to(DEV), _i32([900, 33]), _i32([17, 500])
    want, want2 = layer.decode_typed(qd, lens).clone(), layer.decode_typed(qd, l2).clone()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(5):
        got = layer.decode_typed(qd, lens)
        B.slim_decode_typed(layer.ctx, qd, None, cache, l2, o, B.SLIM_BF16, ws, s.cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(o, want2)
    B.slim_cache_destroy(cache)
    layer.close()


@pytest.mark.parametrize("d,H,t_cap", [(4096, 32, 2200003), (16384, 64, 300007)])
def test_offsets_beyond_32_bits(d, H, t_cap):
    """The second sequence's last rows lie more than 2^32 bytes into the storage."""
    layer = SlimLayer(d, H, d // H, 0.0, "fp4", 2, t_cap, DEV)
    x = _keys(50, d, 3, wide=False).to(DEV)
    layer.append_rows(x, _i32([0, 0]), _i32([0, 0, 50]))
    layer.append_rows(x[:3], _i32([0, t_cap - 3]), _i32([0, 0, 3]))
    both = torch.cat([layer.read_rows(_i32([0, 0]), _i32([0, 0, 50]), 50), layer.read_rows(_i32([0, t_cap - 3]), _i32([0, 0, 3]), 3)])
    assert layer.device_status() == B.SLIM_OK
    want = torch.from_numpy(po.fp4_values(*po.fp4_quantise(x.double().cpu().numpy())))
    assert torch.equal(both.double().cpu(), torch.cat([want, want[:3]]))
    if d == 4096:
        g = torch.Generator().manual_seed(3)
        W = (torch.randn(d, d, generator=g) / d ** 0.5).bfloat16().float().numpy().astype(np.float64)
        layer.set_wkv(W)
        q = torch.randn(2, d, generator=g).bfloat16()
        _check(layer, q, [want.numpy()[:0], want.numpy()], W, H, 0.0, [0, 50])
    layer.close()


@pytest.mark.parametrize("d,H,d_k", [(512, 4, 128), (256, 2, 128), (2816, 22, 128), (1280, 20, 64), (1536, 16, 96), (4096, 32, 128), (500, 5, 100)])
@pytest.mark.parametrize("where", ["first", "tenth", "last"])
def test_keys_beside_a_dominant_one_keep_their_weight(d, H, d_k, where):
    """One key 7 to 17 nats above thousands of others, which alone hold values in most columns: those columns are what the others make of them."""
    lengths, dom = [9000, 20, 9000], {"first": 0, "tenth": 9, "last": 8999}[where]
    g = torch.Generator().manual_seed(d)
    layer = SlimLayer(d, H, d_k, 0.0, "fp4", 3, 9000, DEV)
    layer.set_wkv(np.eye(d))
    # A head's score is its column 0 times a query's only element.  Keys are values of the format with scale 1, so scores are exact.
    gap = 7 + (torch.arange(H) * 3 % 11).float()                                # nats
    x = torch.tensor([0.5, 1, 1.5, 2, 3, 4, 6])[torch.randint(0, 7, (sum(lengths), H, d_k), generator=g)]
    x[:, :, 0] = torch.tensor([-0.5, 0, 0, 0.5])[torch.randint(0, 4, (sum(lengths), H), generator=g)]
    x.view(-1, d)[:, 5::32] = 6                                                 # (a group's largest)
    for s in (0, lengths[0] + lengths[1]):
        x[s + dom] = 0
        x[s + dom, :, 0] = 6
    q = torch.zeros(3, H, d_k)
    q[:, :, 0] = gap * d_k ** 0.5 / 6
    q = q.bfloat16()
    x = x.reshape(-1, d).bfloat16()
    layer.append_rows(x.to(DEV), _i32([0] * 3), _i32(_starts(lengths)))
    o = torch.empty(3, d, device=DEV)
    layer.decode_typed(q.view(3, d).to(DEV), _i32(lengths), o=o)
    K = layer.read_rows(_i32([0] * 3), _i32(_starts(lengths)), sum(lengths)).double()
    assert layer.device_status() == B.SLIM_OK
    for b, (lo, hi) in enumerate(zip(_starts(lengths)[:-1], _starts(lengths)[1:])):
        Kb, qb = K[lo:hi], q[b].to(DEV).double()
        p = torch.softmax(torch.einsum("thc,hc->ht", Kb.view(-1, H, d_k), qb) / d_k ** 0.5, 1)
        for h in range(H):
            c = slice(h * d_k, (h + 1) * d_k)
            want, ua = p[h] @ Kb[:, c], p[h] @ Kb.abs()
            # Scores in float32, up to 25 log2 units: 2^-18, in the sum and beside it.  Probabilities in 11 bits, likewise.  The
            # projection's operands are two terms of 11 bits, steps of 2^-24 of the row's largest; float32 sums of 9000 and d terms in
            # any order, 2^-24 each (their errors are averaged: a hundred steps).
            tol = (2 * 2.0 ** -18 + 2 * 2.0 ** -11 + 100 * 2.0 ** -24) * ua[c] + 2.0 ** -22 * ua.max()
            assert ((o[b, c].double() - want).abs() <= tol).all(), (b, h, float(gap[h]), ((o[b, c].double() - want).abs() / tol).max())
    layer.close()


@pytest.mark.parametrize("d,H", [(4096, 32), (1280, 20)])
def test_rows_are_moved_once_whatever_share_of_them_a_warp_has(d, H):
    """Two numbers of rows that differ by 16, between which a warp's share of a row changes: the fewer rows are not slower."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    few, more = (16 * sms - 8, 16 * sms + 8) if d == 4096 else (32 * sms - 8, 32 * sms + 8)
    layer = SlimLayer(d, H, d // H, 0.0, "fp4", 1, more, DEV)
    x, pos = _keys(more, d, 1).to(DEV), _i32([0])
    out = torch.empty_like(x)

    def call(n, write):
        cu = cus[n]
        if write:
            B.slim_append_rows(layer.ctx, layer.cache, x, pos, cu, n, torch.cuda.current_stream().cuda_stream)
        else:
            B.slim_read_rows(layer.ctx, layer.cache, pos, cu, n, out, torch.cuda.current_stream().cuda_stream)

    def time(n, write):
        t, graph = [], torch.cuda.CUDAGraph()
        call(n, write)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            for _ in range(40):
                call(n, write)
        for _ in range(12):
            e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            e[0].record()
            graph.replay()
            e[1].record()
            torch.cuda.synchronize()
            t.append(e[0].elapsed_time(e[1]) * 25)
        return min(t[2:])

    cus = {n: _i32([0, n]) for n in (few, more)}
    for write in (True, False):
        a, b = time(few, write), time(more, write)
        assert a < 1.15 * b, (write, a, b)
    layer.close()


def test_rows_are_read_right_behind_the_kernels_that_wrote_them():
    """Prompts written, read back and attended over, and a step, again and again without a pause: what each call does behind one."""
    d, H, d_k, n = 1024, 8, 128, 700
    layer, _, _, W = _decode_case(d, H, d_k, 1e4, [0, 0], 720, 2)
    cu, cu_step, zero, lens, st = _i32([0, n, 2 * n]), _i32([0, 1, 2]), _i32([0, 0]), _i32([n + 1, n + 1]), torch.cuda.current_stream().cuda_stream
    sets = [(_keys(2 * n, d, 50 + i, wide=False).to(DEV), _keys(2, d, 90 + i, wide=False).to(DEV)) for i in range(4)]

    def go(i, pause):
        x, new = sets[i % 4]
        steps = [lambda: layer.append_rows(x, zero, cu), lambda: layer.read_rows(zero, cu, 2 * n),
                 lambda: B.slim_values_from_keys(layer.ctx, k, 2 * n, v, st), lambda: layer.prompt_attention(x, k, v, cu, cu, n),
                 lambda: layer.prompt_attention(x, k, v.bfloat16(), cu, cu, n, False), lambda: layer.decode_typed(new, lens, k_new=new)]
        v, out = torch.empty(2 * n, d, device=DEV), []
        for s, step in enumerate(steps):
            r = step()
            if s == 1:
                k = r
            if pause:
                torch.cuda.synchronize()
            out.append(r)
        return [r for r in out if r is not None] + [v]

    layer.prompt_attention(sets[0][0], sets[0][0], sets[0][0], cu, cu, n)
    want = [go(i, True) for i in range(4)]
    got = [go(i, False) for i in range(40)]
    assert layer.device_status() == B.SLIM_OK
    for i, g in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(g, want[i % 4])), i
    layer.close()


def test_calls_without_rows_and_scratch_sized_ahead():
    layer, q, Ks, W = _decode_case(512, 4, 128, 1e4, [20, 0], 64, 2)
    none, x = torch.empty(0, 512, dtype=torch.bfloat16, device=DEV), _keys(6, 512, 1).to(DEV)
    kept = layer.k.clone()
    layer.append_rows(none, _i32([0, 0]), _i32([0, 0, 0]))
    assert layer.read_rows(_i32([0, 0]), _i32([0, 0, 0]), 0).shape == (0, 512) and torch.equal(layer.k, kept)
    for k in (none, none.view(0, 4, 128), none[:, :256].contiguous().view(0, 2, 128), none[:, :128].contiguous()):
        for v in (k, k.float()):
            assert not layer.prompt_attention(x, k, v, _i32([0, 6]), _i32([0, 0]), 0).any()          # no keys: rows of zeros
    assert layer.prompt_attention(none, x, x, _i32([0, 0]), _i32([0, 6]), 6).shape == (0, 512)
    three = torch.empty(0, 3, 128, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError):
        layer.prompt_attention(x, three, three, _i32([0, 6]), _i32([0, 0]), 0)
    # a scratch sized ahead takes a capture of these sizes, and no larger one
    fresh = SlimLayer(512, 4, 128, 1e4, "fp4", 2, 64, DEV)
    cu, o = _i32([0, 6]), torch.empty_like(x)
    with pytest.raises(ValueError):
        fresh.reserve_scratch(prompts=1, q_rows=0, k_rows=6)
    with pytest.raises(ValueError):
        fresh.reserve_scratch(prompts=1, q_rows=6, k_rows=6, kv_heads=3)
    fresh.reserve_scratch(prompts=1, q_rows=6, k_rows=6)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        fresh.prompt_attention(x, x, x, cu, cu, 6, o=o)
    graph.replay()
    assert torch.equal(o, layer.prompt_attention(x, x, x, cu, cu, 6))
    del graph
    fresh.close()
    layer.close()


@pytest.mark.parametrize("dtype", ["fp4", "bf16", "f32"])
def test_layers_of_other_shapes_beside_one_another(dtype):
    """Each layer's calls go on as before when layers of other shapes come after it: limits that a launch needs are not a context's."""
    shapes = [(1280, 20, 64, 1e4, 23), (4096, 32, 128, 1e6, 3), (1536, 16, 96, 0.0, 9), (500, 5, 100, 1e4, 2), (512, 8, 64, 0.0, 40), (256, 2, 128, 1e4, 1)]
    td = torch.float32 if dtype == "f32" else torch.bfloat16
    layers = []
    for d, H, d_k, theta, n in shapes:
        g = torch.Generator().manual_seed(d)
        layer = SlimLayer(d, H, d_k, theta, dtype, n, 64, DEV)
        layer.set_wkv((torch.randn(d, d, generator=g) / d ** 0.5).numpy())
        layer.append_k(torch.randn(n, 40, d, generator=g).to(DEV, td), _i32([0] * n))
        q, lens = torch.randn(n, d, generator=g).to(DEV, td), _i32([40 - i % 9 for i in range(n)])
        layers.append((layer, q, lens, layer.decode(q, lens).clone()))
    for layer, q, lens, want in layers + layers[::-1]:
        assert torch.equal(layer.decode(q, lens), want)
    for layer, *_ in layers:
        layer.close()
