"""Attention over packed prompts against the float64 definition."""
import numpy as np
import pytest
import torch

from oracle import prompt_oracle as po
from paper_2503_05840_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _starts(n, first=0):
    return np.concatenate([[first], first + np.cumsum(n)]).astype(np.int32)


class Case:
    """Inputs of a packed batch with `lead` rows in front of the first and behind the last sequence."""

    def __init__(self, dtype, H, KV, dk, theta, nq, nk, v32=True, seed=0, lead=3, max_k=None):
        g = torch.Generator().manual_seed(seed)
        self.H, self.KV, self.dk, self.theta, self.nq, self.nk = H, KV, dk, theta, nq, nk
        self.f32, self.v32 = dtype == "f32", v32
        td = torch.float32 if self.f32 else torch.bfloat16
        self.tq, self.tk = sum(nq) + 2 * lead, sum(nk) + 2 * lead
        self.cu_q, self.cu_k = _starts(nq, lead), _starts(nk, lead)
        self.q = torch.randn(self.tq, H, dk, generator=g).to(td)
        self.k = torch.randn(self.tk, KV, dk, generator=g).to(td)
        self.v = torch.randn(self.tk, KV, dk, generator=g).to(torch.float32 if v32 else td)
        self.max_k = max(nk) if max_k is None else max_k
        self.ctx = B.slim_create(H * dk, H, dk, theta, B.SLIM_F32 if self.f32 else B.SLIM_BF16)
        if theta:
            B.slim_reserve_positions(self.ctx, max(self.max_k, 1))

    def close(self):
        B.slim_destroy(self.ctx)

    def buffers(self):
        need = B.slim_prompt_workspace_bytes(self.ctx, self.KV, len(self.nq), self.tq, self.tk)
        assert need > 0
        return dict(q=self.q.to(DEV), k=self.k.to(DEV), v=self.v.to(DEV), cu_q=torch.from_numpy(self.cu_q).to(DEV), cu_k=torch.from_numpy(self.cu_k).to(DEV),
                    o=torch.full((self.tq, self.H, self.dk), 7.0, dtype=self.q.dtype, device=DEV), ws=torch.empty(need, dtype=torch.uint8, device=DEV))

    def call(self, b, causal, stream=None):
        st = torch.cuda.current_stream().cuda_stream if stream is None else stream
        B.slim_prompt_attention(self.ctx, b["q"], b["k"], b["v"], B.SLIM_F32 if self.v32 else B.SLIM_BF16, self.KV, b["cu_q"], b["cu_k"], len(self.nq),
                                self.tq, self.tk, self.max_k, causal, b["o"], b["ws"], st)

    def reference(self, causal):
        """(o, allowed difference), rows outside every sequence 7."""
        o, tol = np.full((self.tq, self.H, self.dk), 7.0), np.zeros((self.tq, self.H, self.dk))
        q, k, v = (x.float().numpy() for x in (self.q, self.k, self.v))
        for b in range(len(self.nq)):
            s, t = slice(self.cu_q[b], self.cu_q[b + 1]), slice(self.cu_k[b], self.cu_k[b + 1])
            o[s], pv, qk = po.attention(q[s], k[t], v[t], self.theta, causal)
            # Scores: products and sums of d_k terms in float32, rotations of two float32 products and tables (2^-22 each side),
            # and in bf16 both rotated operands rounded to 11 bits (2^-11 each).  exp and the softmax sum: 2^-20.
            ds = ((self.dk + 16) * 2.0 ** -24 + 2.0 ** -21) * qk + 2.0 ** -20
            if not self.f32:
                ds = ds + (2 * 2.0 ** -11 + 2.0 ** -22) * qk
            # a relative change of every p by at most ds changes the weighted mean by at most 2 ds sum p |v|; probabilities rounded
            # to bf16 (2^-8, in the sum or not: twice), float32 values rounded to bf16, the output rounded once
            rel = 2 * ds[..., None] + (0 if self.f32 else 2 * 2.0 ** -8 + (2.0 ** -8 if self.v32 else 0))
            tol[s] = rel * pv + (2.0 ** -23 if self.f32 else 2.0 ** -8) * np.abs(o[s]) + 1e-30
        return o, tol

    def check(self, causal, b=None):
        b = b or self.buffers()
        self.call(b, causal)
        torch.cuda.synchronize()
        assert B.slim_device_status(self.ctx) == B.SLIM_OK
        got = b["o"].double().cpu().numpy()
        want, tol = self.reference(causal)
        bad = ~(np.abs(got - want) <= tol)
        assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], tol[bad][:5])
        return got


# head layouts, head widths and types; lengths around the tiles of 64 and 128; one token; no token; no key
SHAPES = [
    ("f32", 6, 6, 64, 0.0, True), ("f32", 4, 2, 96, 1e4, True), ("f32", 5, 1, 40, 1e4, False), ("f32", 2, 2, 256, 1e4, True), ("f32", 1, 1, 2, 1e4, True), ("f32", 2, 1, 130, 0.0, False),
    ("bf16", 4, 4, 128, 1e6, True), ("bf16", 8, 2, 128, 1e6, True), ("bf16", 4, 1, 64, 1e4, True), ("bf16", 3, 3, 64, 0.0, False), ("bf16", 4, 4, 96, 1e4, True),
    ("bf16", 6, 3, 96, 0.0, False), ("bf16", 5, 5, 100, 1e4, True), ("bf16", 3, 1, 128, 0.0, False), ("bf16", 2, 2, 18, 1e4, True), ("bf16", 1, 1, 200, 1e4, True),
]


@pytest.mark.parametrize("dtype,H,KV,dk,theta,causal", SHAPES)
@pytest.mark.parametrize("v32", [True, False])
def test_packed_lengths(dtype, H, KV, dk, theta, causal, v32):
    if dtype == "f32" and not v32:
        pytest.skip("float32 contexts take float32 values")
    nq = [1, 0, 130, 63, 257, 5, 128, 2]
    nk = [1, 4, 130, 200, 257, 0, 384, 1]
    c = Case(dtype, H, KV, dk, theta, nq, nk, v32, seed=H * dk)
    c.check(causal)
    c.close()


@pytest.mark.parametrize("n,before", [(1, 0), (1, 1000), (129, 0), (700, 333), (512, 513), (1025, 0)])
@pytest.mark.parametrize("H,KV,dk", [(2, 2, 128), (4, 1, 64)])
def test_one_sequence(n, before, H, KV, dk):
    c = Case("bf16", H, KV, dk, 1e6, [n], [n + before], v32=False, seed=n, lead=0)
    c.check(True)
    c.check(False)
    c.close()


def test_more_queries_than_keys():
    c = Case("bf16", 2, 2, 128, 1e4, [300, 140], [170, 3], v32=False)
    got = c.check(True)
    assert not got[3:3 + 130].any() and not got[303:303 + 137].any()       # they attend nothing
    c.close()


@pytest.mark.parametrize("dtype,H,dk", [("bf16", 2, 128), ("bf16", 2, 40), ("f32", 2, 64)])
def test_queries_in_front_of_the_first_key_attend_all_keys_where_not_causal(dtype, H, dk):
    c = Case(dtype, H, H, dk, 1e4, [90, 300], [60, 17], v32=dtype == "f32", max_k=400)
    c.check(False)
    c.close()
    c = Case(dtype, H, H, dk, 1e4, [300], [2], v32=dtype == "f32")         # the tables end before position -298
    b = c.buffers()
    c.call(b, False)
    assert B.slim_device_status(c.ctx) == B.SLIM_ERR_CAPACITY
    c.close()


@pytest.mark.parametrize("H,dk,v32", [(2, 128, False), (2, 64, True), (2, 96, False)])
def test_huge_values_in_masked_places_have_no_weight(H, dk, v32):
    c = Case("bf16", H, H, dk, 0.0, [140, 30], [140, 30], v32=v32)
    c.v = c.v.float()
    c.v[3 + 100:3 + 140] = 3e38 if not v32 else 3e30       # rows that queries 0 .. 99 do not attend
    c.v[-2:] = 3e38 if not v32 else 3e30                   # behind the last sequence
    c.v = c.v.to(torch.float32 if v32 else torch.bfloat16)
    b = c.buffers()
    c.call(b, True)
    torch.cuda.synchronize()
    got = b["o"].double().cpu().numpy()
    want, tol = c.reference(True)
    rows = np.r_[0:103, 143:got.shape[0]]
    assert (np.abs(got - want)[rows] <= tol[rows]).all()
    c.close()


def test_many_sequences_of_any_length():
    rng = np.random.default_rng(5)
    nq = [int(x) for x in rng.integers(0, 40, 300)]
    nk = [n + int(x) for n, x in zip(nq, rng.integers(0, 90, 300))]
    c = Case("bf16", 2, 1, 64, 1e4, nq, nk, v32=False)
    c.check(True)
    c.close()


@pytest.mark.parametrize("dtype,H,dk", [("f32", 2, 64), ("bf16", 2, 128), ("bf16", 2, 100)])
def test_numbers_that_are_not_finite_stay_with_the_rows_that_attend_them(dtype, H, dk):
    c = Case(dtype, H, H, dk, 1e4, [200, 90], [200, 90], v32=dtype == "f32")
    c.v[3 + 150, 0, 1] = float("nan")          # value of key 150, head 0, one column
    c.k[3 + 170, 1, :] = float("inf")          # key 170, head 1
    c.q[3 + 20, 1, 3] = float("nan")           # query 20, head 1
    c.v[3 + 200 + 89, :, :] = float("-inf")    # last value of the second sequence
    c.k[0] = float("nan")                      # a row in front of the first sequence
    c.v[0] = float("nan")
    b = c.buffers()
    c.call(b, True)
    torch.cuda.synchronize()
    got = b["o"].double().cpu().numpy()
    want, tol = c.reference(True)
    touched = np.zeros(got.shape, dtype=bool)
    touched[3 + 150:203, 0, 1] = touched[3 + 170:203, 1] = touched[23, 1] = touched[3 + 200 + 89] = True
    assert not np.isfinite(got[touched]).any()
    assert (np.abs(got - want)[~touched] <= tol[~touched]).all()
    c.close()


@pytest.mark.parametrize("scale_q,scale_k", [(1e-20, 1e20), (2e4, 1e-6), (1.0, 1e30), (3e-3, 3e4), (1e30, 1e-30)])
def test_magnitudes_beyond_16_bits(scale_q, scale_k):
    c = Case("bf16", 2, 2, 128, 1e4, [140], [140], v32=False)
    c.q, c.k = (c.q.float() * scale_q).bfloat16(), (c.k.float() * scale_k).bfloat16()
    if scale_q * scale_k > 1e3:                # one key takes all the weight: nothing to compare but that it is a value
        b = c.buffers()
        c.call(b, True)
        got = b["o"][3:143].float().cpu()
        assert torch.isfinite(got).all() and (got.abs() <= c.v.float().abs().max()).all()
    else:
        c.check(True)
    c.close()


def test_values_beyond_16_bits():
    c = Case("bf16", 2, 2, 64, 1e4, [150], [150], v32=True)
    c.v = c.v * 1e30
    c.check(True)
    c.close()


def test_starts_that_do_not_ascend_are_reported():
    c = Case("bf16", 2, 2, 64, 1e4, [20, 20, 20], [20, 20, 20], v32=False)
    for cu in ([3, 2, 43, 63], [-1, 23, 43, 63], [3, 23, 43, 67], [3, 2000000000, 43, 63]):
        for which in ("cu_q", "cu_k"):
            b = c.buffers()
            b[which] = torch.tensor(cu, dtype=torch.int32, device=DEV)
            c.call(b, True)
            assert B.slim_device_status(c.ctx) == B.SLIM_ERR_CAPACITY
    b = c.buffers()                            # longer than max_k: left out
    c.max_k = 19
    c.call(b, True)
    assert B.slim_device_status(c.ctx) == B.SLIM_ERR_CAPACITY
    assert (b["o"] == 7).all()
    c.close()


def test_refusals():
    c = Case("bf16", 4, 2, 64, 1e4, [20], [20], v32=False)
    b = c.buffers()
    args = [c.ctx, b["q"], b["k"], b["v"], B.SLIM_BF16, 2, b["cu_q"], b["cu_k"], 1, c.tq, c.tk, 20, True, b["o"], b["ws"]]

    def status(i, x):
        a = list(args)
        a[i] = x
        try:
            B.slim_prompt_attention(*a)
        except B.SlimError as e:
            return e.status
        return B.SLIM_OK

    for i in (1, 2, 3, 6, 7, 13, 14):
        assert status(i, None) == B.SLIM_ERR_INVALID_ARG
    for i, x in ((5, 0), (8, 0), (9, 0), (10, -1), (11, -1), (4, B.SLIM_FP8), (4, B.SLIM_FP4)):
        assert status(i, x) == B.SLIM_ERR_INVALID_ARG
    for i in (1, 2, 3, 13):
        assert status(i, args[i].data_ptr() + 2) == B.SLIM_ERR_INVALID_ARG
    assert status(14, b["ws"].data_ptr() + 128) == B.SLIM_ERR_INVALID_ARG
    assert status(5, 3) == B.SLIM_ERR_UNSUPPORTED
    assert status(8, 5000) == B.SLIM_ERR_UNSUPPORTED
    assert status(9, 1 << 30) == B.SLIM_ERR_UNSUPPORTED
    assert status(11, 1 << 20) == B.SLIM_ERR_CAPACITY              # beyond the position tables
    assert B.slim_prompt_workspace_bytes(c.ctx, 3, 1, 1, 1) == 0
    assert status(11, 20) == B.SLIM_OK
    c.close()
    f = Case("f32", 2, 2, 64, 0.0, [4], [4])
    f.v32 = False
    with pytest.raises(B.SlimError):
        f.call(f.buffers(), True)
    f.close()


def test_captured_and_replayed_on_new_inputs():
    c = Case("bf16", 4, 2, 128, 1e4, [150, 0, 77], [300, 5, 77], v32=False)
    b = c.buffers()
    c.call(b, True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call(b, True)
    d = Case("bf16", 4, 2, 128, 1e4, [10, 120, 97], [10, 120, 250], v32=False, seed=9)
    d.tq, d.tk = c.tq, c.tk
    for name in ("q", "k", "v"):
        x = getattr(d, name)
        y = torch.zeros_like(getattr(c, name))
        y[:x.shape[0]] = x
        setattr(d, name, y)
        b[name].copy_(y)
    b["cu_q"].copy_(torch.from_numpy(d.cu_q))
    b["cu_k"].copy_(torch.from_numpy(d.cu_k))
    b["o"].fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    got = b["o"].double().cpu().numpy()
    want, tol = d.reference(True)
    assert (np.abs(got - want) <= tol).all()
    del graph
    c.close()
    d.close()


def test_two_streams_with_a_workspace_each():
    c = Case("bf16", 4, 4, 128, 1e4, [500, 31], [700, 31], v32=False)
    bufs = [c.buffers() for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for b, s in zip(bufs, streams):
            with torch.cuda.stream(s):
                c.call(b, True, s.cuda_stream)
    torch.cuda.synchronize()
    c.call(bufs[0], True)
    torch.cuda.synchronize()
    assert torch.equal(bufs[0]["o"], bufs[1]["o"])
    c.check(True)
    c.close()


def test_paths_agree():
    c = Case("bf16", 4, 2, 96, 1e4, [333, 1, 64], [400, 1, 64], v32=False)
    a = c.check(True)
    B.slim_set_path(c.ctx, B.SLIM_PATH_GENERIC)
    b = c.check(True)
    want, tol = c.reference(True)
    assert (np.abs(a - b) <= 2 * tol).all()
    c.close()


def test_offsets_beyond_32_bits():
    """More than 2^31 elements, 2^32 bytes, of queries and outputs: the last sequence is checked."""
    H, dk, n, last = 32, 128, 4096, 77
    seqs = 2 ** 31 // (H * dk) // n + 1
    total = seqs * n + last
    ctx = B.slim_create(H * dk, H, dk, 1e4, B.SLIM_BF16)
    B.slim_reserve_positions(ctx, n)
    g = torch.Generator(device=DEV).manual_seed(1)
    q = torch.empty(total, H, dk, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    k, v = (torch.empty(total, 1, dk, dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(2))
    cu = torch.tensor([i * n for i in range(seqs + 1)] + [total], dtype=torch.int32, device=DEV)
    few = torch.zeros(seqs + 2, dtype=torch.int32, device=DEV)         # only the last two sequences have queries
    few[:] = cu
    few[:seqs] = cu[seqs - 1]
    o = torch.empty_like(q)
    ws = torch.empty(B.slim_prompt_workspace_bytes(ctx, 1, seqs + 1, total, total), dtype=torch.uint8, device=DEV)
    B.slim_prompt_attention(ctx, q, k, v, B.SLIM_BF16, 1, few, cu, seqs + 1, total, total, n, True, o, ws, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert B.slim_device_status(ctx) == B.SLIM_OK
    got = o[-last:].double().cpu().numpy()
    alone = torch.empty(last, H, dk, dtype=torch.bfloat16, device=DEV)
    cu1 = torch.tensor([0, last], dtype=torch.int32, device=DEV)
    B.slim_prompt_attention(ctx, q[-last:].clone(), k[-last:].clone(), v[-last:].clone(), B.SLIM_BF16, 1, cu1, cu1, 1, last, last, last, True, alone, ws,
                            torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert np.array_equal(got, alone.double().cpu().numpy())
    B.slim_destroy(ctx)


# few query tiles over many keys: the tiles are split along their keys and joined
SPLIT = [("f32", 6, 6, 64, 0.0, [448], [448]), ("f32", 2, 1, 40, 1e4, [1, 33, 0, 70], [1999, 700, 40, 70]), ("f32", 1, 1, 256, 1e4, [65], [1300]),
         ("bf16", 2, 2, 128, 1e6, [1], [5000]), ("bf16", 4, 1, 64, 1e4, [300, 1], [3000, 2049]), ("bf16", 2, 2, 96, 0.0, [130, 1, 700, 257], [2000, 900, 700, 3500]),
         ("bf16", 8, 2, 128, 0.0, [512], [4096]), ("bf16", 3, 3, 50, 1e4, [90, 200], [1500, 200])]


@pytest.mark.parametrize("dtype,H,KV,dk,theta,nq,nk", SPLIT)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("v32", [True, False])
def test_long_keys_in_pieces(dtype, H, KV, dk, theta, nq, nk, causal, v32):
    if dtype == "f32" and not v32:
        pytest.skip("float32 contexts take float32 values")
    c = Case(dtype, H, KV, dk, theta, nq, nk, v32=v32, seed=dk)
    b = c.buffers()
    first = c.check(causal, b)
    for _ in range(3):                                   # whichever piece comes last, the sums are the same
        b["o"].fill_(7)
        c.call(b, causal)
        torch.cuda.synchronize()
        assert np.array_equal(b["o"].double().cpu().numpy(), first)
    c.close()


@pytest.mark.parametrize("dtype,H,dk", [("bf16", 2, 128), ("f32", 2, 64)])
def test_numbers_that_are_not_finite_in_one_piece(dtype, H, dk):
    """An infinite key and a NaN value far behind: the rows that attend them get NaN, the others what they would get without them, up to
    rounding (those that share a tile of keys with the two are formed another way)."""
    n = 2600
    c = Case(dtype, H, H, dk, 1e4, [n // 4], [n], seed=9)
    b = c.buffers()
    c.check(True, b)
    row = 400                                            # a query; key at its place, a lead of 3 rows
    at = 3 + n - n // 4 + row
    b["k"][at, 0] = float("inf")
    b["v"][at, 1, 5] = float("nan")
    b["o"].fill_(7)
    c.call(b, True)
    torch.cuda.synchronize()
    got = b["o"].double().cpu().numpy()
    lo, hi = slice(3, 3 + row), slice(3 + row, 3 + n // 4)
    ref, tol = c.reference(True)
    assert (np.abs(got[lo] - ref[lo]) <= tol[lo]).all()
    assert np.isnan(got[hi, 0]).all() and np.isnan(got[hi, 1, 5]).all()
    rest = np.delete(got[hi, 1], 5, axis=1)
    assert np.isfinite(rest).all()
    c.close()


@pytest.mark.parametrize("dk", [2, 30, 66, 80, 98, 126])
@pytest.mark.parametrize("theta,v32", [(1e4, True), (1e4, False), (0.0, True), (0.0, False)])
def test_head_widths_between_the_tiles(dk, theta, v32):
    c = Case("bf16", 4, 2, dk, theta, [130, 1, 0, 257, 30], [130, 300, 5, 257, 700], v32=v32, seed=dk)
    c.check(True)
    c.check(False)
    B.slim_set_path(c.ctx, B.SLIM_PATH_GENERIC)          # (the CUDA cores take them too)
    c.check(True)
    c.close()


def test_not_finite_numbers_with_widened_heads():
    c = Case("bf16", 2, 1, 80, 0.0, [200], [200], seed=4)
    b = c.buffers()
    b["k"][3 + 150, 0, 7] = float("inf")
    b["v"][3 + 20, 0, 79] = float("nan")
    c.call(b, True)
    torch.cuda.synchronize()
    got = b["o"].double().cpu().numpy()[3:203]
    ref, tol = c.reference(True)
    ref, tol = ref[3:203], tol[3:203]
    assert (np.abs(got[:20] - ref[:20]) <= tol[:20]).all()
    assert np.isnan(got[20:150, :, 79]).all() and (np.abs(got[20:150, :, :79] - ref[20:150, :, :79]) <= tol[20:150, :, :79]).all()
    with np.errstate(invalid="ignore"):
        s = np.sign(c.q.double().numpy()[3 + 150:203, :, 7])            # the score is s * inf: all the weight on that key, or NaN
    assert np.isnan(got[150:][s > 0]).all() and (np.abs(got[150:][s < 0][:, :79] - 0) < 10).all()
    c.close()


def _beyond_float16(c, starts):
    """A key that float16 cannot hold at these rows, in a column that queries hardly look at: every row that attends one is formed again."""
    c.q[:, :, [1, 1 + c.dk // 2]] *= 2.0 ** -14
    c.k[starts, :, 1] = 20000.0


@pytest.mark.parametrize("H,KV,dk,v32", [(4, 2, 128, False), (4, 1, 128, True), (3, 3, 96, True), (6, 2, 64, False), (2, 1, 80, False), (2, 2, 80, True)])
@pytest.mark.parametrize("causal", [True, False])
def test_rows_formed_again_of_many_items(H, KV, dk, v32, causal):
    """More items than CTAs, some in pieces; all rows of some sequences are formed again, and what a key behind them touches of others."""
    nq = [300, 1, 65, 190, 0, 64] + [70] * 75
    nk = [2600, 900, 65, 190, 5, 20] + [70] * 75
    c = Case("bf16", H, KV, dk, 1e4, nq, nk, v32=v32, seed=dk, max_k=4300)
    _beyond_float16(c, [int(c.cu_k[b]) for b in range(0, len(nk), 3)] + [int(c.cu_k[1]) + 250, int(c.cu_k[4 + 1]) + 11])
    c.check(causal)
    c.close()


def test_rows_formed_again_of_long_keys_do_not_hold_up_the_others():
    """Every row over many keys is formed again; the call ends with all rows written and no wait run out."""
    nq, nk = [300, 40] * 3, [60000, 20] * 3
    c = Case("bf16", 8, 1, 64, 1e4, nq, nk, v32=False, seed=1)
    _beyond_float16(c, [int(x) for x in c.cu_k[:-1]])
    b = c.buffers()
    c.call(b, True)
    torch.cuda.synchronize()
    assert B.slim_device_status(c.ctx) == B.SLIM_OK
    got = b["o"].double().cpu().numpy()
    for s in (1, 4, 5):
        lo = int(c.cu_q[s])
        rows = np.arange(lo + nq[s] - 3, lo + nq[s])
        o, pv, qk = po.attention(c.q[rows].float().numpy(), c.k[c.cu_k[s]:c.cu_k[s + 1]].float().numpy(), c.v[c.cu_k[s]:c.cu_k[s + 1]].float().numpy(), 1e4, True)
        # float32 throughout; the output rounded once
        assert (np.abs(got[rows] - o) <= (2 * (2.0 ** -20 * qk[..., None] + 2.0 ** -18)) * pv + 2.0 ** -8 * np.abs(o)).all()
    c.close()


def test_rows_formed_again_take_the_time_of_the_cuda_cores():
    """Rows that the tensor cores cannot form are formed by tiles as on the path without them (one by one they took 20 times as long and more)."""
    c = Case("bf16", 8, 8, 128, 1e4, [4096], [4096], v32=False, lead=0)
    _beyond_float16(c, [0])
    b = c.buffers()

    def time():
        t = []
        for _ in range(4):
            e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            e[0].record()
            c.call(b, True)
            e[1].record()
            torch.cuda.synchronize()
            t.append(e[0].elapsed_time(e[1]))
        return min(t[1:])

    auto = time()
    B.slim_set_path(c.ctx, B.SLIM_PATH_GENERIC)
    generic = time()
    assert auto < 10 * generic, (auto, generic)
    c.close()


def _scaled(kind, v):
    KV, dk = v.shape[1:]
    if kind == "columns":                                 # of one head, nine orders of magnitude, one column beyond float16
        v *= 10.0 ** -(torch.arange(dk) % 9).float()
        v[:, 0, 3] *= 1e5
    elif kind == "one column":
        v[:, :, dk - 1] *= 1e-8
        v[:, KV - 1, 0] *= 1e20
    elif kind == "heads":
        v *= 10.0 ** -(4.0 * torch.arange(KV))[:, None]
        v[:, 0] = 0
    elif kind == "ends":
        v *= torch.where(torch.arange(dk) % 2 == 0, 1e37, 1e-37)
    else:
        v *= kind


@pytest.mark.parametrize("H,KV,dk", [(2, 2, 64), (6, 3, 128), (2, 2, 96), (4, 2, 80), (3, 3, 50)])
@pytest.mark.parametrize("kind", [1e-5, 1e-7, 1e5, "columns", "one column", "heads", "ends"])
def test_float32_values_of_any_scale(H, KV, dk, kind):
    c = Case("bf16", H, KV, dk, 1e4, [1, 130, 257, 3], [1, 130, 600, 70], v32=True, seed=dk)
    _scaled(kind, c.v)
    b = c.buffers()
    c.call(b, True)
    torch.cuda.synchronize()
    assert B.slim_device_status(c.ctx) == B.SLIM_OK
    got = b["o"].double().cpu().numpy()
    want, tol = c.reference(True)
    # steps of 2^-28 in columns of ordinary size (bf16 outputs end at 2^-133)
    most = np.repeat(c.v.abs().amax(0).double().numpy(), H // KV, axis=0)
    tol = tol + np.where((most >= 2.0 ** -8) & (most <= 4000), 2.0 ** -29, 2.0 ** -134)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], tol[bad][:5])
    c.close()


def test_heads_whose_values_are_zero_or_small_take_no_longer():
    c = Case("bf16", 8, 8, 128, 1e4, [2048], [2048], v32=True, lead=0)
    b = c.buffers()

    def time():
        t = []
        for _ in range(4):
            e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            e[0].record()
            c.call(b, True)
            e[1].record()
            torch.cuda.synchronize()
            t.append(e[0].elapsed_time(e[1]))
        return min(t[1:])

    ordinary = time()
    b["v"][:, 3] = 0
    b["v"][:, 5] *= 1e-7
    b["v"][:, 6] *= 1e7
    assert time() < 3 * ordinary                          # (row by row it was some 200 times)
    assert not b["o"][:, 3].any()
    c.close()


@pytest.mark.parametrize("H,dk", [(2, 64), (1, 128), (2, 96)])
def test_float32_values_and_the_probabilities_beside_them_keep_11_bits(H, dk):
    """Values, then probabilities, half way between two bf16 numbers and of signs that cancel: 8 bits would leave 2^-8."""
    n = 512
    c = Case("bf16", H, H, dk, 0.0, [n], [n], v32=True, lead=0)
    c.q[:], c.k[:] = 0, 0
    even = torch.arange(n) % 2 == 0
    c.v[:] = torch.where(even, 1 + 2.0 ** -8 - 2.0 ** -10, -(1 + 2.0 ** -8 + 2.0 ** -10))[:, None, None]
    b = c.buffers()
    for part in range(2):
        c.call(b, False)
        torch.cuda.synchronize()
        got = b["o"].double().cpu().numpy()
        o, pv, qk = po.attention(c.q.float().numpy(), c.k.float().numpy(), c.v.numpy(), 0.0, False)
        # Scores in float32.  Probabilities: 2^-11, a quarter of the exponentials off by 7.5e-5; values 2^-11; the output in bf16.
        tol = (2 * 2.0 ** -20 * (1 + qk[..., None]) + 2.0 ** -11 + 2 * 7.5e-5 + 2.0 ** -11) * pv + 2.0 ** -8 * np.abs(o)
        assert tol.max() < 0.6 * (2.0 ** -8 if part == 0 else 0.00195 / 1.50195)
        assert (np.abs(got - o) <= tol).all(), (part, np.abs(got - o).max(), tol.min())
        # the odd keys' probability is 0.50195 of the even ones', half way between the bf16 numbers 0.5 and 0.5039
        x, y = {64: (2.953125, 1.8671875), 96: (4.34375, 1.5546875), 128: (5.28125, 1.4765625)}[dk]
        p = float(np.exp(-x * y / dk ** 0.5))
        b["q"][:, :, 0], b["k"][1::2, :, 0] = x, -y
        c.q, c.k = b["q"].cpu(), b["k"].cpu()
        b["v"][0::2], b["v"][1::2] = -p, 1.0
        c.v = b["v"].cpu()
    c.close()


@pytest.mark.parametrize("dk", [64, 96, 128])
@pytest.mark.parametrize("gap", [12, 14, 15.5])
@pytest.mark.parametrize("at", [0, 1000, 5999])
def test_keys_beside_a_dominant_one_keep_their_weight(dk, gap, at):
    """One key above thousands of others, which alone have values: the output is what the others make of them."""
    n = 6000
    c = Case("bf16", 1, 1, dk, 0.0, [130], [n], v32=True, lead=0, seed=dk)
    c.q[:], c.k[:] = 0, 0
    c.q[:, :, 0], c.k[at, 0, 0] = gap * dk ** 0.5 / 8, 8.0
    c.v = 1 + torch.rand(c.v.shape, generator=torch.Generator().manual_seed(1))
    c.v[at] = 0
    b = c.buffers()
    c.call(b, False)
    torch.cuda.synchronize()
    got = b["o"].double().cpu().numpy()
    s = float(c.q[0, 0, 0]) * c.k[:, 0, 0].double() / dk ** 0.5
    p = torch.softmax(s, 0).numpy()
    o = p @ c.v[:, 0].double().numpy()
    # Scores in float32; probabilities: 2^-11 in steps of 2^-31 of the largest, a quarter of the exponentials off by 7.5e-5; values
    # 2^-11; sums of n positive terms in float32 (n / 2 half steps each way average out far below n 2^-26); the output in bf16.
    tol = (2 * 2.0 ** -18 + 2.0 ** -11 + 2 * 7.5e-5 + 2.0 ** -11 + n * 2.0 ** -26 + 2.0 ** -8) * o + n * 2.0 ** -32 * 2
    assert (np.abs(got[:, 0] - o) <= tol).all(), (np.abs(got[:, 0] - o) / tol).max()
    c.close()


def test_replays_take_the_forms_that_their_inputs_need():
    """One captured call with float32 values, replayed on ordinary inputs, on small values, on keys beyond float16, on values that are not
    finite behind the sequences, and on ordinary ones again."""
    c = Case("bf16", 4, 2, 128, 1e4, [300, 70], [900, 70], v32=True)
    b = c.buffers()
    c.call(b, True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call(b, True)
    q, k, v = c.q.clone(), c.k.clone(), c.v.clone()
    for kind in ("ordinary", "small", "keys", "behind", "ordinary"):
        c.q, c.k, c.v = q.clone(), k.clone(), v.clone()
        if kind == "small":
            c.v[:, 1] *= 1e-9
        elif kind == "keys":
            _beyond_float16(c, [3, 3 + 900 + 20])
        elif kind == "behind":
            c.v[-3:], c.k[-3:] = float("nan"), float("inf")
        for name in ("q", "k", "v"):
            b[name].copy_(getattr(c, name))
        b["o"].fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = b["o"].double().cpu().numpy()
        want, tol = c.reference(True)
        assert B.slim_device_status(c.ctx) == B.SLIM_OK
        assert (np.abs(got - want) <= tol).all(), kind
    del graph
    c.close()


def test_numbers_outside_the_sequences_take_no_longer():
    """Rows in front of the first and behind the last sequence hold huge values: what lies between is converted as if they were not there."""
    c = Case("bf16", 8, 8, 128, 1e4, [2048], [2048], v32=True, lead=40)
    b = c.buffers()

    def time():
        t = []
        for _ in range(4):
            e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            e[0].record()
            c.call(b, True)
            e[1].record()
            torch.cuda.synchronize()
            t.append(e[0].elapsed_time(e[1]))
        return min(t[1:])

    ordinary, want = time(), b["o"].clone()
    b["v"][:40], b["v"][-40:] = 1e30, -1e33
    assert time() < 3 * ordinary                          # (all rows by the CUDA cores: some 30 times)
    assert torch.equal(b["o"], want)
    c.close()
