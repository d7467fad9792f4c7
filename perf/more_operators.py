"""What the operators of the prompt phase and of the 4-bit K-cache are measured on.

Four operators that a prompt and its generation use one after another: attention over whole prompts (causal, grouped heads,
packed sequences of different lengths, a part of the keys in the cache already), keys quantised to 4 bits as they are
written into the cache, cached rows read back, and the decode step's attention over a cache held in 4 bits.  `run` computes
them either in a plain form (elementary torch operations, float32, angles in float64) or through the library's entry
points, as `own` says.

The rotation (pair (j, j + d_k/2) turned by -t theta^(-2j/d_k)), the weights W_KV and the 4-bit storage are the ones of
include/slim.h: a row of d keys is d/2 bytes of E2M1 codes (column 2i in the low half of byte i), padded to a multiple of
16 bytes; behind the codes of all rows, each row has one scale byte for 32 columns, padded likewise: the upper bits of a
float16 without its sign.  A group's scale s is the smallest with 6 s >= max |k| (at most 10240), a code the nearest of
0, 0.5, 1, 1.5, 2, 3, 4, 6 times s, ties to the even code."""
import math

import torch

own = False
DEV = "cuda:0"
GROUP = 32
_weights = {}        # W_KV by shape: a program's weights, the same for all inputs
_contexts = {}       # library contexts by shape, which a program makes once


# ------------------------------------------------------------------------------------------------ cases
def _text(numbers):
    return " ".join(str(x) for x in numbers)


def _case(case):
    """The case with its texts of numbers as lists: queries and earlier keys (nq, before) or rows and their places (rows, at)."""
    return {k: [int(x) for x in v.split()] if k in ("nq", "before", "rows", "at") else v for k, v in case.items()}


def listed():
    return [
        # a decoder prompt of a small float32 model without rotation: latency
        dict(name="prompt_f32_448", op="prompt", dtype="f32", H=6, KV=6, dk=64, theta=0.0, causal=True, nq="448", before="0", v32=True),
        # the encoder of a speech model over eight recordings of 1500 frames: every frame attends every other one
        dict(name="prompt_bf16_encoder", op="prompt", dtype="bf16", H=20, KV=20, dk=64, theta=0.0, causal=False, nq="1500 " * 8, before="0 " * 8, v32=False),
        # the next chunks of four long prompts, the keys before them read back from the cache, float32 values as the library forms them
        dict(name="prompt_bf16_chunks", op="prompt", dtype="bf16", H=32, KV=32, dk=128, theta=1.0e6, causal=True, nq="512 512 333 1", before="3584 1024 0 2047", v32=True),
        # a packed batch of prompts of unequal lengths, four query heads a key head
        dict(name="prompt_bf16_packed", op="prompt", dtype="bf16", H=32, KV=8, dk=128, theta=1.0e6, causal=True,
             nq="4096 17 1111 2500 640 129 3001 1 777 1920 350 64", before="0 " * 12, v32=False),
        # one long prompt of the 4096-wide model
        dict(name="prompt_bf16_16k", op="prompt", dtype="bf16", H=32, KV=32, dk=128, theta=1.0e6, causal=True, nq="16384", before="0", v32=False),
        # the newest rows of a serving batch into its paged cache
        dict(name="append_16_rows", op="append", H=32, dk=128, rows="1 " * 16, at=_text(1000 + 37 * i for i in range(16)), page=64),
        # packed prompts into the cache
        dict(name="append_prompts", op="append", H=32, dk=128, rows="4096 17 8191 2500 640 129 3001 1 777 1920 350 16384", at="0 " * 12, page=0),
        # the cached part of one prompt, rows of 1280 keys
        dict(name="read_1000", op="read", H=20, dk=64, rows="1000", at="3", page=0),
        # the cached parts of the chunks of a batch, in pages
        dict(name="read_batch", op="read", H=32, dk=128, rows="3584 1024 0 2047 16000 8191", at="0 5 0 0 100 1", page=64),
        # cross-attention of 64 users over 1500 cached rows
        dict(name="decode_64x1500", op="decode", H=20, dk=64, theta=0.0, B=64, lo=1500, hi=1500, page=0),
        # a serving batch of ragged contexts on the 4096-wide shape
        dict(name="decode_batch16", op="decode", H=32, dk=128, theta=1.0e6, B=16, lo=8192, hi=16384, page=0),
        # one very long context, in pages
        dict(name="decode_128k", op="decode", H=32, dk=128, theta=1.0e6, B=1, lo=131001, hi=131001, page=64),
    ]


def _log(rng, a, b):
    return max(a, min(b, int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "append", "read", "decode", "decode"])
    page = rng.choice([0, 0, 16, 64, 256])
    if op == "prompt":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        H, dk = rng.choice([(32, 128), (32, 128), (16, 128), (20, 64), (12, 96), (8, 64), (10, 100)] if dtype == "bf16" else [(6, 64), (8, 128), (4, 96), (5, 40)])
        KV = rng.choice([k for k in range(1, H + 1) if H % k == 0])
        causal = rng.random() < 0.8
        # no more products than the longest listed case; the shapes that run without tensor cores are held to smaller ones
        most = 2.2e12 / (64 if dtype == "f32" or dk == 100 else 1)
        B = _log(rng, 1, 24)
        top = max(1, min(16384, int(math.sqrt(most / (4.0 * H * dk * B)))))
        hi = _log(rng, min(16, top), top)
        nq = [hi if b == 0 else max(1, int(hi * rng.uniform(0.02, 1.0))) for b in range(B)]
        before = [int(rng.choice([0, 0, rng.uniform(0, 1)]) * (top - n)) if causal else 0 for n in nq]
        return dict(op=op, dtype=dtype, H=H, KV=KV, dk=dk, theta=rng.choice([0.0, 1.0e4, 1.0e6]), causal=causal, nq=_text(nq), before=_text(before), v32=dtype == "f32" or rng.random() < 0.5)
    H, dk = rng.choice([(32, 128), (32, 128), (16, 96), (20, 64), (8, 128), (12, 64), (10, 100)])
    d = H * dk
    if op != "decode":
        B = _log(rng, 1, 32)
        hi = _log(rng, 1, max(1, 38000 * 4096 // (B * d)))
        rows = [hi if b == 0 else int(hi * rng.random()) for b in range(B)]
        return dict(op=op, H=H, dk=dk, rows=_text(rows), at=_text(rng.randint(0, 300) for _ in range(B)), page=page)
    B = _log(rng, 1, 64)
    hi = _log(rng, 1, max(1, min(131072, 16 * 12288 * 4096 // ((64 if dk == 100 else 1) * B * d))))
    return dict(op=op, H=H, dk=dk, theta=rng.choice([0.0, 1.0e4, 1.0e6]), B=B, lo=max(1, int(hi * rng.uniform(0.3, 1.0))), hi=hi, page=page)


def _lengths(c):
    """Ragged context lengths of a case, the first the longest."""
    return [c["hi"] if b == 0 else c["lo"] + int((c["hi"] - c["lo"]) * ((0.6180339887 * b) % 1.0)) for b in range(c["B"])]


def _batch(c):
    return c["B"] if c["op"] == "decode" else len(c["rows"])


def _t_cap(c):
    t = c["hi"] if c["op"] == "decode" else max(a + r for a, r in zip(c["at"], c["rows"]))
    g = c["page"] or 16
    return (t + g - 1) // g * g


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _starts(n):
    """0 and the running sums of n: where packed sequences begin and end."""
    out = [0]
    for x in n:
        out.append(out[-1] + x)
    return out


def _pitch(n):
    return (n + 15) // 16 * 16


def _parts(store, rows, d):
    """The codes [rows, pitch] and scales [rows, pitch] of a 4-bit storage."""
    pc, ps = _pitch(d // 2), _pitch((d + GROUP - 1) // GROUP)
    return store[:rows * pc].view(rows, pc), store[rows * pc:rows * (pc + ps)].view(rows, ps)


def _scale_values():
    """The finite scales, 0 to 10240, as float32; the value's index is its byte."""
    return (torch.arange(0, 0xE3, device=DEV, dtype=torch.int16) << 7).view(torch.float16).float()


def _pack(x):
    """Rows of keys [n, d] in 4 bits: (code bytes [n, d/2], scale bytes [n, groups])."""
    n, d = x.shape
    groups = (d + GROUP - 1) // GROUP
    x = torch.nn.functional.pad(x.float(), (0, groups * GROUP - d)).view(n, groups, GROUP)
    a = x.abs()
    table = _scale_values()
    byte = torch.searchsorted(6.0 * table, a.amax(-1)).clamp(max=table.numel() - 1)
    s = table[byte][..., None]
    # borders between neighbouring codes; a key on one goes to the even code (products of a scale and a border are exact)
    code = ((a > 0.25 * s).byte() + (a >= 0.75 * s).byte() + (a > 1.25 * s).byte() + (a >= 1.75 * s).byte() + (a > 2.5 * s).byte()
            + (a >= 3.5 * s).byte() + (a > 5.0 * s).byte())
    code = torch.where((x < 0) & (code > 0), code + 8, code).view(n, -1)[:, :d]
    return code[:, 0::2] | (code[:, 1::2] << 4), byte.to(torch.uint8)


def _unpack(codes, scales, d):
    """The values of rows of a 4-bit storage, [n, d] float32."""
    n = codes.shape[0]
    c = torch.stack([codes[:, :d // 2] & 15, codes[:, :d // 2] >> 4], -1).view(n, d)
    m = (c & 7).float()
    m = torch.where(m < 4, 0.5 * m, torch.where(m < 6, m - 2, 2 * m - 8))
    s = (scales[:, :(d + GROUP - 1) // GROUP].to(torch.int16) << 7).view(torch.float16).float()
    return torch.where(c > 7, -m, m) * s.repeat_interleave(GROUP, 1)[:, :d]


def _keys(n, d, g, scale, common):
    """Keys with directions of unequal strength, some of them along one that queries share."""
    x = torch.randn(n, d, device=DEV, generator=g)
    x += 0.5 * common * (torch.rand(n, 1, device=DEV, generator=g) < 0.02)
    return (x * scale).bfloat16()


def _wkv(d):
    """W_KV [d][d], bfloat16."""
    if d not in _weights:
        _weights[d] = (torch.randn(d, d, device=DEV, generator=_gen(d)) / math.sqrt(d)).bfloat16()
    return _weights[d]


def _context(c):
    from paper_2503_05840_b200 import binding as B
    kind = {"f32": B.SLIM_F32, "bf16": B.SLIM_BF16}[c["dtype"]] if c["op"] == "prompt" else B.SLIM_FP4
    key = (c["H"], c["dk"], c.get("theta", 0.0), kind)
    if key not in _contexts:
        _contexts[key] = [B.slim_create(c["H"] * c["dk"], c["H"], c["dk"], c.get("theta", 0.0), kind), False]
    if c["op"] == "decode" and not _contexts[key][1]:
        B.slim_set_wkv(_contexts[key][0], _wkv(c["H"] * c["dk"]).float().cpu().numpy())
        _contexts[key][1] = True
    return _contexts[key][0]


class _Cache:
    """The library's view of the state's key storage."""

    def __init__(self, c, s):
        from paper_2503_05840_b200 import binding as B
        self.B, self.ctx = B, _context(c)
        if c["page"]:
            self.cache = B.slim_cache_create_paged(self.ctx, s["store"], s["table"].numel(), c["page"], s["table"], _batch(c), s["table"].shape[1])
        else:
            self.cache = B.slim_cache_create(self.ctx, s["store"], _batch(c), _t_cap(c))

    def __del__(self):
        self.B.slim_cache_destroy(self.cache)


def prepare(case, seed):
    c, g = _case(case), _gen(seed)
    s = {"case": c}
    d = c["H"] * c["dk"]
    if c["op"] == "prompt":
        td = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        nk = [a + b for a, b in zip(c["nq"], c["before"])]
        common = torch.randn(c["dk"], device=DEV, generator=g)
        s["q"] = (torch.randn(sum(c["nq"]), c["H"], c["dk"], device=DEV, generator=g) + 0.3 * common).to(td)
        s["k"] = torch.randn(sum(nk), c["KV"], c["dk"], device=DEV, generator=g)
        s["k"] = (s["k"] + 0.5 * common * (torch.rand(sum(nk), 1, 1, device=DEV, generator=g) < 0.02)).to(td)
        s["v"] = torch.randn(sum(nk), c["KV"], c["dk"], device=DEV, generator=g).to(torch.float32 if c["v32"] else td)
        s["cu_q"], s["cu_k"] = _i32(_starts(c["nq"])), _i32(_starts(nk))
        s["o"] = torch.empty_like(s["q"])
        if own:
            from paper_2503_05840_b200 import binding as B
            s["ctx"] = _context(c)
            B.slim_reserve_positions(s["ctx"], max(nk))
            need = B.slim_prompt_workspace_bytes(s["ctx"], c["KV"], len(nk), sum(c["nq"]), sum(nk))
            s["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV)
        return s
    B, t_cap = _batch(c), _t_cap(c)
    rows = B * t_cap
    scale, common = 0.5 + 1.5 * torch.rand(d, device=DEV, generator=g), torch.randn(d, device=DEV, generator=g)
    s["store"] = torch.zeros(rows * (_pitch(d // 2) + _pitch((d + GROUP - 1) // GROUP)), dtype=torch.uint8, device=DEV)
    if c["page"]:               # pages in any order
        s["table"] = torch.randperm(rows // c["page"], device=DEV, generator=g).int().view(B, t_cap // c["page"]).contiguous()
    if c["op"] != "append":
        codes, scales = _parts(s["store"], rows, d)
        step = max(1, (1 << 27) // d)
        for a in range(0, rows, step):
            n = min(step, rows - a)
            codes[a:a + n, :d // 2], scales[a:a + n, :(d + GROUP - 1) // GROUP] = _pack(_keys(n, d, g, scale, common))
    if c["op"] == "decode":
        s["lengths"] = _i32(_lengths(c))
        s["q"] = (torch.randn(B, d, device=DEV, generator=g) + 0.3 * common).bfloat16()
        s["W_KV"] = _wkv(d)
        s["o"] = torch.empty(B, d, dtype=torch.bfloat16, device=DEV)
    else:
        total = sum(c["rows"])
        s["cu"], s["at"] = _i32(_starts(c["rows"])), _i32(c["at"])
        if c["op"] == "append":
            s["k_new"] = _keys(total, d, g, scale, common)
        s["k"] = torch.empty(total, d, dtype=torch.bfloat16, device=DEV)
    if own:
        s["h"] = h = _Cache(c, s)
        if c["op"] == "decode":
            s["ws"] = torch.empty(h.B.slim_workspace_bytes(h.ctx, B, t_cap), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    c = s["case"]
    if own:
        return _own(s, c)
    return {"prompt": _plain_prompt, "append": _plain_append, "read": _plain_read, "decode": _plain_decode}[c["op"]](s, c)


def _own(s, c):
    from paper_2503_05840_b200 import binding as B
    st = torch.cuda.current_stream().cuda_stream
    if c["op"] == "prompt":
        B.slim_prompt_attention(s["ctx"], s["q"], s["k"], s["v"], B.SLIM_F32 if c["v32"] else B.SLIM_BF16, c["KV"], s["cu_q"], s["cu_k"], len(c["nq"]),
                                s["q"].shape[0], s["k"].shape[0], max(a + b for a, b in zip(c["nq"], c["before"])), c["causal"], s["o"], s["ws"], st)
        return s["o"]
    h = s["h"]
    if c["op"] == "decode":
        B.slim_decode_typed(h.ctx, s["q"], None, h.cache, s["lengths"], s["o"], B.SLIM_BF16, s["ws"], st)
        return s["o"]
    if c["op"] == "append":
        B.slim_append_rows(h.ctx, h.cache, s["k_new"], s["at"], s["cu"], s["k"].shape[0], st)
    B.slim_read_rows(h.ctx, h.cache, s["at"], s["cu"], s["k"].shape[0], s["k"], st)
    return s["k"]


def _rotate(x, pos, c):
    """x [.., T, heads, d_k] float32 at positions pos [.., T]; the angles in 64 bits."""
    if not c["theta"]:
        return x
    half = x.shape[-1] // 2
    freq = c["theta"] ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
    a = pos.double()[..., None] * freq
    cos, sin = a.cos().float()[..., None, :], a.sin().float()[..., None, :]
    x1, x2 = x[..., :half], x[..., half:]
    return torch.cat([x1 * cos + x2 * sin, x2 * cos - x1 * sin], -1)


def _plain_prompt(s, c):
    share = c["H"] // c["KV"]
    q0 = k0 = 0
    for n, before in zip(c["nq"], c["before"]):        # the scores of a packed batch as one matrix would mostly be masked
        m = n + before
        pos = torch.arange(m, device=DEV)
        q = _rotate(s["q"][q0:q0 + n].float(), pos[before:], c).transpose(0, 1).reshape(c["KV"], share * n, c["dk"])
        k = _rotate(s["k"][k0:k0 + m].float(), pos, c).permute(1, 2, 0)
        v = s["v"][k0:k0 + m].float().transpose(0, 1)
        a = torch.matmul(q * (1.0 / math.sqrt(c["dk"])), k).view(c["KV"], share, n, m)
        if c["causal"]:
            a.masked_fill_(pos > pos[before:, None], -math.inf)
        a.sub_(a.amax(-1, keepdim=True)).exp_()
        l = a.sum(-1)
        o = torch.matmul(a.view(c["KV"], share * n, m), v).view(c["H"], n, c["dk"]) / l.view(c["H"], n, 1)
        s["o"][q0:q0 + n] = o.transpose(0, 1)
        q0, k0 = q0 + n, k0 + m
    return s["o"]


def _packed_rows(s, c):
    """The storage row of every packed row."""
    cu = s["cu"].long()
    i = torch.arange(s["k"].shape[0], device=DEV)
    b = torch.searchsorted(cu, i, right=True) - 1
    return _storage_rows(s, c, b, i - cu[b] + s["at"].long()[b])


def _storage_rows(s, c, b, t):
    if not c["page"]:
        return b * _t_cap(c) + t
    return s["table"].long()[b, t // c["page"]] * c["page"] + t % c["page"]


def _plain_append(s, c):
    d, rows = c["H"] * c["dk"], _packed_rows(s, c)
    codes, scales = _parts(s["store"], _batch(c) * _t_cap(c), d)
    code, byte = _pack(s["k_new"])
    codes[rows, :code.shape[1]] = code
    scales[rows, :byte.shape[1]] = byte
    return _plain_read(s, c)


def _plain_read(s, c):
    d, rows = c["H"] * c["dk"], _packed_rows(s, c)
    codes, scales = _parts(s["store"], _batch(c) * _t_cap(c), d)
    s["k"].copy_(_unpack(codes[rows], scales[rows], d))
    return s["k"]


def _plain_decode(s, c):
    B, H, d, T = c["B"], c["H"], c["H"] * c["dk"], c["hi"]
    codes, scales = _parts(s["store"], B * _t_cap(c), d)
    t = torch.arange(T, device=DEV)
    rows = _storage_rows(s, c, torch.arange(B, device=DEV)[:, None], t[None]).view(-1)
    there = t < s["lengths"][:, None]                                             # [B, T]
    K = _unpack(codes[rows], scales[rows], d).view(B, T, d)
    K = torch.where(there[..., None], K, torch.zeros((), device=DEV))
    q = _rotate(s["q"].float().view(B, 1, H, c["dk"]), s["lengths"][:, None] - 1, c)
    k = _rotate(K.view(B, T, H, c["dk"]), t.expand(B, T), c)
    a = torch.matmul(k.permute(0, 2, 1, 3), q.permute(0, 2, 3, 1))[..., 0] * (1.0 / math.sqrt(c["dk"]))      # [B, H, T]
    a = torch.where(there[:, None], a, torch.full((), -math.inf, device=DEV))
    a = (a - a.amax(-1, keepdim=True)).exp()
    u = torch.matmul(a, K) / a.sum(-1, keepdim=True)                              # [B, H, d]
    W = s["W_KV"].float().view(d, H, c["dk"])
    s["o"].copy_(torch.matmul(u.transpose(0, 1), W.transpose(0, 1)).transpose(0, 1).reshape(B, d))
    return s["o"]


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = _case(case)
    d = c["H"] * c["dk"]
    row4 = d / 2 + (d + GROUP - 1) // GROUP
    if c["op"] == "prompt":
        es = 4 if c["dtype"] == "f32" else 2
        pairs = sum(n * b + (n * (n + 1) / 2 if c["causal"] else n * n) for n, b in zip(c["nq"], c["before"]))
        total_q, total_k = sum(c["nq"]), sum(c["nq"]) + sum(c["before"])
        return {"bytes": 2.0 * es * total_q * d + (es + (4 if c["v32"] else es)) * total_k * c["KV"] * c["dk"], "flops": 4.0 * pairs * d}
    if c["op"] == "decode":
        L = sum(_lengths(c))
        return {"bytes": row4 * L + 2.0 * d * d + 4.0 * c["B"] * d, "flops": 2.0 * L * d * (c["H"] + 1) + 2.0 * c["B"] * d * d}
    total = sum(c["rows"])
    return {"bytes": total * ((2 * d + row4 if c["op"] == "append" else 0) + row4 + 2 * d), "flops": 0}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _turned(x, pos, c):
    """Complex rows [heads, T, d_k / 2]: the pair (x_j, x_{j + d_k/2}) as one number, turned by -pos theta_j; x [T, heads, d_k]."""
    half = c["dk"] // 2
    x = x.double().transpose(0, 1)
    z = torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous())
    if c["theta"]:
        w = torch.tensor([c["theta"] ** (-j / half) for j in range(half)], dtype=torch.float64, device=DEV)
        z = z * torch.polar(torch.ones((), dtype=torch.float64, device=DEV), -pos.double()[:, None] * w)
    return z


def _flat(z):
    return torch.cat([z.real, z.imag], -1)


def _stored(s, c, b, first, n):
    """Rows first .. first + n - 1 of sequence b of a 4-bit storage, [n, d] float64."""
    d, t_cap = c["H"] * c["dk"], _t_cap(c)
    total = _batch(c) * t_cap
    pc, ps = _pitch(d // 2), _pitch((d + GROUP - 1) // GROUP)
    t = torch.arange(first, first + n, device=DEV)
    row = s["table"][b].long()[t // c["page"]] * c["page"] + t % c["page"] if c["page"] else b * t_cap + t
    byte = s["store"][:total * pc].view(total, pc)[row][:, :d // 2].int()
    value = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device=DEV)
    out = torch.empty(n, d, dtype=torch.float64, device=DEV)
    out[:, 0::2] = value[byte % 16]
    out[:, 1::2] = value[byte // 16]
    sb = s["store"][total * pc:].view(total, ps)[row].int()
    e, f = sb // 8, (sb % 8).double()
    scale = torch.where(e == 0, f / 8 * 2.0 ** -14, (1 + f / 8) * torch.pow(2.0, e.double() - 15))
    return out * scale[:, torch.arange(d, device=DEV) // GROUP]


def _rounded(x):
    """The 4-bit value of every key of a row, from the definition."""
    out = torch.empty_like(x, dtype=torch.float64)
    scales = torch.tensor([m / 8 * 2.0 ** -14 for m in range(8)] + [(1 + m / 8) * 2.0 ** (e - 15) for e in range(1, 32) for m in range(8)], dtype=torch.float64, device=DEV)
    scales = scales[scales <= 10240]
    for a in range(0, x.shape[1], GROUP):
        k = x[:, a:a + GROUP].double()
        fits = 6 * scales[None] >= k.abs().amax(1, keepdim=True)
        s = torch.where(fits.any(1), scales[fits.int().argmax(1)], scales[-1])[:, None]
        best, gap = torch.zeros_like(k), k.abs()
        for m in (1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0):         # even codes first: an odd one has to be nearer
            near = (k.abs() - m * s).abs()
            best, gap = torch.where(near < gap, m * s, best), torch.minimum(near, gap)
        out[:, a:a + GROUP] = torch.copysign(best, k)
    return out


def exact(case, seed):
    c, s = _case(case), prepare(case, seed)
    d, H = c["H"] * c["dk"], c["H"]
    if c["op"] == "append":
        return torch.cat([_rounded(s["k_new"][a:a + 4096]) for a in range(0, s["k_new"].shape[0], 4096)])
    if c["op"] == "read":
        return torch.cat([_stored(s, c, b, c["at"][b], c["rows"][b]) for b in range(_batch(c))])
    scale = 1.0 / math.sqrt(c["dk"])
    if c["op"] == "prompt":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
        q0 = k0 = 0
        for n, before in zip(c["nq"], c["before"]):
            m = n + before
            at = torch.arange(m, device=DEV)
            zq, zk = _flat(_turned(s["q"][q0:q0 + n], at[before:], c)), _flat(_turned(s["k"][k0:k0 + m], at, c))
            v = s["v"][k0:k0 + m].double()
            for h in range(H):
                kv = h * c["KV"] // H
                for r in range(0, n, 4096):
                    a = zq[h, r:r + 4096] @ zk[kv].T * scale
                    if c["causal"]:
                        a = a.masked_fill(at[None] > before + r + at[:a.shape[0], None], -math.inf)
                    out[q0 + r:q0 + r + a.shape[0], h] = torch.softmax(a, -1) @ v[:, kv]
            q0, k0 = q0 + n, k0 + m
        return out
    out = torch.zeros(c["B"], d, dtype=torch.float64, device=DEV)
    W = s["W_KV"].double()
    for b, L in enumerate(_lengths(c)):
        K = _stored(s, c, b, 0, L)
        zk = _turned(K.view(L, H, c["dk"]), torch.arange(L, device=DEV), c)
        zq = _turned(s["q"][b].view(1, H, c["dk"]), torch.tensor([L - 1], device=DEV), c)
        a = torch.softmax((zk * zq.conj()).real.sum(-1) * scale, -1)              # [H, L]
        u = a @ K
        for h in range(H):
            out[b, h * c["dk"]:(h + 1) * c["dk"]] = u[h] @ W[:, h * c["dk"]:(h + 1) * c["dk"]]
    return out
