"""SlimLayer: a convenience owner of the torch buffers one attention layer
needs (key storage, workspace, output).  It only allocates memory and forwards
to the C-ABI calls of the same names; no arithmetic happens here."""
from __future__ import annotations

import numpy as np
import torch

from . import binding as B


def _device(device) -> torch.device:
    """With its index: a bare "cuda" is the current device, as tensors name it."""
    device = torch.device(device)
    return torch.device("cuda", torch.cuda.current_device()) if device.type == "cuda" and device.index is None else device


class Scratch:
    """Device memory of SlimLayer.prompt_attention, tree_decode, accumulate_weights and evict.  Layers whose calls run one
    after another on a stream may share one.  It grows with the largest call so far; what it grew out of is given back, unless a graph has been
    captured on it."""

    def __init__(self, device):
        self.device = _device(device)
        self.buffers = []        # the one in use last; before it those that captured graphs hold on to
        self.captured = False    # a graph uses the last one
        self.home = None         # the stream that it was allocated on

    def take(self, need: int) -> torch.Tensor:
        """At least `need` bytes for a call on the current stream."""
        if need == 0:
            raise ValueError("unsupported sizes")
        capturing, stream = torch.cuda.is_current_stream_capturing(), torch.cuda.current_stream(self.device)
        if not self.buffers or self.buffers[-1].numel() < need:
            if capturing:
                raise RuntimeError("the layer's scratch has to exist before a capture: reserve_scratch, or make a call of these "
                                   "sizes first")
            if self.buffers and not self.captured:
                self.buffers.pop()
            self.buffers.append(torch.empty(need, dtype=torch.uint8, device=self.device))
            self.captured, self.home = False, stream
        if capturing:
            self.captured = True
        elif stream != self.home:                # the allocator must not hand it out before this call has run
            self.buffers[-1].record_stream(stream)
        return self.buffers[-1]


class SlimLayer:
    def __init__(self, d: int, H: int, d_k: int, rope_theta: float, dtype: str, batch: int, t_cap: int,
                 device: str = "cuda:0", workspace: "torch.Tensor | None" = None, scratch: "Scratch | None" = None):
        if not torch.cuda.is_available():
            raise RuntimeError("SlimLayer needs a CUDA device (there is no CPU fallback)")
        self.device = _device(device)
        if scratch is not None and (not isinstance(scratch, Scratch) or scratch.device != self.device):
            raise ValueError(f"scratch: a Scratch on {self.device} is needed, e.g. another layer's .scratch")
        self.d, self.H, self.d_k, self.batch, self.t_cap = d, H, d_k, batch, t_cap
        self.dtype = dtype
        # type of q, of new key rows and of W_KV; an "fp8" ("fp4") layer keeps only its cache in 8 (4) bits
        self.tdtype = torch.float32 if dtype == "f32" else torch.bfloat16
        with torch.cuda.device(self.device):
            self.ctx = B.slim_create(d, H, d_k, rope_theta, {"f32": B.SLIM_F32, "bf16": B.SLIM_BF16, "fp8": B.SLIM_FP8, "fp4": B.SLIM_FP4}[dtype])
            if dtype in ("fp8", "fp4"):     # codes of all rows, then their exponents (scales): filled through the append calls only
                self.k = torch.zeros(B.slim_cache_bytes(self.ctx, batch, t_cap), dtype=torch.uint8, device=self.device)
            else:
                self.k = torch.zeros((batch, t_cap, d), dtype=self.tdtype, device=self.device)
            self.cache = B.slim_cache_create(self.ctx, self.k, batch, t_cap)
            need = B.slim_workspace_bytes(self.ctx, batch, t_cap)
            if workspace is None:      # layers that run one after another on a stream may share one
                workspace = torch.empty(need, dtype=torch.uint8, device=self.device)
            assert workspace.numel() >= need and workspace.data_ptr() % 256 == 0
            self.workspace = workspace
            self.o = torch.empty((batch, d), dtype=torch.float32, device=self.device)
            self.scratch = Scratch(self.device) if scratch is None else scratch
            self._extra = self.scratch.buffers

    # ---- set-up -------------------------------------------------------------
    def set_weights(self, W_K, W_V, want_wkv: bool = False):
        with torch.cuda.device(self.device):
            return B.slim_set_weights(self.ctx, W_K, W_V, want_wkv)

    def set_wkv(self, W_KV) -> None:
        with torch.cuda.device(self.device):
            B.slim_set_wkv(self.ctx, W_KV)

    def set_path(self, path: int) -> None:
        B.slim_set_path(self.ctx, path)

    def query(self, key: int) -> int:
        return B.slim_query(self.ctx, key)

    # ---- hot path -----------------------------------------------------------
    def append_k(self, k_new: torch.Tensor, positions: torch.Tensor) -> None:
        n_new = k_new.shape[1] if k_new.dim() == 3 else 1
        B.slim_append_k(self.ctx, self.cache, k_new, positions, n_new,
                        torch.cuda.current_stream(self.device).cuda_stream)

    def decode(self, q: torch.Tensor, lengths: torch.Tensor, o: torch.Tensor | None = None) -> torch.Tensor:
        o = self.o if o is None else o
        B.slim_decode(self.ctx, q, self.cache, lengths, o, self.workspace,
                      torch.cuda.current_stream(self.device).cuda_stream)
        return o

    def decode_step(self, q: torch.Tensor, k_new: torch.Tensor, lengths: torch.Tensor,
                    o: torch.Tensor | None = None) -> torch.Tensor:
        o = self.o if o is None else o
        B.slim_decode_step(self.ctx, q, k_new, self.cache, lengths, o, self.workspace,
                           torch.cuda.current_stream(self.device).cuda_stream)
        return o

    def decode_typed(self, q: torch.Tensor, lengths: torch.Tensor, k_new: "torch.Tensor | None" = None,
                     o: "torch.Tensor | None" = None) -> torch.Tensor:
        """decode, or with k_new decode_step, with o in its own type: float32, or bfloat16 (the default of a bf16 layer)."""
        self._arg("q", q, (self.batch, self.d), self.tdtype)
        self._arg("lengths", lengths, (self.batch,), torch.int32)
        if k_new is not None:
            self._arg("k_new", k_new, (self.batch, self.d), self.tdtype)
        if o is None:
            o = torch.empty((self.batch, self.d), dtype=self.tdtype, device=self.device)
        elif o.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError(f"o: float32 or bfloat16 is needed, got {o.dtype}")
        self._arg("o", o, (self.batch, self.d), o.dtype)
        with torch.cuda.device(self.device):
            B.slim_decode_typed(self.ctx, q, k_new, self.cache, lengths, o, B.SLIM_F32 if o.dtype == torch.float32 else B.SLIM_BF16,
                                self.workspace, torch.cuda.current_stream(self.device).cuda_stream)
        return o

    # ---- packed prompts -----------------------------------------------------------
    def prompt_attention(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, cu_k: torch.Tensor, max_k: int,
                         causal: bool = True, o: "torch.Tensor | None" = None) -> torch.Tensor:
        """Attention of packed prompts (binding.slim_prompt_attention): q [rows, H, d_k] (or [rows, d]), k and v [rows, heads, d_k]
        with as many heads as divide H; v float32, or bfloat16 in a layer that is not float32.  Positions below the layer's t_cap are there;
        longer prompts need binding.slim_reserve_positions.  k, v of no rows: every output row is zero."""
        if q.dim() not in (2, 3) or k.dim() not in (2, 3):
            raise ValueError("q, k: [rows, heads, d_k] or [rows, heads * d_k] is needed")
        kv = k.shape[1] if k.dim() == 3 else k.shape[1] // self.d_k
        self._arg("q", q, (q.shape[0],) + ((self.d,) if q.dim() == 2 else (self.H, self.d_k)), self.tdtype)
        self._arg("k", k, (k.shape[0],) + ((kv * self.d_k,) if k.dim() == 2 else (kv, self.d_k)), self.tdtype)
        if v.dtype not in (torch.float32, self.tdtype):
            raise ValueError(f"v: {torch.float32} or {self.tdtype} is needed, got {v.dtype}")
        self._arg("v", v, k.shape if v.dim() == k.dim() else (k.shape[0],) + ((kv * self.d_k,) if v.dim() == 2 else (kv, self.d_k)), v.dtype)
        if cu_q.dim() != 1 or cu_q.numel() < 2:
            raise ValueError("cu_q: [sequences + 1] is needed")
        self._arg("cu_q", cu_q, cu_q.shape, torch.int32)
        self._arg("cu_k", cu_k, cu_q.shape, torch.int32)
        o = torch.empty_like(q) if o is None else self._arg("o", o, q.shape, self.tdtype)
        n = cu_q.numel() - 1
        if q.shape[0] == 0:
            return o
        with torch.cuda.device(self.device):
            ws = self.scratch.take(B.slim_prompt_workspace_bytes(self.ctx, kv, n, q.shape[0], k.shape[0]))
            B.slim_prompt_attention(self.ctx, q, k, v, B.SLIM_F32 if v.dtype == torch.float32 else B.SLIM_BF16, kv, cu_q, cu_k, n, q.shape[0],
                                    k.shape[0], int(max_k), causal, o, ws, torch.cuda.current_stream(self.device).cuda_stream)
        return o

    def append_rows(self, k_new: torch.Tensor, positions: torch.Tensor, cu_rows: torch.Tensor) -> None:
        """Packed rows [rows, d] of the layer's sequences into the cache (binding.slim_append_rows)."""
        self._arg("k_new", k_new, (k_new.shape[0], self.d), self.tdtype)
        self._arg("positions", positions, (self.batch,), torch.int32)
        self._arg("cu_rows", cu_rows, (self.batch + 1,), torch.int32)
        if k_new.shape[0] == 0:
            return
        with torch.cuda.device(self.device):
            B.slim_append_rows(self.ctx, self.cache, k_new, positions, cu_rows, k_new.shape[0], torch.cuda.current_stream(self.device).cuda_stream)

    def read_rows(self, positions: torch.Tensor, cu_rows: torch.Tensor, rows: int, out: "torch.Tensor | None" = None) -> torch.Tensor:
        """`rows` packed rows [rows, d] as the cache holds them (binding.slim_read_rows)."""
        self._arg("positions", positions, (self.batch,), torch.int32)
        self._arg("cu_rows", cu_rows, (self.batch + 1,), torch.int32)
        out = torch.zeros((rows, self.d), dtype=self.tdtype, device=self.device) if out is None else self._arg("out", out, (rows, self.d), self.tdtype)
        if rows == 0:
            return out
        with torch.cuda.device(self.device):
            B.slim_read_rows(self.ctx, self.cache, positions, cu_rows, int(rows), out, torch.cuda.current_stream(self.device).cuda_stream)
        return out

    # ---- drafted tokens, cache budget -------------------------------------------
    def _arg(self, name: str, x: torch.Tensor, shape, dtype) -> torch.Tensor:
        if tuple(x.shape) != tuple(shape) or x.dtype != dtype or x.device != self.device or not x.is_contiguous():
            raise ValueError(f"{name}: a contiguous {dtype} tensor of shape {tuple(shape)} on {self.device} is needed, got "
                             f"{x.dtype} {tuple(x.shape)} on {x.device}" + ("" if x.is_contiguous() else ", not contiguous"))
        return x

    def reserve_scratch(self, n: int = 0, prompts: int = 0, q_rows: int = 0, k_rows: int = 0, kv_heads: "int | None" = None) -> None:
        """Size the scratch for trees of up to n tokens, accumulate_weights and evict at once (before a capture, for instance), and for
        prompt_attention of `prompts` sequences with q_rows rows of queries and k_rows of keys (kv_heads heads, H if None).
        Without it the scratch grows with the calls."""
        sizes = [B.slim_tree_workspace_bytes(self.ctx, self.batch, self.t_cap, i) for i in range(1, n + 1)]
        if n < 0 or 0 in sizes:
            raise ValueError(f"n: 0 to {B.SLIM_MAX_TREE} drafted tokens are possible, got {n}")
        sizes += [B.slim_weights_workspace_bytes(self.ctx, self.batch, self.t_cap), B.slim_evict_workspace_bytes(self.ctx, self.batch, self.t_cap)]
        if prompts or q_rows or k_rows:
            sizes.append(B.slim_prompt_workspace_bytes(self.ctx, self.H if kv_heads is None else kv_heads, prompts, q_rows, k_rows))
            if sizes[-1] == 0:
                raise ValueError(f"prompts: no call has {prompts} sequences, {q_rows} rows of queries and {k_rows} of keys")
        with torch.cuda.device(self.device):
            self.scratch.take(max(sizes))

    def tree_decode(self, q: torch.Tensor, k_tree: torch.Tensor, lengths: torch.Tensor, parents: torch.Tensor,
                    o: torch.Tensor | None = None) -> torch.Tensor:
        """Attention of q.shape[1] drafted tokens a sequence (binding.slim_tree_decode); o has the layer's dtype."""
        if q.dim() != 3:
            raise ValueError("q: [batch, n, d] is needed")
        n, i32 = q.shape[1], torch.int32
        self._arg("q", q, (self.batch, n, self.d), self.tdtype)
        self._arg("k_tree", k_tree, (self.batch, n, self.d), self.tdtype)
        self._arg("lengths", lengths, (self.batch,), i32)
        self._arg("parents", parents, (self.batch, n), i32)
        o = torch.empty_like(q) if o is None else self._arg("o", o, q.shape, self.tdtype)
        with torch.cuda.device(self.device):
            ws = self.scratch.take(B.slim_tree_workspace_bytes(self.ctx, self.batch, self.t_cap, n))
            B.slim_tree_decode(self.ctx, q, k_tree, self.cache, lengths, parents, n, o, ws,
                               torch.cuda.current_stream(self.device).cuda_stream)
        return o

    def tree_verify(self, p: torch.Tensor, q: torch.Tensor, tokens: torch.Tensor, parents: torch.Tensor, r: torch.Tensor):
        """(path [batch, n], count [batch], next_token [batch]) of binding.slim_tree_verify."""
        if p.dim() != 3:
            raise ValueError("p: [batch, n, vocab] is needed")
        b, n, vocab = p.shape
        f32, i32 = torch.float32, torch.int32
        self._arg("p", p, (b, n, vocab), f32)
        self._arg("q", q, (b, n, vocab), f32)
        self._arg("tokens", tokens, (b, n), i32)
        self._arg("parents", parents, (b, n), i32)
        self._arg("r", r, (b, n), f32)
        path, count, nxt = (torch.empty(s, dtype=i32, device=self.device) for s in ((b, n), (b,), (b,)))
        with torch.cuda.device(self.device):
            B.slim_tree_verify(self.ctx, p, q, tokens, parents, r, b, n, vocab, path, count, nxt,
                               torch.cuda.current_stream(self.device).cuda_stream)
        return path, count, nxt

    def tree_commit(self, k_tree: torch.Tensor, lengths: torch.Tensor, path: torch.Tensor, count: torch.Tensor) -> None:
        """Accepted keys into the cache (binding.slim_tree_commit); the caller adds count to lengths after the last layer."""
        if k_tree.dim() != 3:
            raise ValueError("k_tree: [batch, n, d] is needed")
        n, i32 = k_tree.shape[1], torch.int32
        self._arg("k_tree", k_tree, (self.batch, n, self.d), self.tdtype)
        self._arg("lengths", lengths, (self.batch,), i32)
        self._arg("path", path, (self.batch, n), i32)
        self._arg("count", count, (self.batch,), i32)
        with torch.cuda.device(self.device):
            B.slim_tree_commit(self.ctx, self.cache, k_tree, lengths, path, count, n,
                               torch.cuda.current_stream(self.device).cuda_stream)

    def accumulate_weights(self, q: torch.Tensor, lengths: torch.Tensor, acc: torch.Tensor) -> torch.Tensor:
        """acc [batch, t_cap] += the step's probabilities summed over the heads (binding.slim_accumulate_weights)."""
        self._arg("q", q, (self.batch, self.d), self.tdtype)
        self._arg("lengths", lengths, (self.batch,), torch.int32)
        self._arg("acc", acc, (self.batch, self.t_cap), torch.float32)
        with torch.cuda.device(self.device):
            ws = self.scratch.take(B.slim_weights_workspace_bytes(self.ctx, self.batch, self.t_cap))
            B.slim_accumulate_weights(self.ctx, q, self.cache, lengths, acc, ws, torch.cuda.current_stream(self.device).cuda_stream)
        return acc

    def evict(self, lengths: torch.Tensor, acc: torch.Tensor, budget: int, recent: int) -> torch.Tensor:
        """Bring sequences longer than `budget` down to it (binding.slim_evict); returns kept [batch, budget].  The caller
        clamps lengths to the budget after the last layer."""
        self._arg("lengths", lengths, (self.batch,), torch.int32)
        self._arg("acc", acc, (self.batch, self.t_cap), torch.float32)
        kept = torch.empty((self.batch, max(int(budget), 0)), dtype=torch.int32, device=self.device)
        with torch.cuda.device(self.device):
            ws = self.scratch.take(B.slim_evict_workspace_bytes(self.ctx, self.batch, self.t_cap))
            B.slim_evict(self.ctx, self.cache, lengths, acc, int(budget), int(recent), kept, ws,
                         torch.cuda.current_stream(self.device).cuda_stream)
        return kept

    def profile(self, enable: bool) -> None:
        B.slim_profile_enable(self.ctx, enable)

    def profile_read(self):
        return B.slim_profile_read(self.ctx)

    def device_status(self) -> int:
        return B.slim_device_status(self.ctx, torch.cuda.current_stream(self.device).cuda_stream)

    def close(self) -> None:
        if getattr(self, "cache", None):
            B.slim_cache_destroy(self.cache); self.cache = None
        if getattr(self, "ctx", None):
            B.slim_destroy(self.ctx); self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def to_device_keys(K_f32: np.ndarray, dtype: str, device) -> torch.Tensor:
    """Host float32 array holding cache-dtype values -> device tensor of the cache dtype (exact)."""
    t = torch.from_numpy(np.ascontiguousarray(K_f32))
    return t.to(device=device, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
