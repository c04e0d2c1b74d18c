"""Decoding that branches over a paged KV cache: drafted trees and beams.  Thin binding, as in the package's __init__:
torch CUDA tensors go to the C ABI of include/prima.h, all computation happens in the HIP library.

    cache = PagedCache.empty(n_layers, n_pages, page_rows, n_kv_heads, head_dim)
    bits, depth = draft_tree([-1, 0, 0, 1])               # parents of the drafted tokens of a sequence
    step = PagedStep(n_past, n_tok, table, tree, positions)   # one per decode step, for all layers
    q = paged_append(cache, layer, step, k, v, rope=rope, q=q)
    o = tree_attn(cache, layer, step, q)
    tree_accept(cache, step, path, n_accept)              # all layers

    scores, beams, tokens = beam_select(logits, scores)
    table = beam_reorder(cache, table, beams, n_rows)     # all layers
"""
import ctypes as C
from threading import get_ident

import torch

from . import _ffi
from ._ffi import PAGED_MAX_SEQS, TREE_MAX_TOK, BEAM_MAX, PrimaError  # noqa: F401

_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


# the current stream as a number, without the stream object that torch.cuda.current_stream() makes (2.9 us a call)
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _stream(t):
    """The current stream of the device that t is on."""
    return _raw_stream(t.device.index)


def _ints(t, name, dims):
    if not (t.is_cuda and t.dtype == torch.int32 and t.dim() == dims and t.is_contiguous()):
        raise TypeError(f"{name}: need a contiguous {dims}-d CUDA tensor of torch.int32")
    return t


def _counts(values, name, most=2 ** 31 - 1):
    """A ctypes array of host numbers (which by itself would take any modulo 2^32)."""
    values = [int(n) for n in values]
    if values and not 0 <= min(values) <= max(values) <= most:
        raise ValueError(f"{name}: need numbers from 0 to {most}")
    return (C.c_int32 * max(len(values), 1))(*values)


def _check_scratch(t):
    if not (t.is_cuda and t.is_contiguous()):
        raise TypeError("workspace: need a contiguous CUDA tensor")


def _heads(t, name, tokens, heads, D, dtype):
    """[tokens, heads (0: any), D] whose heads follow one another; the tokens may be strided (views of a fused projection).  Returns the distance of two tokens."""
    shape, stride = t.shape, t.stride()
    if t.dtype is not dtype or not t.is_cuda or len(shape) != 3:
        raise TypeError(f"{name}: need a 3-d CUDA tensor of {dtype}")
    n, h, d = shape
    if n != tokens or d != D or (heads and h != heads):
        raise ValueError(f"{name}: shape {tuple(shape)}, need [{tokens}, {heads or 'heads'}, {D}]")
    if n and h and (stride[2] != 1 or (h > 1 and stride[1] != D)):
        raise ValueError(f"{name}: the heads of a token must follow one another")
    return stride[0] if n > 1 else h * D


class PagedCache:
    """Pages of all layers: kv [layers, 2 (K, V), pages, KV heads, rows of a page, head size], float16 or bfloat16.  The last axis must be
    contiguous; the others may be strided (rows in front of heads, say, by a transposed view)."""

    def __init__(self, kv):
        if not (kv.is_cuda and kv.dim() == 6 and kv.shape[1] == 2 and kv.dtype in (torch.float16, torch.bfloat16)):
            raise TypeError("kv: need a CUDA tensor [layers, 2, pages, KV heads, page rows, head size] of float16 or bfloat16")
        if kv.stride(5) != 1:
            raise ValueError("kv: the elements of a row must follow one another")
        self.kv = kv
        self.n_layers, _, self.n_pages, self.n_kv_heads, self.page_rows, self.head_dim = kv.shape
        # an axis of one element has no stride that matters
        D = self.head_dim
        strides = [s if n > 1 else D for n, s in zip(kv.shape, kv.stride())]
        self.layer_stride = strides[0] if self.n_layers > 1 else 0
        at, size = kv.data_ptr(), kv.element_size()
        self._layers = [_ffi.KVPages(at + l * kv.stride(0) * size, at + (l * kv.stride(0) + kv.stride(1)) * size, strides[2], strides[3], strides[4],
                                     self.n_pages, self.page_rows, self.n_kv_heads, D, _DTYPES[kv.dtype]) for l in range(self.n_layers)]
        self._refs = [C.byref(p) for p in self._layers]
        self.scale = D ** -0.5

    @classmethod
    def empty(cls, n_layers, n_pages, page_rows, n_kv_heads, head_dim, dtype=torch.float16, device="cuda"):
        return cls(torch.empty((n_layers, 2, n_pages, n_kv_heads, page_rows, head_dim), dtype=dtype, device=device))


class PagedStep:
    """One decode step: n_tok[b] tokens (0 to 64) for sequence b behind its n_past[b] cached rows (both lists of numbers on the host).
    table   int32 [sequences, pages]: the pages of every sequence in order; entries outside the pool name no page
    tree    int64 [tokens] or None: bit j: the token attends to its sequence's drafted token j (draft_tree makes them; its own bit among
            them).  None: chains
    positions   int32 [tokens] or None: where a token is rotated to.  None: n_past + its index
    Keeps the tensors alive, and the scratch that tree_attn takes where it is given none, for the layers that follow: one per thread and stream, since a call enqueues two
    launches, between which another thread's may come."""

    def __init__(self, n_past, n_tok, table, tree=None, positions=None):
        B = len(n_past)
        if len(n_tok) != B:
            raise ValueError("n_past and n_tok need as many entries")
        _ints(table, "table", 2)
        if table.shape[0] != B:
            raise ValueError("table needs one row per sequence")
        past, tok = _counts(n_past, "n_past"), _counts(n_tok, "n_tok", TREE_MAX_TOK)
        self.n_tokens = sum(tok)
        if tree is not None:
            if not (tree.is_cuda and tree.dtype == torch.int64 and tree.is_contiguous()):
                raise TypeError("tree: need a contiguous CUDA tensor of torch.int64")
            if tree.numel() != self.n_tokens:
                raise ValueError("tree needs one word per token")
        if positions is not None and _ints(positions, "positions", 1).numel() != self.n_tokens:
            raise ValueError("positions needs one entry per token")
        self.n_seqs = B
        self._keep = (table, tree, positions, past, tok)
        ip = C.POINTER(C.c_int32)
        self._step = _ffi.PagedStep(B, table.shape[1], C.cast(past, ip), C.cast(tok, ip), table.data_ptr(),
                                    None if tree is None else tree.data_ptr(), None if positions is None else positions.data_ptr())
        self._ref = C.byref(self._step)
        self._scratch = {}


def draft_tree(parents):
    """parents[i]: the drafted token that token i continues, an earlier one, or -1 (it continues the cached rows).
    Returns (bits, depth): the words of PagedStep's tree as signed 64-bit numbers, and each token's distance from the cached rows."""
    if len(parents) > TREE_MAX_TOK:
        raise ValueError(f"a tree has at most {TREE_MAX_TOK} tokens")
    bits, depth = [], []
    for i, p in enumerate(parents):
        if not -1 <= p < i:
            raise ValueError("a token continues an earlier one, or -1")
        bits.append((bits[p] if p >= 0 else 0) | 1 << i)
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return [b - (1 << 64) if b >> 63 else b for b in bits], depth


def rope_table(n_rows, head_dim, theta, device="cuda"):
    """(cos, sin) of p * theta^(-2i/head_dim): float32 [n_rows, head_dim/2, 2]."""
    out = torch.empty((n_rows, head_dim // 2, 2), dtype=torch.float32, device=device)
    _ffi.check(_ffi.lib().prima_rope_table(n_rows, head_dim, float(theta), out.data_ptr(), _stream(out)), "prima_rope_table")
    return out


def paged_append(cache, layer, step, k, v, rope=None, rope_mode=0, q=None, q_out=None):
    """Rotates and appends the step's keys and values k, v [tokens, KV heads, D] to the pages of `layer`; returns the rotated queries
    (q [tokens, heads, D]; q_out may be q) or None.  All of the cache's type, or float32 beside a float16 cache.  rope: float32 [positions, D/2, 2],
    None: nothing is rotated."""
    D, n, dtype = cache.head_dim, step.n_tokens, k.dtype
    if dtype not in _DTYPES:
        raise TypeError("k: need float32, float16 or bfloat16")
    ldk, ldv = _heads(k, "k", n, cache.n_kv_heads, D, dtype), _heads(v, "v", n, cache.n_kv_heads, D, dtype)
    rope_at, rows = None, 0
    if rope is not None:
        if not (rope.is_cuda and rope.dtype is torch.float32 and rope.is_contiguous() and rope.dim() == 3 and rope.shape[1:] == (D // 2, 2)):
            raise TypeError(f"rope: need a contiguous CUDA tensor of float32 [positions, {D // 2}, 2]")
        rope_at, rows = rope.data_ptr(), rope.shape[0]
    q_at, heads, ldq, out_at, ldo = None, 0, 0, None, 0
    if q is not None:
        ldq, heads = _heads(q, "q", n, 0, D, dtype), q.shape[1]
        if q_out is None:
            q_out, ldo = q.new_empty((n, heads, D)), heads * D
        else:
            ldo = _heads(q_out, "q_out", n, heads, D, dtype)
        q_at, out_at = q.data_ptr(), q_out.data_ptr()
    if n == 0:
        return q_out
    code = _ffi.lib().prima_paged_append(cache._refs[layer], step._ref, _DTYPES[dtype], k.data_ptr(), ldk, v.data_ptr(), ldv, rope_at, rows, rope_mode,
                                         heads, q_at, ldq, out_at, ldo, _stream(k))
    if code:
        raise PrimaError(code, "prima_paged_append")
    return q_out


def tree_attn_workspace_bytes(cache, step, n_heads):
    return _ffi.lib().prima_tree_attn_workspace_bytes(cache._refs[0], step._ref, n_heads)


def tree_attn_plan(cache, step, n_heads, dtype):
    """How tree_attn shares the step out: (few, many, ranges, range_rows), queries of a workgroup in blocks of 16 or of 32 (the kernel that is not used: 0) and,
    per sequence, the ranges its rows are divided into and how many rows each has but the last."""
    few, many, B = C.c_int32(), C.c_int32(), step.n_seqs
    ranges, rows = (C.c_int32 * max(B, 1))(), (C.c_int32 * max(B, 1))()
    _ffi.check(_ffi.lib().prima_tree_attn_plan(cache._refs[0], step._ref, n_heads, _DTYPES[dtype], C.byref(few), C.byref(many), ranges, rows), "prima_tree_attn_plan")
    return few.value, many.value, list(ranges)[:B], list(rows)[:B]


def tree_attn(cache, layer, step, q, o=None, scale=None, workspace=None):
    """Attention of the step's tokens q [tokens, heads, D] over their sequences' rows in the pages of `layer`, the step's own (appended before)
    among them -> o like q.  scale: None: D ** -0.5."""
    D, n, dtype, lib = cache.head_dim, step.n_tokens, q.dtype, _ffi.lib()
    if dtype not in _DTYPES:
        raise TypeError("q: need float32, float16 or bfloat16")
    ldq, heads = _heads(q, "q", n, 0, D, dtype), q.shape[1]
    if o is None:
        o, ldo = q.new_empty((n, heads, D)), heads * D
    else:
        ldo = _heads(o, "o", n, heads, D, dtype)
    if n == 0:
        return o
    stream = _stream(q)
    if workspace is None:  # a step's calls have the same need for every layer of a cache; a graph gets scratch of its own
        key = (get_ident(), stream, heads, D, cache.n_kv_heads)
        capturing = torch.cuda.is_current_stream_capturing()
        workspace = None if capturing else step._scratch.get(key)
        if workspace is None:
            workspace = q.new_empty(max(256, lib.prima_tree_attn_workspace_bytes(cache._refs[layer], step._ref, heads)), dtype=torch.uint8)
            if not capturing:
                step._scratch[key] = workspace
    else:
        _check_scratch(workspace)
    code = lib.prima_tree_attn(cache._refs[layer], step._ref, heads, _DTYPES[dtype], q.data_ptr(), ldq, cache.scale if scale is None else scale, o.data_ptr(), ldo,
                               workspace.data_ptr(), workspace.nbytes, stream)
    if code:
        raise PrimaError(code, "prima_tree_attn")
    return o


def tree_accept(cache, step, path, n_accept):
    """Moves the accepted branch of every sequence's tree to its place, in all layers: row n_past + path[b, i] becomes row n_past + i, i < n_accept[b].
    path int32 [sequences, any], n_accept int32 [sequences], on the GPU."""
    _ints(path, "path", 2)
    _ints(n_accept, "n_accept", 1)
    n, ld = path.shape
    if n != step.n_seqs or n_accept.shape[0] != n:
        raise ValueError("path and n_accept need one row per sequence")
    if ld == 0:
        return
    code = _ffi.lib().prima_tree_accept(cache._refs[0], cache.layer_stride, cache.n_layers, step._ref, path.data_ptr(), ld, n_accept.data_ptr(), _stream(path))
    if code:
        raise PrimaError(code, "prima_tree_accept")


def beam_select_workspace_bytes(n_seqs, n_beams, vocab, n_best):
    return _ffi.lib().prima_beam_select_workspace_bytes(n_seqs, n_beams, vocab, n_best)


def beam_select(logits, scores, n_best=None, done=None, eos=0, workspace=None):
    """The n_best (None: as many as beams) best continuations of every sequence's beams: logits [sequences * beams, vocab], scores float32 [sequences, beams];
    done uint8 [sequences, beams] or None: beams that have ended (token eos, score unchanged, is all they have).
    Returns (scores float32, beams int32, tokens int32), each [sequences, n_best], best first, of equal ones the lowest (beam, token)."""
    if not (logits.is_cuda and logits.dim() == 2 and logits.dtype in _DTYPES and (logits.shape[1] < 2 or logits.stride(1) == 1)):
        raise TypeError("logits: need a 2-d CUDA tensor of float32, float16 or bfloat16 with contiguous rows")
    if not (scores.is_cuda and scores.dim() == 2 and scores.dtype is torch.float32 and scores.is_contiguous()):
        raise TypeError("scores: need a contiguous 2-d CUDA tensor of float32")
    (B, W), (rows, V) = scores.shape, logits.shape
    if rows != B * W:
        raise ValueError("logits needs one row per beam")
    if done is not None and not (done.is_cuda and done.dtype in (torch.uint8, torch.bool) and done.shape == scores.shape and done.is_contiguous()):
        raise TypeError("done: need a contiguous CUDA tensor of uint8 like scores")
    K, lib = W if n_best is None else n_best, _ffi.lib()
    if not (-2 ** 31 <= eos < 2 ** 31 and K < 2 ** 31):
        raise ValueError("eos and n_best need to be 32-bit numbers")
    if workspace is None:
        workspace = scores.new_empty(max(256, lib.prima_beam_select_workspace_bytes(B, W, V, K)), dtype=torch.uint8)
    else:
        _check_scratch(workspace)
    out = scores.new_empty((B, max(K, 0)))
    beams, tokens = torch.empty_like(out, dtype=torch.int32), torch.empty_like(out, dtype=torch.int32)
    code = lib.prima_beam_select(_DTYPES[logits.dtype], logits.data_ptr(), logits.stride(0) if rows > 1 else V, B, W, V, scores.data_ptr(),
                                 None if done is None else done.data_ptr(), eos, K, out.data_ptr(), beams.data_ptr(), tokens.data_ptr(),
                                 workspace.data_ptr(), workspace.nbytes, _stream(scores))
    if code:
        raise PrimaError(code, "prima_beam_select")
    return out, beams, tokens


def beam_reorder(cache, table, parents, n_rows, out=None):
    """The pages of beam searches after a choice: table int32 [sequences * beams, pages], parents int32 [sequences, beams] (the beam that each
    continues), n_rows: a list with the rows of every sequence's beams.  Returns the new table; where several beams continue one, the partly filled
    page is copied, in all layers, into pages of beams that nobody continues."""
    _ints(table, "table", 2)
    _ints(parents, "parents", 2)
    (B, W), (rows, width) = parents.shape, table.shape
    if rows != B * W or len(n_rows) != B:
        raise ValueError("table needs one row per beam, n_rows one entry per sequence")
    if out is None:
        out = torch.empty_like(table)
    elif _ints(out, "out", 2).shape != table.shape:
        raise ValueError("out: need a tensor like table")
    code = _ffi.lib().prima_beam_reorder(cache._refs[0], cache.layer_stride, cache.n_layers, B, W, _counts(n_rows, "n_rows"), parents.data_ptr(),
                                         table.data_ptr(), out.data_ptr(), width, _stream(table))
    if code:
        raise PrimaError(code, "prima_beam_reorder")
    return out
