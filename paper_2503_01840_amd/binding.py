"""ctypes binding of libeagle3.so: argument marshalling only.

Every step of the speculative path runs in the HIP kernels behind the C ABI declared in
include/eagle3.h; this module turns torch tensors into pointers and sizes, allocates output
tensors and the workspace through torch, and passes torch's current stream.  There is no CPU or
torch fallback: a missing library raises.
"""
import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libeagle3.so")
EAGLE3_FP32, EAGLE3_BF16, EAGLE3_FP8 = 0, 1, 2

EXPORTS = ["eagle3_create", "eagle3_destroy", "eagle3_workspace_bytes", "eagle3_set_workspace", "eagle3_set_weights",
           "eagle3_strerror", "eagle3_last_error", "eagle3_profile_begin", "eagle3_profile_read", "eagle3_profile_end",
           "eagle3_fuse_features", "eagle3_draft_expand",
           "eagle3_tree_verify", "eagle3_tree_verify_layers", "eagle3_accept", "eagle3_accept_static", "eagle3_commit", "eagle3_prefill", "eagle3_draft_chain", "eagle3_ttt_attention",
           "eagle3_rope_turns", "eagle3_rope", "eagle3_rope_grad", "eagle3_paged_append", "eagle3_paged_read", "eagle3_paged_attention",
           "eagle3_paged_attention_workspace"]


class Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("hidden", "n_heads", "n_kv_heads", "head_dim", "intermediate", "vocab",
                                         "draft_vocab", "n_layers")] + \
               [("tap_layers", C.c_int32 * 3), ("dtype", C.c_int32), ("rope_theta", C.c_float), ("rms_eps", C.c_float)] + \
               [(n, C.c_int32) for n in ("max_batch", "max_nodes", "max_depth", "max_topk", "max_new")]


class LayerWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down", "norm_attn", "norm_mlp")]


class TargetWeights(C.Structure):
    _fields_ = [("layers", C.POINTER(LayerWeights)), ("embed", C.c_void_p), ("final_norm", C.c_void_p),
                ("lm_head", C.c_void_p)]


class DraftWeights(C.Structure):
    _fields_ = [("w_fc", C.c_void_p), ("layer", LayerWeights), ("norm_embed", C.c_void_p), ("norm_feat", C.c_void_p),
                ("final_norm", C.c_void_p), ("lm_head", C.c_void_p), ("d2t", C.c_void_p)]


class KV(C.Structure):
    _fields_ = [("k", C.POINTER(C.c_void_p)), ("v", C.POINTER(C.c_void_p)), ("kv_indptr", C.c_void_p),
                ("prefix_len", C.c_void_p), ("max_prefix_len", C.c_int32)]


class DraftDebug(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("pool_tok", "pool_parent", "pool_score", "frontier", "chosen")]


class RopeSpec(C.Structure):
    _fields_ = [("turns", C.c_void_p), ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("amplitude", C.c_float)]


class PagedKV(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k", "v", "k_exp", "v_exp", "page_table")] + \
               [(n, C.c_int32) for n in ("dtype", "n_pages", "page_size", "max_pages", "n_kv_heads", "head_dim")]


_lib = None


def lib():
    """Loads libeagle3.so (built in-tree by paper_2503_01840_amd.build); raises if it is not there."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2503_01840_amd.build` "
                               "(there is no fallback path)")
        L = C.CDLL(LIB_PATH)
        L.eagle3_strerror.restype = C.c_char_p
        L.eagle3_last_error.restype = C.c_char_p
        L.eagle3_strerror.argtypes = [C.c_int]
        L.eagle3_create.argtypes = [C.POINTER(Config), C.POINTER(C.c_void_p)]
        L.eagle3_destroy.argtypes = [C.c_void_p]
        L.eagle3_workspace_bytes.argtypes = [C.c_void_p, C.POINTER(C.c_size_t)]
        L.eagle3_set_workspace.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t]
        L.eagle3_set_weights.argtypes = [C.c_void_p, C.POINTER(TargetWeights), C.POINTER(DraftWeights)]
        L.eagle3_profile_begin.argtypes = [C.c_void_p]
        L.eagle3_profile_end.argtypes = [C.c_void_p]
        L.eagle3_profile_read.argtypes = [C.c_void_p, C.c_int, C.POINTER(C.c_double), C.POINTER(C.c_int64),
                                          C.POINTER(C.c_double)]
        L.eagle3_fuse_features.argtypes = [C.c_void_p] + [C.c_void_p] * 3 + [C.c_int32, C.c_void_p, C.c_void_p]
        L.eagle3_draft_expand.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.POINTER(KV), C.c_int32,
                                          C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                          C.POINTER(DraftDebug), C.c_void_p]
        L.eagle3_tree_verify.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.POINTER(KV),
                                         C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.eagle3_tree_verify_layers.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.POINTER(KV),
                                                C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
        L.eagle3_accept.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float,
                                    C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.eagle3_accept_static.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float,
                                           C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.eagle3_commit.argtypes = [C.c_void_p, C.c_int32, C.c_int32] + [C.c_void_p] * 4 + [C.POINTER(KV), C.c_void_p,
                                    C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                    C.c_void_p]
        L.eagle3_prefill.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.POINTER(KV), C.POINTER(KV), C.c_void_p, C.c_void_p,
                                     C.c_void_p]
        L.eagle3_draft_chain.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.POINTER(KV),
                                         C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
        L.eagle3_ttt_attention.argtypes = [C.c_int32] * 6 + [C.c_void_p] * 5
        L.eagle3_rope_turns.argtypes = [C.c_int32, C.c_double, C.c_int32] + [C.c_double] * 4 + [C.c_void_p]
        L.eagle3_rope.argtypes = [C.c_int32] * 3 + [C.POINTER(RopeSpec), C.c_void_p] + \
            [C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64] * 2 + [C.c_void_p]
        L.eagle3_rope_grad.argtypes = L.eagle3_rope.argtypes
        L.eagle3_paged_append.argtypes = [C.POINTER(PagedKV), C.c_int32, C.c_int32] + [C.c_void_p] * 5 + [C.c_int64] * 2 + [C.c_void_p]
        L.eagle3_paged_read.argtypes = L.eagle3_paged_append.argtypes
        L.eagle3_paged_attention.argtypes = [C.POINTER(PagedKV), C.c_int32, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_int32, C.c_float,
                                             C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.eagle3_paged_attention_workspace.argtypes = [C.POINTER(PagedKV), C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_size_t)]
        _lib = L
    return _lib


class Eagle3Error(RuntimeError):
    def __init__(self, code):
        L = lib()
        msg = L.eagle3_strerror(code).decode()
        if code == -4:
            msg += ": " + L.eagle3_last_error().decode()
        super().__init__(f"eagle3 error {code}: {msg}")
        self.code = code


def _check(code):
    if code != 0:
        raise Eagle3Error(code)


def _ptr(t, dtype=None):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device, contiguous tensors only"
    if dtype is not None:
        assert t.dtype == dtype, (t.dtype, dtype)
    return t.data_ptr()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _layer_struct(W, keep):
    s = LayerWeights()
    for n, _ in LayerWeights._fields_:
        t = W.get(n)
        if t is not None:
            keep.append(t)
            setattr(s, n, _ptr(t))
    return s


class KVCache:
    """Per-layer cache tensors [slots, Hkv, d] plus device kv_indptr [B+1] / prefix_len [B] (int32)."""

    def __init__(self, k_layers, v_layers, kv_indptr, prefix_len, max_prefix_len):
        self.k_layers, self.v_layers = list(k_layers), list(v_layers)
        self.kv_indptr, self.prefix_len, self.max_prefix_len = kv_indptr, prefix_len, int(max_prefix_len)
        self._build()

    def set_max_prefix_len(self, n):
        """The host-side bound on prefix_len (sizes launches); to be kept ahead of the device values."""
        self.max_prefix_len = int(n)
        self.c.max_prefix_len = int(n)

    def _build(self):
        n = len(self.k_layers)
        self._k = (C.c_void_p * n)(*[_ptr(t) for t in self.k_layers])
        self._v = (C.c_void_p * n)(*[_ptr(t) for t in self.v_layers])
        self.c = KV(C.cast(self._k, C.POINTER(C.c_void_p)), C.cast(self._v, C.POINTER(C.c_void_p)),
                    _ptr(self.kv_indptr, torch.int32), _ptr(self.prefix_len, torch.int32), self.max_prefix_len)


class Eagle3Context:
    """Owns the library context and its torch-allocated workspace."""

    def __init__(self, shape=None, *, max_batch=1, max_nodes=64, max_depth=8, max_topk=10, max_new=8, device="cuda:0",
                 **dims):
        """`shape`: an object with the model fields of eagle3_config (e.g. eagle3_synth.Eagle3Shape) or None with
        the fields given as keyword arguments."""
        g = (lambda n: dims[n]) if shape is None else (lambda n: dims.get(n, getattr(shape, n, None)))
        cfg = Config()
        for n in ("hidden", "n_heads", "n_kv_heads", "head_dim", "intermediate", "vocab", "draft_vocab", "n_layers"):
            setattr(cfg, n, int(g(n)))
        taps = dims.get("tap_layers", getattr(shape, "taps", None))
        cfg.tap_layers = (C.c_int32 * 3)(*[int(t) for t in taps])
        dt = g("dtype")
        cfg.dtype = EAGLE3_BF16 if dt in ("bf16", EAGLE3_BF16, torch.bfloat16) else EAGLE3_FP32
        cfg.rope_theta, cfg.rms_eps = float(g("rope_theta")), float(g("rms_eps"))
        cfg.max_batch, cfg.max_nodes, cfg.max_depth, cfg.max_topk, cfg.max_new = (int(max_batch), int(max_nodes),
                                                                                  int(max_depth), int(max_topk), int(max_new))
        self.cfg, self.device = cfg, torch.device(device)
        self.storage_dtype = torch.bfloat16 if cfg.dtype == EAGLE3_BF16 else torch.float32
        self._h = C.c_void_p()
        _check(lib().eagle3_create(C.byref(cfg), C.byref(self._h)))
        need = C.c_size_t()
        _check(lib().eagle3_workspace_bytes(self._h, C.byref(need)))
        self.workspace_bytes = need.value
        self._ws = torch.empty(need.value + 256, dtype=torch.uint8, device=self.device)
        off = (-self._ws.data_ptr()) % 256
        _check(lib().eagle3_set_workspace(self._h, self._ws.data_ptr() + off, need.value))
        self._keep = []

    def close(self):
        if self._h:
            lib().eagle3_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def profile_begin(self):
        _check(lib().eagle3_profile_begin(self._h))

    def profile_read(self, kind):
        """(total ms, launches, weight bytes) of the GEMM launches of one kind since profile_begin: 0 = at most 32
        rows, 1 = 33..64 rows with 64-weight-row workgroups, 2 = 33..64 rows with workgroups of 128 or 256 weight rows,
        3 = more than 64 rows (see include/eagle3_measure.h)."""
        ms, n, by = C.c_double(), C.c_int64(), C.c_double()
        _check(lib().eagle3_profile_read(self._h, int(kind), C.byref(ms), C.byref(n), C.byref(by)))
        return ms.value, n.value, by.value

    def profile_end(self):
        _check(lib().eagle3_profile_end(self._h))

    def set_weights(self, target=None, draft=None):
        """target: {"layers": [layer dicts], "embed", "final_norm", "lm_head"}; draft: {"w_fc", "layer": {...},
        "norm_embed", "norm_feat", "final_norm", "lm_head", "d2t"}; tensors on the device in the storage dtype."""
        keep = []
        tw = dw = None
        if target is not None:
            arr = (LayerWeights * len(target["layers"]))(*[_layer_struct(W, keep) for W in target["layers"]])
            assert len(target["layers"]) == self.cfg.n_layers
            tw = TargetWeights(C.cast(arr, C.POINTER(LayerWeights)), _ptr(target["embed"]), _ptr(target["final_norm"]),
                               _ptr(target["lm_head"]))
            keep += [arr, target["embed"], target["final_norm"], target["lm_head"]]
        if draft is not None:
            dw = DraftWeights(_ptr(draft["w_fc"]), _layer_struct(draft["layer"], keep), _ptr(draft["norm_embed"]),
                              _ptr(draft["norm_feat"]), _ptr(draft["final_norm"]), _ptr(draft["lm_head"]),
                              _ptr(draft["d2t"], torch.int32))
            keep += [draft[n] for n in ("w_fc", "norm_embed", "norm_feat", "final_norm", "lm_head", "d2t")]
        _check(lib().eagle3_set_weights(self._h, C.byref(tw) if tw else None, C.byref(dw) if dw else None))
        self._keep += keep


def eagle3_fuse_features(ctx, low, mid, high):
    M, k = low.shape
    g = torch.empty(M, k, dtype=torch.float32, device=low.device)
    _check(lib().eagle3_fuse_features(ctx._h, _ptr(low, torch.float32), _ptr(mid, torch.float32),
                                      _ptr(high, torch.float32), M, _ptr(g), _stream()))
    return g


def eagle3_draft_expand(ctx, g_new, tok_new, draft_kv, depth, topk, n_nodes, debug=False):
    dev = g_new.device
    n_new = g_new.shape[0]
    out = {"tree_tok": torch.empty(n_nodes, dtype=torch.int32, device=dev),
           "parent": torch.empty(n_nodes, dtype=torch.int32, device=dev),
           "depth": torch.empty(n_nodes, dtype=torch.int32, device=dev),
           "score": torch.empty(n_nodes, dtype=torch.float32, device=dev)}
    dbg = None
    if debug:
        pool = 1 + topk + (depth - 1) * topk * topk
        out.update(pool_tok=torch.zeros(pool, dtype=torch.int32, device=dev),
                   pool_parent=torch.zeros(pool, dtype=torch.int32, device=dev),
                   pool_score=torch.zeros(pool, dtype=torch.float32, device=dev),
                   frontier=torch.zeros(max(depth - 1, 1), topk, dtype=torch.int32, device=dev),
                   chosen=torch.zeros(n_nodes - 1, dtype=torch.int32, device=dev))
        dbg = DraftDebug(*[_ptr(out[n]) for n in ("pool_tok", "pool_parent", "pool_score", "frontier", "chosen")])
    _check(lib().eagle3_draft_expand(ctx._h, _ptr(g_new, torch.float32), _ptr(tok_new, torch.int32), n_new,
                                     C.byref(draft_kv.c), depth, topk, n_nodes, _ptr(out["tree_tok"]),
                                     _ptr(out["parent"]), _ptr(out["depth"]), _ptr(out["score"]),
                                     C.byref(dbg) if dbg else None, _stream()))
    return out


def eagle3_tree_verify(ctx, tree_tok, parent, kv, want_hidden=False, logits=None, taps=None):
    B, N = tree_tok.shape
    dev = tree_tok.device
    k, V, L = ctx.cfg.hidden, ctx.cfg.vocab, ctx.cfg.n_layers
    if logits is None:
        logits = torch.empty(B, N, V, dtype=torch.float32, device=dev)
    if taps is None:
        taps = torch.empty(3, B, N, k, dtype=torch.float32, device=dev)
    hidden = torch.empty(L + 1, B, N, k, dtype=torch.float32, device=dev) if want_hidden else None
    _check(lib().eagle3_tree_verify(ctx._h, B, N, _ptr(tree_tok, torch.int32), _ptr(parent, torch.int32),
                                    C.byref(kv.c), _ptr(logits), _ptr(taps), _ptr(hidden), _stream()))
    return (logits, taps, hidden) if want_hidden else (logits, taps)


def eagle3_tree_verify_layers(ctx, tree_tok, parent, kv, x_in, layer_begin, layer_end, want_logits=False):
    """Layers [layer_begin, layer_end) from the residual stream x_in [B,N,k] (None = embeddings).
    Returns (x_out, logits or None)."""
    B, N = tree_tok.shape
    dev = tree_tok.device
    x_out = torch.empty(B, N, ctx.cfg.hidden, dtype=torch.float32, device=dev)
    logits = torch.empty(B, N, ctx.cfg.vocab, dtype=torch.float32, device=dev) if want_logits else None
    _check(lib().eagle3_tree_verify_layers(ctx._h, B, N, _ptr(tree_tok, torch.int32), _ptr(parent, torch.int32),
                                           C.byref(kv.c), _ptr(x_in, torch.float32) if x_in is not None else None,
                                           int(layer_begin), int(layer_end), _ptr(x_out), _ptr(logits), _stream()))
    return x_out, logits


def eagle3_accept(ctx, logits, tree_tok, parent, temperature=0.0, uniforms=None):
    B, N = tree_tok.shape
    dev = tree_tok.device
    accept_len = torch.empty(B, dtype=torch.int32, device=dev)
    path = torch.empty(B, N, dtype=torch.int32, device=dev)
    bonus = torch.empty(B, dtype=torch.int32, device=dev)
    _check(lib().eagle3_accept(ctx._h, B, N, _ptr(logits, torch.float32), _ptr(tree_tok, torch.int32),
                               _ptr(parent, torch.int32), float(temperature),
                               _ptr(uniforms, torch.float32) if uniforms is not None else None, _ptr(accept_len),
                               _ptr(path), _ptr(bonus), _stream()))
    return accept_len, path, bonus


def eagle3_accept_static(logits, tree_tok, parent, temperature=0.0, uniforms=None, out=None):
    """eagle3_accept without a context or workspace (fixed scratch inside the library).  `out` = preallocated
    (accept_len, path, bonus) to make the call allocation-free on the torch side as well."""
    B, N = tree_tok.shape
    dev = tree_tok.device
    if out is None:
        out = (torch.empty(B, dtype=torch.int32, device=dev), torch.empty(B, N, dtype=torch.int32, device=dev),
               torch.empty(B, dtype=torch.int32, device=dev))
    accept_len, path, bonus = out
    _check(lib().eagle3_accept_static(B, N, logits.shape[-1], _ptr(logits, torch.float32), _ptr(tree_tok, torch.int32),
                                      _ptr(parent, torch.int32), float(temperature),
                                      _ptr(uniforms, torch.float32) if uniforms is not None else None, _ptr(accept_len),
                                      _ptr(path), _ptr(bonus), _stream()))
    return accept_len, path, bonus


def eagle3_commit(ctx, tree_tok, path, accept_len, bonus, kv, taps, rows, draft_kv=None, draft_rows=0):
    """Commits the accepted paths: cache rows compacted in place, kv.prefix_len advanced (and draft_kv.prefix_len by
    draft_rows).  Returns (taps_new [3,B,rows,k], tok_new [B,rows], n_new [B])."""
    B, N = tree_tok.shape
    dev = tree_tok.device
    taps_new = torch.zeros(3, B, rows, ctx.cfg.hidden, dtype=torch.float32, device=dev)
    tok_new = torch.zeros(B, rows, dtype=torch.int32, device=dev)
    n_new = torch.zeros(B, dtype=torch.int32, device=dev)
    _check(lib().eagle3_commit(ctx._h, B, N, _ptr(tree_tok, torch.int32), _ptr(path, torch.int32),
                               _ptr(accept_len, torch.int32), _ptr(bonus, torch.int32), C.byref(kv.c),
                               _ptr(kv.prefix_len, torch.int32), _ptr(taps, torch.float32), int(rows), _ptr(taps_new),
                               _ptr(tok_new), _ptr(n_new),
                               _ptr(draft_kv.prefix_len, torch.int32) if draft_kv is not None else None, int(draft_rows),
                               _stream()))
    return taps_new, tok_new, n_new


def eagle3_prefill(ctx, tokens, kv, draft_kv):
    """Runs the prompt through the target (cache, features) and builds the draft cache; advances both prefix_len
    arrays on the device and the host bounds.  Returns (g_last [hidden], logits_last [vocab])."""
    T = tokens.shape[0]
    g_last = torch.empty(ctx.cfg.hidden, dtype=torch.float32, device=tokens.device)
    logits = torch.empty(ctx.cfg.vocab, dtype=torch.float32, device=tokens.device)
    _check(lib().eagle3_prefill(ctx._h, _ptr(tokens, torch.int32), T, C.byref(kv.c), C.byref(draft_kv.c), _ptr(g_last),
                                _ptr(logits), _stream()))
    kv.set_max_prefix_len(kv.max_prefix_len + T)
    draft_kv.set_max_prefix_len(draft_kv.max_prefix_len + T - 1)
    return g_last, logits


def eagle3_draft_chain(ctx, g_new, tok_new, n_new, draft_kv, length):
    """Batched chain drafting.  g_new [B, rows1, k], tok_new [B, rows1], n_new [B].  Returns (chain_tok [B, length+1],
    chain_logp [B, length+1])."""
    B, rows1 = tok_new.shape
    dev = tok_new.device
    chain_tok = torch.empty(B, length + 1, dtype=torch.int32, device=dev)
    chain_logp = torch.empty(B, length + 1, dtype=torch.float32, device=dev)
    _check(lib().eagle3_draft_chain(ctx._h, B, _ptr(g_new, torch.float32), _ptr(tok_new, torch.int32),
                                    _ptr(n_new, torch.int32), rows1, C.byref(draft_kv.c), int(length), _ptr(chain_tok),
                                    _ptr(chain_logp), _stream()))
    return chain_tok, chain_logp


def eagle3_ttt_attention(q, k_steps, v_steps):
    """Training-time-test attention forward.  q [T,H,d], k_steps / v_steps [s+1,T,Hkv,d] (bf16 or fp32) -> fp32 [T,H,d]."""
    T, H, d = q.shape
    s, Hkv = k_steps.shape[0] - 1, k_steps.shape[2]
    dt = EAGLE3_BF16 if q.dtype == torch.bfloat16 else EAGLE3_FP32
    out = torch.empty(T, H, d, dtype=torch.float32, device=q.device)
    _check(lib().eagle3_ttt_attention(dt, T, H, Hkv, d, s, _ptr(q), _ptr(k_steps, q.dtype), _ptr(v_steps, q.dtype), _ptr(out),
                                      _stream()))
    return out


# ---- rotary positions and a cache in pages: calls without a context
# These are called once and more a layer and decoding step, with little for the GPU to do in each: what follows looks at every argument, but puts
# messages together only for those that are refused (a call of eagle3_rope 25 -> 9 us, of which 3.5 are the launch).
def _refuse(what, wanted, t):
    raise ValueError(f"{what}: {wanted} is wanted, got " + (f"{t.dtype} {tuple(t.shape)}, strides {t.stride()}, on {t.device}" if isinstance(t, torch.Tensor) else repr(t)))


def _arg(t, dtype, shape, gpu, what):
    """The address of a dense tensor of this type and shape on GPU number `gpu`."""
    if t.dtype is not dtype or t.get_device() != gpu or t.shape != shape or not t.is_contiguous():
        _refuse(what, f"a dense {dtype} tensor {tuple(shape)} on cuda:{gpu}", t)
    return t.data_ptr()


def _rows_of(t, dtype, gpu, what):
    """(address, rows, heads, d, row stride) of [rows, heads, d] rows, each with its heads one behind the other, any distance apart."""
    if t.dtype is dtype and t.get_device() == gpu and t.dim() == 3:
        n, h, d = t.shape
        s0, s1, s2 = t.stride()
        if s2 == 1 and (s1 == d or h == 1) and (s0 >= h * d or n <= 1):
            return t.data_ptr(), n, h, d, s0 if n > 1 else h * d
    _refuse(what, f"{dtype} rows [rows, heads, d], each with its heads one behind the other, on cuda:{gpu}", t)


def _gpu_of(t, what):
    gpu = t.get_device()
    if gpu < 0:
        _refuse(what, "a tensor on a GPU", t)
    return gpu


# what torch.cuda's functions ask, 2 us sooner (a torch without GPUs has neither, and no tensors that get this far)
_raw_stream, _current_gpu = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))


def _on(gpu, call, *args):
    """The call on that GPU's own current stream, whichever GPU is current."""
    stream = _raw_stream(gpu)
    if gpu == _current_gpu():
        code = call(*args, stream)
    else:
        with torch.cuda.device(gpu):
            code = call(*args, stream)
    if code:
        raise Eagle3Error(code)


class Rope:
    """Rotary angles of a model: the table that eagle3_rope reads, and how pairs are formed.  scaling: "none", "linear" or "parts"
    (include/eagle3.h: eagle3_rope_turns)."""

    def __init__(self, rot_dim, theta, *, interleaved=False, scaling="none", factor=1.0, low=1.0, high=4.0, original_len=8192, amplitude=1.0,
                 device="cuda:0"):
        if scaling not in ("none", "linear", "parts"):
            _refuse("scaling", "none, linear or parts", scaling)
        if rot_dim < 2 or rot_dim % 2:
            _refuse("rot_dim", "an even number of at least 2", rot_dim)
        turns = torch.empty(rot_dim // 2, dtype=torch.float64)
        _check(lib().eagle3_rope_turns(int(rot_dim), float(theta), ("none", "linear", "parts").index(scaling), float(factor), float(low), float(high),
                                       float(original_len), turns.data_ptr()))
        self.turns = turns.to(device)
        self.gpu = _gpu_of(self.turns, "device")
        self.c = RopeSpec(self.turns.data_ptr(), int(rot_dim), int(bool(interleaved)), float(amplitude))


_ROPE_TYPES = {torch.bfloat16: EAGLE3_BF16, torch.float32: EAGLE3_FP32}


def _place(out, x, rows, heads, d, gpu, what):
    """Where x's rotated rows go, its address and row stride: `out`, or a new dense tensor."""
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
        return out, out.data_ptr(), heads * d
    p, n, h, m, stride = _rows_of(out, x.dtype, gpu, what)
    if n != rows or h != heads or m != d:
        _refuse(what, f"[{rows}, {heads}, {d}]", out)
    return out, p, stride


def _rotate(call, rope, positions, q, k, out):
    gpu, dtype = q.get_device(), q.dtype
    code = _ROPE_TYPES.get(dtype)
    if code is None or gpu < 0 or rope.gpu != gpu:
        _refuse("q", "a bf16 or fp32 tensor on the GPU of the table of angles", q)
    qp, rows, H, d, q_stride = _rows_of(q, dtype, gpu, "q")
    pos = _arg(positions, torch.int32, (rows,), gpu, "positions")
    q_out, k_out = out if isinstance(out, (tuple, list)) else (out, None)
    if k is None:
        if k_out is not None:
            _refuse("out of k", "None without k", k_out)
        q_out, qo, qo_stride = _place(q_out, q, rows, H, d, gpu, "out of q")
        _on(gpu, call, code, rows, d, rope.c, pos, H, qp, q_stride, qo, qo_stride, 0, None, 0, None, 0)
        return q_out
    kp, k_rows, Hkv, k_d, k_stride = _rows_of(k, dtype, gpu, "k")
    if k_rows != rows or k_d != d:
        _refuse("k", f"[{rows}, heads, {d}]", k)
    q_out, qo, qo_stride = _place(q_out, q, rows, H, d, gpu, "out of q")
    k_out, ko, ko_stride = _place(k_out, k, rows, Hkv, d, gpu, "out of k")
    _on(gpu, call, code, rows, d, rope.c, pos, H, qp, q_stride, qo, qo_stride, Hkv, kp, k_stride, ko, ko_stride)
    return q_out, k_out


class _Turned(torch.autograd.Function):
    """A rotation for which gradients are wanted: its backward pass is the way back, whose own is the rotation."""

    @staticmethod
    def forward(ctx, call, back, rope, positions, q, k):
        ctx.save_for_backward(positions)
        ctx.turn = back, call, rope
        return _rotate(call, rope, positions, q, k, None)

    @staticmethod
    def backward(ctx, dq, dk=None):
        grads = _turn(*ctx.turn, ctx.saved_tensors[0], dq.contiguous(), None if dk is None else dk.contiguous(), None)
        return None, None, None, None, *((grads, None) if dk is None else grads)


def _turn(call, back, rope, positions, q, k, out):
    wanted = q.requires_grad or (k is not None and k.requires_grad)
    if out is not None:
        wanted = wanted or any(t is not None and t.requires_grad for t in (out if isinstance(out, (tuple, list)) else (out,)))
    if not wanted or not torch.is_grad_enabled():
        return _rotate(call, rope, positions, q, k, out)
    if out is not None:
        _refuse("out", "None where gradients are recorded", out)
    return _Turned.apply(call, back, rope, positions, q, k)


def eagle3_rope(rope, positions, q, k=None, out=None):
    """q [rows, H, d] and k [rows, Hkv, d] (bf16 or fp32, rows any distance apart) turned to their positions (int32 [rows]).  `out`: where
    to, e.g. (q, k) themselves; returns the rotated q, or (q, k).  Recorded for autograd where q or k requires a gradient, which `out` does not allow."""
    L = lib()
    return _turn(L.eagle3_rope, L.eagle3_rope_grad, rope, positions, q, k, out)


def eagle3_rope_grad(rope, positions, dq, dk=None, out=None):
    """The gradients of eagle3_rope's q and k from those of its results."""
    L = lib()
    return _turn(L.eagle3_rope_grad, L.eagle3_rope, rope, positions, dq, dk, out)


_POOL_TYPES = {torch.bfloat16: EAGLE3_BF16, torch.float32: EAGLE3_FP32, torch.float8_e4m3fn: EAGLE3_FP8}


class PagedKVCache:
    """One layer's paged cache: k, v [n_pages, page_size, Hkv, d] (bf16, fp32 or float8_e4m3fn), page_table int32 [B, max_pages]; for
    float8_e4m3fn also the scale exponents k_exp, v_exp uint8 [n_pages, page_size, Hkv]."""

    def __init__(self, k, v, page_table, k_exp=None, v_exp=None):
        gpu = _gpu_of(k, "k")
        if k.dtype not in _POOL_TYPES or k.dim() != 4:
            _refuse("k", "a pool [n_pages, page_size, Hkv, d] of bf16, fp32 or float8_e4m3fn", k)
        fp8 = k.dtype == torch.float8_e4m3fn
        if (k_exp is not None) != fp8 or (v_exp is not None) != fp8:
            _refuse("k_exp, v_exp", "scale exponents for an 8-bit pool, None for any other", k_exp)
        if page_table.dim() != 2:
            _refuse("page_table", "int32 [B, max_pages]", page_table)
        self.k, self.v, self.k_exp, self.v_exp, self.page_table = k, v, k_exp, v_exp, page_table
        self.row_dtype, self.gpu = torch.bfloat16 if fp8 else k.dtype, gpu
        n_pages, page_size, self.heads, self.d = k.shape
        self.B, max_pages = page_table.shape
        self.sizes = (k.dtype, self.heads, self.d, max_pages * page_size)
        exps = [_arg(x, torch.uint8, k.shape[:3], gpu, "scale exponents") if fp8 else None for x in (k_exp, v_exp)]
        self.c = PagedKV(_arg(k, k.dtype, k.shape, gpu, "k"), _arg(v, k.dtype, k.shape, gpu, "v"), *exps,
                         _arg(page_table, torch.int32, page_table.shape, gpu, "page_table"), _POOL_TYPES[k.dtype], n_pages, page_size, max_pages,
                         self.heads, self.d)


def _paged_rows(call, cache, k, v, start, n, rows, row_start):
    gpu, B, i32 = cache.gpu, cache.B, torch.int32
    kp, n_rows, heads, d, stride = _rows_of(k, cache.row_dtype, gpu, "k rows")
    if heads != cache.heads or d != cache.d:
        _refuse("k rows", f"[rows, {cache.heads}, {cache.d}]", k)
    if v.dtype is not k.dtype or v.get_device() != gpu or v.shape != k.shape or (v.stride() != k.stride() and _rows_of(v, k.dtype, gpu, "v rows")[4] != stride):
        _refuse("v rows", f"what the k rows are ({k.dtype} {tuple(k.shape)}, strides {k.stride()}, on {k.device})", v)
    vp = v.data_ptr()
    if rows is None:
        rows = n_rows // B
        if row_start is not None:
            _refuse("rows", "with row_start the most rows of a sequence", rows)
    if row_start is None and n_rows != B * rows:
        _refuse("k rows", f"{rows} rows for each of {B} sequences", k)
    _on(gpu, call, cache.c, B, rows, None if start is None else _arg(start, i32, (B,), gpu, "start"), None if n is None else _arg(n, i32, (B,), gpu, "n"),
        None if row_start is None else _arg(row_start, i32, (B,), gpu, "row_start"), kp, vp, n_rows, stride)


def eagle3_paged_append(cache, k_new, v_new, start, n_new=None, rows=None, row_start=None):
    """Writes k_new, v_new [n_rows, Hkv, d] behind the sequences' first start[b] tokens: n_new[b] rows each (None: `rows`, by default
    n_rows / B), sequence b's from row row_start[b] (None: b * rows) on.  Nothing is recorded for autograd, here and in the calls below."""
    _paged_rows(lib().eagle3_paged_append, cache, k_new, v_new, start, n_new, rows, row_start)


def eagle3_paged_read(cache, start=None, n=None, rows=None, row_start=None, out=None):
    """Tokens start[b] .. start[b] + n[b] - 1 (None: from 0; `rows` of them) as dense rows.  `out`: (k, v) [n_rows, Hkv, d], of which only the
    rows read are written; by default zeros with `rows` rows of every sequence.  Returns (k, v)."""
    if out is None:
        if rows is None or row_start is not None:
            _refuse("rows", "without out, rows and no row_start", rows)
        out = tuple(torch.zeros(cache.B * rows, cache.heads, cache.d, dtype=cache.row_dtype, device=cache.k.device) for _ in range(2))
    _paged_rows(lib().eagle3_paged_read, cache, out[0], out[1], start, n, rows, row_start)
    return tuple(out)


_workspaces = {}                                              # bytes by sizes: the layers of a step ask for the same


def _attention_workspace(cache, B, H, max_kv_len):
    key = (cache.sizes, B, H, max_kv_len)
    need = _workspaces.get(key)
    if need is None:
        n = C.c_size_t()
        _check(lib().eagle3_paged_attention_workspace(cache.c, B, H, max_kv_len, n))
        if len(_workspaces) >= 256:
            _workspaces.clear()
        need = _workspaces[key] = n.value
    return need


def eagle3_paged_attention(cache, q, kv_len, max_kv_len, scale=None, out=None, want_lse=False):
    """q [B, H, d] over each sequence's first kv_len[b] <= max_kv_len tokens; scale: 1 / sqrt(d) by default.  Returns out [B, H, d], with
    want_lse also the log of the softmax's sum, fp32 [B, H]."""
    gpu, B, dtype, L = cache.gpu, cache.B, cache.row_dtype, lib()
    qp, n, H, d, stride = _rows_of(q, dtype, gpu, "q")
    if n != B or d != cache.d:
        _refuse("q", f"[{B}, heads, {cache.d}]", q)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        to = out.data_ptr()
    else:
        to = _arg(out, dtype, (B, H, d), gpu, "out")
    lse = q.new_empty((B, H), dtype=torch.float32) if want_lse else None
    need = _attention_workspace(cache, B, H, max_kv_len)
    ws = q.new_empty(need, dtype=torch.uint8) if need else None
    _on(gpu, L.eagle3_paged_attention, cache.c, B, H, qp, stride, _arg(kv_len, torch.int32, (B,), gpu, "kv_len"), max_kv_len,
        d ** -0.5 if scale is None else scale, to, None if lse is None else lse.data_ptr(),
        None if ws is None else ws.data_ptr(), need)
    return (out, lse) if want_lse else out
