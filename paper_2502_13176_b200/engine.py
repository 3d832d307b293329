"""Convenience layer over the binding: owns the device buffers of one budgeted cache and drives
allocate -> prompt (attention, scores, bulk evict) -> decode steps.  Memory management and call
sequencing only; every computation happens inside libbaklava.so."""
import numpy as np
import torch

from . import binding as bk
from . import workloads as wl


def shape_of(w):
    return bk.make_shape(w.L, w.Hq, w.Hkv, w.D, w.page, w.n_sink, w.recent_num, w.recent_den)


def norm_rope(shape, q, k, positions, inv_freq, q_weight=None, k_weight=None, eps=1e-6, flags=0):
    """Queries [B, Hq, T, D] and keys [B, Hkv, T, D] (any views with contiguous rows, e.g. of the projection's output)
    as attention takes them: normed per head where a weight is given, rotated to their positions (int32 [B, T]); new
    contiguous tensors.  For a decode step T = 1: `.squeeze(2)` is the [B, H, D] of `DecodeSession.step`."""
    qo = torch.zeros(q.shape, dtype=q.dtype, device=q.device)
    ko = torch.zeros(k.shape, dtype=k.dtype, device=k.device)
    bk.baklava_qk_norm_rope(shape, q, k, positions, inv_freq, q_weight, k_weight, eps, qo, ko, flags)
    return qo, ko


def verify(target, draft, tokens, parent, u_accept, u_sample, n_nodes=None, distinct=False):
    """Which drafted tokens stand (speculative sampling over a tree, from given uniform numbers).  target, draft: float32 or
    bf16 [B, T, V] probabilities (draft None: the children were chosen, not drawn); tokens, parent: int32 [B, T]; u_accept:
    float32 [B, T], u_sample: float32 [B]; `distinct`: siblings were drawn without replacement.  Returns device tensors (path
    [B, T], n_path [B], next_token [B], status [1]), as `DecodeSession.commit` takes the first two."""
    B, T, _ = target.shape
    path, rest = torch.empty((B, T), dtype=torch.int32, device=target.device), torch.zeros((2 * B + 1,), dtype=torch.int32, device=target.device)
    n_path, token, status = rest[:B], rest[B:2 * B], rest[2 * B:]
    bk.baklava_tree_verify(target, draft, tokens, parent, n_nodes, u_accept, u_sample, path, n_path, token, status,
                           bk.VERIFY_DISTINCT if distinct else 0)
    return path, n_path, token, status


class DecodeSession:
    def __init__(self, w, device="cuda", layers=None, chunk_tokens=0, uniform=False, alloc=None, importance=None,
                 total_tokens=None, kv_dtype=bk.KV_BF16):
        """`alloc` = (t, r_num, r_den) overrides the workload's Algorithm 2 parameters, `importance` its
        synthetic importances, `total_tokens` its budget (e.g. the dense length for a reference run)."""
        self.w, self.device = w, torch.device(device)
        self.shape = shape_of(w)
        self.scales = wl.kv_scales(w)
        self.importance = wl.importance(w).numpy() if importance is None else np.asarray(importance, dtype=np.float64)
        t, r_num, r_den = (w.t, w.r_num, w.r_den) if alloc is None else alloc
        total = w.total_pages * w.page if total_tokens is None else int(total_tokens)
        self.cap, self.off, self.stride = bk.baklava_allocate(
            self.shape, self.importance, t, 0 if uniform else r_num, r_den, total,
            w.min_pages * w.page, w.max_pages * w.page)
        self.kv_dtype = kv_dtype
        kv_scale = {bk.KV_FP8_E4M3: wl.kv_fp8_scales, bk.KV_INT4: wl.kv_int4_scales}.get(kv_dtype)
        self.cache = bk.Cache(self.shape, self.cap, self.off, self.stride, w.B, self.device, kv_dtype=kv_dtype,
                              kv_scale=kv_scale and kv_scale(w, self.scales))
        self.lb, self.le = (0, w.L) if layers is None else layers
        n_sm = torch.cuda.get_device_properties(self.device).multi_processor_count
        self.plan = bk.baklava_decode_plan(self.shape, self.cap, w.B, self.lb, self.le, self.stride,
                                           chunk_tokens=chunk_tokens, n_sm=n_sm, kv_dtype=kv_dtype).to(self.device)
        self.ws = bk.decode_workspace(self.plan, self.device)
        nl = self.le - self.lb
        self.out = torch.zeros((nl, w.B, w.Hq, w.D), dtype=torch.bfloat16, device=self.device)
        self.lse = torch.zeros((nl, w.B, w.Hq), dtype=torch.float32, device=self.device)
        self.t = 0                                   # position of the next `step`; None after a `commit`: the device has it, per sequence
        self.prompt_error = None

    def prefill_synthetic(self, prompt_len=None, data=None):
        """Fill every head from the workload's dense synthetic prompt through baklava_evict, a layer at a time.
        `prompt_len` (B ints) keeps only that many tokens of each sequence's prompt; `data` is a copy of the
        workload with another seed (another prompt through the same heads)."""
        w = self.w if data is None else data
        ews = torch.empty((bk.baklava_evict_workspace_size(self.shape, w.B, 1, w.T),), dtype=torch.uint8,
                          device=self.device)
        plen = None if prompt_len is None else torch.tensor(list(prompt_len), dtype=torch.int32, device=self.device)
        for l in range(self.lb, self.le):
            k, v = wl.dense_kv_layer(w, l, self.scales, self.device)
            sc = wl.prefill_scores(w, l, self.device)
            bk.baklava_evict_varlen(self.shape, self.cache, l, l + 1, k, v, sc, w.T, plen, 0, w.Hkv * w.T, w.T, 1, ews)
            torch.cuda.synchronize(self.device)
        self.t = w.T
        self.t_seq = plen

    def prefill_layer(self, l, q, k, v, prompt_len=None):
        """One layer of a real prompt: causal attention (its output [B, Hq, T, D] is returned), the attention every token
        received as its score (from the same rows' log-sum-exp), and the bulk eviction into the layer's slabs.
        q: bf16 [B, Hq, T, D], k, v: bf16 [B, Hkv, T, D], contiguous; prompt_len: device int32 [B] or None."""
        w = self.w
        B, T = w.B, q.shape[2]
        if not 0 <= l < w.L:
            raise ValueError("layer %d of %d" % (l, w.L))
        for what, x, heads in (("q", q, w.Hq), ("k", k, w.Hkv), ("v", v, w.Hkv)):
            # (attention takes any strides; the scores and the eviction read the same tensors densely)
            if x.shape != (B, heads, T, w.D) or not x.is_contiguous():
                raise ValueError("%s: expected a contiguous [%d, %d, %d, %d], got %s with strides %s"
                                 % (what, B, heads, T, w.D, tuple(x.shape), x.stride()))
        out = torch.zeros(q.shape, dtype=q.dtype, device=self.device)
        lse = torch.empty((B, w.Hq, T), dtype=torch.float32, device=self.device)
        bk.baklava_prefill_attn(self.shape, q, k, v, prompt_len, out, lse, self.cache.status)
        score = torch.empty((B, w.Hkv, T), dtype=torch.float32, device=self.device)
        ws = torch.empty((max(bk.baklava_prefill_workspace_size(self.shape, B, T),
                              bk.baklava_evict_workspace_size(self.shape, B, 1, T)),), dtype=torch.uint8, device=self.device)
        bk.baklava_prefill_scores(self.shape, q, k, prompt_len, B, T, score, ws, lse=lse)
        err = ws[:4].view(torch.int32).clone()                        # (the eviction uses the workspace next)
        self.prompt_error = err if self.prompt_error is None else self.prompt_error | err
        bk.baklava_evict_varlen(self.shape, self.cache, l, l + 1, k, v, score, T, prompt_len, 0, w.Hkv * T, T, 1, ws)
        self.t = T
        self.t_seq = prompt_len
        return out

    def step(self, q, k_new, v_new, flags=0):
        """One decode step for the session's layer range, all sequences at position `t`; returns the output tensor (device, bf16).
        After a `commit` the positions are what that returned: the next step is `step_varlen`'s (or `t` is set anew)."""
        if self.t is None and not flags & bk.FLAG_NO_APPEND:
            raise RuntimeError("a commit has moved the sequences on: step_varlen with the positions that it returned")
        bk.baklava_decode_attn(self.shape, self.cache, q, k_new, v_new, self.t or 0, self.out, self.lse, flags,
                               self.plan, self.ws)
        if not (flags & bk.FLAG_NO_APPEND):
            self.t += 1
        return self.out

    def step_varlen(self, q, k_new, v_new, t_pos, flags=0):
        """One decode step with per-sequence positions `t_pos` (device int32 [B]; negative = idle)."""
        bk.baklava_decode_attn_varlen(self.shape, self.cache, q, k_new, v_new, t_pos, self.out, self.lse, flags,
                                      self.plan, self.ws)
        return self.out

    def per_layer_plans(self, chunk_tokens=0, overlap=True):
        """One plan and workspace per layer, for callers that run attention layer by layer (as a model does).
        With `overlap` (the calls after the first will carry BAKLAVA_FLAG_OVERLAP_PREV) and no chunk length given,
        chunks of 1024 tokens: consecutive layers' kernels then share the GPU, and what counts is the fixed cost
        per chunk, not that one layer's chunks fill one wave."""
        if overlap and chunk_tokens == 0:
            chunk_tokens = 1024
        n_sm = torch.cuda.get_device_properties(self.device).multi_processor_count
        self.layer_plans = []
        for l in range(self.lb, self.le):
            plan = bk.baklava_decode_plan(self.shape, self.cap, self.w.B, l, l + 1, self.stride, chunk_tokens=chunk_tokens,
                                          n_sm=n_sm, kv_dtype=self.kv_dtype).to(self.device)
            self.layer_plans.append((plan, bk.decode_workspace(plan, self.device)))

    def step_layers(self, q, k_new, v_new, t_pos, flags=0, overlap=True):
        """One decode step as one call per layer; t_pos: device int32 [B] (so that the sequence of calls can be
        captured in a CUDA graph and replayed with the positions advanced on the device).  q / k_new / v_new of
        every layer must be complete before the first call is enqueued when `overlap` is set."""
        for i, (plan, ws) in enumerate(self.layer_plans):
            # every layer has its own heads, inputs and workspace, and all inputs are complete before the first
            # call: from the second layer on a call may start beside the previous layer's tail
            fl = flags | (bk.FLAG_OVERLAP_PREV if overlap and i > 0 else 0)
            bk.baklava_decode_attn_varlen(self.shape, self.cache, q[i:i + 1], k_new[i:i + 1], v_new[i:i + 1], t_pos,
                                          self.out[i:i + 1], self.lse[i:i + 1], fl, plan, ws)
        return self.out

    def drafts(self, T, max_path=None):
        """Room for steps with trees of up to T drafted tokens, accepted paths of up to `max_path` (T): the nodes' queries, keys
        and values of every layer (`tree_q` [layers, B, Hq, T, D], `tree_k`, `tree_v` [layers, B, Hkv, T, D]: the model writes
        them, e.g. through baklava_qk_norm_rope), outputs, log-sum-exps, one plan per layer, workspaces."""
        w, nl = self.w, self.le - self.lb
        n_sm = torch.cuda.get_device_properties(self.device).multi_processor_count
        bf = dict(dtype=torch.bfloat16, device=self.device)
        self.tree_T, self.max_path = T, T if max_path is None else max_path
        self.tree_q, self.tree_out = (torch.zeros((nl, w.B, w.Hq, T, w.D), **bf) for _ in range(2))
        self.tree_k, self.tree_v = (torch.zeros((nl, w.B, w.Hkv, T, w.D), **bf) for _ in range(2))
        self.tree_lse = torch.zeros((nl, w.B, w.Hq, T), dtype=torch.float32, device=self.device)
        self.tree_plans = [bk.baklava_tree_plan(self.shape, self.cap, w.B, l, T, n_sm=n_sm, kv_dtype=self.kv_dtype).to(self.device)
                           for l in range(self.lb, self.le)]
        # (the layers follow one another on the stream and share a workspace)
        self.tree_ws = torch.empty((max(int(p.info.ws_bytes) for p in self.tree_plans),), dtype=torch.uint8, device=self.device)
        self.commit_ws = bk.tree_commit_workspace(self.shape, self.plan, self.max_path, self.device)

    def tree_layer(self, l, parent, n_nodes=None):
        """Attention of the drafted tree over layer l's slabs and over the nodes' ancestors; returns [B, Hq, T, D].  parent:
        device int32 [B, T]; n_nodes: device int32 [B] or None."""
        if not self.lb <= l < self.le:
            raise ValueError("layer %d of %d .. %d" % (l, self.lb, self.le - 1))
        i = l - self.lb
        bk.baklava_tree_attn(self.shape, self.cache, self.tree_q[i], self.tree_k[i], self.tree_v[i], parent, n_nodes, self.tree_out[i],
                             self.tree_lse[i], self.tree_plans[i], self.tree_ws)
        return self.tree_out[i]

    def commit(self, path, n_path, t_pos, flags=0):
        """The accepted path (as `verify` returned it) into all layers' slabs: scores, append, eviction.  t_pos: device int32 [B],
        the position of each path's first token; returns the next step's (of `tree_layer` and `commit`, or of `step_varlen`).  4-bit
        rows have the bits that a decode step gives them."""
        t_next = torch.empty_like(t_pos)
        bk.baklava_tree_commit(self.shape, self.cache, self.tree_q, self.tree_k, self.tree_v, self.tree_lse, path, n_path, self.max_path,
                               t_pos, t_next, flags | bk.FLAG_ROW_QUOTIENT, self.plan, self.commit_ws)
        self.t = None
        return t_next

    def retained_kv_bytes(self):
        """Bytes of K and V in valid rows of the session's layers: what one step must read."""
        n = int(self.cache.len[:, self.lb:self.le].sum().item())
        return n * bk.kv_row_bytes(self.w.D, self.kv_dtype)

    def check_status(self):
        code = int(self.cache.status.item())
        if code:
            raise RuntimeError("device status word = %d" % code)
        if self.prompt_error is not None and int(self.prompt_error.item()):
            raise RuntimeError("the prompt scores gave up a wait")
