"""Outer LSP loop (Algorithm 1 lines 3-11) on the HIP library.

Host side of the scheduler: per iteration it obtains the step's logits from
the caller (the stand-in for the denoiser), runs lsp_confidence, the flip
bookkeeping and lsp_commit, optionally lsp_attn_step per layer, and stops when
no sequence has an active position left.  The only device-to-host traffic is
the termination test, polled every `poll` steps.
"""
from __future__ import annotations

import torch

from . import (BY_PLACE, AttnLayerTable, LayerTable, LspError, ProgressPoll, _commit_out, _need, attn_key_weights_layers, attn_key_weights_workspace_bytes,
               attn_step_layers, commit_step, confidence, confidence_workspace_bytes, kv_evict, kv_evict_workspace_bytes, kv_gather_append,
               lm_head_confidence, lm_head_confidence_workspace_bytes, token_scores, token_scores_workspace_bytes)


def _need_on(device, name, t, *rest, **kw):
    """_need, on this device: what a step finds out later has changed the caller's state by then."""
    _need(name, t, *rest, **kw)
    if t is not None and t.device != device:
        raise LspError(f"decode_loop: {name} is on {t.device}, the sequences are on {device}")


class _Scores:
    """What the committed tokens' positions are told about them: buffers of one entry per token of the caller's, filled as `tokens` is."""

    def __init__(self, buffers, tokens, V):
        B, T = tokens.shape
        unknown = set(buffers) - {"logprob", "entropy", "alt_id", "alt_logprob"}
        if unknown or not buffers:
            raise LspError(f"decode_loop: scores are logprob, entropy, alt_id and alt_logprob, got {sorted(buffers)}")
        if ("alt_id" in buffers) != ("alt_logprob" in buffers):
            raise LspError("decode_loop: alt_id and alt_logprob come together")
        self.K = buffers["alt_id"].shape[-1] if "alt_id" in buffers else 0
        if "alt_id" in buffers and not 1 <= self.K <= 32:
            raise LspError(f"decode_loop: 1 to 32 alternatives, got {self.K}")
        for k, t in buffers.items():
            _need_on(tokens.device, f"scores['{k}']", t, torch.int32 if k == "alt_id" else torch.float32, (B, T, self.K) if k.startswith("alt") else (B, T))
        self.buffers, self.out, self.workspace = buffers, None, None
        self.place = torch.arange(T, device=tokens.device)

    def look(self, z, top1_id, suffix_len):
        if self.out is None:
            f = dict(dtype=torch.float32, device=z.device)
            B, S = top1_id.shape
            # (zeros: what lies behind the active rows is gathered, though not kept)
            self.out = (torch.zeros((B, S), **f), torch.zeros((B, S), **f), *((torch.zeros((B, S, self.K), dtype=torch.int32, device=z.device),
                        torch.zeros((B, S, self.K), **f)) if self.K else (None, None)))
            self.workspace = torch.empty(max(16, token_scores_workspace_bytes(*z.shape, self.K)), dtype=torch.uint8, device=z.device)
        token_scores(z, top1_id, suffix_len, num_alt=self.K, out=self.out, workspace=self.workspace)

    def keep(self, prefix_len, commit_len):
        """Of the tokens just committed, which are the last commit_len[b] before prefix_len[b]."""
        row = self.place - (prefix_len - commit_len).unsqueeze(1)
        new = (row >= 0) & (row < commit_len.unsqueeze(1))
        row = row.clamp(0, self.out[0].shape[1] - 1)
        for k, src in zip(("logprob", "entropy", "alt_id", "alt_logprob"), self.out):
            to = self.buffers.get(k)
            if to is not None and to.dim() == 2:
                to.copy_(torch.where(new, torch.gather(src, 1, row), to))
            elif to is not None:
                to.copy_(torch.where(new.unsqueeze(2), torch.gather(src, 1, row.unsqueeze(2).expand(to.shape)), to))


class _Budget:
    """Caches that are cut back by accumulated attention weight.  Their rows are no longer the sequence's positions: cache_len counts them."""

    def __init__(self, keep, high=None, first=0, recent=0, decay=1.0, cache_len=None, weights=None, positions=None):
        self.kw = dict(keep=int(keep), high=int(keep if high is None else high), first=int(first), recent=int(recent))
        self.decay, self.cache_len, self.weights, self.positions, self.ready = float(decay), cache_len, weights, positions, False

    def start(self, table, prefix_len, suffix_len):
        if self.cache_len is None:
            self.cache_len = prefix_len.clone()
        k = self.kw
        if not (0 < k["keep"] <= min(k["high"], table.C) and min(k["first"], k["recent"]) >= 0 and k["first"] + k["recent"] <= k["keep"] and 0 <= self.decay <= 1):
            raise LspError(f"decode_loop: cache_budget needs 0 < keep <= high, first + recent <= keep and 0 <= decay <= 1, got {k}, decay {self.decay}")
        shape = (table.n, table.B, table.Hkv, table.C)
        if self.weights is None:
            self.weights = torch.zeros(shape, device=prefix_len.device)
        dev = prefix_len.device
        _need_on(dev, "cache_len", self.cache_len, torch.int32, (table.B,))
        if self.cache_len.data_ptr() in (prefix_len.data_ptr(), suffix_len.data_ptr()):
            raise LspError("decode_loop: cache_len is a buffer of its own")
        _need_on(dev, "weights", self.weights, torch.float32, shape)
        if self.positions is None and k["recent"] > 0:
            self.positions = torch.full(shape, BY_PLACE, dtype=torch.int32, device=dev)
        _need_on(dev, "positions", self.positions, torch.int32, shape, optional=True)
        left, rows = torch.stack([suffix_len.max(), (suffix_len + self.cache_len).max()]).tolist()
        if max(rows, left + self.kw["high"]) > table.C:
            raise LspError(f"decode_loop: a cache of {table.C} rows has no room for {left} more positions on {self.kw['high']} rows (high), or on those there are")

    def weigh(self, attn, suffix_len):
        d = attn.desc
        if not self.ready:
            self.workspace = torch.empty(max(16, attn_key_weights_workspace_bytes(d.dtype, d.B, d.S, d.Hq, d.Hkv, d.D, d.C, attn.n)), dtype=torch.uint8,
                                         device=suffix_len.device)
        attn_key_weights_layers(attn, self.cache_len, suffix_len, self.weights, decay=self.decay, workspace=self.workspace)

    def append(self, table, commit_len, prefix_len):
        if not self.ready:
            dev = commit_len.device
            self.rows = torch.arange(table.S, dtype=torch.int32, device=dev).expand(table.B, table.S).contiguous()
            self.appended = torch.empty(table.B, dtype=torch.int32, device=dev)
            self.evict_workspace = torch.empty(max(16, kv_evict_workspace_bytes(table, **self.kw)), dtype=torch.uint8, device=dev)
            self.ready = True
        kv_gather_append(self.rows, commit_len, self.cache_len, table, appended=self.appended)
        kv_evict(self.weights, self.cache_len, table, workspace=self.evict_workspace, positions=self.positions,
                 token_len=None if self.positions is None else prefix_len, **self.kw)


def decode_loop(logits_fn, bitmap, V, tau, window, min_commit, snap_enabled,
                prefix_len, suffix_len, tokens, kv_layers=None, gen_len=None, run_attention=False,
                poll=1, max_steps=100000, stop_after=None, observer=None, timed=False, commit_kw=None,
                graph=False, lm_head_weight=None, flip_window=None, flip_trace=False, state=None, scores=None, cache_budget=None):
    """logits_fn(step, prefix_len) -> device logits [B,S,V].  prefix_len,
    suffix_len, tokens and the caches in kv_layers (list of dicts q?, k_suf,
    v_suf, k_cache, v_cache) are updated in place.
    run_attention: also run the attention of every layer, behind the step's logits_fn, over what is
    then in the buffers of kv_layers; the outputs stay inside.
    commit_kw: extra keyword arguments of commit() (adaptive, alpha, beta, max_commit).
    stop_after: leave the loop after that many steps even if positions remain.
    observer(step, logits, conf, commit_out): called after every step's commit
    (the tensors are reused by the next step: copy what is to be kept).
    timed: bracket every step's library calls with HIP events on the current
    stream and return their sum as lsp_ms (the logits callback is outside).
    lm_head_weight [V,K] (bf16): logits_fn then returns the step's HIDDEN states
    [B,S,K] and lsp_lm_head_confidence takes the place of lsp_confidence (the
    logits are never stored).
    graph: launch every step after the first from ONE captured HIP graph (all
    sequence state lives in device memory and no entry point reads it on the
    host, so the same graph serves every step); the first step runs eagerly.
    The step's logits must then sit at one address: a tensor that logits_fn
    returns elsewhere is copied there (outside the timed region).
    flip_window: (lo, hi) committed positions of a sequence, inclusive, inside which its
    flips also count towards the mid-generation window of Section 4.3.4 (default: 25 %-75 %
    of the generation length).  flip_trace: keep every step's per-sequence counts.
    state: the dict an earlier call returned under "state" (one that stop_after ended, or
    whose tensors were saved and loaded back): the call then continues that generation -
    same generation start, last-seen ids and flip counters, step numbers going on from
    where it stopped - so that stopping and resuming walks exactly like one uninterrupted
    call.  The sequence state itself (lengths, tokens, caches) is the caller's as always.
    scores: dict of buffers that take, for every committed token at its place in `tokens`, what the logits it was chosen from
    say about it (lsp_token_scores): "logprob", "entropy" (fp32 [B,T]), "alt_id", "alt_logprob" (int32 and fp32 [B,T,K], K up
    to 32); any of them.  Needs the logits, so not together with lm_head_weight.
    cache_budget: dict(keep[, high, first, recent, decay, cache_len, weights, positions]): caches of bounded length (run_attention and
    kv_layers needed).  After every step, sequences with more than `high` (default: keep) cached rows are cut back to the `keep`
    that received most attention, per layer and KV head, beside the first `first` rows and those of the newest `recent` tokens (lsp_attn_key_weights,
    lsp_kv_evict_positions); decay: what is left of a weight at the next step (default 1).  The caches' lengths are then cache_len (int32 [B],
    updated in place; default: a copy of prefix_len), and prefix_len counts tokens alone; weights fp32 [layers,B,Hkv,C] are those that
    the prompt's rows begin with (default 0), positions int32 of that shape the cached rows' tokens, which `recent` goes by (default: BY_PLACE, the
    cached rows are in order and end with the newest token, which is also what is to be behind the cached rows).  A cache has to have room for `high` rows and all that is to be generated.  state
    carries these on (those of cache_budget are not looked at then).
    A sequence that still has active positions but commits nothing (min_commit = 0, or its
    cache / token buffer is full) would never finish: the loop raises LspError instead.
    Returns dict(steps, flips, flip_denominator, window_flips, window_denominator, committed,
    state[, flip_trace: int32 [steps,B,2]][, lsp_ms, lsp_ms_steps][, cache_len]); steps, the flip counts
    and committed are totals since the generation began (earlier calls included)."""
    dev = prefix_len.device
    B = prefix_len.shape[0]
    G = int(gen_len if gen_len is not None else suffix_len.max().item())
    if state is None:
        base = prefix_len.clone()
        last_id = torch.full((B, G), -1, dtype=torch.int32, device=dev)
        counters = torch.zeros(4, dtype=torch.int64, device=dev)
        steps = 0
    else:
        base, last_id, counters, steps = state["base"], state["last_id"], state["counters"], int(state["steps"])
        if (tuple(base.shape) != (B,) or base.dtype != prefix_len.dtype or tuple(last_id.shape) != (B, G)
                or last_id.dtype != torch.int32 or tuple(counters.shape) != (4,) or counters.dtype != torch.int64
                or any(t.device != dev for t in (base, last_id, counters)) or steps < 0):
            raise LspError("decode_loop: state does not belong to this batch (shapes, dtypes or device differ)")
    first = steps
    if flip_window is None:
        flip_window = (-(-G // 4), (3 * G) // 4)
    step_counts = torch.zeros((B, 2), dtype=torch.int32, device=dev) if flip_trace else None
    trace = []
    if min_commit < 1 and stop_after is None:
        raise LspError("decode_loop needs min_commit >= 1 (Section 3.2: at least one token per iteration) "
                       "unless stop_after bounds the number of steps")
    said = budget = None
    if scores is not None:
        if lm_head_weight is not None:
            raise LspError("decode_loop: scores need the logits, which the fused output head does not store")
        said = _Scores(scores, tokens, V)
    if cache_budget is not None:
        if not run_attention or kv_layers is None:
            raise LspError("decode_loop: a cache budget goes by the attention of kv_layers (run_attention)")
        kept = {} if state is None or "cache_len" not in state else {k: state.get(k) for k in ("cache_len", "weights", "positions")}
        budget = _Budget(**{**cache_budget, **kept})
        if kept and budget.positions is None and budget.kw["recent"] > 0:
            raise LspError("decode_loop: this state's caches were cut back without positions (recent = 0): nothing says which of their rows are recent")
    elif kv_layers is not None and state is not None and "cache_len" in state:
        raise LspError("decode_loop: this state's caches were cut back (cache_len): it goes on with a cache_budget")
    # Lengths of another type or place are no error with nothing to do.
    ordinary = all(t.is_cuda and t.dtype == torch.int32 and t.is_contiguous() for t in (prefix_len, suffix_len, base)) and counters.is_contiguous()
    progress = None
    if ordinary:
        progress = ProgressPoll()
        progress.start(suffix_len, None, prefix_len, base, counters)
    table = None
    if kv_layers is not None:       # (built while the first test is under way)
        table = LayerTable(*[[L[k] for L in kv_layers] for k in ("k_suf", "v_suf", "k_cache", "v_cache")])
    if budget is not None:
        budget.start(table, prefix_len, suffix_len)
    cached = prefix_len if budget is None else budget.cache_len
    out = conf = None
    attn_out = None
    events = []
    zbuf = step_graph = None
    totals = None   # positions committed and the counters, where the last test has seen the final ones
    ws = None   # workspace of the reduction or the fused output head: allocated by the first (eager) step, then reused

    def one_step(z):
        nonlocal out, conf, attn_out, ws
        if run_attention and kv_layers is not None:
            if attn_out is None:     # one output per layer (a denoiser consumes each of them), allocated once
                q = kv_layers[0]["q"]
                outs = torch.empty((len(kv_layers), *q.shape), dtype=q.dtype, device=q.device)
                attn_out = AttnLayerTable(*[[L[k] for L in kv_layers] for k in ("q", "k_suf", "v_suf", "k_cache", "v_cache")],
                                          list(outs.unbind(0)))
            attn_step_layers(attn_out, cached, suffix_len)     # every layer in one launch
            if budget is not None:
                budget.weigh(attn_out, suffix_len)
        if lm_head_weight is None:
            if ws is None:
                ws = torch.empty(confidence_workspace_bytes(*z.shape), dtype=torch.uint8, device=dev)
            conf = confidence(z, suffix_len, out=conf, workspace=ws)
        else:
            if ws is None:
                ws = torch.empty(lm_head_confidence_workspace_bytes(z.shape[0], z.shape[1], V), dtype=torch.uint8, device=dev)
            conf = lm_head_confidence(z, lm_head_weight, suffix_len, out=conf, workspace=ws)
        if said is not None:
            said.look(z, conf[0], suffix_len)
        if out is None:
            out = _commit_out(*conf[0].shape, dev)
        commit_step(conf[2], conf[0], bitmap, V, tau, window, min_commit, snap_enabled, prefix_len, suffix_len,
                    base, last_id, counters, flip_window, step_counts, tokens=tokens, layers=table if budget is None else None, C=tokens.shape[1], out=out,
                    **(commit_kw or {}))
        if said is not None:
            said.keep(prefix_len, out["commit_len"])
        if budget is not None:
            budget.append(table, out["commit_len"], prefix_len)

    while True:
        if (steps - first) % poll == 0:
            # positions left, and whether a sequence that has some committed nothing
            if out is None and not ordinary:
                left, stalled = int(suffix_len.max().item()), False
            else:
                if out is not None:
                    progress.start(suffix_len, out["commit_len"], prefix_len, base, counters)
                left, stalled, *totals = progress.wait()
            if left == 0:
                break
            if stalled and min_commit >= 1:
                raise LspError(f"decode_loop: a sequence with active positions committed nothing at step {steps - 1} "
                               f"(status_flags {out['status_flags'].tolist()}): cache or token buffer full")
        if stop_after is not None and steps - first >= stop_after:
            break
        assert steps < max_steps
        z = logits_fn(steps, prefix_len)
        if graph:
            if zbuf is None:
                zbuf = z
            elif z.data_ptr() != zbuf.data_ptr():
                zbuf.copy_(z)
                z = zbuf
        if graph and steps - first >= 1 and step_graph is None:   # one-time set-up, not part of a step
            step_graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(step_graph):
                one_step(zbuf)
        if timed:
            events.append((torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)))
            events[-1][0].record()
        if graph and steps - first >= 1:
            step_graph.replay()
        else:
            one_step(z)
        if timed:
            events[-1][1].record()
        if step_counts is not None:
            trace.append(step_counts.clone())
        if observer is not None:
            observer(steps, z, conf, out)
        steps += 1
        totals = None
    if totals is None:
        *c, committed = torch.cat([counters, (prefix_len - base).sum().view(1)]).tolist()
    else:
        committed, *c = totals
    res = dict(steps=steps, flips=c[0], flip_denominator=c[1], window_flips=c[2], window_denominator=c[3],
               committed=committed, state=dict(base=base, last_id=last_id, counters=counters, steps=steps))
    if budget is not None:
        res["cache_len"] = budget.cache_len
        res["state"].update(cache_len=budget.cache_len, weights=budget.weights)
        if budget.positions is not None:
            res["state"]["positions"] = budget.positions
    if flip_trace:
        res["flip_trace"] = torch.stack(trace).cpu() if trace else torch.zeros((0, B, 2), dtype=torch.int32)
    if timed:
        torch.cuda.synchronize()
        res["lsp_ms_steps"] = [a.elapsed_time(b) for a, b in events]
        res["lsp_ms"] = sum(res["lsp_ms_steps"])
    return res
