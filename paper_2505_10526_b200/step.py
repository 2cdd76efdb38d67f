"""One verify step = massv_verify_attn + massv_accept + massv_kv_commit.

``VerifyStep`` owns the descriptors, the scratch buffers and the output tensors
for a fixed geometry, so that a step is three C-ABI calls and nothing else.  All
arithmetic happens inside ``libmassv.so``.

What a serving loop adds around them is switched on per step object: ``rope``
turns the block's queries and keys first (massv_rotary), ``n_groups`` lets groups of
sequences share a prefix (massv_verify_attn_shared), ``rules`` puts biases, penalties and
grammars on the logits and keeps the history they read (massv_accept_logits,
massv_history_add).
"""
from __future__ import annotations

import torch

from . import binding as mv

# tensors that change every step (the rest - page pools, page table, lengths,
# LM-head weights - is resident state)
STEP_INPUTS = ("q", "k_new", "v_new", "hidden", "draft_tokens", "draft_probs", "u_accept", "u_sample")


class VerifyStep:
    def __init__(self, batch, gamma, n_q_heads, n_kv_heads, head_dim, hidden, vocab, temperature,
                 max_pages_per_seq, num_pages, device="cuda", kv_chunk=0, scale=0.0, window=0,
                 attn_kernel=0, want_logits=False, want_probs=False, want_attn_f32=False,
                 rope=None, n_groups=0, rules=False):
        """``rope``: None, or the keyword arguments of ``rope_desc`` from ``rot_dim`` on together with ``turns``
        (massv_rope_frequencies); the step's inputs may then hold ``pos_delta`` (int32 [B]).
        ``n_groups`` > 0: the inputs hold ``group_start`` and ``shared_lens``; ``attn_kernel`` and ``kv_chunk`` are not used then.
        ``rules``: the inputs hold ``rules`` (``logit_rules``), and ``run`` adds the emitted tokens to the history that they read, or to
        ``output_bits`` and ``counts`` of the inputs where these are given."""
        self.device = torch.device(device)
        self.B, self.gamma, self.R = batch, gamma, gamma + 1
        self.T = float(temperature)
        self.adesc = mv.attn_desc(batch, gamma, n_q_heads, n_kv_heads, head_dim, max_pages_per_seq, num_pages,
                                  scale=scale, kv_chunk=kv_chunk, window=window, kernel=attn_kernel)
        self.cdesc = mv.accept_desc(batch, gamma, hidden, vocab, temperature)
        dev = self.device
        self.n_groups, self.rules, self.vocab = n_groups, bool(rules), vocab
        if n_groups and mv.massv_verify_attn_shared_workspace_size(self.adesc, n_groups) == 0:
            raise ValueError("massv: groups that share a prefix take no window, at most 256 groups and 2,048 sequences, and no more blocks than massv_verify_attn_shared counts "
                             "(include/massv.h)")
        self.attn_ws = mv.alloc_workspace(mv.massv_verify_attn_shared_workspace_size(self.adesc, n_groups) if n_groups
                                          else mv.massv_verify_attn_workspace_size(self.adesc), dev)
        self.accept_ws = mv.alloc_workspace(mv.massv_accept_logits_workspace_size(self.cdesc) if rules
                                            else mv.massv_accept_workspace_size(self.cdesc), dev)
        self.rope = None
        if rope is not None:
            how = dict(rope)
            self.turns = how.pop("turns")
            self.rope = mv.rope_desc(batch, self.R, n_q_heads, n_kv_heads, head_dim, **how)
            self.q_turned = torch.empty((batch, self.R, n_q_heads, head_dim), dtype=torch.bfloat16, device=dev)
            self.k_turned = torch.empty((batch, self.R, n_kv_heads, head_dim), dtype=torch.bfloat16, device=dev)
        self.attn_out = torch.empty((batch, self.R, n_q_heads, head_dim), dtype=torch.bfloat16, device=dev)
        self.attn_out_f32 = torch.empty_like(self.attn_out, dtype=torch.float32) if want_attn_f32 else None
        self.lse = torch.empty((batch, self.R, n_q_heads), dtype=torch.float32, device=dev) if want_attn_f32 else None
        # tokens and accepted lengths share one buffer, so that a host reads both back with one copy
        self._out_blob = torch.empty((batch * self.R + batch,), dtype=torch.int32, device=dev)
        self.out_tokens = self._out_blob[:batch * self.R].view(batch, self.R)
        self.accept_len = self._out_blob[batch * self.R:]
        self.logits = torch.empty((batch, self.R, vocab), dtype=torch.float32, device=dev) if want_logits or rules else None
        self.stats = torch.empty((mv.massv_shard_stats_words(self.cdesc),), dtype=torch.float32, device=dev) if rules else None
        self.probs = (torch.empty((batch, self.R, vocab), dtype=torch.float32, device=dev)
                      if want_probs and temperature > 0 else None)
        self.dev_status = torch.zeros((1,), dtype=torch.int32, device=dev)
        self._staging = None
        self._host_out = None

    @classmethod
    def for_workload(cls, cfg, w, **kw):
        return cls(cfg.batch, cfg.gamma, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cfg.hidden, cfg.vocab,
                   cfg.temperature, w["page_table"].shape[1], w["k_pages"].shape[0],
                   device=w["k_pages"].device, **{"window": getattr(cfg, "window", 0), **kw})

    # -- the calls -------------------------------------------------------------------
    def rotate(self, w):
        """The block's queries and keys at positions seq_lens + j (+ pos_delta), into the step's own buffers."""
        mv.massv_rotary(self.rope, self.turns, w["q"], w["k_new"], self.q_turned, self.k_turned, None, w["seq_lens"], w.get("pos_delta"))

    def attn(self, w):
        q, k = (self.q_turned, self.k_turned) if self.rope is not None else (w["q"], w["k_new"])
        if self.n_groups:
            mv.massv_verify_attn_shared(self.adesc, w["group_start"], w["shared_lens"], q, k, w["v_new"], w["k_pages"], w["v_pages"],
                                        w["page_table"], w["seq_lens"], self.attn_out, self.attn_out_f32, self.lse,
                                        self.attn_ws, self.dev_status)
            return
        mv.massv_verify_attn(self.adesc, q, k, w["v_new"], w["k_pages"], w["v_pages"],
                             w["page_table"], w["seq_lens"], self.attn_out, self.attn_out_f32, self.lse,
                             self.attn_ws, self.dev_status)

    def accept(self, w):
        sampling = self.T > 0
        if self.rules:
            # the logits of all rows, then the rules over them in place with the acceptance behind
            mv.massv_shard_lm_head(self.cdesc, 1, 0, w["hidden"], w["lm_head"], self.logits, self.stats, self.dev_status)
            mv.massv_accept_logits(self.cdesc, w["rules"], self.logits, self.logits, w["draft_tokens"],
                                   w.get("draft_probs") if sampling else None, w.get("u_accept") if sampling else None,
                                   w.get("u_sample") if sampling else None, self.out_tokens, self.accept_len,
                                   self.probs, self.accept_ws, self.dev_status)
            return
        mv.massv_accept(self.cdesc, w["hidden"], w["lm_head"], w["draft_tokens"],
                        w.get("draft_probs") if sampling else None, w.get("u_accept") if sampling else None,
                        w.get("u_sample") if sampling else None, self.out_tokens, self.accept_len,
                        self.logits, self.probs, self.accept_ws, self.dev_status)

    def commit(self, seq_lens, rollback=False):
        mv.massv_kv_commit(self.B, self.gamma, None if rollback else self.accept_len, seq_lens, self.dev_status)

    def record(self, w):
        """The step's emitted tokens into the history that the rules read; nothing to do where they read none."""
        bits, counts = w.get("output_bits"), w.get("counts")
        own_bits, own_counts = getattr(w["rules"], "history", (None, None))
        if bits is None:
            bits, counts = own_bits, own_counts if counts is None else counts
        elif counts is None and own_bits is not None and bits.data_ptr() == own_bits.data_ptr():
            counts = own_counts
        if bits is not None:
            mv.massv_history_add(self.vocab, self.out_tokens, self.accept_len, bits, counts, self.dev_status)

    def run(self, w, commit=True):
        """Enqueue one whole step on the current stream (no synchronisation)."""
        if self.rope is not None:
            self.rotate(w)
        self.attn(w)
        self.accept(w)
        if commit:
            self.commit(w["seq_lens"])
            if self.rules:
                self.record(w)

    # -- end-to-end step with host buffers ----------------------------------------------
    def host_inputs_like(self, tensors):
        """Pinned host buffers for per-step inputs, shaped like ``tensors`` (a dict of name ->
        tensor): a ``HostInputs`` dict whose values are views of ONE pinned allocation, mirrored by
        ONE device allocation, so that ``run_host`` moves a step's inputs with a single copy however
        many tensors they are.  The caller writes each step's inputs into the returned views in place.
        Several sets may exist side by side (say, one with and one without the draft distributions)."""
        return HostInputs(tensors, self.device)

    def _host_result(self):
        if self._host_out is None:
            self._host_out_blob = torch.empty(self._out_blob.shape, dtype=torch.int32).pin_memory()
            n_tok = self.B * self.R
            self._host_out = (self._host_out_blob[:n_tok].view(self.B, self.R), self._host_out_blob[n_tok:])
        return self._host_out

    def run_host(self, host_inputs, resident, commit=False):
        """One step whose per-step inputs start in pinned host memory and whose result (tokens and
        accepted lengths) ends in pinned host memory.  ``host_inputs`` is what ``host_inputs_like``
        returned (one copy up, one copy down) or any dict of pinned tensors (one copy per tensor);
        ``resident`` holds everything that already lives on the device.  Returns (out_tokens,
        accept_len) host tensors after synchronising."""
        w = dict(resident)
        out = self._host_result()
        if isinstance(host_inputs, HostInputs):
            host_inputs.dev_blob.copy_(host_inputs.host_blob, non_blocking=True)
            w.update(host_inputs.dev_views)
        else:
            if self._staging is None or set(self._staging) != set(host_inputs):
                self._staging = {k: torch.empty_like(v, device=self.device) for k, v in host_inputs.items()}
            for k, v in host_inputs.items():
                self._staging[k].copy_(v, non_blocking=True)
                w[k] = self._staging[k]
        self.run(w, commit=commit)
        self._host_out_blob.copy_(self._out_blob, non_blocking=True)
        torch.cuda.current_stream().synchronize()
        return out

    def host_bytes_per_step(self, host_inputs):
        if isinstance(host_inputs, HostInputs):
            h2d = host_inputs.host_blob.numel()     # the whole staging buffer goes up, padding included
        else:
            h2d = sum(v.numel() * v.element_size() for v in host_inputs.values())
        d2h = self.out_tokens.numel() * 4 + self.accept_len.numel() * 4
        return h2d, d2h


class HostInputs(dict):
    """name -> pinned host view; ``host_blob`` / ``dev_blob`` are the two allocations behind the
    views and ``dev_views`` the device-side tensors of the same names."""

    def __init__(self, tensors, device, align=256):
        layout, off = {}, 0
        for k, v in tensors.items():
            nbytes = v.numel() * v.element_size()
            layout[k] = (off, nbytes, v.dtype, tuple(v.shape))
            off = (off + nbytes + align - 1) // align * align
        self.host_blob = torch.empty((max(off, align),), dtype=torch.uint8).pin_memory()
        self.dev_blob = torch.empty((max(off, align),), dtype=torch.uint8, device=device)
        view = lambda blob: {k: blob[o:o + n].view(dt).view(shape) for k, (o, n, dt, shape) in layout.items()}
        super().__init__(view(self.host_blob))
        self.dev_views = view(self.dev_blob)
        for k, v in tensors.items():
            self[k].copy_(v)
