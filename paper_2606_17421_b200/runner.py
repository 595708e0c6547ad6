"""Drive the library over a workload with synthetic inputs (benchmarks and demos).

Holds no arithmetic of the method: it creates a context, fills rotation keys and ciphertexts with
seeded uniform residues (a fresh ciphertext or a switching key is indistinguishable from that, and
the kernels' work does not depend on the values), draws fp32 weights ~ N(0, 0.02^2), and calls the
C ABI.  Correctness is established elsewhere (tests compare with the CPU reference).
"""
from __future__ import annotations

import numpy as np
import torch

from . import bifrost as bf
from . import workloads as wl


def _uniform_residues(gen: torch.Generator, moduli, lead_shape, N: int, device) -> torch.Tensor:
    """int64 tensor [*lead_shape, len(moduli), N], slice m uniform in [0, moduli[m])."""
    out = torch.empty((*lead_shape, len(moduli), N), dtype=torch.int64, device=device)
    for m, q in enumerate(moduli):
        out[..., m, :] = torch.randint(0, int(q), (*lead_shape, N), generator=gen, device=device, dtype=torch.int64)
    return out


class TrustedHalf:
    """The trusted domain's part of a decode step, on a GPU of its own in earnest: in every layer the new token's keys and values
    appended to a cache in 4 bits and attention over it, behind the last layer the vocabulary projection from 4-bit weights.
    What it would get by decryption (rows of q, k and v; the last hidden state) is drawn once and stands in for it."""

    def __init__(self, name: str, seqs: int = 1, context: int = 512, room: int = 512, group: int = 64, page_tokens: int = 64, seed: int = 0,
                 device: str = "cuda:0", stream: torch.cuda.Stream | None = None):
        if seqs < 1 or context < 1 or room < 1:
            raise ValueError("a sequence, a token of its prompt and room for a step's token are the least")
        m = self.model = wl.DECODERS[name]
        self.layers, self.seqs, self.context, self.most = wl.WORKLOADS[name].n_repeat, seqs, context, context + room
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.stream = stream or torch.cuda.Stream(device=self.device)
        with torch.cuda.stream(self.stream):
            gen = torch.Generator(device=self.device)
            gen.manual_seed(seed)
            self.ctx = bf.bf_trusted_create(0, self.stream.cuda_stream)
            max_pages = wl.ceil_div(self.most, page_tokens)
            n_pages = seqs * max_pages
            self.pool = torch.zeros((self.layers, n_pages, m.kv_heads, bf.bf_kv4_block_bytes(m.head_dim, group, page_tokens)),
                                    dtype=torch.uint8, device=self.device)
            self.tables = torch.full((seqs, max_pages), -1, dtype=torch.int32, device=self.device)
            self.lengths = torch.zeros(seqs, dtype=torch.int32, device=self.device)
            self.refs = torch.zeros(n_pages, dtype=torch.int32, device=self.device)
            self.cache = bf.bf_kv4_cache.of(self.pool, self.tables, self.lengths, self.refs, m.head_dim, group, page_tokens)
            # lists that kernels read in later steps are made once, on the stream that reads them
            self.all_seqs = torch.arange(seqs, dtype=torch.int32, device=self.device)
            self.prompt_counts = torch.full((seqs,), context, dtype=torch.int32, device=self.device)
            rows = torch.randn((seqs, m.heads + 2 * m.kv_heads, m.head_dim), generator=gen, device=self.device).bfloat16()
            self.qkv, (self.q, self.k, self.v) = rows, rows.split([m.heads, m.kv_heads, m.kv_heads], 1)
            self.attended = torch.empty((seqs, m.heads, m.head_dim), dtype=torch.bfloat16, device=self.device)
            self.hidden = torch.randn((seqs, m.hidden), generator=gen, device=self.device).bfloat16()
            self.logits = torch.empty((seqs, m.vocab), dtype=torch.float32, device=self.device)
            codes, scales = wl.gen_q4_weights(seed, "vocab", m.vocab, m.hidden, group)
            self.codes, self.scales = torch.from_numpy(codes).to(self.device), torch.from_numpy(scales).to(self.device)
            self.head = bf.bf_q4_matrix.of(self.codes, self.scales, None, m.hidden, group)
            self.length = 0
            self._prompt(gen)

    def _prompt(self, gen):
        """Fills the cache with `context` tokens of every sequence."""
        self._grow(self.context, self.prompt_counts)
        m, n = self.model, self.seqs * self.context
        starts = torch.arange(self.seqs + 1, dtype=torch.int32, device=self.device) * self.context
        for layer in range(self.layers):
            k, v = torch.randn((2, n, m.kv_heads, m.head_dim), generator=gen, device=self.device).bfloat16()
            bf.bf_kv4_append(self.ctx, self.cache, layer, None, starts, self.seqs, self.context, bf.bf_rows.of(k), bf.bf_rows.of(v))
        bf.bf_trusted_status(self.ctx)

    def _grow(self, tokens: int, counts=None):
        bf.bf_kv4_grow(self.ctx, self.cache, None, counts, self.seqs)
        self.length += tokens

    def begin(self):
        """Room for the step's token.  A cache that is full starts over from the prompt's length (and keeps its bytes)."""
        if self.length == self.most:
            bf.bf_kv4_free(self.ctx, self.cache, self.all_seqs, self.seqs)
            self.length = 0
            self._grow(self.context, self.prompt_counts)
        self._grow(1)

    def attend(self, layer: int):
        """Between the q/k/v product of a layer and its output product."""
        m = self.model
        bf.bf_kv4_append(self.ctx, self.cache, layer, None, None, self.seqs, 1, bf.bf_rows.of(self.k), bf.bf_rows.of(self.v))
        bf.bf_kv4_attention(self.ctx, self.cache, layer, None, None, self.seqs, 1, self.length, bf.bf_rows.of(self.q), m.heads,
                            bf.bf_rows.of(self.attended), m.head_dim ** -0.5)

    def finish(self):
        """Logits of the step."""
        bf.bf_q4_linear(self.ctx, self.head, bf.bf_rows.of(self.hidden), self.seqs, bf.bf_rows.of(self.logits))

    def close(self):
        """Raises what the kernels found wrong; the context is gone either way."""
        try:
            bf.bf_trusted_status(self.ctx)
        finally:
            bf.bf_trusted_destroy(self.ctx)


class WorkloadRunner:
    """One context per workload; per layer: weights (cached when the budget allows), input and
    output ciphertext buffers."""

    def __init__(self, name: str, seed: int = 0, device: str = "cuda:0", cache: bool = True,
                 cache_budget_bytes: int | None = None, stream: torch.cuda.Stream | None = None,
                 fuse_shared_inputs: bool = True, fold_in_ciphertext: bool = False, compact_cache: bool = False,
                 pack: str | None = None, moddown: str | None = None, hoist: str | None = None, coef_bits: int = 0,
                 lanes: int | None = None, q4_group: int = 0, trusted: TrustedHalf | None = None):
        self.w = wl.WORKLOADS[name]
        ps = wl.PARAM_SETS[self.w.params]
        self.N, self.primes, self.P, self.scale = ps["N"], list(ps["primes"]), ps["special"], ps["scale"]
        self.r = len(self.primes)
        self.plan = self.w.plan
        if pack or moddown or hoist:         # the workload's plan with another packing / key-switch variant
            self.plan = wl.PlanSpec(self.plan.D, self.plan.tau, self.plan.b, self.plan.g,
                                    pack or self.plan.pack, moddown or self.plan.moddown, hoist or self.plan.hoist)
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        # a stream of our own: the legacy default stream cannot be captured, which would keep the
        # library from replaying its launch sequences as CUDA graphs
        self.stream = stream or torch.cuda.Stream(device=self.device)
        torch.cuda.set_stream(self.stream)
        self.gen = torch.Generator(device=self.device)
        self.gen.manual_seed(seed)
        self.ctx = bf.bf_ctx_create(self.N, self.primes + [self.P], self.r, self.scale,
                                    bf.bf_plan(self.plan.D, self.plan.tau, self.plan.b, self.plan.g,
                                               (bf.BF_PLAN_COMPLEX_PACK if self.plan.pack == "complex" else 0) |
                                               (bf.BF_PLAN_MODDOWN_PER_OUTPUT if self.plan.moddown == "per_output" else 0) |
                                               (bf.BF_PLAN_DOUBLE_HOIST if self.plan.hoist == "double" else 0)),
                                    self.stream.cuda_stream)
        if compact_cache:           # weights count for the bytes of their words in the cache budget, not for 8 a word
            bf.bf_set_compact_cache(self.ctx, True)
        self.compact_cache = compact_cache
        if lanes:                   # concurrent key-switch chains (the library's default otherwise)
            bf.bf_set_lanes(self.ctx, lanes)
        if coef_bits:               # weights resident as rounded 64- or 32-bit coefficients, transformed on every call
            bf.bf_set_coefficient_cache(self.ctx, coef_bits)
        self.coef_bits = coef_bits
        # bytes an encoded coefficient has over all primes it is held in (with double hoisting the special prime too)
        held = self.primes + ([self.P] if self.plan.hoist == "double" else [])
        self.word_bytes = sum(4 if q < 2 ** 32 else 5 if q < 2 ** 40 else 8 for q in held)
        budget = cache_budget_bytes if cache_budget_bytes is not None else self.w.cache_budget_bytes
        if budget:
            bf.bf_set_cache_budget(self.ctx, int(budget))
        # calls: projections that read the same activation stacked into one (q/k/v, gate/up), each with its baby/giant split
        D = self.plan.D
        if fuse_shared_inputs:
            fused = wl.fuse_shared_inputs(self.w.layers, D)
            units = [wl.Layer(nm, d_in, sum(m.d_out for m in members), members[0].input) for nm, d_in, members in fused]
            members_of = {nm: members for nm, _, members in fused}
        else:
            units = list(self.w.layers)
            members_of = {L.name: [L] for L in units}
        self.splits = {L.name: self.w.split_of(L.name, self.plan) for L in units}
        # rotation keys for every split in use: uniform residues over the extended basis
        steps = []
        for b, g in sorted(set(self.splits.values()) | {(self.plan.b, self.plan.g)}):
            steps += [k * self.plan.tau for k in range(1, b)] + [j * b * self.plan.tau for j in range(1, g)]
        self.fold_in_ciphertext = fold_in_ciphertext
        if fold_in_ciphertext:      # the variant that sums the tau partial results on the device
            steps += [1 << i for i in range(self.plan.tau.bit_length() - 1)]
        n = self.N // 2
        self.rot_steps = sorted({s % n for s in steps if s % n})
        basis = self.primes + [self.P]
        if self.rot_steps:
            keys = _uniform_residues(self.gen, basis, (len(self.rot_steps), self.r, 2), self.N, self.device)
            bf.bf_load_eval_keys(self.ctx, self.rot_steps, len(self.rot_steps), keys)
            del keys
        self.key_bytes = len(self.rot_steps) * self.r * 2 * self.N * sum(5 if q < 2 ** 40 else 8 for q in basis)
        # layers
        self.trusted = trusted
        self.layers = []
        for rep in range(self.w.n_repeat):
            for L in units:
                n_in, n_out = wl.ceil_div(L.d_in, D), wl.ceil_div(L.d_out, self.plan.rows_per_ct)
                W, q4 = None, None
                if q4_group:            # a quantised checkpoint: what is encoded comes from 4 bits, and what is not cached stays in them
                    parts = [wl.gen_q4_weights(seed, f"{m.name}.{rep}", m.d_out, m.d_in, q4_group) for m in members_of[L.name]]
                    q4_data = [torch.from_numpy(np.concatenate(a, axis=0)).to(self.device) for a in zip(*parts)]
                    q4 = (bf.bf_q4_matrix.of(*q4_data, None, L.d_in, q4_group), q4_data)
                else:
                    W = torch.from_numpy(np.concatenate(
                        [wl.gen_weights(seed, f"{m.name}.{rep}", m.d_out, m.d_in) for m in members_of[L.name]], axis=0)
                    ).to(self.device)
                handle = None
                b, g = self.splits[L.name]
                if cache:
                    try:
                        handle = bf.bf_encode_weights_q4(self.ctx, q4[0], b, g) if q4 else \
                            bf.bf_encode_weights_split(self.ctx, W, L.d_out, L.d_in, b, g)
                    except bf.BifrostError as e:
                        if e.code != bf.BF_ERR_OOM:
                            raise
                if handle is None:      # the on-the-fly path runs under the plan's own split
                    b, g = self.plan.b, self.plan.g
                ct_in = _uniform_residues(self.gen, self.primes, (n_in, 2), self.N, self.device)
                ct_out = torch.empty((n_out, 2, self.r, self.N), dtype=torch.int64, device=self.device)
                ct_low = torch.empty((n_out, 2, self.r - 1, self.N), dtype=torch.int64, device=self.device)
                self.layers.append(dict(layer=L, rep=rep, n_in=n_in, n_out=n_out, b=b, g=g, W=W, q4=q4, handle=handle,
                                        ct_in=ct_in, ct_out=ct_out, ct_low=ct_low,
                                        pt_bytes=n_in * n_out * (D // self.plan.tau) * self.N * self.word_bytes,
                                        resident_bytes=n_in * n_out * (D // self.plan.tau) * self.N *
                                        (coef_bits // 8 if coef_bits else self.word_bytes) if handle else 0))
        torch.cuda.synchronize()

    # ------------------------------------------------------------------ one decode token
    def step(self):
        """All linear layers of the workload once: the product and its rescale per layer (device buffers), as the one
        call that does both unless the in-ciphertext fold sits between them or the weights come from 4 bits.  With a trusted half,
        its attention follows the products of each layer that make q, k and v (the first, and those that read the same input) and its
        projection the last of all, in that order on whatever streams the two have: one waits for the other, and the step is over when
        the runner's stream has reached its end."""
        after = self._ends_of_qkv() if self.trusted else ()
        if self.trusted:
            self._in_turn(self.trusted.begin)
        for i, e in enumerate(self.layers):
            self._call(e)
            if i in after:
                self._in_turn(self.trusted.attend, e["rep"])
        if self.trusted:
            self._in_turn(self.trusted.finish)

    def _ends_of_qkv(self):
        """The calls with which q, k and v of a transformer layer are there: of those at its start that read one input, the last."""
        ends, rep, tag = [], None, ""
        for i, e in enumerate(self.layers):
            if e["rep"] != rep:
                rep, tag = e["rep"], e["layer"].input
                ends.append(i)
            elif tag and e["layer"].input == tag:
                ends[-1] = i
            else:
                tag = ""
        return set(ends)

    def _in_turn(self, part, *args):
        """A part of the trusted half's work behind what the runner's stream has, and before what it gets next."""
        apart = self.trusted.stream != self.stream
        if apart:
            self.trusted.stream.wait_stream(self.stream)
        part(*args)
        if apart:
            self.stream.wait_stream(self.trusted.stream)

    def _call(self, e):
        L = e["layer"]
        if e["q4"] and not e["handle"]:
            bf.bf_linear_q4(self.ctx, e["ct_in"], e["n_in"], e["q4"][0], e["ct_out"], e["n_out"])
            if self.fold_in_ciphertext:
                bf.bf_fold(self.ctx, e["ct_out"], e["n_out"])
            bf.bf_rescale(self.ctx, e["ct_out"], e["ct_low"], e["n_out"], self.r)
            return
        if not self.fold_in_ciphertext:
            bf.bf_linear_rescaled(self.ctx, e["ct_in"], e["n_in"], e["handle"], None if e["handle"] else e["W"],
                                  L.d_out, L.d_in, e["ct_low"], e["n_out"])
            return
        bf.bf_linear(self.ctx, e["ct_in"], e["n_in"], e["handle"], None if e["handle"] else e["W"],
                     L.d_out, L.d_in, e["ct_out"], e["n_out"])
        bf.bf_fold(self.ctx, e["ct_out"], e["n_out"])
        bf.bf_rescale(self.ctx, e["ct_out"], e["ct_low"], e["n_out"], self.r)

    def make_host_buffers(self):
        for e in self.layers:
            e["h_in"] = e["ct_in"].cpu().pin_memory()
            e["h_out"] = torch.empty((e["n_out"], 2, self.r - 1, self.N), dtype=torch.int64).pin_memory()

    def step_host(self):
        """The products (with fp32 or cached weights) through the host-buffer entry point: ciphertexts travel host -> device -> host."""
        for e in self.layers:
            L = e["layer"]
            bf.bf_linear_host(self.ctx, e["h_in"], e["n_in"], e["handle"], None if e["handle"] else e["W"],
                              L.d_out, L.d_in, e["h_out"], e["n_out"])

    def host_bytes_per_step(self):
        h2d = sum(e["n_in"] * 2 * self.r * self.N * 8 for e in self.layers)
        d2h = sum(e["n_out"] * 2 * (self.r - 1) * self.N * 8 for e in self.layers)
        return h2d, d2h

    def cached_pt_bytes(self):
        return sum(e["pt_bytes"] for e in self.layers if e["handle"])

    def resident_bytes(self):
        """Bytes the cached weights have (differs from the streamed bytes when they are kept as coefficients)."""
        return sum(e["resident_bytes"] for e in self.layers)

    def total_pt_bytes(self):
        return sum(e["pt_bytes"] for e in self.layers)

    def n_fallback_layers(self):
        return sum(1 for e in self.layers if not e["handle"])

    def transforms_weights_per_call(self, e) -> bool:
        """The call of layer entry e transforms its weights (encoded on the fly, or kept as coefficients)."""
        return not e["handle"] or bool(self.coef_bits)

    def close(self):
        bf.bf_ctx_destroy(self.ctx)
        self.layers = []
