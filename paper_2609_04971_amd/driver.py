"""Periodic BeaconKV eviction across decoding steps (Algorithm 2's phase
machine) on the library's kernels, for all layers of a model at once.

Layers are stacked into the batch dimension: "batch" here is layers * B, so
every call covers every layer (one FPS launch for every query buffer of the
model, one eviction launch for every kv-head of the model).  The caller owns
the decode loop and supplies, per step, the new token's keys and values and
the step's queries before and after RoPE (a model computes both anyway);
this module keeps the per-head state of Algorithm 2 and makes the calls:

  * prefill: the prompt's keys and values fill the cache; each query head's
    buffer starts as FPS(prompt queries, n_beacon) (Appendix D.2).
  * while L <= B_max - n_recent: the step's pre-RoPE query joins the head's
    buffer; a buffer that reaches B_Q^max = n_beacon + n_recent is compressed
    to B_Q^min = n_beacon by FPS (Section 4.2, Eq. fps_q).
  * at L = B_max - n_recent: the beacon set becomes FPS(buffer, n_beacon),
    frozen, and also widened into the fp32 beacon layout scoring reads; the
    recent set starts empty.
  * while B_max - n_recent < L <= B_max: the step's post-RoPE query joins the
    recent set (and its pre-RoPE form is kept for the merge below).
  * at L = B_max: bkv_evict_ex scores every cached key with the group's
    beacons (rotated to the current step) and recent queries, keeps
    B_min = 7/8 B_max (Section 5.1), compacts K and V; then the buffer is
    the beacon set plus the recent queries, compressed by FPS to n_beacon.

mode "rpc" is the recent-queries-only baseline on the same kernels: no
buffer, no beacons (C = 0), the last n_recent queries before each eviction.
mode "ns" keeps running-mean beacons instead of the FPS buffer: every
step's pre-RoPE queries join the nearest of G * n_beacon slots per kv-head
(bkv_beacon_update), and evictions score with those beacons as they stand.
mode "initial" is the Initial+Recent baseline of Table 3: the first
n_beacon queries of each query head (the prompt's) are frozen as its
beacons for good, next to the same recent window.
mode "mass" ranks by what tokens were attended to: the prompt's and every
step's attention (bkv_attend) adds its weights to the tokens' mass, and
evictions keep the prefix, the last n_recent tokens and the largest masses
(bkv_evict_mass).  It needs no query buffers; prefill takes the prompt's
post-RoPE queries.

attention=True has step() compute the step's attention over the cache, in
every mode and before any eviction, into `out` [LB, Hq, D] (and `lse`); mode
"mass" always does.  share_prefix gives the sequences of each layer a prefix
that is held once and never evicted (bkv_attend_shared): the B sequences are
samples of one prompt, and what each of them writes is its own cache.

cache="mx" holds keys and values in 4 bits (bkv_store_mx), in every mode: tokens
are stored as they come, attention reads the 4-bit rows (bkv_attend_mx), and
evictions move them (bkv_evict_mass_mx, bkv_compact_mx).  The scoring modes
score each layer on its keys' plain values, read back (bkv_load_mx) into one
layer's scratch.  window > 0, with attention=True: a step sees the last `window`
cached tokens up to its own and the first `sinks` ones (bkv_attend_window); it
counts cached tokens, so those that evictions took leave the window.

compaction "fill" evicts with bkv_score, bkv_topk and bkv_compact_fill
instead of bkv_evict_ex: the cache keeps the same rows but only the kept
rows past B_min move (into the evicted rows below it), so rows are no
longer in token order; `kept` then holds, for each row, the row it came
from (what bkv_compact_fill calls src_of), which is also what `kept` means
for the order-preserving compaction.

Everything that computes runs in the library's kernels; this module only
slices the caller's tensors and appends rows to them (the writes a serving
engine makes to its own cache).
"""
from __future__ import annotations

import torch

import paper_2609_04971_amd as bkv


class PeriodicEviction:
    def __init__(self, layers: int, B: int, Hq: int, Hkv: int, D: int, B_max: int, rope_table, n_beacon: int = 16,
                 n_recent: int = 16, n_prefix: int = 0, mode: str = "beacon", dtype=torch.bfloat16,
                 device="cuda", record: bool = False, timing: bool = False, compaction: str = "order",
                 attention: bool = False, cache: str = "plain", window: int = 0, sinks: int = 0):
        """rope_table(t) -> (cos, sin), fp32 [D/2] device tensors of the
        model's rotate-half RoPE at absolute position t (the beacons are
        rotated to the step at which eviction runs).  record keeps every
        call's inputs and outputs in `events`; timing brackets every library
        call with HIP events on the current stream, in `times`."""
        if mode not in ("beacon", "rpc", "ns", "initial", "mass"):
            raise ValueError("mode is 'beacon', 'rpc', 'ns', 'initial' or 'mass'")
        if B_max % 8:
            raise ValueError("B_max must be a multiple of 8 (B_min = 7/8 B_max)")
        if compaction not in ("order", "fill"):
            raise ValueError("compaction is 'order' or 'fill'")
        if cache not in ("plain", "mx"):
            raise ValueError("cache is 'plain' or 'mx'")
        if cache == "mx" and compaction == "fill" and mode != "mass":
            raise ValueError("the scoring modes compact a 4-bit cache in order")
        window, sinks = bkv._i32(window, "window"), bkv._i32(sinks, "sinks")
        if window < 0 or sinks < 0:
            raise ValueError("window and sinks are not negative")
        if window and (not attention or mode == "mass"):
            raise ValueError("a window needs attention=True, and sums no weights for mode 'mass'")
        if window and compaction == "fill":
            raise ValueError("a window needs the tokens in order")
        self.window, self.sinks = window, sinks
        self.compaction = compaction
        self.mode = mode
        self.layers = layers
        self.LB, self.Hq, self.Hkv, self.D = layers * B, Hq, Hkv, D
        self.G = Hq // Hkv
        self.B_max, self.B_min = B_max, 7 * B_max // 8
        self.nb = 0 if mode in ("rpc", "mass") else n_beacon
        self.nr = n_recent
        if self.B_max - self.nr <= self.B_min:
            raise ValueError("the recent window must fit between B_min and B_max")
        self.record = record
        self.rope_table = rope_table
        dt, dev = dtype, device
        LB = self.LB
        self.dt = dt
        self.K = self.V = self.cache = None  # keys and values, or both in 4 bits
        if cache == "plain":
            self.K = torch.zeros(LB, Hkv, B_max, D, dtype=dt, device=dev)
            self.V = torch.zeros_like(self.K)
        self.L = 0  # cached tokens per head
        self.t = 0  # absolute position of the next token
        nb, nr = self.nb, self.nr
        if mode == "beacon":
            self.obs = torch.zeros(LB, Hq, nb + nr, D, dtype=dt, device=dev)  # pre-RoPE buffer
            self.obs_len = 0
        self.beacons = torch.zeros(LB, Hkv, self.G * nb, D, dtype=torch.float32, device=dev)
        self.counts = torch.zeros(LB, Hkv, self.G * nb, dtype=torch.int32, device=dev)
        self.recent_rope = torch.zeros(LB, Hq, nr, D, dtype=dt, device=dev)
        self.recent_pre = torch.zeros(LB, Hq, nr, D, dtype=dt, device=dev)
        self.n_rec = 0
        self.dims = bkv.dims(B=LB, Hq=Hq, Hkv=Hkv, D=D, N=B_max, N_cap=B_max, W=nr, C=self.G * nb,
                             budget=self.B_min, n_prefix=n_prefix, dtype="bf16" if dt == torch.bfloat16 else "fp32")
        self.mass = torch.zeros(LB, Hkv, B_max, dtype=torch.float32, device=dev) if mode == "mass" else None
        if cache == "mx":
            self.cache = bkv.mx_cache(self.dims, device=dev)
            if mode != "mass":  # scoring, one layer at a time
                self.ldims = self.dims.replace(B=B)
                self.lkeys = torch.empty(B, Hkv, B_max, D, dtype=dt, device=dev)
                self.lws = bkv.workspace(self.ldims, bkv.OP_SCORE, device=dev)
        self.ws = bkv.mass_workspace(self.dims, device=dev) if mode == "mass" else \
            bkv.workspace(self.dims, bkv.OP_EVICT if cache == "plain" else bkv.OP_COMPACT, device=dev)
        self.kept = torch.empty(LB, Hkv, self.B_min, dtype=torch.int32, device=dev)
        # top-k output before filling
        self.sel = torch.empty_like(self.kept) if compaction == "fill" and mode != "mass" else None
        self.scores = None if mode == "mass" else torch.empty(LB, Hkv, B_max, dtype=torch.float32, device=dev)
        self.attention = attention or mode == "mass"
        self.prefix = None  # (keys, values) of share_prefix
        if self.attention:
            self.adims = self.dims.replace(N=0)  # the cache as it stands
            self.out = torch.zeros(LB, Hq, D, dtype=dt, device=dev)
            self.lse = torch.zeros(LB, Hq, dtype=torch.float32, device=dev)
            self.aws = bkv.attend_workspace(self.dims, 1, mode == "mass", device=dev)
        self.events = []  # (kind, details) of the calls made, when recording
        self.timing = timing
        self.times = []   # (kind, start event, end event), when timing

    # ---- helpers --------------------------------------------------------------
    def _log(self, kind, **kw):
        if self.record:
            self.events.append((kind, kw))

    def _call(self, kind, fn):
        if not self.timing:
            fn()
            return
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        fn()
        e1.record()
        self.times.append((kind, e0, e1))

    def _compress(self, n: int, why: str):
        picks = torch.empty(self.LB, self.Hq, min(self.nb, n), dtype=torch.int32, device=self.obs.device)
        src = self.obs[:, :, :n].clone() if self.record else None
        self._call("fps_" + why, lambda: bkv.fps_gather(self.obs, self.nb, n=n, picks=picks))
        self.obs_len = min(self.nb, n)
        self._log("fps", why=why, src=src, picks=picks)

    # ---- attention over the cache --------------------------------------------------
    def share_prefix(self, K, V):
        """Keys and values [layers, Hkv, P, D] of a prompt that the B sequences of
        every layer share: held once, seen by every query, never evicted.  Before
        prefill; the sequences' own tokens start at position P."""
        if not self.attention:
            raise ValueError("a shared prefix needs attention=True or mode 'mass'")
        if self.cache is not None or self.window:
            raise ValueError("a shared prefix goes with a plain cache and no window")
        if self.t != 0:
            raise ValueError("the prefix comes before every other token")
        if K.shape != V.shape or K.dim() != 4 or tuple(K.shape[:2]) != (self.layers, self.Hkv) or K.shape[3] != self.D:
            raise ValueError(f"the prefix is [layers, Hkv, P, D], got {tuple(K.shape)} and {tuple(V.shape)}")
        if any(x.dtype != self.K.dtype or x.device != self.K.device for x in (K, V)):
            raise ValueError(f"the prefix must be {self.K.dtype} on {self.K.device}, as the cache is")
        self.t = K.shape[2]
        if self.t:
            self.prefix = (K.contiguous(), V.contiguous())
            self.aws = bkv.attend_workspace(self.dims, 1, self.mass is not None, self.layers, self.t, device=K.device)

    def _attend(self, q, out, lse, ws):
        self.adims.N = self.L
        kw = {"lse": lse, "mass": self.mass, "causal": True}
        if self.cache is not None:
            kw |= {"window": self.window, "sinks": self.sinks}
            self._call("attend", lambda: bkv.attend_mx(self.adims, q, self.cache, out, ws, **kw))
        elif self.window:
            self._call("attend", lambda: bkv.attend_window(self.adims, q, self.K, self.V, out, ws, self.window, sinks=self.sinks,
                                                           lse=lse))
        elif self.prefix is None:
            self._call("attend", lambda: bkv.attend(self.adims, q, self.K, self.V, out, ws, **kw))
        else:
            self._call("attend", lambda: bkv.attend_shared(self.adims, q, *self.prefix, self.K, self.V, out, ws, **kw))

    # ---- the phase machine -----------------------------------------------------
    def prefill(self, K, V, q_pre, q_rope=None):
        """Prompt keys/values [LB, Hkv, T, D] and pre-RoPE queries [LB, Hq, T, D].
        With attention, and where the post-RoPE queries q_rope [LB, Hq, T, D]
        are given (mode "mass" needs them), returns the prompt's causal
        attention [LB, Hq, T, D]."""
        T = K.shape[2]
        if T > self.B_max - self.nr:
            raise ValueError("the prompt must end before the recent window")
        if self.mode == "mass" and q_rope is None:
            raise ValueError("mode 'mass' needs the prompt's post-RoPE queries")
        if self.attention and q_rope is not None:
            want = (self.LB, self.Hq, T, self.D)
            if tuple(q_rope.shape) != want or q_rope.dtype != self.dt or q_rope.device != self.kept.device:
                raise ValueError(f"q_rope must be {want}, {self.dt} on {self.kept.device}: got {tuple(q_rope.shape)}, "
                                 f"{q_rope.dtype} on {q_rope.device}")
        if self.cache is not None:
            self._call("store", lambda: bkv.store_mx(self.dims, K.contiguous(), V.contiguous(), self.cache))
        else:
            self.K[:, :, :T] = K
            self.V[:, :, :T] = V
        self.L = T
        self.t = T + (self.prefix[0].shape[2] if self.prefix else 0)
        if self.mass is not None:
            self.mass.zero_()
        out = None
        if self.attention and q_rope is not None:
            q = q_rope.contiguous()
            out = torch.empty_like(q)
            groups, P = (self.layers, self.prefix[0].shape[2]) if self.prefix else (0, 0)
            ws = bkv.attend_workspace(self.dims, T, self.mass is not None, groups, P, device=q.device)
            self._attend(q, out, None, ws)
        if self.mode == "ns":
            # bkv_beacon_update takes queries t-major, so consecutive prompt
            # chunks give the same running means as one call; chunks keep
            # each call's element count within the library's 32-bit limit
            tc = max(1, (2 ** 31 - 1) // (self.LB * self.Hq * self.D))
            for t0 in range(0, T, tc):
                qc = q_pre[:, :, t0:t0 + tc].contiguous()
                self._call("beacon_update", lambda: bkv.beacon_update(self.dims, qc, self.beacons, self.counts))
        if self.mode == "initial":
            # every one of the first min(n_beacon, T) rows is picked (m >= n): the
            # gather widens them into the beacon layout and sets their counts
            self._call("beacon_widen", lambda: bkv.fps_gather(
                q_pre, self.nb, n=min(self.nb, T), dst=self.beacons.view(self.LB, self.Hq, self.nb, self.D),
                counts=self.counts.view(self.LB, self.Hq, self.nb)))
        if self.mode == "beacon":
            picks = torch.empty(self.LB, self.Hq, min(self.nb, T), dtype=torch.int32, device=K.device)
            self._call("fps_prefill", lambda: bkv.fps_gather(q_pre, self.nb, dst=self.obs, picks=picks))
            self.obs_len = min(self.nb, T)
            self._log("fps", why="prefill", src=q_pre.clone() if self.record else None, picks=picks)
        return out

    def step(self, k, v, q_pre, q_rope):
        """One decoding step: k, v [LB, Hkv, D]; q_pre, q_rope [LB, Hq, D].
        Returns True when the step evicted."""
        # the step's rows: the token into the cache, its queries into the
        # buffer (up to the freeze) or into the recent set (after it)
        L, nb, nr = self.L + 1, self.nb, self.nr
        writes = []
        if self.cache is None:
            writes = [(self.K, self.L, k), (self.V, self.L, v)]
        else:
            self._call("store", lambda: bkv.store_mx(self.dims, k.unsqueeze(2).contiguous(), v.unsqueeze(2).contiguous(), self.cache,
                                                     self.L))
        recent = self.B_max - nr < L <= self.B_max and self.mode != "mass"
        if recent:
            writes += [(self.recent_rope, self.n_rec, q_rope), (self.recent_pre, self.n_rec, q_pre)]
        elif self.mode == "beacon":
            writes.append((self.obs, self.obs_len, q_pre))
        bkv.append_rows(writes)
        self.L = L
        self.t += 1
        if self.attention:
            q = q_rope.reshape(self.LB, self.Hq, 1, self.D).contiguous()
            self._attend(q, self.out.unsqueeze(2), self.lse.unsqueeze(2), self.aws)
        if self.mode == "ns":
            q_new = q_pre.reshape(self.LB, self.Hq, 1, self.D).contiguous()
            self._call("beacon_update", lambda: bkv.beacon_update(self.dims, q_new, self.beacons, self.counts))
        if self.mode == "beacon":
            if L <= self.B_max - nr:
                self.obs_len += 1
                if self.obs_len >= nb + nr:
                    self._compress(self.obs_len, "fill")
            if L == self.B_max - nr:
                # freeze: the buffer's FPS selection is the beacon set, kept
                # pre-RoPE in the buffer's first rows and widened for scoring
                self._compress(self.obs_len, "freeze")
                self._call("beacon_widen", lambda: bkv.fps_gather(
                    self.obs, nb, n=self.obs_len, dst=self.beacons.view(self.LB, self.Hq, nb, self.D),
                    counts=self.counts.view(self.LB, self.Hq, nb)))
                self.n_rec = 0
        if recent:
            self.n_rec += 1
        if L == self.B_max:
            self._evict()
            return True
        return False

    def _evict_mx(self, rc, rs):
        """Scores of every layer's keys as the 4-bit cache holds them, one
        selection, one compaction."""
        B = self.ldims.B
        for i in range(self.layers):
            at = slice(i * B, (i + 1) * B)
            bkv.load_mx(self.ldims, bkv.MxCache(*(x[at] for x in self.cache)), self.lkeys, None)
            bkv.score(self.ldims, self.lkeys, self.recent_rope[at], self.beacons[at], self.counts[at], self.scores[at], self.lws,
                      rope_cos=rc, rope_sin=rs)
        bkv.topk(self.dims, self.scores, self.kept)
        bkv.compact_mx(self.dims, self.cache, self.kept, self.ws)

    def _evict(self):
        pre = None
        if self.record:
            pre = (self.K.clone(), self.V.clone()) if self.cache is None else bkv.MxCache(*(x.clone() for x in self.cache))
        if self.mode == "mass":
            mass = self.mass.clone() if self.record else None
            kw = {"kept": self.kept, "fill": self.compaction == "fill"}
            if self.cache is None:
                self._call("evict", lambda: bkv.evict_mass(self.dims, self.K, self.V, self.mass, self.ws, **kw))
            else:
                self._call("evict", lambda: bkv.evict_mass_mx(self.dims, self.cache, self.mass, self.ws, **kw))
            self._log("evict", before=pre, mass=mass, kept=self.kept.clone())
            self.L = self.B_min
            return
        rc, rs = self.rope_table(self.t - 1)  # beacons rotated to the current step
        if self.cache is not None:
            self._call("evict", lambda: self._evict_mx(rc, rs))
        elif self.compaction == "order":
            self._call("evict", lambda: bkv.evict(self.dims, self.K, self.V, self.recent_rope, self.beacons,
                                                  self.counts, self.ws, kept=self.kept, scores=self.scores,
                                                  rope_cos=rc, rope_sin=rs))
        else:
            def evict_fill():
                bkv.score(self.dims, self.K, self.recent_rope, self.beacons, self.counts, self.scores, self.ws,
                          rope_cos=rc, rope_sin=rs)
                bkv.topk(self.dims, self.scores, self.sel)
                bkv.compact_fill(self.dims, self.K, self.V, self.sel, self.kept, self.ws)
            self._call("evict", evict_fill)
        self._log("evict", before=pre, q_win=self.recent_rope.clone() if self.record else None,
                  beacons=self.beacons.clone() if self.record else None,
                  counts=self.counts.clone() if self.record else None, rope=(rc, rs), kept=self.kept.clone(),
                  scores=self.scores.clone() if self.record else None)
        self.L = self.B_min
        if self.mode == "beacon":
            # the buffer becomes the beacon set plus the recent queries, then FPS
            n = self.obs_len
            self.obs[:, :, n:n + self.n_rec] = self.recent_pre[:, :, :self.n_rec]
            self._compress(n + self.n_rec, "merge")
        self.n_rec = 0
