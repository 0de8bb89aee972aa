"""Caller-side plumbing around libttkv: allocates the tiers' record pools
(torch tensors: HBM or pinned host memory), fills the ttkv_cache descriptor and
forwards to the C ABI.  No arithmetic of the method lives here; every step of
the hot path runs in the library's kernels."""
import ctypes as C
import functools
from dataclasses import dataclass

import numpy as np
import torch

from . import binding as B


@dataclass
class TierConfig:
    k_fmt: str                 # 'f16' | 'bf16' | 'i8' | 'i4' | 'i4t' (keys of the last tier: int4 grouped over 128 tokens per channel)
    v_fmt: str                 # the same, or 'i4c' (last tier, >= 2 query heads per KV head: int4 as 'i4', stored channel-major per 32 tokens)
    capacity: int              # eviction threshold in tokens (L_fast for tier 0)
    block_tokens: int          # B_blk
    ring_blocks: int           # records per sequence ring
    mem: str = "device"        # 'device' | 'host'
    paged_seed: int = None     # not None: shuffled block table over a shared pool (paged KV)
    summary: bool = False      # keep mean-key summaries (block identification)
    weights: bool = False      # keep what attention has given each token (add_weights, evict_light)


_Q_FMT = {torch.float16: B.F16, torch.bfloat16: B.BF16}
_SRC_FMT = {torch.float16: B.F16, torch.bfloat16: B.BF16, torch.float32: B.F32}
# The current stream's handle without a torch.cuda.Stream object around it (2 us of a step's 14 on the host).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)   # (its users hold device tensors: the runtime is up)

_SECTION_BYTES = {"f16": (256, 0), "bf16": (256, 0), "i8": (128, 8), "i4": (64, 8), "i4t": (64, 4), "i4c": (64, 8)}


def _on_own_device(method):
    """The call runs with the object's device current (the default stream's handle means the current device's)."""
    @functools.wraps(method)
    def call(self, *args, **kw):
        index = self.device.index
        if index is None or _current_device() == index:
            return method(self, *args, **kw)
        with torch.cuda.device(index):
            return method(self, *args, **kw)
    return call


def _stream_of(device):
    if _raw_stream is None or device.index is None:
        return torch.cuda.current_stream(device).cuda_stream
    return _raw_stream(device.index)


def _on(x, device):
    """A tensor, or an object with a device, is on `device` (that may be "cuda", the current one)."""
    return x.device == device or (x.device.type == device.type and None in (device.index, x.device.index))


def _heads(x, shape, device):
    """A tensor of `shape`, [sequence][token][head][128], as the library's strided view."""
    seq, token, head, channel = x.stride()
    assert x.shape == shape and channel == 1 and (x.device == device or _on(x, device)), (x.shape, shape, x.stride(), x.device)
    return B.ttkv_heads(x.data_ptr(), _SRC_FMT[x.dtype], shape[2], seq, token, head)


@functools.lru_cache(128)
def _int64s(n):
    return C.c_int64 * n


def _host_int64(x, n):
    """None, or n host integers as the library takes them."""
    if x is None or n == 0:
        return None
    a = np.ascontiguousarray(x, np.int64)
    assert a.shape == (n,), a.shape
    try:
        return _int64s(n).from_buffer(a)                  # (half the time of a.ctypes)
    except TypeError:                                     # read-only
        return _int64s(n).from_buffer(a.copy())


def _device_positions(x, n_seq, n_tokens, device):
    if x is not None:
        assert x.dtype == torch.int64 and x.shape == (n_seq, n_tokens) and x.is_contiguous() and _on(x, device)
    return x


class Rotary:
    """Norm per head and position rotation of queries and keys (ttkv_norm_rope; in TieredCache.append_rotated).
    freq: radians per token of each pair (64-bit; its length is half the number of channels that turn, a multiple of 8 up to
    64); interleaved: pairs (2 i, 2 i + 1) instead of (i, i + len(freq)); norm: RMS norm of both queries and keys, or a pair of
    truth values for each; q_weight, k_weight: the norms' weights [128] (None: ones)."""

    def __init__(self, freq, interleaved=False, magnitude=1.0, norm=False, q_weight=None, k_weight=None, eps=1e-6, device="cuda:0"):
        self.device = torch.device(device)
        self.freq = np.ascontiguousarray(freq, np.float64)
        assert self.freq.ndim == 1
        weights = []
        for w in (q_weight, k_weight):
            if w is not None:
                assert w.shape == (128,), w.shape
                w = w.detach().to(self.device, torch.float32).contiguous().clone()
            weights.append(w)
        self.q_weight, self.k_weight = weights
        norm_q, norm_k = norm if isinstance(norm, (tuple, list)) else (norm, norm)
        self.r = B.ttkv_rope(2 * len(self.freq), int(interleaved), int(bool(norm_q)) + 2 * int(bool(norm_k)), eps, magnitude,
                             self.freq.ctypes.data, B._p(weights[0]), B._p(weights[1]))
        self.h = B.ttkv_create()

    @staticmethod
    def frequencies(rotary_dim=128, base=10000.0):
        return base ** (-np.arange(0, rotary_dim, 2, dtype=np.float64) / rotary_dim)

    def close(self):
        if self.h is not None:
            torch.cuda.synchronize(self.device)
            B.ttkv_destroy(self.h)
            self.h = None

    @_on_own_device
    def apply(self, q=None, k=None, first_pos=None, positions=None, q_out=None, k_out=None, dtype=None):
        """q [B][T][Hq][128] and / or k [B][T][Hkv][128], any strides but the last, f16 / bf16 / f32 -> (q_out, k_out), new tensors
        of `dtype` (None: the input's) unless given (an output may be its own input).  Token i of sequence b is at
        positions[b][i] (int64 on the device), or first_pos[b] + i (host integers; None: i).  Up to 64 sequences (B)."""
        dev = self.device
        qv = qo = kv = ko = None
        if k is not None:
            if k_out is None:
                k_out = torch.empty_like(k, dtype=dtype, memory_format=torch.contiguous_format)
            shape = k.shape
            n, T, _, channels = shape
            assert channels == 128
            kv, ko = _heads(k, shape, dev), _heads(k_out, shape, dev)
        else:
            k_out = None
            n, T = q.shape[:2]
        if q is not None:
            if q_out is None:
                q_out = torch.empty_like(q, dtype=dtype, memory_format=torch.contiguous_format)
            shape = (n, T, q.shape[2], 128)
            qv, qo = _heads(q, shape, dev), _heads(q_out, shape, dev)
        else:
            q_out = None
        B.ttkv_norm_rope(self.h, self.r, qv, qo, kv, ko, n, T, _host_int64(first_pos, n), _device_positions(positions, n, T, dev), _stream_of(dev))
        return q_out, k_out


class TieredCache:
    def __init__(self, batch, n_q_heads, n_kv_heads, tiers, device="cuda:0", softmax_scale=None, n_slots=0, prefix=None, members=None):
        self.B, self.Hq, self.Hkv = batch, n_q_heads, n_kv_heads
        self.cfg = list(tiers)
        self.device = torch.device(device)
        self.n_slots = n_slots
        self.device_topk = True           # step() with select_k: the chosen ids stay on the device (ttkv_decode_step_topk)
        self.one_call_step = True         # step(): append + attend through ttkv_decode_step; False: the two calls
        self.host_demote_direct = False   # True: evictions into a host tier are stored by the kernels (no staging, no copies)
        self.host_append_direct = True    # bulk appends to a host tier are stored by the kernels; False: staging record + copies
        self.h = B.ttkv_create()
        self.c = B.ttkv_cache()
        c = self.c
        c.batch, c.n_q_heads, c.n_kv_heads, c.head_dim, c.n_tiers = batch, n_q_heads, n_kv_heads, 128, len(self.cfg)
        c.softmax_scale = float(softmax_scale) if softmax_scale is not None else 1.0 / float(np.sqrt(128.0))
        self._keep = []          # tensors / arrays the descriptor points into
        self.start, self.len, self.pool, self.table = [], [], [], []
        self.weights = []                 # per tier None, or fp32 [record][KV head][block token] beside the tier's records
        self._weighed = [np.zeros(batch, np.int64) for _ in self.cfg]   # lifetime ordinal behind the newest token weighed
        self._weighted = [t for t, cfg in enumerate(self.cfg) if cfg.weights]
        self._weighs = [False] * len(self.cfg)   # add_weights keeps the tier's weights (otherwise the caller does, who knows what they wrote)
        self.evicted = np.zeros(batch, np.int64)   # tokens of each sequence that evict_light dropped since it began (they still count as positions)
        self._thinned = False             # some of `evicted` may not be 0
        for t, cfg in enumerate(self.cfg):
            T = c.tier[t]
            T.k_fmt, T.v_fmt = B.FMT_NAMES[cfg.k_fmt], B.FMT_NAMES[cfg.v_fmt]
            T.mem = B.MEM_HOST_PINNED if cfg.mem == "host" else B.MEM_DEVICE
            T.block_tokens, T.capacity_tokens, T.ring_blocks = cfg.block_tokens, cfg.capacity, cfg.ring_blocks
            T.pool_blocks = batch * cfg.ring_blocks
            rec = B.ttkv_record_bytes(c, t)
            assert rec > 0
            nbytes = T.pool_blocks * rec
            if cfg.mem == "host":
                pool = torch.zeros(nbytes, dtype=torch.uint8, pin_memory=True)
            else:
                pool = torch.zeros(nbytes, dtype=torch.uint8, device=self.device)
            T.data = pool.data_ptr()
            start = np.zeros(batch, np.int64)
            ln = np.zeros(batch, np.int64)
            T.start, T.len = start.ctypes.data, ln.ctypes.data
            table = None
            if cfg.paged_seed is not None:
                table = np.random.Generator(np.random.Philox(cfg.paged_seed)).permutation(T.pool_blocks).astype(np.int32)
                table = np.ascontiguousarray(table.reshape(batch, cfg.ring_blocks))
                tdev = torch.from_numpy(table).to(self.device)
                T.block_table, T.block_table_dev = table.ctypes.data, tdev.data_ptr()
                self._keep.append(tdev)
            if cfg.summary:
                ksum = torch.zeros(T.pool_blocks * n_kv_heads * 128, dtype=torch.float32, device=self.device)
                kmu = torch.zeros(T.pool_blocks * n_kv_heads * 128, dtype=torch.float16, device=self.device)
                T.k_sum, T.k_summary = ksum.data_ptr(), kmu.data_ptr()
                self._keep += [ksum, kmu]
                self.ksum, self.kmu = ksum, kmu
            self.weights.append(torch.zeros(T.pool_blocks, n_kv_heads, cfg.block_tokens, dtype=torch.float32, device=self.device)
                                if cfg.weights else None)
            self.start.append(start)
            self.len.append(ln)
            self.pool.append(pool)
            self.table.append(table)
        self.copy_stream = torch.cuda.Stream(device=self.device)
        self.ws = None
        self.ws_parts = 0
        # Parts per row of a launch of up to 256 workgroups, the most that the library cuts into items of 128 tokens where the
        # workspace holds their partials.  Every workspace does: one token more than such a launch takes, or all blocks
        # where only some are selected, counts fewer parts.
        self._few_parts = max(0, 256 // max(1, n_kv_heads * -(-n_q_heads // (16 * n_kv_heads))) - (batch - 1))
        self.demote_ws = None
        self._demote_need = None          # bytes of staging that evictions into a host tier want (constant for a cache)
        self._parts_age = None            # dense steps since the parts per row were last counted (None: never)
        self._until_evict = 0             # steps until some sequence's tier 0 can have filled (0: ask the library)
        self.sel_blocks = self.sel_count = self.sel_scratch = None
        self.out = torch.empty(batch, n_q_heads, 128, dtype=torch.float32, device=self.device)
        self.lse = torch.empty(batch, n_q_heads, dtype=torch.float32, device=self.device)
        self._shared = {}                 # stream -> workspace, out and lse of attend_shared
        self._streams_ws = {}             # (use, stream) -> workspace
        self.prefix = self.members = None
        if prefix is not None:
            self.share(prefix, members)

    def share(self, prefix, members=None):
        """Attend the tokens of `prefix`, a TieredCache of batch 1 with its tiers in HBM, in front of every sequence's own
        from now on (members: truth values, the sequences that do; None: all).  prefix None: no longer.  A prefix has none itself."""
        if prefix is not None:
            assert prefix.B == 1 and (prefix.Hq, prefix.Hkv) == (self.Hq, self.Hkv) and _on(prefix, self.device)
            assert prefix.prefix is None and prefix is not self, "a prefix is attended without its own"
            assert self.n_slots == 0, "a prefix goes with host tiers read in place"
        if members is not None:
            members = np.ascontiguousarray(np.asarray(members, bool), np.int32)
            assert members.shape == (self.B,)
        self.prefix, self.members = prefix, members
        self._parts_age = None

    def close(self):
        if self.h is not None:
            torch.cuda.synchronize(self.device)
            B.ttkv_destroy(self.h)
            self.h = None

    # ------------------------------------------------------------------ streams
    def _compute(self):
        return _stream_of(self.device)

    def _copy(self, overlap=True):
        return self.copy_stream.cuda_stream if overlap else self._compute()

    # ------------------------------------------------------------------ calls
    def record_bytes(self, t):
        return B.ttkv_record_bytes(self.c, t)

    def locate(self, b, pos):
        return B.ttkv_locate(self.c, b, pos)

    def stats(self):
        return B.ttkv_get_stats(self.h)

    def append(self, tier, k, v, seq=-1, through_tiers=False):
        """k, v: device tensors [B][Hkv][n][128] (seq=-1) or [Hkv][n][128], f16 / bf16 / f32."""
        fmt = _SRC_FMT[k.dtype]
        assert k.is_contiguous() and v.is_contiguous() and k.shape == v.shape and k.dtype == v.dtype
        n = k.shape[-2]
        self._parts_age = None            # lengths jump: count the parts again at the next step
        self._until_evict = 0
        self._ended()
        self._unweighed()
        if self.cfg[tier].mem == "host" and self.host_append_direct:
            # no staging: the conversion kernels store into the pinned records
            B.ttkv_quantize_append_host(self.h, self.c, tier, seq, k, v, fmt, n, int(through_tiers), None, 0, self._compute())
        elif self.cfg[tier].mem == "host":
            need = B.ttkv_append_host_workspace_bytes(self.c, tier, seq, n)
            ws = torch.empty(need, dtype=torch.uint8, device=self.device)
            B.ttkv_quantize_append_host(self.h, self.c, tier, seq, k, v, fmt, n, int(through_tiers), ws, need, self._compute())
            torch.cuda.current_stream(self.device).synchronize()   # ws goes out of scope
        else:
            B.ttkv_quantize_append(self.h, self.c, tier, seq, k, v, fmt, n, int(through_tiers), self._compute())

    @_on_own_device
    def append_rotated(self, rotary, k, v, q=None, q_out=None, counts=None, first_pos=None, positions=None, tier=0, seq=-1):
        """Keys normed and rotated on their way into an fp16 / bf16 tier, values beside them, the queries normed and rotated in the
        same launch (ttkv_rope_append).  k, v [B][T][Hkv][128], q [B][T][Hq][128], any strides but the last, f16 / bf16 / f32;
        seq >= 0: one sequence's, B = 1.  counts: tokens of each sequence (host integers; None: T).  Positions as in
        Rotary.apply; neither given: behind the tokens held (prefix included) and those that evict_light dropped; a sequence that holds none begins anew
        (begin_anew).  Returns q_out (a new tensor unless given; rows behind a
        sequence's count are not written, a new tensor's hold anything)."""
        n, T = (self.B, k.shape[1]) if seq < 0 else (1, k.shape[1])
        assert rotary.device == self.device or _on(rotary, self.device)
        dev = self.device
        qv = qo = None
        if q is not None:
            if q_out is None:
                q_out = torch.empty_like(q, dtype=torch.bfloat16 if self.cfg[tier].k_fmt == "bf16" else torch.float16,
                                         memory_format=torch.contiguous_format)
            shape = (n, T, self.Hq, 128)
            qv, qo = _heads(q, shape, dev), _heads(q_out, shape, dev)
        self._ended()
        if first_pos is None and positions is None and (self.prefix is not None or self._thinned):
            first_pos = sum(self.len) + self.evicted
            if self.prefix is not None:
                self.prefix._ended()
                ahead = int(sum(x[0] for x in self.prefix.len) + self.prefix.evicted[0])
                first_pos = first_pos + (1 if self.members is None else self.members) * ahead
            first_pos = first_pos if seq < 0 else first_pos[seq:seq + 1]
        shape = (n, T, self.Hkv, 128)
        self._unweighed()
        B.ttkv_rope_append(self.h, self.c, tier, seq, rotary.r, qv, qo, _heads(k, shape, dev), _heads(v, shape, dev), T, _host_int64(counts, n),
                           _host_int64(first_pos, n), _device_positions(positions, n, T, dev), self._compute())
        self._parts_age = None            # lengths jump: count the parts again at the next step
        self._until_evict = 0
        return q_out

    def begin_anew(self, seq=-1):
        """Sequence seq (-1: every one) ends: no tier holds a token of it any more, and the next ones begin at position 0, or right behind the prefix.
        (Setting its lengths in all tiers to 0 by hand comes to the same.)"""
        assert -1 <= seq < self.B
        rows = slice(None) if seq < 0 else slice(seq, seq + 1)
        for held in self.len:
            held[rows] = 0
        self._ended()
        self._parts_age = None            # lengths jump: count the parts again at the next step
        self._until_evict = 0

    def _ended(self):
        """Before tokens are appended: of a sequence that holds none evict_light has dropped none."""
        if self._thinned:
            self.evicted[sum(self.len) == 0] = 0
            self._thinned = bool(self.evicted.any())

    def demote(self, overlap=True):
        """Cascade eviction through all tiers (Alg. 1, last lines)."""
        if self._demote_need is None:
            self._demote_need = max([B.ttkv_demote_workspace_bytes(self.c, t) for t in range(len(self.cfg) - 1)], default=0)
        need = 0 if self.host_demote_direct else self._demote_need
        if need and (self.demote_ws is None or self.demote_ws.numel() < need):
            self.demote_ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        self._unweighed()
        B.ttkv_evict(self.h, self.c, self.demote_ws if need else None, need, self._compute(), self._copy(overlap))

    def _workspace(self, parts):
        if self.ws is None or parts > self.ws_parts or self.ws_slots != self.n_slots:
            parts = max(parts + 16, int(parts * 1.25), self._few_parts)
            need = B.ttkv_workspace_bytes(self.c, parts, self.n_slots)
            assert need > 0
            if self.ws is not None:       # it may come from another stream than the one whose work still uses it
                self.ws.record_stream(torch.cuda.current_stream(self.device))
            self.ws = torch.empty(need, dtype=torch.uint8, device=self.device)
            self.ws_parts, self.ws_slots = parts, self.n_slots
        return self.ws

    def decode(self, q, selected=None, overlap=True, new=None):
        """q [B][Hq][128] f16/bf16 on the device.  selected: None or (sel_blocks, sel_count) pinned int32 tensors.
        new: None, or (k_new, v_new) [B][Hkv][1][128] of the step's token, appended to tier 0 by the same call."""
        if new is not None:
            self._ended()
            self._unweighed()
        if self.prefix is not None:
            assert selected is None, "blocks are not selected behind a prefix"
            return self._decode_shared(q, new)
        q_fmt = _Q_FMT[q.dtype]
        assert q.is_contiguous() and q.shape == (self.B, self.Hq, 128)
        sb = sc = None
        stride = 0
        if selected is not None:
            sb, sc = selected
            stride = sb.shape[1]
        # Parts per row: counted by the library.  A dense decode step adds one token per sequence, i.e. at most one
        # part per tier every 128 steps, and the workspace is sized with 16 parts to spare: inside step() the count is
        # therefore refreshed only every 64 steps (the library still checks the workspace on every call).
        if selected is None and new is not None and self.ws is not None and self._parts_age is not None and self._parts_age < 64 \
                and self.ws_slots == self.n_slots:
            self._parts_age += 1
            ws = self.ws
        else:
            if new is not None:
                self.len[0] += 1            # size the workspace for the lengths the attention may see
            parts = B.ttkv_count_parts(self.h, self.c, sb, sc, stride, self.n_slots)
            if new is not None:
                self.len[0] -= 1
            if parts < 0:
                raise B.TTKVError(B.ERR_INVALID_ARG, "ttkv_count_parts")
            ws = self._workspace(max(parts, 1))
            self._parts_age = 0 if (selected is None and new is not None) else None
        if new is not None:
            k_new, v_new = new
            fmt = _Q_FMT[k_new.dtype]
            assert k_new.is_contiguous() and v_new.is_contiguous() and k_new.dtype == v_new.dtype
            assert k_new.shape == v_new.shape == (self.B, self.Hkv, 1, 128)
            try:
                B.ttkv_decode_step(self.h, self.c, q, q_fmt, k_new, v_new, fmt, self.out, self.lse, sb, sc, stride, ws, ws.numel(),
                                   self.n_slots, self._compute(), self._copy(overlap))
            except B.TTKVError as e:
                if e.status != B.ERR_WORKSPACE or self._parts_age in (None, 0):
                    raise
                self._parts_age = None    # the split changed under a cached count (nothing was enqueued): count and go again
                return self.decode(q, selected, overlap, new)
        else:
            B.ttkv_decode_attn(self.h, self.c, q, q_fmt, self.out, self.lse, sb, sc, stride, ws, ws.numel(), self.n_slots,
                               self._compute(), self._copy(overlap))
        return self.out, self.lse

    @_on_own_device
    def _decode_shared(self, q, new):
        """decode() of a cache with a prefix (ttkv_decode_step_shared)."""
        q_fmt = _Q_FMT[q.dtype]
        assert q.is_contiguous() and q.shape == (self.B, self.Hq, 128) and _on(q, self.device)
        assert self.prefix.prefix is None, "a prefix is attended without its own"
        k_new, v_new = new if new is not None else (None, None)
        fmt = q_fmt
        if new is not None:
            fmt = _Q_FMT[k_new.dtype]
            assert k_new.is_contiguous() and v_new.is_contiguous() and k_new.dtype == v_new.dtype
            assert k_new.shape == v_new.shape == (self.B, self.Hkv, 1, 128) and _on(k_new, self.device) and _on(v_new, self.device)
        members = None if self.members is None else self.members.ctypes.data
        if torch.cuda.is_current_stream_capturing():   # a graph keeps its workspace, whatever this one's grows to
            ws = torch.empty(B.ttkv_workspace_bytes(self.c, self._count_shared(new is not None), 0), dtype=torch.uint8, device=self.device)
            B.ttkv_decode_step_shared(self.h, self.c, self.prefix.c, members, q, q_fmt, k_new, v_new, fmt, self.out, self.lse, ws, ws.numel(),
                                      self._compute())
            self._parts_age = None
            return self.out, self.lse
        # parts per row: counted anew every 64 steps, as in decode(), or when the library finds the workspace too small
        if new is None or self.ws is None or self._parts_age is None or self._parts_age >= 64:
            self._workspace(self._count_shared(new is not None))
            self._parts_age = 0 if new is not None else None
        else:
            self._parts_age += 1
        while True:
            try:
                B.ttkv_decode_step_shared(self.h, self.c, self.prefix.c, members, q, q_fmt, k_new, v_new, fmt, self.out, self.lse, self.ws,
                                          self.ws.numel(), self._compute())
                return self.out, self.lse
            except B.TTKVError as e:
                if e.status != B.ERR_WORKSPACE or self._parts_age in (None, 0):
                    raise
                self._workspace(self._count_shared(new is not None))
                self._parts_age = 0

    def _count_shared(self, with_token):
        """Parts per row that a step's workspace holds."""
        if with_token:
            self.len[0] += 1            # size the workspace for the lengths the attention may see
        own = B.ttkv_count_parts(self.h, self.c, None, None, 0, 0)
        if with_token:
            self.len[0] -= 1
        lead = B.ttkv_prefix_parts(self.h, self.prefix.c, self.B if self.members is None else int(self.members.sum()))
        if own < 0 or lead < 0:
            raise B.TTKVError(B.ERR_INVALID_ARG, "ttkv_count_parts" if own < 0 else "ttkv_prefix_parts")
        return max(1, max(own, self._few_parts) + lead)

    @_on_own_device
    def attend_shared(self, q):
        """Queries of any number of sequences over this cache of batch 1 as their shared prefix: q [n][Hq][128] f16 / bf16 ->
        out [n][Hq][128], lse [n][Hq] fp32 (ttkv_shared_attn; kept for the next call on the same stream, like those of decode(); a call
        that is captured into a graph has tensors of its own).  Calls on several streams may overlap."""
        q_fmt = _Q_FMT[q.dtype]
        n = q.shape[0]
        assert q.is_contiguous() and q.shape == (n, self.Hq, 128) and _on(q, self.device)
        assert self.prefix is None, "a prefix is attended without its own"
        if torch.cuda.is_current_stream_capturing():
            out, lse = self._shared_results(n)
            ws = self._shared_workspace(n)
            B.ttkv_shared_attn(self.h, self.c, q, q_fmt, n, out, lse, ws, ws.numel(), self._compute())
            return out, lse
        # Every stream has its own, so that calls on two of them may overlap, and what a larger call replaces belongs to the
        # stream that used it: its memory is handed out again behind that stream's work only.
        stream = self._compute()
        kept = self._shared.get(stream)
        if kept is None or kept[1].shape[0] != n:
            kept = self._shared[stream] = (kept[0] if kept else self._shared_workspace(n), *self._shared_results(n))
        ws, out, lse = kept
        try:
            B.ttkv_shared_attn(self.h, self.c, q, q_fmt, n, out, lse, ws, ws.numel(), stream)
        except B.TTKVError as e:
            if e.status != B.ERR_WORKSPACE:
                raise
            ws = self._shared_workspace(n)   # more sequences or parts than any call before: nothing was enqueued
            self._shared[stream] = ws, out, lse
            B.ttkv_shared_attn(self.h, self.c, q, q_fmt, n, out, lse, ws, ws.numel(), stream)
        return out, lse

    def _shared_results(self, n):
        return (torch.empty(n, self.Hq, 128, dtype=torch.float32, device=self.device),
                torch.empty(n, self.Hq, dtype=torch.float32, device=self.device))

    def _shared_workspace(self, n):
        need = B.ttkv_shared_workspace_bytes(self.h, self.c, n)
        return torch.empty(max(256, need), dtype=torch.uint8, device=self.device)

    # ------------------------------------------------------------------ chunks of new tokens
    def _with_workspace(self, use, call, need):
        """call(workspace, bytes) with the workspace that `use` has on the current stream, a larger one where the library asks for it
        (nothing was enqueued then).  What a larger one replaces is handed out again behind that stream's work only; a call
        that is captured into a graph has one of its own."""
        if torch.cuda.is_current_stream_capturing():
            ws = torch.empty(need(), dtype=torch.uint8, device=self.device)
            return call(ws, ws.numel())
        key = use, self._compute()
        ws = self._streams_ws.get(key)
        try:
            return call(ws, 0 if ws is None else ws.numel())
        except B.TTKVError as e:
            if e.status != B.ERR_WORKSPACE:
                raise
        ws = self._streams_ws[key] = torch.empty(need() * 5 // 4, dtype=torch.uint8, device=self.device)
        return call(ws, ws.numel())

    @_on_own_device
    def attend_chunk(self, q, counts=None, out=None, lse=None, seq=-1, dtype=None):
        """Attention of the newest tokens' queries, q [B][T][Hq][128] f16 / bf16 (any strides but the last), over every tier, and the prefix
        of a cache that has one; the tokens themselves are in the cache already (append, append_rotated).  Causal: each query sees the tokens up to its own.
        counts: new tokens of each sequence (host integers; None: T); seq >= 0: one sequence's, B = 1.  Returns out (a new tensor of
        `dtype`, None: q's, f16 or bf16, unless given) and lse [B][T][Hq] fp32 (a new tensor unless given, contiguous); rows
        behind a sequence's count are not written (ttkv_chunk_attn)."""
        n, T = (self.B if seq < 0 else 1), q.shape[1]
        shape = (n, T, self.Hq, 128)
        if out is None:
            out = torch.empty_like(q, dtype=dtype, memory_format=torch.contiguous_format)
        if lse is None:
            lse = torch.empty(shape[:3], dtype=torch.float32, device=self.device)
        assert lse.shape == shape[:3] and lse.is_contiguous() and lse.dtype == torch.float32 and _on(lse, self.device)
        assert self.prefix is None or self.prefix.prefix is None, "a prefix is attended without its own"
        qv, ov, each = _heads(q, shape, self.device), _heads(out, shape, self.device), _host_int64(counts, n)
        prefix = None if self.prefix is None else self.prefix.c
        members = None if self.members is None else self.members.ctypes.data
        stream = self._compute()
        self._with_workspace("chunk", lambda ws, size: B.ttkv_chunk_attn(self.h, self.c, seq, prefix, members, qv, ov, lse, T, each, ws, size, stream),
                             lambda: B.ttkv_chunk_workspace_bytes(self.h, self.c, seq, prefix, members, T, each))
        return out, lse

    def prefill(self, rotary, q, k, v, counts=None, first_pos=None, positions=None, seq=-1, dtype=None, overlap=True):
        """A chunk of new tokens from the projections: norm and rotation -> append -> attend -> evict.  q [B][T][Hq][128], k, v
        [B][T][Hkv][128], arguments as in append_rotated and attend_chunk; tier 0's ring has room for what it holds and the chunk.  A chunk
        that is refused leaves the cache as it was."""
        held = self.len[0].copy()
        rotated = self.append_rotated(rotary, k, v, q=q, counts=counts, first_pos=first_pos, positions=positions, seq=seq)
        try:
            out, lse = self.attend_chunk(rotated, counts, seq=seq, dtype=dtype)
        except Exception:
            self.len[0][:] = held
            raise
        self.demote(overlap)
        return out, lse

    # ------------------------------------------------------------------ weights of tokens
    def _unweighed(self):
        """Before tokens come into a tier, from outside or down the cascade: what lies behind the newest token that each tier holds has not been
        weighed (tokens may have been taken back, a sequence may have ended)."""
        for t in self._weighted:
            np.minimum(self._weighed[t], self.start[t] + self.len[t], out=self._weighed[t])

    @_on_own_device
    def add_weights(self, q, lse, counts=None, fresh=None, tier=0, seq=-1):
        """Adds to self.weights[tier] what the newest tokens' queries give each token (ttkv_add_weights): q [B][T][Hq][128] (or [B][Hq][128]
        of a decode step) and lse [B][T][Hq] ([B][Hq]) as attend_chunk or step had and returned them, before the tokens lie elsewhere
        (evicted).  fresh: so many of each sequence's newest tokens begin at 0 (host integers; None: those appended since the last call)."""
        assert self.weights[tier] is not None, "the tier keeps no weights"
        n = self.B if seq < 0 else 1
        if q.dim() == 3:
            q = q.unsqueeze(1)
        T = q.shape[1]
        assert lse.numel() == n * T * self.Hq and lse.is_contiguous() and lse.dtype == torch.float32 and _on(lse, self.device)
        rows = slice(None) if seq < 0 else slice(seq, seq + 1)
        end = (self.start[tier] + self.len[tier])[rows]
        if fresh is None:
            newer = sum((x[rows] for x in self.len[:tier]), np.zeros(n, np.int64))
            fresh = np.maximum(0, end - self._weighed[tier][rows]) + newer
        qv, each, begin, stream = _heads(q, (n, T, self.Hq, 128), self.device), _host_int64(counts, n), _host_int64(fresh, n), self._compute()
        self._with_workspace("weights", lambda ws, size: B.ttkv_add_weights(self.h, self.c, tier, seq, qv, lse, T, each, begin, self.weights[tier], ws, size, stream),
                             lambda: B.ttkv_weights_workspace_bytes(self.h, self.c, tier, seq, T, each, begin))
        self._weighed[tier][rows] = end
        self._weighs[tier] = True

    @_on_own_device
    def evict_light(self, keep, recent, tier=0, swap=False):
        """Frees the tier's oldest blocks, as many as leave every sequence at least `keep` tokens: per KV head the tokens of least weight go, the
        `recent` newest stay, the others have been weighed (ttkv_evict_light; where add_weights keeps the tier's weights, tokens that came after it and
        are not among the recent ones are refused).  swap: nothing goes; the light tokens lie in the oldest blocks afterwards, for demote()."""
        assert self.weights[tier] is not None, "the tier keeps no weights"
        if self._weighs[tier]:            # tokens that were not weighed have what their places held before
            held, bt = self.len[tier], self.cfg[tier].block_tokens
            if ((held - keep >= bt) & (self.start[tier] + held - self._weighed[tier] > recent)).any():
                raise B.TTKVError(B.ERR_INVALID_ARG, "ttkv_evict_light: tokens in front of the recent ones were not weighed")
        held, stream = self.len[tier].copy(), self._compute()
        self._with_workspace("light", lambda ws, size: B.ttkv_evict_light(self.h, self.c, tier, keep, recent, swap, self.weights[tier], ws, size, stream),
                             lambda: B.ttkv_evict_light_workspace_bytes(self.h, self.c, tier, keep, recent))
        self.evicted += held - self.len[tier]
        self._thinned = bool(self.evicted.any())
        self._parts_age = None            # lengths jump: count the parts again at the next step
        self._until_evict = 0

    def select(self, q, k):
        q_fmt = _Q_FMT[q.dtype]
        stride = self._select_buffers(k)
        B.ttkv_select_blocks(self.h, self.c, q, q_fmt, k, self.sel_blocks, self.sel_count, stride, self.sel_scratch,
                             self.sel_scratch.numel(), self._compute())
        return self.sel_blocks, self.sel_count

    def _select_buffers(self, k):
        stride = max(1, k)
        if self.sel_blocks is None or self.sel_blocks.shape[1] != stride:
            self.sel_blocks = torch.zeros(self.B, stride, dtype=torch.int32, pin_memory=True)
            self.sel_count = torch.zeros(self.B, dtype=torch.int32, pin_memory=True)
            self.sel_scratch = torch.empty(self.B * (1024 * 4 + (stride + 1) * 4) + 512, dtype=torch.uint8, device=self.device)
        return stride

    def step_topk(self, q, k_new, v_new, k):
        """append -> identify + top-k + attend with the chosen ids left on the device (no host round trip)."""
        assert self.prefix is None, "blocks are not selected behind a prefix"
        q_fmt = _Q_FMT[q.dtype]
        fmt = _Q_FMT[k_new.dtype]
        assert q.is_contiguous() and k_new.is_contiguous() and v_new.is_contiguous()
        assert k_new.shape == v_new.shape == (self.B, self.Hkv, 1, 128)
        stride = self._select_buffers(k)
        self._ended()
        self._unweighed()
        # The split of a selection is planned inside the call, which refuses a workspace that is too small for it before
        # anything is enqueued: the workspace is sized once from a dense plan's parts and grows when it is refused (no
        # run is cut finer than into items of 128 tokens, which bounds it).
        self._parts_age = None
        if self.ws is None or self.ws_slots != self.n_slots:
            self.len[0] += 1
            parts = B.ttkv_count_parts(self.h, self.c, None, None, 0, 0)
            self.len[0] -= 1
            self._workspace(max(parts, 1))
        while True:
            try:
                B.ttkv_decode_step_topk(self.h, self.c, q, q_fmt, k_new, v_new, fmt, self.out, self.lse, k, self.sel_blocks,
                                        self.sel_count, stride, self.sel_scratch, self.sel_scratch.numel(), self.ws,
                                        self.ws.numel(), self._compute())
                break
            except B.TTKVError as e:
                if e.status != B.ERR_WORKSPACE or self.ws_parts > sum(int(n.max()) // 64 + 2 for n in self.len):
                    raise
                self._workspace(2 * self.ws_parts)
        return self.out, self.lse

    def _evict_if_due(self, overlap):
        """Alg. 1's eviction check after a step that appended one token per sequence.  A tier below the first only grows
        when the one above evicts, so nothing can be due before some sequence's tier 0 has filled: until then the
        library is not asked (every call validates the whole descriptor)."""
        self._until_evict -= 1
        if self._until_evict > 0:
            return
        self.demote(overlap)
        self._until_evict = max(1, int((self.cfg[0].capacity - self.len[0]).min()))

    def step(self, q, k_new, v_new, select_k=None, overlap=True):
        """One decode step (Alg. 1): append -> [identify blocks] -> attend -> evict.  k_new, v_new [B][Hkv][1][128]."""
        if select_k is not None and self.device_topk and self.one_call_step and self.n_slots == 0:
            out, lse = self.step_topk(q, k_new, v_new, select_k)
            self._evict_if_due(overlap)
            return out, lse
        if not self.one_call_step:
            self.append(0, k_new, v_new)
            sel = self.select(q, select_k) if select_k is not None else None
            out, lse = self.decode(q, sel, overlap)
        else:
            sel = self.select(q, select_k) if select_k is not None else None
            out, lse = self.decode(q, sel, overlap, new=(k_new, v_new))
        self._evict_if_due(overlap)
        return out, lse

    def step_rotated(self, rotary, q, k, v, first_pos=None, positions=None, overlap=True):
        """One decode step from the projections: norm and rotation -> append -> attend (the prefix too) -> evict.  q [B][1][Hq][128],
        k, v [B][1][Hkv][128] and the positions as in append_rotated.  A step that is refused leaves the cache as it was."""
        assert q.shape == (self.B, 1, self.Hq, 128) and k.shape == v.shape == (self.B, 1, self.Hkv, 128), "one token of every sequence"
        until, held = self._until_evict, self.len[0].copy()
        rotated = self.append_rotated(rotary, k, v, q=q, first_pos=first_pos, positions=positions)
        self._until_evict = until         # one token per sequence: nothing jumped
        try:
            out, lse = self.decode(rotated.view(self.B, self.Hq, 128), None, overlap)
        except Exception:
            self.len[0][:] = held         # refused: nor is the token held (its row lies behind the live ones)
            raise
        self._evict_if_due(overlap)
        return out, lse

    # ------------------------------------------------------------------ inspection (layout decoding only)
    def dump_tier(self, t, b):
        """Live rows of tier t, sequence b, oldest first, as raw bytes:
        {'k': uint8 [Hkv][n][kc], 'k_meta': uint8 [Hkv][n][km], 'v': ..., 'v_meta': ...}."""
        torch.cuda.synchronize(self.device)
        cfg = self.cfg[t]
        bt, ring = cfg.block_tokens, cfg.ring_blocks
        kc, km = _SECTION_BYTES[cfg.k_fmt]
        vc, vm = _SECTION_BYTES[cfg.v_fmt]
        head_bytes = bt * (kc + km + vc + vm)
        pool = self.pool[t].cpu().numpy().reshape(-1, self.Hkv, head_bytes)
        o = int(self.start[t][b]) + np.arange(int(self.len[t][b]), dtype=np.int64)
        r = (o // bt) % ring
        rec = self.table[t][b][r] if self.table[t] is not None else b * ring + r
        row = o % bt
        out, off = {}, 0
        for name, w in (("k", kc), ("k_meta", km), ("v", vc), ("v_meta", vm)):
            sec = pool[:, :, off:off + bt * w].reshape(pool.shape[0], self.Hkv, bt, w)
            out[name] = np.ascontiguousarray(sec[rec, :, row].transpose(1, 0, 2)) if w else None
            off += bt * w
        return out

    def dump_summary(self, t, b, block_id):
        torch.cuda.synchronize(self.device)
        ring = self.cfg[t].ring_blocks
        r = block_id % ring
        rec = int(self.table[t][b][r]) if self.table[t] is not None else b * ring + r
        return self.kmu.view(-1, self.Hkv, 128)[rec].cpu().numpy().view(np.uint16)
