"""PyTorch-side marshalling for libviscache: allocates the outputs and the
workspace that the C ABI asks for and passes device addresses and the current
stream.  No computation happens here."""
from __future__ import annotations

import ctypes
import struct

import torch
from torch.autograd import forward_ad as _forward

from . import (VC_ERR_WORKSPACE, VC_PRUNE_EVENTS, VC_Q8_BLOCK, VisCacheError, _int32, lib, VC_Q8_E4M3, VC_Q8_INT8, VC_RANK_GLOBAL, make_params, make_prune_io, make_shape, prune_with_io, vc_cache,
               vc_decode_shape, vc_mass_cache, vc_norm, vc_q8cache, vc_qcache, vc_rope, vc_rows, viscache_append_kv, viscache_budget, viscache_decode_attn,
               viscache_decode_plan, viscache_decode_step, viscache_decode_step_noalloc,
               viscache_decode_step_planned, viscache_decode_step_q4,
               viscache_decode_step_workspace_bytes,
               viscache_decode_workspace_bytes, viscache_mass_attend_workspace_bytes,
               viscache_mass_evict_workspace_bytes, viscache_out_rows, viscache_prune_workspace_bytes,
               viscache_q8_append, viscache_q8_attend_workspace_bytes, viscache_quantize_rows)


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _addr(t: torch.Tensor | None) -> int:
    return 0 if t is None or t.numel() == 0 else t.data_ptr()


class PruneCall:
    """One PruneKV problem: shape, parameters, per-layer outputs, workspace.

    k_in / v_in: per-layer bf16 tensors [sum_b Hkv*n_b, d]; q_win: per-layer
    fp32 tensors [B, Hq, W, d] (window scores) or [sum_b Hq*(n_b+W), d]
    (prefill scores); k_text: per-layer bf16 [B, Hkv, W, d] (prefill scores
    only).  `run()` enqueues viscache_prune on the current stream."""

    def __init__(self, B, L, Hq, Hkv, d, W, n_vis, params, k_in, v_in, q_win, with_drop=False, k_text=None):
        self.B, self.L, self.Hq, self.Hkv, self.d, self.W = B, L, Hq, Hkv, d, W
        self.n_vis = [int(x) for x in n_vis]
        self.params = params
        self.shape = make_shape(B, L, Hq, Hkv, d, W, self.n_vis)
        self.k, self.n_surv, self.h = viscache_budget(self.shape, params)
        self.rows = viscache_out_rows(self.shape, params)
        dev = k_in[0].device
        vdt = torch.float32 if params.v_out_fp32 else torch.bfloat16
        self.k_in, self.v_in, self.q_win = list(k_in), list(v_in), list(q_win)
        self.k_text = list(k_text) if k_text is not None else None
        self.k_out, self.v_out, self.idx_out, self.drop_out = [], [], [], []
        for l in range(L):
            nrow = self.rows[l * (B + 1) + B]
            self.k_out.append(torch.empty((nrow, d), dtype=torch.bfloat16, device=dev))
            self.v_out.append(torch.empty((nrow, d), dtype=vdt, device=dev))
            self.idx_out.append(torch.empty((nrow,), dtype=torch.int32, device=dev))
            if with_drop:
                ndrop = sum(Hkv * (self.n_surv[b * L + l] - self.k[b * L + l]) for b in range(B)) if l < self.h else 0
                self.drop_out.append(torch.empty((ndrop,), dtype=torch.int32, device=dev))
        self.ws_bytes = viscache_prune_workspace_bytes(self.shape, params)
        self.ws = torch.empty((self.ws_bytes,), dtype=torch.uint8, device=dev)
        self._io = None

    @property
    def global_rank(self) -> bool:
        return self.params.rank_mode == VC_RANK_GLOBAL

    def _prune_io(self):
        """The call's vc_prune_io, built once (the buffers never move)."""
        if self._io is None:
            a = lambda ts: [_addr(t) for t in ts]
            self._io = make_prune_io(a(self.k_in), a(self.v_in), a(self.q_win), a(self.k_out), a(self.v_out),
                                     a(self.idx_out), a(self.drop_out) if self.drop_out else None,
                                     a(self.k_text) if self.k_text is not None else None)
        return self._io

    def run(self, events=None) -> None:
        """Enqueue viscache_prune on the current stream; with `events`
        (VC_PRUNE_EVENTS torch.cuda.Event objects created with
        enable_timing=True, or raw hipEvent_t handles as ints) the stages are
        bracketed (viscache_prune_staged)."""
        handles = None
        if events is not None:
            assert len(events) == VC_PRUNE_EVENTS
            handles = []
            for e in events:
                if isinstance(e, int):
                    handles.append(e)
                    continue
                if e.cuda_event == 0:
                    e.record()  # materialise the handle
                handles.append(e.cuda_event)
        prune_with_io(self.shape, self.params, self._prune_io(), self.ws.data_ptr(), self.ws_bytes, _stream(),
                      handles)

    def unit_rows(self, l: int, b: int, g: int):
        """Row range of (layer, sequence, kv head) in layer l's outputs."""
        k = self.k[b * self.L + l]
        r0 = self.rows[l * (self.B + 1) + b] + g * k
        return r0, r0 + k

    def unit_drop_rows(self, l: int, b: int, g: int):
        r = self.n_surv[b * self.L + l] - self.k[b * self.L + l]
        base = sum(self.Hkv * (self.n_surv[bb * self.L + l] - self.k[bb * self.L + l]) for bb in range(b))
        return base + g * r, base + (g + 1) * r


class DecodeCache:
    """A decode cache pool over L layers x B sequences x Hkv heads.  Unit
    u = (l*B + b)*Hkv + g owns `cap[u]` rows starting at row_off[u]."""

    def __init__(self, L, B, Hq, Hkv, d, caps, device):
        self.shape = vc_decode_shape(B, L, Hq, Hkv, d)
        self.L, self.B, self.Hq, self.Hkv, self.d = L, B, Hq, Hkv, d
        caps = [int(c) for c in caps]
        offs, o = [], 0
        for c in caps:
            offs.append(o)
            o += c
        self.total_rows = o
        self.max_cap = max(caps) if caps else 0
        self.k_pool = torch.zeros((max(o, 1), d), dtype=torch.bfloat16, device=device)
        self.v_pool = torch.zeros((max(o, 1), d), dtype=torch.bfloat16, device=device)
        self.row_off = torch.tensor(offs, dtype=torch.int64, device=device)
        self.cap = torch.tensor(caps, dtype=torch.int32, device=device)
        self.len = torch.zeros(len(caps), dtype=torch.int32, device=device)
        self.offs_host, self.caps_host = offs, caps
        self.ws_bytes = viscache_decode_workspace_bytes(self.shape, self.max_cap)
        self.ws = torch.empty((max(self.ws_bytes, 256),), dtype=torch.uint8, device=device)
        # The fused step keeps arrival counters in its workspace: zero-filled once.
        self.step_ws_bytes = viscache_decode_step_workspace_bytes(self.shape, self.max_cap)
        self.step_ws = torch.zeros((max(self.step_ws_bytes, 256),), dtype=torch.uint8, device=device)
        self.c = vc_cache(self.k_pool.data_ptr(), self.v_pool.data_ptr(), self.row_off.data_ptr(),
                          self.cap.data_ptr(), self.len.data_ptr())

    def append(self, k_new: torch.Tensor, v_new: torch.Tensor) -> None:
        viscache_append_kv(self.shape, self.c, k_new.data_ptr(), v_new.data_ptr(), _stream())

    def attend(self, q: torch.Tensor, out: torch.Tensor, scale: float) -> None:
        viscache_decode_attn(self.shape, self.c, q.data_ptr(), out.data_ptr(), scale, self.max_cap,
                             self.ws.data_ptr(), self.ws_bytes, _stream())

    def step(self, k_new: torch.Tensor, v_new: torch.Tensor, q: torch.Tensor, out: torch.Tensor,
             scale: float) -> None:
        """append + attend in one launch (viscache_decode_step)."""
        viscache_decode_step(self.shape, self.c, k_new.data_ptr(), v_new.data_ptr(), q.data_ptr(),
                             out.data_ptr(), scale, self.max_cap, self.step_ws.data_ptr(), self.step_ws_bytes,
                             _stream())

    def step_noalloc(self, k_new: torch.Tensor, v_new: torch.Tensor, q: torch.Tensor, out: torch.Tensor,
                     scale: float) -> None:
        """step() through viscache_decode_step_noalloc: no workspace, the
        library's own scratch."""
        viscache_decode_step_noalloc(self.shape, self.c, k_new.data_ptr(), v_new.data_ptr(), q.data_ptr(),
                                     out.data_ptr(), scale, self.max_cap, _stream())

    def step_layers(self, k_new: torch.Tensor, v_new: torch.Tensor, q: torch.Tensor, out: torch.Tensor,
                    scale: float) -> None:
        """The same decode step as L launches, one per layer (the loop of a
        model that attends layer by layer): viscache_decode_step on each
        layer's units, with the layer's slices of the pool tables, inputs and
        outputs.  The launches are ordered on one stream, so they share one
        step workspace."""
        if not hasattr(self, "_layer_caches"):
            per = self.B * self.Hkv
            self.layer_shape = vc_decode_shape(self.B, 1, self.Hq, self.Hkv, self.d)
            self._layer_caches = [
                vc_cache(self.k_pool.data_ptr(), self.v_pool.data_ptr(), self.row_off[l * per:].data_ptr(),
                         self.cap[l * per:].data_ptr(), self.len[l * per:].data_ptr()) for l in range(self.L)]
            # One row bound for all layers.  The workgroups it leaves idle in a
            # layer of small capacities cost nothing: with each layer's own
            # bound a step over 28 layers of a 3136-token pruned cache takes
            # 307 us as with one for all, of a 12.5k one 367 against 365.
            self.layer_ws_bytes = max(viscache_decode_step_workspace_bytes(self.layer_shape, self.max_cap), 256)
            self.layer_ws = torch.zeros((self.layer_ws_bytes,), dtype=torch.uint8, device=self.k_pool.device)
        for l in range(self.L):
            viscache_decode_step(self.layer_shape, self._layer_caches[l], k_new[l].data_ptr(), v_new[l].data_ptr(),
                                 q[l].data_ptr(), out[l].data_ptr(), scale, self.max_cap,
                                 self.layer_ws.data_ptr(), self.layer_ws_bytes, _stream())

    def quantize(self, nq) -> None:
        """Quantise every pool row to 4 bits (viscache_quantize_rows) and let
        unit u read its first nq[u] rows (rounded down to the 32-row tile)
        from the codes in later q4 steps; the rows stay in the bf16 pools."""
        dev = self.k_pool.device
        rows, d = self.k_pool.shape
        self.qk = torch.empty((rows, d // 2), dtype=torch.uint8, device=dev)
        self.qv = torch.empty((rows, d // 2), dtype=torch.uint8, device=dev)
        self.qkm = torch.empty((rows, d // 32, 2), dtype=torch.float32, device=dev)
        self.qvm = torch.empty((rows, d // 32, 2), dtype=torch.float32, device=dev)
        viscache_quantize_rows(d, rows, self.k_pool.data_ptr(), self.qk.data_ptr(), self.qkm.data_ptr(), _stream())
        viscache_quantize_rows(d, rows, self.v_pool.data_ptr(), self.qv.data_ptr(), self.qvm.data_ptr(), _stream())
        self.nq = torch.as_tensor([int(x) for x in nq], dtype=torch.int32).to(dev)
        self.qc = vc_qcache(self.qk.data_ptr(), self.qkm.data_ptr(), self.qv.data_ptr(), self.qvm.data_ptr(),
                            self.row_off.data_ptr(), self.nq.data_ptr())

    def plan(self, max_rows=None, hint=True) -> None:
        """Builds the piece table of this cache on the host
        (viscache_decode_plan) and keeps a device copy for step_planned.  The
        length hint: the current lengths (hint True), none (False), or the
        given sequence."""
        self.plan_rows = self.max_cap if max_rows is None else int(max_rows)
        if hint is True:
            lens = self.len.cpu().tolist()
        elif hint is False or hint is None:
            lens = None
        else:
            lens = [int(x) for x in hint]
        blob = viscache_decode_plan(self.shape, self.caps_host, self.offs_host, self.plan_rows, lens)
        host = torch.frombuffer(bytearray(blob), dtype=torch.uint8)
        self.plan_dev = host.to(self.k_pool.device)
        self.plan_bytes = len(blob)

    def step_planned(self, k_new: torch.Tensor, v_new: torch.Tensor, q: torch.Tensor, out: torch.Tensor,
                     scale: float, q4: bool = False, max_rows=None) -> None:
        """step() (or step_q4() with q4) over the piece table of plan()
        (viscache_decode_step_planned)."""
        rows = self.plan_rows if max_rows is None else int(max_rows)
        viscache_decode_step_planned(self.shape, self.c, self.qc if q4 else None, self.plan_dev.data_ptr(),
                                     self.plan_bytes, k_new.data_ptr(), v_new.data_ptr(), q.data_ptr(),
                                     out.data_ptr(), scale, rows, self.step_ws.data_ptr(), self.step_ws_bytes,
                                     _stream())

    def step_q4(self, k_new: torch.Tensor, v_new: torch.Tensor, q: torch.Tensor, out: torch.Tensor,
                scale: float) -> None:
        """step() with each unit's quantised rows read from the 4-bit codes
        (viscache_decode_step_q4); quantize() first."""
        viscache_decode_step_q4(self.shape, self.c, self.qc, k_new.data_ptr(), v_new.data_ptr(), q.data_ptr(),
                                out.data_ptr(), scale, self.max_cap, self.step_ws.data_ptr(), self.step_ws_bytes,
                                _stream())


# ---- the 8-bit cache and the rotary positions ---------------------------------
# A call of a few microseconds on the GPU is soon bound by what is done for it
# here, so a tensor is looked at once and its vc_rows is packed as bytes.

_pack_rows = struct.Struct("5q").pack
assert ctypes.sizeof(vc_rows) == struct.calcsize("5q")
_pack_norm = struct.Struct("fi2q").pack
assert ctypes.sizeof(vc_norm) == struct.calcsize("fi2q")
_current_device = getattr(torch._C, "_cuda_getDevice", None)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_BF16, _FP32 = torch.bfloat16, torch.float32
_changed = torch._C._increment_version  # tensors written through their addresses


def _refuse(t, name, shape, typ, index):
    raise ValueError(f"{name}: {tuple(t.shape)} {t.dtype} on {t.device}, need {tuple(shape)} {typ} on GPU {index}")


def _take(t: torch.Tensor, name: str, shape, typ, index: int, head_major: bool = False) -> bytes:
    """The vc_rows of a tensor [L, B, n, H, d] ([L, B, H, n, d] with head_major) of
    this type and GPU and, unless that is known (None), this shape, its rows
    contiguous."""
    if (shape is not None and t.shape != shape) or t.dtype is not typ or t.get_device() != index or index < 0:
        shape = t.shape if shape is None else shape
        _refuse(t, name, shape, typ, index)
    s = t.stride()
    if s[4] != 1:
        raise ValueError(f"{name}: rows must be contiguous")
    if head_major:
        return _pack_rows(t.data_ptr(), s[0], s[1], s[3], s[2])
    return _pack_rows(t.data_ptr(), s[0], s[1], s[2], s[3])


def _ints(t, name: str, shape, index: int) -> int:
    """Address of a contiguous int32 tensor of this shape, unless that is known (0 for None)."""
    if t is None:
        return 0
    if (shape is not None and t.shape != shape) or t.dtype is not torch.int32 or t.get_device() != index or not t.is_contiguous():
        _refuse(t, name, t.shape if shape is None else shape, "contiguous int32", index)
    return t.data_ptr()


def _enqueue(name: str, f, index: int, *args) -> None:
    """f(*args, stream): the current stream of GPU `index`, as the current device."""
    if _current_device() == index:
        st = f(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            st = f(*args, _raw_stream(index))
    if st:
        raise VisCacheError(st, name)


def _no_tangents(*tensors) -> None:
    """Refuses tensors that carry a tangent (forward-mode autograd, which a call through
    addresses would leave as it was)."""
    for t in tensors:
        if t is not None and _forward.unpack_dual(t).tangent is not None:
            raise ValueError("a tensor carries a tangent: forward-mode autograd does not see the rotation")


class Rope:
    """Rotary positions with several axes (viscache_rope): head dim d, `rot`
    rotated channels (all by default), `sections` frequencies for time, height
    and width (one axis by default)."""

    def __init__(self, d: int, rot: int | None = None, theta: float = 1e6, sections=None, layout: int = 0,
                 pairing: int = 0, scale: float = 1.0, inv_freq=None):
        self.d, rot = int(d), int(d if rot is None else rot)
        sections = (rot // 2, 0, 0) if sections is None else tuple(int(x) for x in sections)
        self._freq = None
        if inv_freq is not None:
            if len(inv_freq) != rot // 2:
                raise ValueError(f"inv_freq: {len(inv_freq)} frequencies, need {rot // 2}")
            self._freq = (ctypes.c_double * (rot // 2))(*[float(x) for x in inv_freq])
        elif theta > 0:  # once, not in every call
            self._freq = (ctypes.c_double * (rot // 2))(*[float(theta) ** (-2.0 * i / rot) for i in range(rot // 2)])
        # By (fp32, inverse).
        self._params = [[vc_rope(rot, (ctypes.c_int32 * 3)(*sections), layout, pairing, fp32, inverse, scale, theta,
                                 self._freq) for inverse in (0, 1)] for fp32 in (0, 1)]
        self._address = [[ctypes.addressof(p) for p in row] for row in self._params]
        self._shapes = {}
        self._f = lib().viscache_rope

    def apply(self, pos, q=None, k=None, q_out=None, k_out=None, inverse: bool = False, count=None):
        """Rotates q [L, B, n, Hq, d] and k [L, B, n, Hkv, d] (either may be
        None; both bf16 or fp32) by pos int32 [3, B, n] into q_out and k_out, by
        default in place, on the current stream of their GPU.  count int32 [B]:
        the tokens of each sequence.  `inverse` turns back, which is the
        gradient.  Returns (q_out, k_out).  In one call Hq is a multiple of Hkv and at
        most 16 times it; other heads take a call for q and one for k.

        Autograd does not see the rotation, so tensors that require grad are refused
        where it records, and tensors with a tangent (a program calls this in the forward,
        backward and jvp of an autograd function of its own, or under no_grad); outputs
        count as changed in place."""
        if ((q is not None and q.requires_grad) or (k is not None and k.requires_grad) or
                (q_out is not None and q_out.requires_grad) or (k_out is not None and k_out.requires_grad)):
            if torch.is_grad_enabled():
                raise ValueError("a tensor requires grad: autograd does not see the rotation")
        if _forward._current_level >= 0:
            _no_tangents(q, k, q_out, k_out)
        return self._turn(pos, q, k, q_out, k_out, inverse, count)

    def _turn(self, pos, q, k, q_out, k_out, inverse=False, count=None):
        ref = q if q is not None else k
        if ref is None:
            raise ValueError("nothing to rotate")
        typ, index = ref.dtype, ref.get_device()
        L, B, n, Hq, d = was = ref.shape
        if (typ is not _BF16 and typ is not _FP32) or d != self.d:
            _refuse(ref, "q" if q is not None else "k", ref.shape[:-1] + (self.d,), "bf16 or fp32", max(index, 0))
        qi = qo = ki = ko = None
        Hkv = Hq  # of the one that there is
        if q is not None:
            qi = _take(q, "q", None, typ, index)
            qo = qi if q_out is None else _take(q_out, "q_out", was, typ, index)
        if k is not None:
            if k is not ref:
                was = k.shape
                Hkv = was[3] if len(was) == 5 else 0
                if was != (L, B, n, Hkv, d):
                    _refuse(k, "k", (L, B, n, "heads", d), typ, index)
            ki = _take(k, "k", None, typ, index)
            ko = ki if k_out is None else _take(k_out, "k_out", was, typ, index)
        cnt = _ints(count, "count", (B,), index)
        at = _ints(pos, "pos", (3, B, n), index)
        q_out, k_out = q if q_out is None else q_out, k if k_out is None else k_out
        if L == 0 or B == 0 or n == 0:
            return q_out, k_out
        key = (L, B, Hq, Hkv)
        shape = self._shapes.get(key)
        if shape is None:
            shape = vc_decode_shape(B, L, Hq, Hkv, d)
            shape = self._shapes[key] = ctypes.addressof(shape), shape
        _enqueue("viscache_rope", self._f, index, shape[0], self._address[typ is _FP32][bool(inverse)], n, at, cnt, qi,
                 qo, ki, ko)
        out = q_out, k_out
        _changed(out if q is not None and k is not None else (q_out,) if k is None else (k_out,))
        return out


class NormRope:
    """Norm of every query and key head, its weights and a rotation in one pass
    (viscache_norm_rope), and their gradient.  rope: the Rope that turns the normed
    rows."""

    def __init__(self, rope: Rope, eps: float = 1e-6):
        self.rope, self.d, self.eps = rope, rope.d, float(eps)
        self._bytes = {}
        self._lib = lib()

    def _weight(self, w, name, L, typ, index) -> int:
        """Address of contiguous weights [L, d]."""
        if w.shape != (L, self.d) or w.dtype is not typ or w.get_device() != index or not w.is_contiguous():
            _refuse(w, name, (L, self.d), f"contiguous {typ}", index)
        return w.data_ptr()

    def _call(self, pos, q, k, q_weight, k_weight, count):
        """What both directions look at: the shape's address, (L, B, n), the rows' type
        and GPU, the norm, and the addresses of pos and count."""
        ref = q if q is not None else k
        if ref is None:
            raise ValueError("no rows")
        if (q is None) != (q_weight is None) or (k is None) != (k_weight is None):
            raise ValueError("rows without their weights, or weights without their rows")
        typ, index = ref.dtype, ref.get_device()
        L, B, n, Hq, d = ref.shape
        if (typ is not _BF16 and typ is not _FP32) or d != self.d:
            _refuse(ref, "q" if q is not None else "k", ref.shape[:-1] + (self.d,), "bf16 or fp32", max(index, 0))
        Hkv = Hq  # of the one that there is
        if k is not None and k is not ref:
            Hkv = k.shape[3] if k.dim() == 5 else 0
            if k.shape != (L, B, n, Hkv, d):
                _refuse(k, "k", (L, B, n, "heads", d), typ, index)
        w = q_weight if q_weight is not None else k_weight
        wtyp = w.dtype
        if wtyp is not _BF16 and wtyp is not _FP32:
            _refuse(w, "q_weight" if q is not None else "k_weight", (L, self.d), "bf16 or fp32", index)
        at = _ints(pos, "pos", (3, B, n), index), _ints(count, "count", (B,), index)
        norm = _pack_norm(self.eps, wtyp is _FP32, 0 if q is None else self._weight(q_weight, "q_weight", L, wtyp, index),
                          0 if k is None else self._weight(k_weight, "k_weight", L, wtyp, index))
        shapes, key = self.rope._shapes, (L, B, Hq, Hkv)
        shape = shapes.get(key)
        if shape is None:
            shape = vc_decode_shape(B, L, Hq, Hkv, d)
            shape = shapes[key] = ctypes.addressof(shape), shape
        return shape[0], (L, B, n), typ, index, norm, at

    @staticmethod
    def _no_grad(*tensors) -> None:
        if torch.is_grad_enabled():
            for t in tensors:
                if t is not None and t.requires_grad:
                    raise ValueError("a tensor requires grad: autograd does not see the normed rotation")
        if _forward._current_level >= 0:
            _no_tangents(*tensors)

    def apply(self, pos, q=None, k=None, q_weight=None, k_weight=None, q_out=None, k_out=None, inverse: bool = False,
              count=None):
        """Norms q [L, B, n, Hq, d] and k [L, B, n, Hkv, d] (either may be None; both
        bf16 or fp32), multiplies them by their layers' q_weight and k_weight [L, d]
        (bf16 or fp32, both of one type) and turns them by pos int32 [3, B, n] into q_out
        and k_out, by default in place.  Every other argument, heads, streams and
        autograd as for Rope.apply: tensors that require grad are refused where it
        records, those with a tangent too, and a program calls apply and grad in an
        autograd function of its own.  Returns (q_out, k_out)."""
        self._no_grad(q, k, q_weight, k_weight, q_out, k_out)
        shape, (L, B, n), typ, index, norm, at = self._call(pos, q, k, q_weight, k_weight, count)
        qi = qo = ki = ko = None
        out = []
        if q is not None:
            qi = _take(q, "q", None, typ, index)
            qo = qi if q_out is None else _take(q_out, "q_out", q.shape, typ, index)
            q_out = q if q_out is None else q_out
            out.append(q_out)
        if k is not None:
            ki = _take(k, "k", None, typ, index)
            ko = ki if k_out is None else _take(k_out, "k_out", k.shape, typ, index)
            k_out = k if k_out is None else k_out
            out.append(k_out)
        if L == 0 or B == 0 or n == 0:
            return q_out, k_out
        _enqueue("viscache_norm_rope", self._lib.viscache_norm_rope, index, shape,
                 self.rope._address[typ is _FP32][bool(inverse)], norm, n, *at, qi, qo, ki, ko)
        _changed(out)
        return q_out, k_out

    def grad(self, pos, q=None, k=None, q_weight=None, k_weight=None, q_dout=None, k_dout=None, q_din=None, k_din=None,
             inverse: bool = False, count=None):
        """The gradient of apply with the same pos, q, k, weights, inverse and count, of
        which q and k are what went in: from the outputs' gradients q_dout and k_dout
        (the rows' type) to the rows' gradients, in q_din and k_din (by default new
        tensors; q or q_dout itself is allowed; rows of tokens past count are left as
        they were, in new tensors zeros), and the weights', new fp32 tensors [L, d].
        Sums are formed in an order that depends on the shape and count alone.
        Returns (q_din, k_din, q_dweight, k_dweight), None for a side without rows."""
        self._no_grad(q, k, q_weight, k_weight, q_dout, k_dout, q_din, k_din)
        shape, (L, B, n), typ, index, norm, at = self._call(pos, q, k, q_weight, k_weight, count)
        if (q is None) != (q_dout is None) or (k is None) != (k_dout is None):
            raise ValueError("rows without their outputs' gradients, or gradients without rows")
        new = torch.zeros_like if count is not None else torch.empty_like
        side, out, dw = [], [], []
        for x, w, g, o, name in ((q, q_weight, q_dout, q_din, "q"), (k, k_weight, k_dout, k_din, "k")):
            if x is None:
                side += (None, None, None, 0)
                out.append(None)
                dw.append(None)
                continue
            xr, gr = _take(x, name, None, typ, index), _take(g, name + "_dout", x.shape, typ, index)
            if o is None:
                o = new(x, memory_format=torch.contiguous_format)
            w = torch.empty_like(w, dtype=_FP32)  # contiguous, as the weights are
            side += (xr, gr, _take(o, name + "_din", x.shape, typ, index), w.data_ptr())
            out.append(o)
            dw.append(w)
        if L == 0:
            return (*out, *dw)
        if B == 0 or n == 0:
            return (*out, *[None if w is None else w.zero_() for w in dw])
        need = self._bytes.get((shape, n))
        if need is None:
            if len(self._bytes) >= 4096:
                self._bytes.clear()
            need = self._bytes[shape, n] = self._lib.viscache_norm_rope_grad_workspace_bytes(shape, n)
        # Of this call alone: the allocator orders its reuse after the stream's work.
        ws = (q if k is None else k).new_empty((max(need, 1),), dtype=torch.uint8)
        _enqueue("viscache_norm_rope_grad", self._lib.viscache_norm_rope_grad, index, shape,
                 self.rope._address[typ is _FP32][bool(inverse)], norm, n, *at, *side, ws.data_ptr(), need)
        _changed([o for o in out if o is not None])
        return (*out, *dw)


class _Attends:
    """What caches share whose attention takes a workspace: shape, device, row bound."""

    def _shaped(self, L, B, Hq, Hkv, d, caps, device) -> list:
        self.L, self.B, self.Hq, self.Hkv, self.d = L, B, Hq, Hkv, d
        self.shape = vc_decode_shape(B, L, Hq, Hkv, d)
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index if self.device.type == "cuda" else -1
        self.units = L * B * Hkv
        caps = [int(c) for c in caps]
        if len(caps) != self.units or min(caps, default=0) < 0:
            raise ValueError(f"{len(caps)} capacities, need {self.units}, none negative")
        self.max_cap = max(caps)
        self._ws, self._ws_of, self._kept = None, {}, []
        self._shape_at = ctypes.addressof(self.shape)
        self._lib = lib()
        return caps

    def _bind(self, need, buffers) -> list:
        """The buffers by the names and (shape, type) of `need`, as attributes; their addresses."""
        for name, (shape, t) in need.items():
            b = buffers[name]
            if b.shape != shape or b.dtype is not t or b.device != self.device or not b.is_contiguous():
                _refuse(b, name, shape, f"contiguous {t}", self._index)
            setattr(self, name, b)
        return [buffers[name].data_ptr() for name in need]

    def _workspace(self, n: int, max_rows: int):
        """(address, bytes) of the workspace, grown when a call needs more than any
        before it (a call that is captured into a graph must have run once)."""
        ws = self._ws_of.get((n, max_rows))
        if ws is None:
            need = self._needs(n, max_rows)
            had = 0 if self._ws is None else self._ws.numel()
            if self._ws is None or had < need:
                if torch.cuda.is_current_stream_capturing():
                    raise RuntimeError("the workspace is too small: run the call once before it is captured")
                # By half at least, so that all that are kept come to three times the largest.
                self._ws = torch.empty((max(need, had + had // 2),), dtype=torch.uint8, device=self.device)
                self._kept.append(self._ws)  # a graph captured before this goes on using the one it knows
                self._ws_of.clear()
            elif len(self._ws_of) >= 4096:  # bounds that change with every call
                self._ws_of.clear()
            ws = self._ws_of[n, max_rows] = self._ws.data_ptr(), self._ws.numel()
        return ws

    def _bound(self, max_rows) -> int:
        """The row bound of a call: no unit holds more rows than it has room for."""
        return self.max_cap if max_rows is None else min(_int32(max_rows), self.max_cap)


class Q8Cache(_Attends):
    """A decode cache in 8 bits (viscache_q8_*) over L layers x B sequences x
    Hkv heads: unit u = (l*B + b)*Hkv + g has room for caps[u] rows.  format:
    "int8" or "e4m3".  `buffers`: the cache's tensors by name (k_codes, v_codes,
    k_scale, v_scale, k_tail, v_tail, row_off, cap, len), laid out as vc_q8cache
    has them, where a program keeps them itself; row_off and cap have to hold the
    units' first rows, whole blocks one unit after the other, and caps (they are
    not read back to be checked).

    How a call's rows go to workgroups, and which units single tokens start with,
    follow from the capacities, not from the lengths, which only the device knows;
    a program that knows a bound well below the capacities passes it as max_rows
    (8 units with room for 32000 rows and 1024 in each: a step 15.0 us, 11.3 with
    max_rows = 1088; attention 12.2, 10.1).

    A program may lower `len` itself to take rows back, to a multiple of 64 or
    within the open block; no other length can be gone back to.

    Calls go to the current stream of the cache's device.  Calls that attend
    share one workspace and must not overlap."""

    FORMATS = {"int8": (VC_Q8_INT8, torch.int8), "e4m3": (VC_Q8_E4M3, torch.float8_e4m3fn)}

    def __init__(self, L, B, Hq, Hkv, d, caps, device, format: str = "e4m3", buffers=None):
        caps = self._shaped(L, B, Hq, Hkv, d, caps, device)
        code, typ = self.FORMATS[format]
        self.format = format
        offs, o = [], 0
        for c in caps:
            offs.append(o)
            o += (c + VC_Q8_BLOCK - 1) // VC_Q8_BLOCK
        nblk = max(o, 1)
        need = {"k_codes": ((nblk, VC_Q8_BLOCK, d), typ), "v_codes": ((nblk, d, VC_Q8_BLOCK), typ),
                "k_scale": ((nblk,), torch.float32), "v_scale": ((nblk,), torch.float32),
                "k_tail": ((self.units, VC_Q8_BLOCK, d), torch.bfloat16),
                "v_tail": ((self.units, VC_Q8_BLOCK, d), torch.bfloat16),
                "row_off": ((self.units,), torch.int64), "cap": ((self.units,), torch.int32),
                "len": ((self.units,), torch.int32)}
        if buffers is None:
            buffers = {name: torch.zeros(shape, dtype=t, device=self.device) for name, (shape, t) in need.items()}
            buffers["row_off"] = torch.tensor(offs, dtype=torch.int64, device=self.device) * VC_Q8_BLOCK
            buffers["cap"] = torch.tensor(caps, dtype=torch.int32, device=self.device)
        at = self._bind(need, buffers)
        # Attention starts on the units with the most room first.
        order = sorted(range(self.units), key=lambda u: -caps[u])
        self.order = torch.tensor(order, dtype=torch.int32, device=self.device) if len(set(caps)) > 1 else None
        self.c = vc_q8cache(code, *at, 0 if self.order is None else self.order.data_ptr())
        self._cache_at = ctypes.addressof(self.c)

    def _needs(self, n: int, max_rows: int) -> int:
        return viscache_q8_attend_workspace_bytes(self.shape, n, max_rows)

    def append(self, k, v, count=None, head_major: bool = False) -> None:
        """Appends k, v bf16 [L, B, n, Hkv, d] ([L, B, Hkv, n, d] with
        head_major); count int32 [L*B]: the rows of each layer and sequence."""
        kr, vr, n = self._pair(k, v, head_major, _BF16)
        cnt = _ints(count, "count", (self.L * self.B,), self._index)
        if n == 0:
            return
        _enqueue("viscache_q8_append", self._lib.viscache_q8_append, self._index, self._shape_at, self._cache_at, kr,
                 vr, n, cnt, 0)

    def _pair(self, k, v, head_major, typ):
        """The descriptors of keys and values [L, B, n, Hkv, d] (or [L, B, Hkv, n, d]), and n."""
        was = k.shape
        n = was[3 if head_major else 2]
        want = (self.L, self.B, self.Hkv, n, self.d) if head_major else (self.L, self.B, n, self.Hkv, self.d)
        if was != want:
            _refuse(k, "k", want, typ, self._index)
        return (_take(k, "k", None, typ, self._index, head_major), _take(v, "v", want, typ, self._index, head_major),
                _int32(n))

    def load_pruned(self, pc: "PruneCall") -> None:
        """Appends what pc.run() left in its outputs (bf16 values): every
        layer's kept rows, a launch or two a layer.  Evicted layers get none.  Refused,
        with nothing appended, where a unit has too little room (the lengths are read
        back for that, so not in a capture)."""
        if (pc.L, pc.B, pc.Hkv, pc.d) != (self.L, self.B, self.Hkv, self.d) or pc.params.v_out_fp32:
            raise ValueError("the pruned cache has another shape, or fp32 values")
        per = self.B * self.Hkv
        one = vc_decode_shape(self.B, 1, self.Hq, self.Hkv, self.d)
        count = torch.tensor([[pc.k[b * pc.L + l] for b in range(pc.B)] for l in range(pc.L)], dtype=torch.int32)
        off = torch.tensor([[pc.unit_rows(l, b, g)[0] * self.d for b in range(pc.B) for g in range(pc.Hkv)]
                            for l in range(pc.L)], dtype=torch.int64)
        most = count.amax(dim=1).tolist()
        if any(m and t.get_device() != self._index for m, t in zip(most, pc.k_out)):
            raise ValueError("the pruned cache is on another device")
        room = (self.cap - self.len).cpu().view(self.L, self.B, self.Hkv)
        lacks = ((count[..., None] > room) & (count[..., None] > 0)).flatten().nonzero().flatten()
        if len(lacks):
            u = int(lacks[0])
            raise ValueError(f"unit {u} has room for {max(int(room.flatten()[u]), 0)} rows of "
                             f"{int(count.flatten()[u // self.Hkv])}, and {len(lacks) - 1} others have too little")
        count, off = count.to(self.device), off.to(self.device)
        with torch.cuda.device(self._index):
            stream = _raw_stream(self._index)
            for l in range(pc.L):
                if most[l] == 0:
                    continue
                c = vc_q8cache(self.c.format, self.c.k_codes, self.c.v_codes, self.c.k_scale, self.c.v_scale,
                               self.k_tail[l * per:].data_ptr(), self.v_tail[l * per:].data_ptr(),
                               self.row_off[l * per:].data_ptr(), self.cap[l * per:].data_ptr(),
                               self.len[l * per:].data_ptr(), 0)
                k = vc_rows(pc.k_out[l].data_ptr(), 0, 0, self.d, 0)
                v = vc_rows(pc.v_out[l].data_ptr(), 0, 0, self.d, 0)
                viscache_q8_append(one, c, k, v, most[l], count[l].data_ptr(), off[l].data_ptr(), stream)

    def read(self, k, v, max_rows=None, head_major: bool = False) -> None:
        """Reads rows [0, len) of every unit back into k, v (bf16 or fp32)
        [L, B, rows, Hkv, d] ([L, B, Hkv, rows, d] with head_major); rows behind
        them are left as they were.  max_rows: by default, as many as k holds."""
        typ = k.dtype
        if typ is not _BF16 and typ is not _FP32:
            _refuse(k, "k", k.shape, "bf16 or fp32", self._index)
        kr, vr, rows = self._pair(k, v, head_major, typ)
        m = rows if max_rows is None else _int32(max_rows)
        if m > rows:
            raise ValueError(f"max_rows {m} exceeds the {rows} rows of k")
        if rows == 0:
            return
        _enqueue("viscache_q8_read", self._lib.viscache_q8_read, self._index, self._shape_at, self._cache_at, m, kr, vr,
                 0, int(typ is _FP32))

    def attend(self, q, out, scale: float, count=None, causal: bool = True, max_rows=None) -> None:
        """Attention of q bf16 [L, B, n, Hq, d] over the cache into out (bf16 or
        fp32, the same shape); count int32 [B]: the queries of each sequence.
        max_rows: rows past it are not attended (by default, and at most, the largest
        capacity)."""
        was = q.shape
        n = was[2]
        want = (self.L, self.B, n, self.Hq, self.d)
        if was != want:
            _refuse(q, "q", want, _BF16, self._index)
        fp32 = out.dtype is _FP32
        qr, outr = _take(q, "q", None, _BF16, self._index), _take(out, "out", want, _FP32 if fp32 else _BF16, self._index)
        cnt = _ints(count, "count", (self.B,), self._index)
        if n == 0:
            return
        rows = self._bound(max_rows)
        ws = self._workspace(n, rows)
        _enqueue("viscache_q8_attend", self._lib.viscache_q8_attend, self._index, self._shape_at, self._cache_at, qr,
                 outr, n, cnt, int(causal), int(fp32), scale, rows, ws[0], ws[1])

    def step(self, q, k, v, out, scale: float, rope: Rope | None = None, pos=None, q_out=None, k_out=None,
             max_rows=None) -> None:
        """A serving step: rotates q and k by pos int32 [3, B, n] (with `rope`),
        appends k and v and attends q.  One token (n = 1) is a single call
        (viscache_q8_step), which turns q and k on its way; several tokens are three
        calls, and so is one whose rotated rows are asked for, in q_out or k_out.
        q, k and v are left as they are, unless one of those is q or k.  max_rows as
        for attend; it bounds what is attended, not what is appended."""
        n, index, most = q.shape[2], self._index, self._bound(max_rows)
        if n != 1 or (rope is not None and (q_out is not None or k_out is not None)):
            # All of it is looked at before anything is appended.
            want = (self.L, self.B, n, self.Hq, self.d)
            _take(q, "q", want, _BF16, index)
            _take(out, "out", want, _FP32 if out.dtype is _FP32 else _BF16, index)
            self._pair(k, v, False, _BF16)
            if k.shape[2] != n:
                raise ValueError(f"{k.shape[2]} new rows for {n} queries")
            if rope is not None:
                q_out = torch.empty_like(q) if q_out is None else q_out
                k_out = torch.empty_like(k) if k_out is None else k_out
            if n > 0:
                # Without a workspace attention launches nothing and says so last.
                fp32, qr = out.dtype is _FP32, _take(q if rope is None else q_out, "q_out", want, _BF16, index)
                st = self._lib.viscache_q8_attend(self._shape_at, self._cache_at, qr, _take(out, "out", None, out.dtype, index),
                                                  n, 0, 1, int(fp32), scale, most, 0, 0, 0)
                if st != VC_ERR_WORKSPACE:
                    raise VisCacheError(st, "viscache_q8_attend")
                self._workspace(n, most)
            if rope is not None:
                q, k = rope._turn(pos, q, k, q_out, k_out)
            self.append(k, v)
            self.attend(q, out, scale, max_rows=most)
            return
        want, kv = (self.L, self.B, 1, self.Hq, self.d), (self.L, self.B, 1, self.Hkv, self.d)
        fp32 = out.dtype is _FP32
        rows = (_take(q, "q", want, _BF16, index), _take(k, "k", kv, _BF16, index), _take(v, "v", kv, _BF16, index),
                _take(out, "out", want, _FP32 if fp32 else _BF16, index))
        turn, at = 0, 0
        if rope is not None:
            if rope.d != self.d or pos is None:
                raise ValueError("the rotation is of another head dim, or has no positions")
            turn, at = rope._address[0][0], _ints(pos, "pos", (3, self.B, 1), index)
        ws = self._workspace(1, most)
        _enqueue("viscache_q8_step", self._lib.viscache_q8_step, index, self._shape_at, self._cache_at, turn, at, *rows,
                 int(fp32), scale, most, ws[0], ws[1])


class MassCache(_Attends):
    """A bf16 decode cache that keeps what its rows were given (viscache_mass_*) over L
    layers x B sequences x Hkv heads: unit u = (l*B + b)*Hkv + g has room for caps[u]
    rows, and `mass` holds for each row the attention weight it got so far.  `buffers`:
    the cache's tensors by name (k_pool, v_pool [rows, d], mass [rows], row_off, cap,
    len), where a program keeps them itself; row_off and cap have to hold the units'
    first rows, one unit after the other, and caps (they are not read back to be
    checked).

    How a call's rows go to workgroups, and which units single tokens start with, follow
    from the capacities, not from the lengths, which only the device knows; a program
    that knows a bound well below the capacities passes it as max_rows.

    Calls go to the current stream of the cache's device.  Calls on one cache share a
    workspace and must not overlap.  Autograd records nothing of them, whether their
    tensors require grad or not: outputs and masses are numbers without a history."""

    def __init__(self, L, B, Hq, Hkv, d, caps, device, buffers=None):
        caps = self._shaped(L, B, Hq, Hkv, d, caps, device)
        offs, o = [], 0
        for c in caps:
            offs.append(o)
            o += c
        rows, units = max(o, 1), self.units
        need = {"k_pool": ((rows, d), _BF16), "v_pool": ((rows, d), _BF16), "mass": ((rows,), _FP32),
                "row_off": ((units,), torch.int64), "cap": ((units,), torch.int32), "len": ((units,), torch.int32)}
        if buffers is None:
            buffers = {name: torch.zeros(shape, dtype=t, device=self.device) for name, (shape, t) in need.items()}
            buffers["row_off"] = torch.tensor(offs, dtype=torch.int64, device=self.device)
            buffers["cap"] = torch.tensor(caps, dtype=torch.int32, device=self.device)
        at = self._bind(need, buffers)
        # Attention of single tokens starts on the units with the most room first.
        order = sorted(range(units), key=lambda u: -caps[u])
        self.order = torch.tensor(order, dtype=torch.int32, device=self.device) if len(set(caps)) > 1 else None
        self.c = vc_mass_cache(*at, 0 if self.order is None else self.order.data_ptr())
        self._cache_at = ctypes.addressof(self.c)

    def _needs(self, n: int, max_rows: int) -> int:
        """Of n queries, or (-1) of an eviction."""
        if n < 0:
            return viscache_mass_evict_workspace_bytes(self.shape, max_rows)
        return viscache_mass_attend_workspace_bytes(self.shape, n, max_rows)

    def attend(self, q, out, scale: float, k=None, v=None, count=None, decay: float = 1.0, max_rows=None) -> None:
        """Attention of q bf16 [L, B, n, Hq, d] over the cache into out (bf16 or fp32,
        the same shape), every row's mass fading by `decay` and growing by what the row
        was given.  With k and v bf16 [L, B, n, Hkv, d] their rows are appended first (a
        serving step); without them the cache's newest rows are the queries' own.  count
        int32 [B]: the tokens of each sequence.  max_rows: rows past it are not attended
        (by default, and at most, the largest capacity)."""
        was = q.shape
        n, index = was[2], self._index
        want = (self.L, self.B, n, self.Hq, self.d)
        if was != want:
            _refuse(q, "q", want, _BF16, index)
        fp32 = out.dtype is _FP32
        qr, outr = _take(q, "q", None, _BF16, index), _take(out, "out", want, _FP32 if fp32 else _BF16, index)
        if (k is None) != (v is None):
            raise ValueError("keys without values, or values without keys")
        kr = vr = None
        if k is not None:
            kv = (self.L, self.B, n, self.Hkv, self.d)
            kr, vr = _take(k, "k", kv, _BF16, index), _take(v, "v", kv, _BF16, index)
        cnt = _ints(count, "count", (self.B,), index)
        if n == 0:
            return
        rows = self._bound(max_rows)
        ws = self._workspace(n, rows)
        _enqueue("viscache_mass_attend", self._lib.viscache_mass_attend, index, self._shape_at, self._cache_at, kr, vr,
                 qr, outr, n, cnt, int(fp32), scale, decay, rows, ws[0], ws[1])

    def evict(self, keep, sinks: int = 0, recent: int = 0, to: "MassCache | None" = None, index=None,
              max_rows=None) -> None:
        """Every unit keeps keep[u] (int32 [units]) of its rows: the first `sinks`, the
        last `recent` and of the others those of the largest mass (ties to the lower
        index), in order, with their masses; in place, or into `to`, a cache of the
        same shape with rows of its own, which bounds keep by its capacities and leaves
        this one as it was.  index int32 [units, rows]: where the kept rows came from
        (entries past them are left as they were).  max_rows: rows past it are evicted
        (by default, and at most, the largest capacity)."""
        at, idx = _ints(keep, "keep", (self.units,), self._index), _ints(index, "index", None, self._index)
        if keep is None:
            raise ValueError("keep: the rows that each unit keeps")
        if index is not None and (index.dim() != 2 or index.shape[0] != self.units):
            _refuse(index, "index", (self.units, "rows"), "contiguous int32", self._index)
        if to is not None and (to.L, to.B, to.Hkv, to.d, to.device) != (self.L, self.B, self.Hkv, self.d, self.device):
            raise ValueError("the other cache has another shape or device")
        wide = 0 if index is None else index.shape[1]
        rows = self._bound(max_rows)
        ws = self._workspace(-1, rows)
        _enqueue("viscache_mass_evict", self._lib.viscache_mass_evict, self._index, self._shape_at, self._cache_at,
                 None if to is None else to._cache_at, at, _int32(sinks), _int32(recent), rows, idx, wide, ws[0], ws[1])


__all__ = ["PruneCall", "DecodeCache", "Q8Cache", "Rope", "NormRope", "MassCache", "make_params"]
