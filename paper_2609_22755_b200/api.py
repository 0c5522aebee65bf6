"""User-facing wrapper: one object per packed batch that owns the plan and the device buffers and runs the
forward + backward of the local attention compute phase through the C ABI.

Only marshalling lives here. ``step_device`` runs on tensors already resident on the GPU; ``step_host`` is the
end-to-end call (nsp_attn_step_host): Q, K, V, dO come from (pinned) host tensors and O, LSE, dQ, dK, dV go back to
host tensors; the library makes the copies on a second stream under the kernels where the data dependencies allow.
With ``rope`` the queries and keys are rotated by their positions on the way in and the gradients dQ and dK on the way back, in
place, as the backward pass has left them: gradients in bf16 are then rounded a second time (``dq_dtype`` and ``dkv_dtype`` "f32"
have one rounding, to fp32).
"""
from __future__ import annotations

from . import binding as B


class Rotary:
    """Rotary positions of a model: frequencies (float64, radians per position), which elements of a head are pairs, and the
    factor on sine and cosine. kind, scale, trained_tokens, fast_turns, slow_turns: scaling for long contexts (see
    nsp_rope_frequencies)."""

    def __init__(self, rot_dim, base=10000.0, layout=B.NSP_ROPE_HALF, **scaling):
        self.inv_freq, self.magnitude = B.nsp_rope_frequencies(rot_dim, base, **scaling)
        self.layout = layout

    def rotate(self, xs, ys, positions, inverse=False, stream=None):
        """See nsp_rope; inverse: the way back of gradients."""
        B.nsp_rope(xs, ys, positions, self.inv_freq, layout=self.layout, magnitude=self.magnitude, inverse=inverse, stream=stream)


def packed_runs(workload):
    """The dense pieces of a batch's packed tensors: (first segment, segments behind the last, tokens, hq, hkv) of every maximal
    range of consecutive segments with equal head counts."""
    runs, L = [], workload.lengths
    for s in range(workload.n_seg):
        hq, hkv = int(workload.hq[s]), int(workload.hkv[s])
        if runs and runs[-1][3:] == (hq, hkv):
            first, _, tokens = runs[-1][:3]
            runs[-1] = (first, s + 1, tokens + int(L[s]), hq, hkv)
        else:
            runs.append((s, s + 1, int(L[s]), hq, hkv))
    return runs


class NspAttention:
    def __init__(self, workload, device="cuda:0", dq_dtype="bf16", dkv_dtype="f32", stream=None, rope=None, positions=None):
        """rope: a Rotary; q and k are then the unrotated ones, and dq and dk their gradients. positions: int64 tensor with one
        entry per packed token (default: every segment counts from 0)."""
        import torch

        self.torch = torch
        self.w = workload
        self.dev = torch.device(device)
        torch.cuda.set_device(self.dev)
        self.stream = stream
        self.plan = B.nsp_plan_tiles(workload.cu_seqlens, workload.hq, workload.hkv, workload.head_dim, stream=stream)
        qe, kve, le = self.plan.q_elems, self.plan.kv_elems, self.plan.lse_elems
        bf, f32 = torch.bfloat16, torch.float32
        mk = lambda n, dt: torch.empty(n, dtype=dt, device=self.dev)
        self.q, self.k, self.v, self.do = mk(qe, bf), mk(kve, bf), mk(kve, bf), mk(qe, bf)
        self.o, self.lse = mk(qe, bf), mk(le, f32)
        self.dq = mk(qe, f32 if dq_dtype == "f32" else bf)
        self.dk = mk(kve, f32 if dkv_dtype == "f32" else bf)
        self.dv = mk(kve, f32 if dkv_dtype == "f32" else bf)
        self.ws = torch.empty(max(self.plan.bwd_ws_bytes, 256), dtype=torch.uint8, device=self.dev)
        self.scale = workload.softmax_scale
        self.rope = rope
        if rope is not None:
            self._prepare_rope(positions)

    def _prepare_rope(self, positions):
        t, w, D = self.torch, self.w, self.w.head_dim
        if positions is None:
            positions = t.cat([t.arange(int(n)) for n in w.lengths] or [t.empty(0, dtype=t.int64)])
        total = int(w.lengths.sum())
        if positions.dtype != t.int64 or positions.shape != (total,):
            raise ValueError("positions: int64, one entry per packed token")
        self.positions = positions.to(self.dev)
        self.q_rot, self.k_rot = t.empty_like(self.q), t.empty_like(self.k)
        qo, ko, cu = w.q_offsets(), w.kv_offsets(), w.cu_seqlens

        def views(q, k):  # of every run, query and key side by side
            out = []
            for first, last, n, hq, hkv in packed_runs(w):
                out += [q[qo[first]:qo[last]].view(n, hq, D), k[ko[first]:ko[last]].view(n, hkv, D)]
            return out

        self._run_positions = [p for first, last, n, hq, hkv in packed_runs(w) for p in [self.positions[cu[first]:cu[last]]] * 2]
        self._rope_in, self._rope_out = views(self.q, self.k), views(self.q_rot, self.k_rot)
        self._rope_grads = views(self.dq, self.dk)

    # ---- data movement
    def load(self, host):
        """Copy Q, K, V, dO from host tensors (dict with keys q, k, v, do)."""
        for name, dst in (("q", self.q), ("k", self.k), ("v", self.v), ("do", self.do)):
            dst.copy_(host[name], non_blocking=True)
        return sum(host[n].numel() * host[n].element_size() for n in ("q", "k", "v", "do"))

    def store(self, host_out):
        """Copy O, LSE, dQ, dK, dV to host tensors (dict with keys o, lse, dq, dk, dv)."""
        n = 0
        for name, src in (("o", self.o), ("lse", self.lse), ("dq", self.dq), ("dk", self.dk), ("dv", self.dv)):
            host_out[name].copy_(src, non_blocking=True)
            n += src.numel() * src.element_size()
        return n

    def alloc_host_outputs(self):
        t = self.torch
        return {name: t.empty(src.shape, dtype=src.dtype, pin_memory=True)
                for name, src in (("o", self.o), ("lse", self.lse), ("dq", self.dq), ("dk", self.dk), ("dv", self.dv))}

    # ---- compute
    def _qk(self):
        """The queries and keys that attention reads."""
        return (self.q, self.k) if self.rope is None else (self.q_rot, self.k_rot)

    def _rotate_in(self):
        if self.rope is not None:
            self.rope.rotate(self._rope_in, self._rope_out, self._run_positions, stream=self.stream)

    def forward(self):
        self._rotate_in()
        q, k = self._qk()
        B.nsp_attn_fwd(self.plan, q, k, self.v, self.o, self.lse, self.scale, stream=self.stream)

    def backward(self, recompute=None):
        """recompute: optional uint8 flags per segment (see nsp_recompute_mark): O and LSE of a flagged segment are
        not read, the backward pass recomputes what it needs of them. With ``rope`` the rotated queries and keys are the
        forward pass's; where there are flags they are made anew, so that q and k are all that a flagged segment needs."""
        if recompute is not None:
            self._rotate_in()
        q, k = self._qk()
        if recompute is None:
            B.nsp_attn_bwd(self.plan, q, k, self.v, self.o, self.do, self.lse, self.dq, self.dk, self.dv,
                           self.scale, self.ws, stream=self.stream)
        else:
            need = B.nsp_plan_recompute_ws_bytes(self.plan)
            if self.ws.numel() < need:
                self.ws = self.torch.empty(need, dtype=self.torch.uint8, device=self.dev)
            B.nsp_attn_bwd_recompute(self.plan, recompute, q, k, self.v, self.o, self.do, self.lse, self.dq,
                                     self.dk, self.dv, self.scale, self.ws, stream=self.stream)
        if self.rope is not None:
            self.rope.rotate(self._rope_grads, self._rope_grads, self._run_positions, inverse=True, stream=self.stream)

    def step_device(self):
        self.forward()
        self.backward()

    def step_host(self, host_in, host_out):
        """End to end: host tensors in (dict with q, k, v, do), host tensors out (dict with o, lse, dq, dk, dv), through
        the library's host-buffer entry point nsp_attn_step_host: the copies run on the plan's second stream, so that
        dO travels to the device while the forward pass runs and O / LSE travel back while the backward pass runs.
        The device copies live in a workspace of this object's own (not in the tensors step_device uses).
        Returns (host-to-device bytes, device-to-host bytes). The call returns without waiting for the device. Not with
        ``rope``: that entry point takes queries and keys as attention reads them."""
        if self.rope is not None:
            raise B.NspError(B.NSP_ERR_UNSUPPORTED, "step_host with rope")
        if getattr(self, "_host_ws", None) is None:
            dq_dt = B.NSP_F32 if host_out["dq"].dtype == self.torch.float32 else B.NSP_BF16
            dkv_dt = B.NSP_F32 if host_out["dk"].dtype == self.torch.float32 else B.NSP_BF16
            need = B.nsp_plan_step_host_ws_bytes(self.plan, dq_dt, dkv_dt)
            self._host_ws = self.torch.empty(max(need, 256), dtype=self.torch.uint8, device=self.dev)
        return B.nsp_attn_step_host(self.plan, host_in["q"], host_in["k"], host_in["v"], host_in["do"], host_out["o"],
                                    host_out["lse"], host_out["dq"], host_out["dk"], host_out["dv"], self.scale,
                                    self._host_ws, stream=self.stream)

    def status(self):
        return B.nsp_device_status(self.plan)
