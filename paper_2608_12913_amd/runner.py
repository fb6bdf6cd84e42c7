"""Device buffers for one verification problem and calls through the C ABI.

PyTorch only allocates device memory and provides the stream; every step of the
verification runs in libdcd's kernels (through :mod:`paper_2608_12913_amd.dcd`).
"""
from __future__ import annotations

import numpy as np
import torch

from . import dcd


def _dev(a: np.ndarray, device) -> torch.Tensor:
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:  # bf16 bit patterns
        return torch.from_numpy(a.view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(a).to(device)


class DeviceProblem:
    """Inputs, outputs and workspace of one problem, resident on `device`."""

    def __init__(self, *, hp, hq, wp, wq, bias_p, bias_q, parents, tokens, B, N, V, dtype,
                 theta, s, T=1.0, draft_probs=None, u_acc=None, u_res=None, device="cuda:0",
                 row_outputs=True, norm_p=None, norm_q=None, norm_eps=0.0):
        self.device = torch.device(device)
        dv = lambda a: None if a is None else _dev(a, self.device)  # noqa: E731
        self.B, self.N, self.V = B, N, V
        self.hp, self.hq, self.wp, self.wq = dv(hp), dv(hq), dv(wp), dv(wq)
        self.bias_p = dv(None if bias_p is None else np.asarray(bias_p, np.float32))
        self.bias_q = (self.bias_p if bias_q is bias_p
                       else dv(None if bias_q is None else np.asarray(bias_q, np.float32)))
        self.parents = dv(np.asarray(parents, np.int32).reshape(B, N))
        self.tokens = dv(np.asarray(tokens, np.int32).reshape(B, N))
        self.draft_probs = dv(None if draft_probs is None else np.asarray(draft_probs, np.float32))
        self.u_acc = dv(None if u_acc is None else np.asarray(u_acc, np.float32))
        self.u_res = dv(None if u_res is None else np.asarray(u_res, np.float32))
        # norm_p / norm_q: scales of the models' final RMS normalisation; hp / hq are
        # then the rows before it
        self.norm_p, self.norm_q = dv(norm_p), dv(norm_q)
        final_norm = norm_p is not None
        self.problem = dcd.make_problem(B, N, V, hp.shape[1], hq.shape[1], dtype, theta, s, T,
                                        final_norm, norm_eps)
        R = B * N
        i32 = dict(dtype=torch.int32, device=self.device)
        f32 = dict(dtype=torch.float32, device=self.device)
        self.accept_len = torch.empty(B, **i32)
        self.accept_path = torch.empty(B, N, **i32)
        self.next_token = torch.empty(B, **i32)
        self.status = torch.empty(B, **i32)
        self.row_argmax = torch.empty(R, **i32) if row_outputs else None
        self.row_stats = torch.empty(R, 8, **f32) if row_outputs else None
        self.node_stats = torch.empty(R, 6, **f32) if row_outputs else None
        self.row_argmax_expert = torch.empty(R, **i32) if row_outputs else None
        self.row_kl = torch.empty(R, 2, **f32) if row_outputs else None
        self.ws_bytes = dcd.workspace_bytes(self.problem)
        if self.ws_bytes == 0:
            raise dcd.DcdError(dcd.DCD_ERR_SHAPE)
        # zero-filled once: its first words are the call count the library keeps
        self.workspace = torch.zeros(self.ws_bytes, dtype=torch.uint8, device=self.device)
        self.inputs = dcd.make_inputs(self.hp, self.hq, self.wp, self.wq, self.bias_p, self.bias_q,
                                      self.parents, self.tokens, self.norm_p, self.norm_q)
        self.outputs = dcd.make_outputs(self.accept_len, self.accept_path, self.next_token,
                                        self.status, self.row_argmax, self.row_stats,
                                        self.node_stats, self.row_argmax_expert, self.row_kl)

    @classmethod
    def from_case(cls, case, tokens, draft_probs=None, device="cuda:0", row_outputs=True,
                  **overrides):
        kw = dict(hp=case.hp, hq=case.hq, wp=case.wp, wq=case.wq, bias_p=case.bias,
                  bias_q=case.bias, parents=case.parents, tokens=tokens, B=case.B, N=case.N,
                  V=case.V, dtype=case.dtype, theta=case.theta, s=case.s, T=case.T,
                  draft_probs=draft_probs, u_acc=case.u_acc, u_res=case.u_res, device=device,
                  row_outputs=row_outputs)
        kw.update(overrides)
        return cls(**kw)

    def set_tokens(self, tokens):
        self.tokens.copy_(torch.from_numpy(np.asarray(tokens, np.int32).reshape(self.B, self.N)))

    def launch(self, mode: str, stream=None) -> None:
        """Enqueue one verification on `stream` (default: torch's current stream)."""
        if stream is None:
            stream = torch.cuda.current_stream(self.device)
        if mode == "greedy":
            dcd.verify_greedy(self.problem, self.inputs, self.outputs, self.workspace,
                              self.ws_bytes, stream)
        else:
            dcd.verify_sample(self.problem, self.inputs, self.draft_probs, self.u_acc, self.u_res,
                              self.outputs, self.workspace, self.ws_bytes, stream)

    def propose(self, u, want_probs=True) -> dict:
        """dcd_propose on this problem's heads (the expert slots hold one drafter head,
        the amateur slots the other); synchronous, host copies of the outputs."""
        R, V = self.B * self.N, self.V
        i32 = dict(dtype=torch.int32, device=self.device)
        u = torch.from_numpy(np.asarray(u, np.float32)).to(self.device)
        tokens, argmax = torch.empty(R, **i32), torch.empty(R, **i32)
        probs = torch.empty(R, V, dtype=torch.float32, device=self.device) if want_probs else None
        dcd.propose(self.problem, self.inputs, u, tokens, probs, argmax, self.workspace,
                    self.ws_bytes, torch.cuda.current_stream(self.device))
        torch.cuda.synchronize(self.device)
        out = dict(tokens=tokens.cpu().numpy(), argmax=argmax.cpu().numpy())
        if probs is not None:
            out["probs"] = probs.cpu().numpy()
        return out

    def launch_lmhead(self, mode: str, stream=None) -> None:
        """Enqueue only the LM-head projection stage (the dominant kernel)."""
        if stream is None:
            stream = torch.cuda.current_stream(self.device)
        dcd.lmhead_partials(self.problem, self.inputs, mode == "sample", self.workspace,
                            self.ws_bytes, stream)

    def run(self, mode: str) -> dict:
        """One synchronous verification; returns host copies of every output."""
        self.launch(mode)
        torch.cuda.synchronize(self.device)
        out = dict(accept_len=self.accept_len.cpu().numpy(),
                   accept_path=self.accept_path.cpu().numpy(),
                   next_token=self.next_token.cpu().numpy(), status=self.status.cpu().numpy())
        if self.row_argmax is not None:
            out.update(row_argmax=self.row_argmax.cpu().numpy(),
                       row_stats=self.row_stats.cpu().numpy(),
                       node_stats=self.node_stats.cpu().numpy(),
                       row_argmax_expert=self.row_argmax_expert.cpu().numpy(),
                       row_kl=self.row_kl.cpu().numpy())
        return out


class DraftHead:
    """A drafter's LM head held in 8-bit codes, with the buffers for up to `max_rows` hidden states:
    a token per row, drawn with that row's rules, and the distribution it was drawn from.

    w: [V, d] bf16 or fp32 (a tensor, or numpy as in :class:`DeviceProblem`); its codes and scales
    are made here, once.  A step is three kernels' calls (codes of the hidden states, logits,
    sampling); it allocates nothing and can be captured into a graph.  Calls share the buffers: run
    them in stream order.
    """

    def __init__(self, w, bias=None, *, max_rows, logits_dtype="f32", device="cuda:0"):
        w = (w if torch.is_tensor(w) else _dev(w, device)).to(device).contiguous()
        self.device = w.device
        self.V, self.d = w.shape
        self.max_rows, self.logits_dtype = int(max_rows), logits_dtype
        if bias is not None:
            bias = torch.as_tensor(bias).to(self.device, torch.float32).contiguous()
            if bias.shape != (self.V,):
                raise ValueError(f"bias {tuple(bias.shape)} for {self.V} tokens")
        self.bias = bias
        groups = -(-self.d // 128)
        u8 = dict(dtype=torch.uint8, device=self.device)
        f32 = dict(dtype=torch.float32, device=self.device)
        self.w, self.w_scale = torch.empty(self.V, self.d, **u8), torch.empty(-(-self.V // 128), groups, **f32)
        self.h, self.h_scale = torch.empty(self.max_rows, self.d, **u8), torch.empty(self.max_rows, groups, **f32)
        self.logits = torch.empty(self.max_rows, self.V, device=self.device,
                                  dtype=torch.bfloat16 if logits_dtype == "bf16" else torch.float32)
        self.ws_bytes = dcd.sample_workspace_bytes(dcd.make_sample_problem(self.max_rows, self.V, logits_dtype))
        if self.ws_bytes == 0:
            raise dcd.DcdError(dcd.DCD_ERR_SHAPE)
        self.workspace = torch.empty(self.ws_bytes, **u8)
        stream = torch.cuda.current_stream(self.device)
        with torch.cuda.device(self.device):
            dcd.quantize_fp8(w, self.w, self.w_scale, rows=self.V, cols=self.d, dtype=self._name(w), block_rows=128,
                             stream=stream)
        stream.synchronize()  # `w` may go; any stream may use the codes

    @staticmethod
    def _name(t) -> str:
        if t.dtype not in (torch.bfloat16, torch.float32):
            raise ValueError(f"{t.dtype}: bf16 or fp32")
        return "bf16" if t.dtype == torch.bfloat16 else "f32"

    def _take(self, name, t, shape, dtype=None):
        """`t` as the library takes it: on this device, contiguous, of this shape and type."""
        if t is None:
            return None
        if (t.device != self.w.device or tuple(t.shape) != shape or not t.is_contiguous()
                or (dtype is not None and t.dtype != dtype)):
            raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)} on {t.device}, wanted "
                             f"{dtype or 'bf16 or fp32'} {shape}, contiguous, on {self.w.device}")
        return t

    def launch(self, h, u, tokens, probs=None, *, temperature=None, top_k=None, top_p=None,
               min_p=None, logprob=None, kept=None, stream=None) -> None:
        """Enqueue one step on `stream` (default: torch's current stream): h [rows, d] bf16 or fp32,
        u [rows] and the rules (each None or [rows]); tokens int32 and, where given, probs [rows, V], logprob and
        kept are written, each dense.  tokens and probs may be a :class:`DeviceProblem`'s tokens and
        draft_probs [B * N, V], where row b * N + i proposes node i of sequence b: one step then draws all
        of their rows (node i of every sequence alone lies N rows apart: draw into buffers of the
        step's own and copy)."""
        rows = int(h.shape[0])
        if rows > self.max_rows:
            raise ValueError(f"{rows} rows, room for {self.max_rows}")
        f32, i32 = torch.float32, torch.int32
        h = self._take("h", h, (rows, self.d))
        u = self._take("u", u, (rows,), f32)
        tokens = self._take("tokens", tokens.view(-1), (rows,), i32)
        rules = [self._take(n, t, (rows,), d) for n, t, d in
                 (("temperature", temperature, f32), ("top_k", top_k, i32), ("top_p", top_p, f32), ("min_p", min_p, f32))]
        outs = [self._take(n, t, s, d) for n, t, s, d in
                (("probs", probs, (rows, self.V), f32), ("logprob", logprob, (rows,), f32), ("kept", kept, (rows,), i32))]
        if stream is None:
            stream = torch.cuda.current_stream(self.device)
        with torch.cuda.device(self.device):  # (its default stream is NULL: the current device's)
            dcd.quantize_fp8(h, self.h, self.h_scale, rows=rows, cols=self.d, dtype=self._name(h), stream=stream)
            dcd.logits_fp8(dcd.make_fp8_problem(rows, self.V, self.d, self.logits_dtype),
                           dcd.make_fp8_inputs(self.h, self.h_scale, self.w, self.w_scale, self.bias),
                           self.logits, stream)
            dcd.sample(dcd.make_sample_problem(rows, self.V, self.logits_dtype),
                       dcd.make_sample_inputs(self.logits, u, *rules), dcd.make_sample_outputs(tokens, *outs),
                       self.workspace, self.ws_bytes, stream)

    def propose(self, h, u, *, want_probs=True, **rules) -> dict:
        """One synchronous step on numpy (or torch) inputs; returns host copies of the outputs."""
        h = (h if torch.is_tensor(h) else _dev(h, self.device)).to(self.device).contiguous()
        rows = int(h.shape[0])
        dv = lambda a, t: None if a is None else torch.as_tensor(a).to(self.device, t).contiguous()  # noqa: E731
        rules = {n: dv(a, torch.int32 if n == "top_k" else torch.float32) for n, a in rules.items()}
        i32, f32 = dict(dtype=torch.int32, device=self.device), dict(dtype=torch.float32, device=self.device)
        out = dict(tokens=torch.empty(rows, **i32), kept=torch.empty(rows, **i32), logprob=torch.empty(rows, **f32))
        if want_probs:
            out["probs"] = torch.empty(rows, self.V, **f32)
        self.launch(h, dv(u, torch.float32), out["tokens"], out.get("probs"), logprob=out["logprob"],
                    kept=out["kept"], **rules)
        torch.cuda.synchronize(self.device)
        return {n: t.cpu().numpy() for n, t in out.items()}
