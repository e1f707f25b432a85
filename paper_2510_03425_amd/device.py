"""Device-memory plumbing for the C ABI: uploads a model's compressed weights, LoRA
adapters and token ids into torch tensors on the GPU, fills the ABI structs with their
addresses, owns the workspace, and calls the entry points on torch's current stream.

PyTorch is used only for device allocations and the stream handle; every step of the
training step runs inside ``libmebp.so``.
"""
from __future__ import annotations

import ctypes as C
import functools
from typing import List, Optional

import numpy as np
import torch

from mebp_inputs import PROJ, Config, Inputs

from . import _lib as L

ACT_CODE = {"silu": 0, "gelu_tanh": 1}


def make_config(cfg: Config) -> L.MebpConfig:
    return L.MebpConfig(
        n_layers=cfg.n_layers, hidden=cfg.hidden, n_heads=cfg.n_heads, n_kv_heads=cfg.n_kv_heads,
        head_dim=cfg.head_dim, ffn=cfg.ffn, vocab=cfg.vocab, act=ACT_CODE[cfg.act], rms_eps=cfg.rms_eps,
        rope_theta_global=cfg.rope_theta_global, rope_theta_local=cfg.rope_theta_local,
        window=cfg.window, global_every=cfg.global_every, group=cfg.group, lora_rank=cfg.lora_rank,
        lora_alpha=cfg.lora_alpha, lora_mask=cfg.lora_mask(), arch=cfg.arch_flags)


# the handle alone: a torch.cuda.Stream of it takes 2.6 us to make (no public name: absent in other builds of torch)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def stream_handle() -> int:
    """torch's current stream on the current device."""
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _dev(a: np.ndarray, device) -> torch.Tensor:
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        a = a.view(np.int16)
    return torch.from_numpy(a).to(device)


def ptr(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


# ---------------------------------------------------------------- operators on logits
LOGIT_TYPE = {torch.float32: L.MEBP_F32, torch.float16: L.MEBP_F16, torch.bfloat16: L.MEBP_BF16}


def _on_device(f):
    """Runs with the first tensor's device current: the library launches there, on torch's
    current stream of that device."""
    @functools.wraps(f)
    def g(z, *a, **kw):
        if not z.is_cuda:
            raise ValueError("logits must be on the GPU")
        if z.get_device() == torch.cuda.current_device():
            return f(z, *a, **kw)
        with torch.cuda.device(z.device):
            return f(z, *a, **kw)
    return g


def _on_model_device(f):
    """Runs a method with the model's device current."""
    @functools.wraps(f)
    def g(self, *a, **kw):
        with torch.cuda.device(self.norm_final.device):
            return f(self, *a, **kw)
    return g


def logits_struct(z: torch.Tensor, like: Optional[torch.Tensor] = None) -> L.MebpLogits:
    """[rows][vocab] logits (or their gradient, on the device of ``like``) whose columns follow
    one another."""
    dtype = LOGIT_TYPE.get(z.dtype)
    if dtype is None or z.dim() != 2 or (z.stride(1) != 1 and z.shape[1] > 1):
        raise ValueError("logits must be a fp32, fp16 or bf16 matrix with contiguous rows")
    if like is not None and z.get_device() != like.get_device():
        raise ValueError(f"dz must be on {like.device}")
    rows, vocab = z.shape
    return L.MebpLogits(z.data_ptr(), z.stride(0) if rows > 1 else vocab, rows, vocab, dtype)


def _operand(t: Optional[torch.Tensor], dtype, shape, like: torch.Tensor, what: str) -> int:
    """Address of an operand, None as NULL."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != like.get_device():
        raise ValueError(f"{what} must be contiguous {dtype} {tuple(shape)} on {like.device}")
    return t.data_ptr()


def _logits_ws(ws: Optional[torch.Tensor], z: torch.Tensor, top_k: int):
    """The given workspace, or one that lives until the stream is done with it."""
    if ws is None:
        n = L.mebp_logits_workspace_bytes(z.shape[0], z.shape[1], top_k)
        ws = torch.empty(max(n, 256), dtype=torch.uint8, device=z.device)
    elif ws.get_device() != z.get_device() or not ws.is_contiguous():
        raise ValueError(f"workspace must be contiguous on {z.device}")
    return ws, ws.nbytes


def _scores(z: torch.Tensor, n: int, targets, top_k: int, out: Optional[dict]):
    """The outputs of a scoring call over n rows (made where `out` is None), and the struct of them."""
    f32, one = torch.float32, (n,)
    if out is None:
        names = ["lse", "entropy"] + (["logp"] if targets is not None else [])
        out = {k: torch.empty(n, dtype=f32, device=z.device) for k in names}
        if top_k > 0:
            out["top_ids"] = torch.empty((n, top_k), dtype=torch.int32, device=z.device)
            out["top_logp"] = torch.empty((n, top_k), dtype=f32, device=z.device)
    get = out.get
    return out, L.MebpTokenScores(
        _operand(get("logp"), f32, one, z, "logp"), _operand(get("lse"), f32, one, z, "lse"),
        _operand(get("entropy"), f32, one, z, "entropy"), _operand(get("top_ids"), torch.int32, (n, top_k), z, "top_ids"),
        _operand(get("top_logp"), f32, (n, top_k), z, "top_logp"))


def _distill(z: torch.Tensor, n: int, ids, logits, temperature, alpha, targets, row_weight) -> L.MebpDistill:
    k = 1 if ids is None else ids.shape[-1]
    return L.MebpDistill(_operand(ids, torch.int32, (n, k), z, "ids"), _operand(logits, torch.float32, (n, k), z, "logits"),
                         _operand(targets, torch.int32, (n,), z, "targets"),
                         _operand(row_weight, torch.float32, (n,), z, "row_weight"), k, temperature, alpha)


@_on_device
def token_logprobs(z: torch.Tensor, targets: Optional[torch.Tensor] = None, top_k: int = 0, temperature: float = 1.0,
                   out: Optional[dict] = None, ws: Optional[torch.Tensor] = None) -> dict:
    """``mebp_token_logprobs`` of logits [rows][vocab]: a dict of fp32 ``logp`` (with int32
    ``targets``), ``lse``, ``entropy`` [rows] and, with ``top_k``, int32 ``top_ids`` and ``top_logp``
    [rows][top_k]. ``out``: the wanted ones of these as tensors to write into."""
    n = z.shape[0]
    out, s = _scores(z, n, targets, top_k, out)
    zs = logits_struct(z)
    ws, nb = _logits_ws(ws, z, top_k)
    L.mebp_token_logprobs(zs, _operand(targets, torch.int32, (n,), z, "targets"), temperature, top_k, s, ws.data_ptr(),
                          nb, stream_handle())
    return out


@_on_device
def token_logprobs_backward(z: torch.Tensor, targets: Optional[torch.Tensor], lse: torch.Tensor,
                            entropy: Optional[torch.Tensor], d_logp: Optional[torch.Tensor],
                            d_entropy: Optional[torch.Tensor] = None, dz: Optional[torch.Tensor] = None,
                            temperature: float = 1.0) -> torch.Tensor:
    """``mebp_token_logprobs_backward``: the gradient w.r.t. the logits, into ``dz`` (any logits
    type; ``z`` itself for one in place) or a new tensor of their type."""
    n = (z.shape[0],)
    if dz is None:
        dz = torch.empty(z.shape, dtype=z.dtype, device=z.device)
    f32 = torch.float32
    L.mebp_token_logprobs_backward(logits_struct(z), _operand(targets, torch.int32, n, z, "targets"), temperature,
                                   _operand(lse, f32, n, z, "lse"), _operand(entropy, f32, n, z, "entropy"),
                                   _operand(d_logp, f32, n, z, "d_logp"), _operand(d_entropy, f32, n, z, "d_entropy"),
                                   logits_struct(dz, z), stream_handle())
    return dz


@_on_device
def distill_topk(z: torch.Tensor, ids: Optional[torch.Tensor], logits: Optional[torch.Tensor], row_loss: Optional[torch.Tensor] = None,
                 dz: Optional[torch.Tensor] = None, temperature: float = 1.0, alpha: float = 1.0,
                 targets: Optional[torch.Tensor] = None, row_weight: Optional[torch.Tensor] = None,
                 ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``mebp_distill_topk``: the loss of each row against a teacher's int32 ``ids`` and fp32
    ``logits`` [rows][k] (None: hard labels alone, alpha 0), and its gradient into ``dz`` where that is given."""
    n = z.shape[0]
    if row_loss is None:
        row_loss = torch.empty(n, dtype=torch.float32, device=z.device)
    d = _distill(z, n, ids, logits, temperature, alpha, targets, row_weight)
    zs = logits_struct(z)
    ws, nb = _logits_ws(ws, z, 0)
    L.mebp_distill_topk(zs, d, _operand(row_loss, torch.float32, (n,), z, "row_loss"),
                        None if dz is None else logits_struct(dz, z), ws.data_ptr(), nb, stream_handle())
    return row_loss


class DeviceModel:
    """A model's inputs resident in HBM plus the ABI structs that point at them."""

    def __init__(self, inp: Inputs, device: str = "cuda"):
        cfg = inp.cfg
        self.cfg = cfg
        self.inp = inp
        self.device = device
        self.ccfg = make_config(cfg)
        self.L = len(inp.base)
        if self.L != cfg.n_layers:
            # a truncated input set (per-layer or LM-head-only use); with no layer at all the
            # config still needs one for validation, and train_step is refused
            self.ccfg.n_layers = max(self.L, 1)
        self.keep: List[torch.Tensor] = []
        self.base = (L.MebpLayerBase * self.L)()
        self.lora = (L.MebpLayerLora * self.L)()
        self.grads = (L.MebpLayerLoraGrad * self.L)()
        self.dA: List[dict] = []
        self.dB: List[dict] = []
        for l in range(self.L):
            for i, p in enumerate(PROJ):
                q4, sb = inp.base[l][p]
                tq, ts = _dev(q4, device), _dev(sb, device)
                self.keep += [tq, ts]
                self.base[l].w[i].q4 = tq.data_ptr()
                self.base[l].w[i].scale = ts.data_ptr()
            na, nm = _dev(inp.norm_attn[l], device), _dev(inp.norm_mlp[l], device)
            self.keep += [na, nm]
            self.base[l].norm_attn = na.data_ptr()
            self.base[l].norm_mlp = nm.data_ptr()
            ex = inp.extra
            if ex.get("bias") and ex["bias"][l] is not None:
                for i, p in enumerate(("q", "k", "v")):
                    tb = _dev(ex["bias"][l][p], device)
                    self.keep.append(tb)
                    self.base[l].bias[i] = tb.data_ptr()
            if ex.get("qk_norm") and ex["qk_norm"][l] is not None:
                tq, tk = (_dev(w, device) for w in ex["qk_norm"][l])
                self.keep += [tq, tk]
                self.base[l].q_norm, self.base[l].k_norm = tq.data_ptr(), tk.data_ptr()
            if ex.get("post_norm") and ex["post_norm"][l] is not None:
                ta, tm = (_dev(w, device) for w in ex["post_norm"][l])
                self.keep += [ta, tm]
                self.base[l].post_attn_norm, self.base[l].post_mlp_norm = ta.data_ptr(), tm.data_ptr()
            dA, dB = {}, {}
            for i, p in enumerate(PROJ):
                if p not in inp.lora[l]:
                    continue
                A, B = inp.lora[l][p]
                tA, tB = _dev(A, device), _dev(B, device)
                self.keep += [tA, tB]
                self.lora[l].A[i] = tA.data_ptr()
                self.lora[l].B[i] = tB.data_ptr()
                gA = torch.empty(A.shape, dtype=torch.float32, device=device)
                gB = torch.empty(B.shape, dtype=torch.float32, device=device)
                dA[p], dB[p] = gA, gB
                self.grads[l].dA[i] = gA.data_ptr()
                self.grads[l].dB[i] = gB.data_ptr()
            self.dA.append(dA)
            self.dB.append(dB)
        self.emb = None
        if inp.emb is not None:
            eq, es = _dev(inp.emb[0], device), _dev(inp.emb[1], device)
            self.keep += [eq, es]
            self.emb = L.MebpQ4(q4=eq.data_ptr(), scale=es.data_ptr())
            self.norm_final = _dev(inp.norm_final, device)
        if inp.ids is not None:
            self.ids = _dev(inp.ids, device)
        self.B, self.T = cfg.batch, cfg.seq
        self.N = self.B * self.T
        self.ws_bytes = L.mebp_workspace_bytes(self.ccfg, self.B, self.T)
        if self.ws_bytes == 0:
            raise L.MebpError(L.MEBP_EINVAL, "invalid config for workspace sizing")
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        self.loss = torch.zeros(1, dtype=torch.float32, device=device)
        self.ckpt = None
        self.distill_ws = None

    # ------------------------------------------------------------------ entry points
    def layer_forward(self, l: int, x_in: torch.Tensor, x_out: torch.Tensor):
        L.mebp_layer_forward_ckpt(self.ccfg, l, self.base[l], self.lora[l], ptr(x_in), ptr(x_out), self.B,
                                  self.T, ptr(self.ws), self.ws_bytes, stream_handle())

    def layer_backward(self, l: int, x_ckpt: torch.Tensor, dy: torch.Tensor, dx: Optional[torch.Tensor]):
        L.mebp_layer_recompute_backward(self.ccfg, l, self.base[l], self.lora[l], ptr(x_ckpt), ptr(dy), ptr(dx),
                                        self.grads[l], self.B, self.T, ptr(self.ws), self.ws_bytes,
                                        stream_handle())

    def lm_head(self, x_last: torch.Tensor, dx_last: torch.Tensor):
        L.mebp_lm_head_ce_backward(self.ccfg, self.emb, ptr(self.norm_final), ptr(x_last), ptr(self.ids), self.B,
                                   self.T, ptr(self.loss), ptr(dx_last), ptr(self.ws), self.ws_bytes,
                                   stream_handle())

    def embed(self, x0: torch.Tensor):
        L.mebp_embed(self.ccfg, self.emb, ptr(self.ids), self.B, self.T, ptr(x0), stream_handle())

    def alloc_ckpt(self):
        if self.ckpt is None:
            self.ckpt = torch.empty((self.L + 1, self.N, self.cfg.hidden), dtype=torch.float32,
                                    device=self.device)
        return self.ckpt

    def train_step(self, dx0: Optional[torch.Tensor] = None):
        if self.L == 0:
            raise ValueError("this input set has no layers")
        ck = self.alloc_ckpt()
        L.mebp_train_step(self.ccfg, self.emb, self.base, ptr(self.norm_final), self.lora, ptr(self.ids), self.B,
                          self.T, ptr(ck), ptr(self.loss), self.grads, ptr(dx0), ptr(self.ws), self.ws_bytes,
                          stream_handle())

    def train_step_offload(self, ckpt_host: torch.Tensor, ring: torch.Tensor, dx0: Optional[torch.Tensor] = None):
        """The step with checkpoints in pinned host memory ``ckpt_host`` [(L+1)][N][d] and a
        device ring ``ring`` [slots][N][d]."""
        if self.L == 0:
            raise ValueError("this input set has no layers")
        L.mebp_train_step_offload(self.ccfg, self.emb, self.base, ptr(self.norm_final), self.lora, ptr(self.ids),
                                  self.B, self.T, ptr(ckpt_host), ptr(ring), ring.shape[0], ptr(self.loss), self.grads,
                                  ptr(dx0), ptr(self.ws), self.ws_bytes, stream_handle())

    # ---------------------------------------------------------------- operators on the head's logits
    def _head_ws(self, rows: int, top_k: int = 0):
        """A workspace of the head's calls, which lives until the stream is done with it."""
        n = L.mebp_head_workspace_bytes(self.ccfg, rows, top_k)
        if n == 0:
            raise L.MebpError(L.MEBP_EINVAL, "invalid shape for the head's workspace")
        return torch.empty(n, dtype=torch.uint8, device=self.device), n

    @_on_model_device
    def lm_head_logits(self, x: torch.Tensor, dtype: torch.dtype = torch.float32) -> torch.Tensor:
        """Logits [rows][vocab] of hidden states x [rows][d] fp32, in fp32 or fp16."""
        rows = x.shape[0]
        z = torch.empty((rows, self.cfg.vocab), dtype=dtype, device=x.device)
        ws, nb = self._head_ws(rows)
        L.mebp_lm_head_logits(self.ccfg, self.emb, ptr(self.norm_final), self._x(x), rows, logits_struct(z), ptr(ws), nb,
                              stream_handle())
        return z

    @_on_model_device
    def lm_head_logits_backward(self, x: torch.Tensor, dz: torch.Tensor) -> torch.Tensor:
        """The gradient w.r.t. x of bf16 gradients w.r.t. its logits."""
        rows = x.shape[0]
        dx = torch.empty_like(x)
        ws, nb = self._head_ws(rows)
        L.mebp_lm_head_logits_backward(self.ccfg, self.emb, ptr(self.norm_final), self._x(x), rows, logits_struct(dz, x),
                                       ptr(dx), ptr(ws), nb, stream_handle())
        return dx

    @_on_model_device
    def lm_head_logprobs(self, x: torch.Tensor, targets: Optional[torch.Tensor] = None, top_k: int = 0,
                         temperature: float = 1.0, out: Optional[dict] = None) -> dict:
        """`token_logprobs` of the head's logits of x, which are never held at once."""
        rows = x.shape[0]
        out, s = _scores(x, rows, targets, top_k, out)
        ws, nb = self._head_ws(rows, top_k)
        L.mebp_lm_head_logprobs(self.ccfg, self.emb, ptr(self.norm_final), self._x(x), rows,
                                _operand(targets, torch.int32, (rows,), x, "targets"), temperature, top_k, s, ptr(ws), nb,
                                stream_handle())
        return out

    @_on_model_device
    def lm_head_distill(self, x: torch.Tensor, dx: torch.Tensor, ids: Optional[torch.Tensor], logits: Optional[torch.Tensor],
                        temperature: float = 1.0, alpha: float = 1.0, targets: Optional[torch.Tensor] = None,
                        row_weight: Optional[torch.Tensor] = None, row_loss: Optional[torch.Tensor] = None):
        """Loss (into self.loss) and gradient of distilling the head's logits of x (`distill_topk`)."""
        rows = x.shape[0]
        d = _distill(x, rows, ids, logits, temperature, alpha, targets, row_weight)
        ws, nb = self._head_ws(rows)
        L.mebp_lm_head_distill_backward(self.ccfg, self.emb, ptr(self.norm_final), self._x(x), rows, d, ptr(self.loss),
                                        _operand(row_loss, torch.float32, (rows,), x, "row_loss"),
                                        _operand(dx, torch.float32, (rows, self.cfg.hidden), x, "dx"), ptr(ws), nb,
                                        stream_handle())

    @_on_model_device
    def train_step_distill(self, ids: Optional[torch.Tensor], logits: Optional[torch.Tensor], temperature: float = 1.0,
                           alpha: float = 1.0, targets: Optional[torch.Tensor] = None, row_weight: Optional[torch.Tensor] = None,
                           row_loss: Optional[torch.Tensor] = None, dx0: Optional[torch.Tensor] = None):
        """`train_step` against a teacher's int32 ids and fp32 logits [N][k], in the model's workspace where
        that is large enough (as it is for many tokens), else in one that the first such step makes."""
        if self.L == 0:
            raise ValueError("this input set has no layers")
        ck = self.alloc_ckpt()
        d = _distill(ck, self.N, ids, logits, temperature, alpha, targets, row_weight)
        need = L.mebp_distill_step_workspace_bytes(self.ccfg, self.B, self.T)
        ws = self.ws
        if need > self.ws_bytes:
            if self.distill_ws is None or self.distill_ws.numel() < need:
                self.distill_ws = torch.empty(need, dtype=torch.uint8, device=self.device)
            ws = self.distill_ws
        L.mebp_train_step_distill(self.ccfg, self.emb, self.base, ptr(self.norm_final), self.lora, ptr(self.ids), self.B,
                                  self.T, d, ptr(ck), ptr(self.loss),
                                  _operand(row_loss, torch.float32, (self.N,), ck, "row_loss"), self.grads, ptr(dx0),
                                  ptr(ws), ws.numel(), stream_handle())

    def _x(self, x: torch.Tensor) -> int:
        return _operand(x, torch.float32, (x.shape[0], self.cfg.hidden), self.norm_final, "x")

    def grad_probe(self) -> torch.Tensor:
        """First and last layers' LoRA gradients, concatenated (a cheap result fingerprint)."""
        parts = [t.reshape(-1) for l in {0, self.L - 1} for d in (self.dA[l], self.dB[l]) for t in d.values()]
        return torch.cat(parts) if parts else torch.zeros(1, device=self.device)

    def ws_view(self, slot: int, dtype: torch.dtype, shape) -> torch.Tensor:
        """A view of a workspace intermediate (tests)."""
        off = L.mebp_workspace_offset(self.ccfg, self.B, self.T, slot)
        n = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
        return self.ws[off:off + n].view(dtype).view(*shape)


def slot_index(name: str) -> int:
    i = 0
    while True:
        s = L.mebp_workspace_slot_name(i)
        if s is None:
            raise KeyError(name)
        if s == name:
            return i
        i += 1
