"""Losses over a policy's logits, with their gradients: what a training loop does with its rewards.

    lp = token_logprobs(logits, tokens, lengths=lengths)                 # differentiable, float32 [B, T]
    r = policy_loss_grad(logits, tokens, old_lp, advantages, ref_logprobs=ref_lp, kl_coef=0.04,
                         lengths=lengths)                                # value and gradient in one pass
    logits.backward(r.grad)                                              # on into the model
    policy_loss(...).backward()                                          # the same through autograd

`token_logprobs`, `policy_loss`, `preference_loss` and `distillation_loss` return tensors that torch can
differentiate in the logits; their backward pass reads the logits a second time.  The functions whose
names end in `_grad` return the gradient at once.  For the policy loss and the distillation this is
one pass over the logits: half to two thirds of the traffic of the other way.

Common arguments
  logits       [B, T, V], or [N, V] for packed positions (then one sequence of N); float32, bfloat16 or
               float16, any strides over B and T (views like model_output[:, :-1] are read in place)
  tokens       [B, T] or [N], int32 or int64: the token that position t scores (for a causal model the
               one behind it: input_ids[:, 1:])
  lengths      [B]: position t of sequence b counts if t < lengths[b].  Not for packed positions
  mask         bool or uint8, of the tokens' shape: a position counts if it is not 0
  temperature  divides the logits
  out          where the gradient goes (default: a new tensor); may be the logits themselves, which then
               count as changed in place: what has saved them for a backward pass raises there
  grad_scale   the gradient is that of grad_scale * loss (loss scaling, gradient accumulation)
  status       int32 [1] on the GPU; TB_DEV_TOKEN_RANGE / TB_DEV_LENGTH_RANGE are OR-ed into it

What stands at positions that do not count has no part in anything; what is returned for them is 0.
Gradients are for reverse mode, and of first order; logits with a forward-mode tangent are refused.
Everything runs on the current stream of the logits' GPU, and nothing synchronises.  See
include/tensorloss.h for the formulas and for what wrong ids and infinite logits give.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from . import binding as _b
from .binding import TensorBLEUError

TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
AVERAGES = {"token": 0, "sequence": 1, "sum": 2}
PAIRS = {"sigmoid": 0, "hinge": 1, "ipo": 2}
TEACHER_MOST = 1024

EXPORTS = [
    "tensorloss_distill", "tensorloss_distill_grad", "tensorloss_policy", "tensorloss_preference",
    "tensorloss_token_logprobs", "tensorloss_token_logprobs_grad", "tensorloss_workspace_bytes",
]

_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class tb_logits_t(ctypes.Structure):
    _fields_ = [("data", _vp), ("seq_stride", _i64), ("pos_stride", _i64), ("B", _i32), ("T", _i32),
                ("V", _i32), ("type", _i32), ("temperature", _f32)]


class tb_positions_t(ctypes.Structure):
    _fields_ = [("tokens", _vp), ("token_stride", _i64), ("token_bytes", _i32), ("lengths", _vp),
                ("mask", _vp)]


class tb_gradient_t(ctypes.Structure):
    _fields_ = [("data", _vp), ("seq_stride", _i64), ("pos_stride", _i64), ("scale", _f32)]


class tb_policy_t(ctypes.Structure):
    _fields_ = [("old_logprobs", _vp), ("ref_logprobs", _vp), ("advantages", _vp), ("each", _i32),
                ("average", _i32), ("clip_low", _f32), ("clip_high", _f32), ("kl_coef", _f32),
                ("entropy_coef", _f32)]


class tb_preference_t(ctypes.Structure):
    _fields_ = [("ref_logprobs", _vp), ("kind", _i32), ("beta", _f32), ("label_smoothing", _f32)]


class tb_teacher_t(ctypes.Structure):
    _fields_ = [("ids", _vp), ("logits", _vp), ("id_bytes", _i32), ("type", _i32), ("K", _i32),
                ("average", _i32)]


class PolicyLoss(NamedTuple):
    terms: torch.Tensor        # float32 [4]: loss, mean KL, share of clipped positions, mean entropy
    grad: torch.Tensor
    logprobs: torch.Tensor     # float32, of the tokens' shape

    @property
    def loss(self) -> torch.Tensor:
        return self.terms[0]


class PreferenceLoss(NamedTuple):
    terms: torch.Tensor        # float32 [3]: loss, share of pairs with a positive margin, mean margin
    grad: torch.Tensor
    sequence_logprobs: torch.Tensor   # float32 [B]
    margins: torch.Tensor      # float32 [B / 2]

    @property
    def loss(self) -> torch.Tensor:
        return self.terms[0]


class DistillationLoss(NamedTuple):
    terms: torch.Tensor        # float32 [1]: loss
    grad: torch.Tensor
    row_loss: torch.Tensor     # float32, one for each position

    @property
    def loss(self) -> torch.Tensor:
        return self.terms[0]


_lib = None


def _library() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        lib = _b.load_library()
        p = ctypes.POINTER
        head = [p(tb_logits_t), p(tb_positions_t)]
        end = [_vp, _vp, ctypes.c_size_t, _vp]                 # status, workspace, its size, stream
        for name, rest in (
                ("token_logprobs", [_vp] * 5),
                ("token_logprobs_grad", [_vp, _vp, _vp, _i64, _i64, _vp, p(tb_gradient_t), _vp]),
                ("policy", [p(tb_policy_t), p(tb_gradient_t)] + [_vp] * 5 + end),
                ("preference", [p(tb_preference_t), p(tb_gradient_t)] + [_vp] * 5 + end),
                ("distill", [p(tb_teacher_t), p(tb_gradient_t)] + [_vp] * 4 + end),
                ("distill_grad", [p(tb_teacher_t), _vp, _vp, _vp, p(tb_gradient_t), _vp])):
            f = getattr(lib, "tensorloss_" + name)
            f.restype, f.argtypes = ctypes.c_int, head + rest
        lib.tensorloss_workspace_bytes.restype = ctypes.c_size_t
        lib.tensorloss_workspace_bytes.argtypes = [_i32, _i32]
        _lib = lib
    return _lib


_host = None


def native():
    """The native marshalling module (built with the library; raises if it has not been).  Its functions
    return None for what they leave to the code here."""
    global _host
    if _host is None:
        _library()
        try:
            from . import _loss_host as module
        except ImportError as e:
            raise TensorBLEUError("the module _loss_host does not load: run `python -m "
                                  f"paper_2510_05485_amd.build` first ({e})") from e
        _host = module
    return _host


def workspace_bytes(B: int, T: int) -> int:
    return int(_library().tensorloss_workspace_bytes(B, T))


def _named(table, key, what):
    if key not in table:
        raise TensorBLEUError(f"{what} must be one of {', '.join(table)} (got {key!r})")
    return table[key]


def _on(t: torch.Tensor, device, name: str) -> None:
    if not isinstance(t, torch.Tensor) or t.device != device:
        raise TensorBLEUError(f"{name} must be a tensor on the logits' GPU "
                              f"(got {getattr(t, 'device', type(t).__name__)})")


def _refuse_tangent(logits: torch.Tensor) -> None:
    if torch.autograd.forward_ad.unpack_dual(logits).tangent is not None:
        raise TensorBLEUError("the losses have no forward-mode derivative (the logits carry a tangent)")


class _Call:
    """A call's logits and positions, checked, as the C structs; keeps what was converted alive."""

    def __init__(self, logits, tokens, lengths, mask, temperature, status):
        if not isinstance(logits, torch.Tensor) or not logits.is_cuda:
            raise TensorBLEUError("logits must live on the GPU "
                                  f"(got {getattr(logits, 'device', type(logits).__name__)})")
        if logits.dtype not in TYPES:
            raise TensorBLEUError(f"logits must be float32, bfloat16 or float16 (got {logits.dtype})")
        if logits.dim() not in (2, 3) or logits.shape[-1] < 1:
            raise TensorBLEUError(f"expected logits [B, T, V] or [N, V] (got {tuple(logits.shape)})")
        _refuse_tangent(logits)
        logits = logits.detach()
        if logits.shape[-1] > 1 and logits.stride(-1) != 1:
            logits = logits.contiguous()
        self.logits, self.device, self.shape = logits, logits.device, tuple(logits.shape[:-1])
        self.packed = logits.dim() == 2
        self.B, self.T = (1, self.shape[0]) if self.packed else self.shape
        self.V = int(logits.shape[-1])
        if self.B * self.T >= 2 ** 31 - 1 or self.V >= 2 ** 31:
            raise TensorBLEUError("too many positions or tokens for 32-bit counts")
        self.keep = []
        at = tb_positions_t()
        if tokens is not None:
            _on(tokens, self.device, "tokens")
            if tokens.dtype not in (torch.int32, torch.int64) or tuple(tokens.shape) != self.shape:
                raise TensorBLEUError(f"tokens must be int32 or int64 of shape {self.shape} "
                                      f"(got {tokens.dtype} {tuple(tokens.shape)})")
            if self.T > 1 and tokens.stride(-1) != 1:
                tokens = self._kept(tokens.contiguous())
            at.tokens, at.token_bytes = tokens.data_ptr(), tokens.element_size()
            at.token_stride = self.T if self.packed else tokens.stride(0)
        if lengths is not None:
            if self.packed:
                raise TensorBLEUError("lengths are for logits [B, T, V]; packed positions take a mask")
            _on(lengths, self.device, "lengths")
            if lengths.dtype not in (torch.int32, torch.int64) or tuple(lengths.shape) != (self.B,):
                raise TensorBLEUError(f"lengths must be int32 or int64 of shape {(self.B,)} "
                                      f"(got {lengths.dtype} {tuple(lengths.shape)})")
            if lengths.dtype == torch.int64:       # (wrong ones stay wrong when they are narrowed)
                lengths = lengths.clamp(-1, self.T + 1).to(torch.int32)
            at.lengths = self._kept(lengths.contiguous()).data_ptr()
        if mask is not None:
            _on(mask, self.device, "mask")
            if mask.dtype not in (torch.bool, torch.uint8) or tuple(mask.shape) != self.shape:
                raise TensorBLEUError(f"mask must be bool or uint8 of shape {self.shape} "
                                      f"(got {mask.dtype} {tuple(mask.shape)})")
            at.mask = self._kept(mask.contiguous()).data_ptr()
        self.at = at
        l = tb_logits_t()
        l.data = logits.data_ptr()
        l.seq_stride, l.pos_stride = (0, logits.stride(0)) if self.packed else logits.stride()[:2]
        l.B, l.T, l.V, l.type, l.temperature = self.B, self.T, self.V, TYPES[logits.dtype], float(temperature)
        if not 0.0 < l.temperature < float("inf"):
            raise TensorBLEUError(f"temperature must be positive and finite (got {temperature})")
        self.l = l
        if status is not None:
            _on(status, self.device, "status")
            if status.dtype != torch.int32 or status.numel() != 1:
                raise TensorBLEUError("status must be an int32 tensor of one element")
        self.status = status

    def _kept(self, t):
        self.keep.append(t)
        return t

    def values(self, t, name, shape=None):
        """The pointer of a float32 tensor over the positions (or of another shape)."""
        shape = self.shape if shape is None else shape
        _on(t, self.device, name)
        if t.dtype != torch.float32 or tuple(t.shape) != tuple(shape):
            raise TensorBLEUError(f"{name} must be float32 of shape {tuple(shape)} "
                                  f"(got {t.dtype} {tuple(t.shape)})")
        return self._kept(t.detach().contiguous()).data_ptr()

    def gradient(self, out, scale):
        x = self.logits
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        else:
            _on(out, self.device, "out")
            if out.dtype != x.dtype or out.shape != x.shape or (self.V > 1 and out.stride(-1) != 1):
                raise TensorBLEUError(f"out must be {x.dtype} of shape {tuple(x.shape)} with consecutive "
                                      f"values in a row (got {out.dtype} {tuple(out.shape)})")
            if out.requires_grad and out.is_leaf and torch.is_grad_enabled():
                raise TensorBLEUError("out must not require a gradient")
        g = tb_gradient_t()
        g.data = out.data_ptr()
        g.seq_stride, g.pos_stride = (0, out.stride(0)) if self.packed else out.stride()[:2]
        g.scale = float(scale)
        return out, g

    @staticmethod
    def written(out, to):
        """The caller's tensor `out` has been written over: torch's checks of saved tensors notice it.
        (Tensors of inference mode count no versions and are not saved.)"""
        if out is not None and not to.is_inference():
            torch.autograd.graph.increment_version(to)

    def new(self, *shape):
        return torch.empty(*shape, dtype=torch.float32, device=self.device)

    def run(self, entry, *args, workspace=False):
        def c(a):
            if isinstance(a, torch.Tensor):
                return a.data_ptr()
            return ctypes.byref(a) if isinstance(a, ctypes.Structure) else a
        args = [c(a) for a in args]
        with torch.cuda.device(self.device):
            if workspace:
                n = workspace_bytes(self.B, self.T)
                w = torch.empty(n, dtype=torch.uint8, device=self.device)
                args += [w.data_ptr(), n]
            args.append(int(torch.cuda.current_stream().cuda_stream))
            rc = getattr(_library(), entry)(ctypes.byref(self.l), ctypes.byref(self.at), *args)
        _b._check(rc, entry)


def _needs_grad(logits) -> bool:
    if not isinstance(logits, torch.Tensor):
        return False
    _refuse_tangent(logits)                # (not to be seen any more inside a Function's forward)
    return torch.is_grad_enabled() and logits.requires_grad


# ---- log-probabilities --------------------------------------------------------------------------

def _score(call, want_entropy, keep_state):
    lp = call.new(call.shape)
    entropy = call.new(call.shape) if want_entropy else None
    state = call.new(*call.shape, 4) if keep_state else None
    call.run("tensorloss_token_logprobs", lp, entropy, state, call.status)
    return lp, entropy, state


def _rows_gradient(call, state, d_lp, d_entropy, d_strides, upstream):
    out, g = call.gradient(None, 1.0)
    # (hooks on saved tensors give back the same values, in what strides they like)
    state = call.values(state, "the rows' state", (*call.shape, 4))
    over = call.shape if d_strides[1] else (call.B,)
    d_lp = call.values(d_lp, "d_lp", over)
    d_entropy = None if d_entropy is None else call.values(d_entropy, "d_entropy", over)
    call.run("tensorloss_token_logprobs_grad", state, d_lp, d_entropy, *d_strides, upstream, g)
    return out


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, lengths, mask, temperature, want_entropy, status):
        call = _Call(logits, tokens, lengths, mask, temperature, status)
        lp, entropy, state = _score(call, want_entropy, True)
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(logits, tokens, lengths, mask, state)
        ctx.temperature = temperature
        return (lp, entropy) if want_entropy else lp

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_lp, d_entropy=None):
        none = (None,) * 6
        if d_lp is None and d_entropy is None:
            return (None, *none)
        logits, tokens, lengths, mask, state = ctx.saved_tensors
        call = _Call(logits, tokens, lengths, mask, ctx.temperature, None)
        as32 = lambda d: None if d is None else d.to(torch.float32).contiguous()
        d_lp, d_entropy = as32(d_lp), as32(d_entropy)
        if d_lp is None:
            d_lp = torch.zeros_like(d_entropy)
        return (_rows_gradient(call, state, d_lp, d_entropy, (call.T, 1), None), *none)


def token_logprobs(logits, tokens, *, lengths=None, mask=None, temperature: float = 1.0,
                   want_entropy: bool = False, status: Optional[torch.Tensor] = None):
    """float32 log-probabilities of `tokens` (their shape), and with want_entropy a tuple of these and
    the entropies of the rows.  Differentiable in the logits."""
    found = native().logprobs(logits, tokens, lengths, mask, temperature, status, want_entropy)
    if found is not None:
        return found
    if _needs_grad(logits):
        return _TokenLogprobs.apply(logits, tokens, lengths, mask, temperature, want_entropy, status)
    lp, entropy, _ = _score(_Call(logits, tokens, lengths, mask, temperature, status), want_entropy, False)
    return (lp, entropy) if want_entropy else lp


# ---- policy loss --------------------------------------------------------------------------------

def _policy(call, old_logprobs, advantages, ref_logprobs, clip_low, clip_high, kl_coef, entropy_coef,
            average, grad, keep):
    p = tb_policy_t()
    p.old_logprobs = call.values(old_logprobs, "old_logprobs")
    _on(advantages, call.device, "advantages")
    p.each = 1 if call.packed or advantages.dim() == 2 else 0
    p.advantages = call.values(advantages, "advantages", call.shape if p.each else (call.B,))
    p.average = _named(AVERAGES, average, "average")
    p.clip_low, p.clip_high = float(clip_low), float(clip_high)
    p.kl_coef, p.entropy_coef = float(kl_coef), float(entropy_coef)
    if not (p.clip_low >= 0 and p.clip_high >= 0 and p.kl_coef >= 0 and p.entropy_coef == p.entropy_coef):
        raise TensorBLEUError("clip_low, clip_high and kl_coef must not be negative")
    if ref_logprobs is not None:
        p.ref_logprobs = call.values(ref_logprobs, "ref_logprobs")
    elif p.kl_coef != 0:
        raise TensorBLEUError("kl_coef needs ref_logprobs")
    terms, lp = call.new(4), call.new(call.shape)
    state, d_lp, d_entropy = (call.new(*call.shape, 4), call.new(call.shape), call.new(call.shape)) \
        if keep else (None,) * 3
    call.run("tensorloss_policy", p, grad, terms, lp, state, d_lp, d_entropy, call.status, workspace=True)
    return terms, lp, state, d_lp, d_entropy if p.entropy_coef != 0 else None


class _PolicyLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, lengths, mask, temperature, status, *policy):
        call = _Call(logits, tokens, lengths, mask, temperature, status)
        terms, _, state, d_lp, d_entropy = _policy(call, *policy, None, True)
        ctx.save_for_backward(logits, tokens, lengths, mask, state, d_lp, d_entropy)
        ctx.temperature = temperature
        return terms[0].clone()

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_loss):
        logits, tokens, lengths, mask, state, d_lp, d_entropy = ctx.saved_tensors
        call = _Call(logits, tokens, lengths, mask, ctx.temperature, None)
        grad = _rows_gradient(call, state, d_lp, d_entropy, (call.T, 1), d_loss.to(torch.float32))
        return (grad, *(None,) * 13)


def policy_loss(logits, tokens, old_logprobs, advantages, *, ref_logprobs=None, lengths=None, mask=None,
                clip_low: float = 0.2, clip_high: float = 0.2, kl_coef: float = 0.0,
                entropy_coef: float = 0.0, average: str = "token", temperature: float = 1.0,
                status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The clipped policy loss as a scalar that torch can differentiate: the average over positions of
    -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl_coef kl - entropy_coef H  with
    r = exp(lp - old_logprobs) and kl = exp(ref_logprobs - lp) - (ref_logprobs - lp) - 1.

    old_logprobs, ref_logprobs: float32 of the tokens' shape; advantages: float32 [B], or one for each
    position.  average: "token" (over all positions that count), "sequence" (the mean of sequences'
    means) or "sum"."""
    loss = native().policy(logits, tokens, lengths, mask, temperature, status, None, None, old_logprobs, advantages,
                           ref_logprobs, clip_low, clip_high, kl_coef, entropy_coef, AVERAGES.get(average))
    if loss is not None:
        return loss
    policy = (old_logprobs, advantages, ref_logprobs, clip_low, clip_high, kl_coef, entropy_coef, average)
    if _needs_grad(logits):
        return _PolicyLoss.apply(logits, tokens, lengths, mask, temperature, status, *policy)
    return _policy(_Call(logits, tokens, lengths, mask, temperature, status), *policy, None, False)[0][0]


def policy_loss_grad(logits, tokens, old_logprobs, advantages, *, ref_logprobs=None, lengths=None,
                     mask=None, clip_low: float = 0.2, clip_high: float = 0.2, kl_coef: float = 0.0,
                     entropy_coef: float = 0.0, average: str = "token", temperature: float = 1.0,
                     grad_scale: float = 1.0, out: Optional[torch.Tensor] = None,
                     status: Optional[torch.Tensor] = None) -> PolicyLoss:
    """policy_loss and its gradient in the logits, in one pass over them."""
    found = native().policy(logits, tokens, lengths, mask, temperature, status, out, float(grad_scale), old_logprobs,
                            advantages, ref_logprobs, clip_low, clip_high, kl_coef, entropy_coef,
                            AVERAGES.get(average))
    if found is not None:
        return PolicyLoss(*found)
    call = _Call(logits, tokens, lengths, mask, temperature, status)
    to, g = call.gradient(out, grad_scale)
    terms, lp, *_ = _policy(call, old_logprobs, advantages, ref_logprobs, clip_low, clip_high, kl_coef,
                            entropy_coef, average, g, False)
    call.written(out, to)
    return PolicyLoss(terms, to, lp)


# ---- preference loss ----------------------------------------------------------------------------

def _preference(call, ref_logprobs, beta, kind, label_smoothing, grad, keep):
    if call.packed or call.B % 2:
        raise TensorBLEUError("expected logits [B, T, V] with an even B: the first half is chosen, the "
                              "second rejected")
    p = tb_preference_t()
    p.ref_logprobs = call.values(ref_logprobs, "ref_logprobs")
    p.kind, p.beta, p.label_smoothing = _named(PAIRS, kind, "kind"), float(beta), float(label_smoothing)
    if not 0 < p.beta < float("inf"):
        raise TensorBLEUError(f"beta must be positive and finite (got {beta})")
    if not 0 <= p.label_smoothing <= 0.5 or (p.label_smoothing and kind != "sigmoid"):
        raise TensorBLEUError("label_smoothing must lie in [0, 0.5], and is for the sigmoid loss")
    terms, lp, margins = call.new(3), call.new(call.B), call.new(call.B // 2)
    state, d_sequence = (call.new(*call.shape, 4), call.new(call.B)) if keep else (None, None)
    call.run("tensorloss_preference", p, grad, terms, lp, margins, state, d_sequence, call.status,
             workspace=True)
    return terms, lp, margins, state, d_sequence


class _PreferenceLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, lengths, mask, temperature, status, *preference):
        call = _Call(logits, tokens, lengths, mask, temperature, status)
        terms, _, _, state, d_sequence = _preference(call, *preference, None, True)
        ctx.save_for_backward(logits, tokens, lengths, mask, state, d_sequence)
        ctx.temperature = temperature
        return terms[0].clone()

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_loss):
        logits, tokens, lengths, mask, state, d_sequence = ctx.saved_tensors
        call = _Call(logits, tokens, lengths, mask, ctx.temperature, None)
        grad = _rows_gradient(call, state, d_sequence, None, (1, 0), d_loss.to(torch.float32))
        return (grad, *(None,) * 9)


def preference_loss(logits, tokens, ref_logprobs, *, lengths=None, mask=None, beta: float = 0.1,
                    kind: str = "sigmoid", label_smoothing: float = 0.0, temperature: float = 1.0,
                    status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The loss of paired log ratios as a scalar that torch can differentiate.  The first half of the
    sequences is chosen, the second rejected (sequence i against i + B/2).  With h the chosen
    sequence's sum of lp - ref_logprobs less the rejected one's (for "ipo" of their means):
    "sigmoid"  -(1 - e) log sigmoid(beta h) - e log sigmoid(-beta h), e = label_smoothing;
    "hinge"  max(0, 1 - beta h);  "ipo"  (h - 1 / (2 beta))^2;  averaged over the pairs.

    ref_logprobs: float32 of the tokens' shape (token_logprobs of the reference model)."""
    loss = native().preference(logits, tokens, lengths, mask, temperature, status, None, None, ref_logprobs, beta,
                               PAIRS.get(kind), label_smoothing)
    if loss is not None:
        return loss
    preference = (ref_logprobs, beta, kind, label_smoothing)
    if _needs_grad(logits):
        return _PreferenceLoss.apply(logits, tokens, lengths, mask, temperature, status, *preference)
    return _preference(_Call(logits, tokens, lengths, mask, temperature, status), *preference, None, False)[0][0]


def preference_loss_grad(logits, tokens, ref_logprobs, *, lengths=None, mask=None, beta: float = 0.1,
                         kind: str = "sigmoid", label_smoothing: float = 0.0, temperature: float = 1.0,
                         grad_scale: float = 1.0, out: Optional[torch.Tensor] = None,
                         status: Optional[torch.Tensor] = None) -> PreferenceLoss:
    """preference_loss and its gradient in the logits."""
    found = native().preference(logits, tokens, lengths, mask, temperature, status, out, float(grad_scale), ref_logprobs,
                                beta, PAIRS.get(kind), label_smoothing)
    if found is not None:
        return PreferenceLoss(*found)
    call = _Call(logits, tokens, lengths, mask, temperature, status)
    to, g = call.gradient(out, grad_scale)
    terms, lp, margins, *_ = _preference(call, ref_logprobs, beta, kind, label_smoothing, g, False)
    call.written(out, to)
    return PreferenceLoss(terms, to, lp, margins)


# ---- distillation -------------------------------------------------------------------------------

def _teacher(call, teacher_ids, teacher_logits, average):
    for t, name in ((teacher_ids, "teacher_ids"), (teacher_logits, "teacher_logits")):
        _on(t, call.device, name)
        if t.dim() != len(call.shape) + 1 or tuple(t.shape[:-1]) != call.shape or \
                not 1 <= t.shape[-1] <= TEACHER_MOST or t.shape != teacher_ids.shape:
            raise TensorBLEUError(f"{name} must be {[*call.shape, 'K']} with K in 1..{TEACHER_MOST} "
                                  f"(got {tuple(t.shape)})")
    if teacher_ids.dtype not in (torch.int32, torch.int64) or teacher_logits.dtype not in TYPES:
        raise TensorBLEUError("teacher_ids must be int32 or int64, teacher_logits float32, bfloat16 or "
                              f"float16 (got {teacher_ids.dtype}, {teacher_logits.dtype})")
    q = tb_teacher_t()
    q.ids = call._kept(teacher_ids.contiguous()).data_ptr()
    q.logits = call._kept(teacher_logits.detach().contiguous()).data_ptr()
    q.id_bytes, q.type, q.K = teacher_ids.element_size(), TYPES[teacher_logits.dtype], teacher_ids.shape[-1]
    q.average = _named(AVERAGES, average, "average")
    return q


def _distill(call, q, grad, keep):
    terms, rows = call.new(1), call.new(call.shape)
    state, d_row = (call.new(*call.shape, 4), call.new(call.shape)) if keep else (None, None)
    call.run("tensorloss_distill", q, grad, terms, rows, state, d_row, call.status, workspace=True)
    return terms, rows, state, d_row


class _DistillationLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, teacher_ids, teacher_logits, lengths, mask, temperature, status, average):
        call = _Call(logits, None, lengths, mask, temperature, status)
        terms, _, state, d_row = _distill(call, _teacher(call, teacher_ids, teacher_logits, average), None, True)
        ctx.save_for_backward(logits, teacher_ids, teacher_logits, lengths, mask, state, d_row)
        ctx.temperature, ctx.average = temperature, average
        return terms[0].clone()

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_loss):
        logits, teacher_ids, teacher_logits, lengths, mask, state, d_row = ctx.saved_tensors
        call = _Call(logits, None, lengths, mask, ctx.temperature, None)
        q = _teacher(call, teacher_ids, teacher_logits, ctx.average)
        out, g = call.gradient(None, 1.0)
        state, d_row = call.values(state, "the rows' state", (*call.shape, 4)), call.values(d_row, "d_row")
        call.run("tensorloss_distill_grad", q, state, d_row, d_loss.to(torch.float32), g)
        return (out, *(None,) * 7)


def distillation_loss(logits, teacher_ids, teacher_logits, *, lengths=None, mask=None,
                      temperature: float = 1.0, average: str = "token",
                      status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Kullback-Leibler divergence from a teacher's best logits, as a scalar that torch can
    differentiate: the average over positions of temperature^2 sum q (log q - log p[id]) with q the
    softmax of the K entries of teacher_logits [..., K] over the temperature, and p that of the logits.

    An entry of -inf is none, whatever its id; a position without entries adds 0."""
    loss = native().distill(logits, lengths, mask, temperature, status, None, None, teacher_ids, teacher_logits,
                            AVERAGES.get(average))
    if loss is not None:
        return loss
    if _needs_grad(logits):
        return _DistillationLoss.apply(logits, teacher_ids, teacher_logits, lengths, mask, temperature,
                                       status, average)
    call = _Call(logits, None, lengths, mask, temperature, status)
    return _distill(call, _teacher(call, teacher_ids, teacher_logits, average), None, False)[0][0]


def distillation_loss_grad(logits, teacher_ids, teacher_logits, *, lengths=None, mask=None,
                           temperature: float = 1.0, average: str = "token", grad_scale: float = 1.0,
                           out: Optional[torch.Tensor] = None,
                           status: Optional[torch.Tensor] = None) -> DistillationLoss:
    """distillation_loss and its gradient in the logits, in one pass over them."""
    found = native().distill(logits, lengths, mask, temperature, status, out, float(grad_scale), teacher_ids,
                             teacher_logits, AVERAGES.get(average))
    if found is not None:
        return DistillationLoss(*found)
    call = _Call(logits, None, lengths, mask, temperature, status)
    q = _teacher(call, teacher_ids, teacher_logits, average)
    to, g = call.gradient(out, grad_scale)
    terms, rows, *_ = _distill(call, q, g, False)
    call.written(out, to)
    return DistillationLoss(terms, to, rows)
