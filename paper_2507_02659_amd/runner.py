"""Device-memory plumbing around the C ABI: uploads a batch with PyTorch-ROCm, owns output buffers, calls the step.

PyTorch is used for device allocations, host<->device copies and the stream only.  No arithmetic of the
verification path happens here; every stage runs in libotverify's kernels.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import itertools
from dataclasses import dataclass
from typing import Optional

import numpy as np
import torch

from . import binding as ot


def _to_device(x: np.ndarray, dtype: str, device) -> torch.Tensor:
    """float32 array, or uint16 bfloat16 bit patterns, to a device tensor of the same bits."""
    if dtype == "bf16":
        return torch.from_numpy(np.ascontiguousarray(x).view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(device)


def read_device(ptr: int, count: int, np_dtype) -> np.ndarray:
    """Copies `count` elements from a raw device address (used for the library's workspace view)."""
    out = np.empty(count, dtype=np_dtype)
    if count:
        hip = C.CDLL("libamdhip64.so")
        hip.hipMemcpy.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int]
        hip.hipMemcpy.restype = C.c_int
        rc = hip.hipMemcpy(out.ctypes.data, C.c_void_p(ptr), out.nbytes, 2)  # hipMemcpyDeviceToHost
        if rc != 0:
            raise RuntimeError(f"hipMemcpy failed with {rc}")
    return out


@dataclass
class QuantWeights:
    """A target head of 4-bit weights as device tensors: W[k, v] = scales[k // group, v] * (code[k, v] - zeros[k // group, v])."""

    codes: torch.Tensor                             # uint8 [d / 2, V_t]: hidden index 2 i in the low four bits of row i, 2 i + 1 in the high ones
    scales: torch.Tensor                            # bfloat16 or float16 [ceil(d / group), V_t]
    zeros: Optional[torch.Tensor] = None            # uint8 [ceil(d / group), V_t], 0..15; None: 8
    group: int = 128

    def check(self):
        (half, V_t), n = self.codes.shape, -(-2 * self.codes.shape[0] // self.group)
        if self.codes.dtype != torch.uint8 or self.scales.dtype not in (torch.bfloat16, torch.float16):
            raise TypeError("codes are uint8, scales bfloat16 or float16")
        if tuple(self.scales.shape) != (n, V_t) or (self.zeros is not None and tuple(self.zeros.shape) != (n, V_t)):
            raise ValueError(f"scales and zeros of {2 * half} x {V_t} weights in groups of {self.group} are [{n}, {V_t}]")
        if self.zeros is not None and self.zeros.dtype != torch.uint8:
            raise TypeError("zeros are uint8")


class Verifier:
    """One library context plus (optionally) one n-gram cache, for batches of a fixed model shape.

    Work is enqueued on `stream` (None: the default stream).  Inputs have to be ready on it; outputs are allocated and ready on it."""

    _numbers = itertools.count()

    def __init__(self, *, d, V_t, V_d, dtype: str, W, direct_map, max_batch, max_k, max_ngram_len=2,
                 device="cuda:0", stream: Optional[torch.cuda.Stream] = None, draft_side: int = ot.OT_DRAFT_SIDE_AUTO):
        if not torch.cuda.is_available():
            raise RuntimeError("otverify needs a GPU: there is no CPU path")
        self.device = torch.device(device)
        self.dtype = dtype
        self.d, self.V_t, self.V_d = d, V_t, V_d
        self.stream = stream
        self._number = next(self._numbers)          # of this verifier, never used again
        torch.cuda.set_device(self.device)
        if self.device == torch.device("cuda"):     # as its tensors will say
            self.device = torch.device("cuda", torch.cuda.current_device())
        common = dict(d=d, V_t=V_t, V_d=V_d, max_batch=max_batch, max_k=max_k, max_ngram_len=max_ngram_len, direct_map=direct_map,
                      dtype=ot.OT_BF16 if dtype == "bf16" else ot.OT_F32, stream=None if stream is None else stream.cuda_stream,
                      draft_side=draft_side)
        self.ctx = None
        if isinstance(W, QuantWeights):
            W.check()
            self._here(codes=W.codes, scales=W.scales, zeros=W.zeros)
            assert tuple(W.codes.shape) == (d // 2, V_t)
            torch.cuda.synchronize(self.device)
            self.ctx = ot.ot_verify_init_quantized(codes=W.codes, scales=W.scales, zeros=W.zeros, group=W.group,
                                                   scale_dtype=ot.OT_F16 if W.scales.dtype == torch.float16 else ot.OT_BF16, **common)
        else:
            W_dev = W if isinstance(W, torch.Tensor) else _to_device(W, dtype, self.device)
            assert tuple(W_dev.shape) == (d, V_t)
            torch.cuda.synchronize(self.device)
            self.ctx = ot.ot_verify_init(W=W_dev, **common)
            del W_dev                               # init keeps a private re-tiled copy
        self.cache = None
        self._keep = None

    @classmethod
    def for_case(cls, case, **kw) -> "Verifier":
        kw.setdefault("max_batch", max(1, case.B))
        kw.setdefault("max_k", int(case.k.max()) if case.B else 0)
        kw.setdefault("max_ngram_len", case.max_ngram_len)
        W = case.W
        if W is None:                               # logits-only cases still need an LM head to create a context
            W = np.zeros((case.d, case.V_t), dtype=np.float32 if case.dtype == "f32" else np.uint16)
        v = cls(d=case.d, V_t=case.V_t, V_d=case.V_d, dtype=case.dtype, W=W, direct_map=case.direct_map, **kw)
        v.set_cache(case.ngram_key_off, case.ngram_key_ids, case.ngram_target_ids)
        return v

    @classmethod
    def quantized(cls, weights: QuantWeights, **kw) -> "Verifier":
        """A verifier whose target head has 4-bit weights; the other arguments are the constructor's."""
        half, V_t = weights.codes.shape
        return cls(d=2 * half, V_t=V_t, dtype="bf16", W=weights, **kw)

    def set_cache(self, key_off, key_ids, target_ids):
        if self.cache is not None:
            ot.ot_ngram_cache_destroy(self.cache)
        self.cache = ot.ot_ngram_cache_build(self.ctx, key_off, key_ids, target_ids)

    def close(self):
        if self.cache is not None:
            ot.ot_ngram_cache_destroy(self.cache)
            self.cache = None
        if self.ctx is not None:
            ot.ot_verify_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ------------------------------------------------------------------ batches
    def upload(self, case) -> dict:
        """Device copies of one batch's inputs and fresh output buffers."""
        dev = self.device
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(dev)
        inp = {
            "B": case.B, "M": case.M, "K": case.K, "step": case.step, "seed": case.seed,
            "row_off_host": np.ascontiguousarray(case.row_off, dtype=np.int32),
            "row_off": i32(case.row_off),
            "hidden": None if case.hidden is None else _to_device(case.hidden, case.dtype, dev),
            "target_logits": None if case.target_logits is None else _to_device(case.target_logits, "f32", dev),
            "draft_logits": _to_device(case.draft_logits, case.dtype, dev),
            "draft_ids": i32(case.draft_ids),
            "temperature": torch.from_numpy(np.ascontiguousarray(case.temperature, dtype=np.float32)).to(dev),
            "draft_temperature": None if case.draft_temperature is None else
            torch.from_numpy(np.ascontiguousarray(case.draft_temperature, dtype=np.float32)).to(dev),
            "seq_id": torch.from_numpy(np.ascontiguousarray(case.seq_id, dtype=np.uint64).view(np.int64)).to(dev),
        }
        inp["out"] = self.alloc_outputs(case.B, case.M)
        return inp

    def alloc_outputs(self, B: int, M: int) -> dict:
        dev = self.device
        out = {n: torch.full((max(B, 1),), -7, dtype=torch.int32, device=dev) for n in ot.OUT_INT_B}
        out.update({n: torch.full((max(M, 1),), -7, dtype=torch.int32, device=dev) for n in ot.OUT_INT_M})
        out.update({n: torch.full((max(M, 1),), -7.0, dtype=torch.float32, device=dev) for n in ot.OUT_F32_M})
        return out

    def step(self, inp: dict, *, from_logits: bool = False, use_cache: bool = True, step: Optional[int] = None):
        """Enqueues one ot_verify_step on the context's stream (asynchronous)."""
        sin = ot.make_step_in(B=inp["B"], step=inp["step"] if step is None else step, row_off=inp["row_off"],
                              row_off_host=inp["row_off_host"], hidden=inp["hidden"], draft_logits=inp["draft_logits"],
                              draft_ids=inp["draft_ids"], temperature=inp["temperature"],
                              draft_temperature=inp["draft_temperature"], seq_id=inp["seq_id"], seed=inp["seed"])
        sout = ot.make_step_out(inp["out"])
        cache = self.cache if use_cache else None
        if from_logits:
            ot.ot_verify_step_from_logits(self.ctx, cache, sin, inp["target_logits"], sout)
        else:
            ot.ot_verify_step(self.ctx, cache, sin, sout)

    def distill_loss(self, inp: dict, *, from_logits: bool = False, lam: float = 0.2, lambda_mode: int = ot.OT_LAMBDA_FIXED,
                     ngram_term: int = ot.OT_NGRAM_TERM_NLL, accepted_only: bool = False, with_qprime: bool = False,
                     sync: bool = True) -> Optional[dict]:
        """Enqueues ot_distill_loss after a step on `inp`; with sync, waits and returns its outputs as numpy arrays."""
        buf = self._loss_buffers(inp, with_qprime)
        sin = ot.make_step_in(B=inp["B"], step=inp["step"], row_off=inp["row_off"], row_off_host=inp["row_off_host"],
                              hidden=inp["hidden"], draft_logits=inp["draft_logits"], draft_ids=inp["draft_ids"],
                              temperature=inp["temperature"], draft_temperature=inp["draft_temperature"],
                              seq_id=inp["seq_id"], seed=inp["seed"])
        ot.ot_distill_loss(self.ctx, sin, ot.make_step_out(inp["out"]), inp["target_logits"] if from_logits else None,
                           lam=lam, lambda_mode=lambda_mode, ngram_term=ngram_term, accepted_only=accepted_only, buffers=buf)
        if not sync:
            return None
        self.synchronize()
        res = {n: t.cpu().numpy()[:inp["M"]] for n, t in buf.items() if n != "totals"}
        totals = buf["totals"].cpu().numpy()
        res.update(loss_dm=float(totals[0]), loss_ngram=float(totals[1]), n_dm=int(totals[2]), n_ngram_tokens=int(totals[3]),
                   loss=float(totals[4]))
        return res

    def _loss_buffers(self, inp: dict, with_qprime: bool) -> dict:
        M = max(inp["M"], 1)
        own = ("loss_buffers", M, with_qprime, self._number)   # a batch may go through several verifiers, each on its stream and with its V_t
        buf = inp.get(own)
        if buf is None:
            dev = self.device
            with self._on_stream():                 # the loss writes them there: filled anywhere else, they could be filled after it
                buf = {"kind": torch.full((M,), -7, dtype=torch.int32, device=dev),
                       "totals": torch.full((5,), -7.0, dtype=torch.float64, device=dev)}
                buf.update({n: torch.full((M,), -7.0, dtype=torch.float64, device=dev) for n in ("kl", "nll", "weight")})
                if with_qprime:
                    buf["qprime"] = torch.full((M, self.V_t), -7.0, dtype=torch.float32, device=dev)
            inp[own] = buf
        inp["loss_buffers", M, with_qprime] = buf   # the last call's
        return buf

    def distill_loss_grad(self, inp: dict, *, from_logits: bool = False, lam: float = 0.2, lambda_mode: int = ot.OT_LAMBDA_FIXED,
                          ngram_term: int = ot.OT_NGRAM_TERM_NLL, accepted_only: bool = False, with_qprime: bool = False,
                          grad_loss: Optional[torch.Tensor] = None) -> dict:
        """Enqueues ot_distill_loss_grad after a step on `inp`.  Returns device tensors: "grad", the gradient of grad_loss * loss (a float32
        tensor of one element; None: 1) with respect to the draft logits [K, V_d], and the loss's outputs (the same buffers every call)."""
        if grad_loss is not None and (grad_loss.dtype != torch.float32 or grad_loss.numel() != 1):
            raise ValueError("grad_loss is one float32")
        zq = inp["draft_logits"]                    # the gradient is allocated like them
        if zq.dtype != self._type() or zq.dim() != 2 or zq.size(0) != inp["K"] or zq.size(1) != self.V_d:
            raise ValueError(f"draft logits are [{inp['K']}, {self.V_d}] of the verifier's type, not {tuple(zq.shape)} {zq.dtype}")
        if self.stream is not None or zq.device != self.device or (grad_loss is not None and grad_loss.device != self.device):
            self._here(draft_logits=zq, grad_loss=grad_loss)
        buf = self._loss_buffers(inp, with_qprime)
        grad = self._empty(zq.shape, zq.dtype)
        sin = ot.make_step_in(B=inp["B"], step=inp["step"], row_off=inp["row_off"], row_off_host=inp["row_off_host"],
                              hidden=inp["hidden"], draft_logits=inp["draft_logits"], draft_ids=inp["draft_ids"],
                              temperature=inp["temperature"], draft_temperature=inp["draft_temperature"],
                              seq_id=inp["seq_id"], seed=inp["seed"])
        out, at = inp["out"], ot._ptr               # of the step's outputs, what the loss reads
        sout = ot.ot_step_out(n_mapped=at(out["n_mapped"]), n_accept=at(out["n_accept"]), mapped_ids=at(out["mapped_ids"]),
                              span_start=at(out["span_start"]), span_len=at(out["span_len"]), p_tok=at(out["p_tok"]))
        ot.ot_distill_loss_grad(self.ctx, sin, sout, inp["target_logits"] if from_logits else None, lam=lam,
                                lambda_mode=lambda_mode, ngram_term=ngram_term, accepted_only=accepted_only, buffers=buf,
                                grad_loss=grad_loss, grad=grad)
        return dict(buf, grad=grad)

    # ------------------------------------------------------------------ logits and log-probabilities
    def _on_stream(self):
        """Makes the verifier's stream the current one."""
        return contextlib.nullcontext() if self.stream is None else torch.cuda.stream(self.stream)

    def _empty(self, shape, dtype) -> torch.Tensor:
        """Memory for outputs that work on the verifier's stream writes."""
        if self.stream is None:
            return torch.empty(shape, dtype=dtype, device=self.device)
        with self._on_stream():
            return torch.empty(shape, dtype=dtype, device=self.device)

    def _type(self):
        return torch.bfloat16 if self.dtype == "bf16" else torch.float32

    def _here(self, **tensors):
        """Refuses tensors that are not on the verifier's device, where their addresses mean nothing.  Of the others the allocator learns that
        the verifier's stream uses them: the caller may drop them before the work there is done."""
        for name, t in tensors.items():
            if t is not None:
                if t.device != self.device:
                    raise ValueError(f"{name} is on {t.device}, the verifier on {self.device}")
                if self.stream is not None:
                    t.record_stream(self.stream)

    def lm_head(self, hidden: torch.Tensor) -> torch.Tensor:
        """Logits [M, V_t] (float32) of hidden rows [M, d] through the verifier's head (ot_lm_head)."""
        if hidden.dtype != self._type() or hidden.dim() != 2 or hidden.shape[1] != self.d:
            raise ValueError(f"hidden rows are [M, {self.d}] of the verifier's type, not {tuple(hidden.shape)} {hidden.dtype}")
        if self.stream is not None or hidden.device != self.device:
            self._here(hidden=hidden)
        M = hidden.shape[0]
        logits = self._empty((M, self.V_t), torch.float32)
        ot.ot_lm_head(self.ctx, M, hidden, logits, self.V_t)
        return logits

    def _logprob_in(self, logits, tokens, temperature, row_off, n_top, given_rows_only):
        M, V = logits.shape
        if logits.dtype not in (torch.bfloat16, torch.float32) or (V > 1 and logits.stride(1) != 1):
            raise ValueError("logits are [M, V] bfloat16 or float32 with neighbouring ids next to each other")
        n_tok = 0
        if tokens is not None:
            if tokens.dtype != torch.int32 or tokens.shape[0] != M or tokens.dim() > 2:
                raise ValueError(f"tokens are int32 [{M}] or [{M}, n]")
            n_tok = 1 if tokens.dim() == 1 else tokens.shape[1]
        B = M if row_off is None else row_off.numel() - 1
        if temperature is not None and (temperature.dtype != torch.float32 or temperature.numel() != B):
            raise ValueError(f"temperatures are {B} float32")
        if row_off is not None and row_off.dtype != torch.int32:
            raise ValueError("row_off is int32")
        dev = self.device                           # (a call of one row is bound by the host)
        if (self.stream is not None or row_off is not None or logits.device != dev or (tokens is not None and tokens.device != dev)
                or (temperature is not None and temperature.device != dev)):
            self._here(logits=logits, tokens=tokens, temperature=temperature, row_off=row_off)
        # rows may lie further apart than V, and overlap nothing: one row alone may have any stride
        return ot.ot_logprob_in(M, V, ot.OT_BF16 if logits.dtype == torch.bfloat16 else ot.OT_F32, n_tok, n_top, 1 if given_rows_only else 0, B, 0,
                                logits.stride(0) if M > 1 else V, logits.data_ptr(), ot._ptr(tokens), ot._ptr(temperature), ot._ptr(row_off))

    def token_logprobs(self, logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, *, temperature: Optional[torch.Tensor] = None,
                       row_off: Optional[torch.Tensor] = None, n_top: int = 0, given_rows_only: bool = False) -> dict:
        """Log-probabilities of the given tokens (int32 [M] or [M, n], -1: none), entropy and the n_top most likely ids of every row of logits
        [M, V] (ot_token_logprobs).  Returns device tensors: logprob (shaped like tokens), entropy, row_max, row_sumexp and, with n_top,
        top_ids and top_logprobs.  temperature: one per row, or per sequence of row_off."""
        given = self._logprob_in(logits, tokens, temperature, row_off, n_top, given_rows_only)
        return self._token_logprobs(given, tokens)

    def _token_logprobs(self, given, tokens) -> dict:
        # a call of one row is bound by the host: one allocation for all outputs, whose addresses are known without asking for them
        M, n_top, n_tok = given.M, given.n_top, given.n_tok
        at_top = (3 + n_tok) * M
        memory = self._empty((at_top + 2 * n_top * M,), torch.float32)
        p, one, part = memory.data_ptr(), (M,), memory.as_strided
        out = {"entropy": part(one, (1,), 0), "row_max": part(one, (1,), M), "row_sumexp": part(one, (1,), 2 * M)}
        if tokens is not None:
            out["logprob"] = part(tokens.shape, (1,) if tokens.dim() == 1 else (n_tok, 1), 3 * M)
        if n_top:
            out["top_logprobs"] = part((M, n_top), (n_top, 1), at_top)
            out["top_ids"] = memory.view(torch.int32).as_strided((M, n_top), (n_top, 1), at_top + n_top * M)
        ot.ot_token_logprobs(self.ctx, given, ot.ot_logprob_out(p + 12 * M if n_tok else None, p, p + 4 * M, p + 8 * M, p + 4 * at_top if n_top else None,
                                                                p + 4 * (at_top + n_top * M) if n_top else None))
        return out

    def _statistic(self, forward, name, M):
        """Address of a statistic that token_logprobs left."""
        t = forward.get(name)
        if t is None or t.dtype != torch.float32 or t.dim() != 1 or t.numel() != M or not t.is_contiguous():
            raise ValueError(f"forward holds {name}, float32 [{M}]")
        if self.stream is not None or t.device != self.device:
            self._here(**{name: t})
        return t.data_ptr()

    def token_logprobs_grad(self, logits: torch.Tensor, tokens: Optional[torch.Tensor], forward: dict, *, grad_logprob: Optional[torch.Tensor] = None,
                            grad_entropy: Optional[torch.Tensor] = None, temperature: Optional[torch.Tensor] = None,
                            row_off: Optional[torch.Tensor] = None, given_rows_only: bool = False) -> torch.Tensor:
        """Gradient of sum grad_logprob * logprob + sum grad_entropy * entropy with respect to the logits, in their type
        (ot_token_logprobs_grad).  forward: what token_logprobs returned for the same arguments."""
        given = self._logprob_in(logits, tokens, temperature, row_off, 0, given_rows_only)
        M = given.M
        if grad_logprob is not None and (tokens is None or grad_logprob.dtype != torch.float32 or grad_logprob.shape != tokens.shape):
            raise ValueError(f"grad_logprob is float32 {None if tokens is None else tuple(tokens.shape)}")
        if grad_entropy is not None and (grad_entropy.dtype != torch.float32 or grad_entropy.dim() != 1 or grad_entropy.numel() != M):
            raise ValueError(f"grad_entropy is float32 [{M}]")
        if self.stream is not None or (grad_logprob is not None and grad_logprob.device != self.device) or (
                grad_entropy is not None and grad_entropy.device != self.device):
            self._here(grad_logprob=grad_logprob, grad_entropy=grad_entropy)
        stats = ot.ot_logprob_out(None, None if grad_entropy is None else self._statistic(forward, "entropy", M), self._statistic(forward, "row_max", M),
                                  self._statistic(forward, "row_sumexp", M), None, None)
        grad = self._empty(logits.shape, logits.dtype)
        ot.ot_token_logprobs_grad(self.ctx, given, stats, grad_logprob, grad_entropy, grad, given.V)
        return grad

    def step_logprobs(self, inp: dict, *, from_logits: bool = False, n_top: int = 0, at_temperature: bool = True) -> dict:
        """Log-probabilities of the tokens that the last step on `inp` emitted, with entropy and alternatives, from the logits it left
        (from_logits: those it was given).  Rows without an emitted token hold 0, no alternatives.  at_temperature: under the step's
        temperatures (greedy sequences at 1), else at 1."""
        M, tokens = inp["M"], inp["out"]["out_tokens"]
        w = ot.ot_verify_workspace(self.ctx)
        given = ot.make_logprob_in(M=M, V=self.V_t, dtype=ot.OT_F32, logits=inp["target_logits"] if from_logits else w.logits, ld=self.V_t if from_logits else w.ld_logits,
                                   tokens=tokens, n_tok=1, n_top=n_top, temperature=inp["temperature"] if at_temperature else None,
                                   row_off=inp["row_off"] if at_temperature else None, B=inp["B"], given_rows_only=True)
        return self._token_logprobs(given, tokens[:M])

    def synchronize(self):
        if self.stream is not None:
            self.stream.synchronize()
        else:
            torch.cuda.synchronize(self.device)

    def results(self, inp: dict) -> dict:
        """Synchronises and returns the outputs as numpy arrays trimmed to [B] / [M]."""
        self.synchronize()
        B, M = inp["B"], inp["M"]
        res = {}
        for n, t in inp["out"].items():
            a = t.cpu().numpy()
            res[n] = a[:B] if n in ot.OUT_INT_B else a[:M]
        return res

    def workspace(self, M: int, K: int, with_logits: bool = False) -> dict:
        """Row statistics (and optionally the logits) the last step left in the library's workspace."""
        self.synchronize()
        v = ot.ot_verify_workspace(self.ctx)
        ws = {
            "row_max": read_device(v.row_max, M, np.float32),
            "row_sumexp": read_device(v.row_sumexp, M, np.float64),
            "row_argmax": read_device(v.row_argmax, M, np.int32),
            "draft_row_max": read_device(v.draft_row_max, K, np.float32),
            "draft_row_sumexp": read_device(v.draft_row_sumexp, K, np.float64),
            "draft_row_argmax": read_device(v.draft_row_argmax, K, np.int32),
        }
        if with_logits:
            ws["logits"] = read_device(v.logits, M * int(v.ld_logits), np.float32).reshape(M, int(v.ld_logits))
        return ws

    def run_case(self, case, **kw) -> dict:
        inp = self.upload(case)
        self.step(inp, from_logits=case.hidden is None, **kw)
        return self.results(inp)
