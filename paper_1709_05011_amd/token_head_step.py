"""The output side of a token model on the device: RMS norm with the residual's addition, a classifier over the vocabulary (a 1x1 convolution over one
pixel per token), the log probabilities of given tokens, and the way back to the norm's inputs with an AdamW update of the classifier and the
norm's scale.  Every operator is a call into the C library; this module only owns buffers and the order of calls, and torch is used for device memory.

    head = TokenHeadStep(width=1024, vocab=32000, dtype=lc.LC_BF16)
    logprob, entropy, dx = head.step(x, residual, tokens, dlogprob)     # dlogprob: the loss's gradient with respect to each log probability
    logprob, entropy, ids, top = head.score(x, residual, tokens, top=5) # one token or many, nothing is updated
    total, codes, scales = head.packed(x, residual)                     # the norm's output in 8 bits, for a product or a wire that takes it so

Calls share one set of buffers, for as many rows as any of them has had; results are kept apart for the last eight of (rows, top).  What a captured call
works in stays with the object.  Calls of one object follow one another: one on another stream than the last waits for it there (a graph's replays and
other threads have to see to that themselves).

The vocabulary is padded to a multiple of 8 rows of the classifier (what the bf16 products take without copies); the pad's logits are never read and their
gradient stays zero.
"""
from __future__ import annotations

from typing import Dict, Optional, Tuple

import torch

from . import larsconv as lc


KEPT_SETS = 8


class TokenHeadStep:
    def __init__(self, width: int, vocab: int, dtype: int = lc.LC_BF16, states_in_8_bits: bool = False, eps: float = 1e-5, lr: float = 1e-3,
                 beta1: float = 0.9, beta2: float = 0.95, adam_eps: float = 1e-8, weight_decay: float = 0.1, device: str = "cuda:0"):
        lc.lib()                     # fails here, loudly, when the library has not been built
        self.dev, self.width, self.vocab, self.dtype, self.eps = device, width, vocab, dtype, eps
        self.type = torch.bfloat16 if dtype == lc.LC_BF16 else torch.float32
        self.padded = (vocab + 7) // 8 * 8
        self.lr, self.betas, self.adam_eps, self.weight_decay, self.steps = lr, (beta1, beta2), adam_eps, weight_decay, 0
        f32 = dict(dtype=torch.float32, device=device)
        self.params: Dict[str, torch.Tensor] = {"w": torch.zeros((self.padded, width), **f32), "gamma": torch.ones(width, **f32)}
        self.grads = {k: torch.zeros_like(p) for k, p in self.params.items()}
        self.w_lowp = torch.zeros((self.padded, width), dtype=self.type, device=device) if dtype == lc.LC_BF16 else None
        names = list(self.params)
        lists = [[d[k] for k in names] for d in (self.params, self.grads)]
        lowp = [self.w_lowp, None] if self.w_lowp is not None else None
        self.states_in_8_bits = states_in_8_bits
        sizes = [self.params[k].numel() for k in names]
        if states_in_8_bits:
            self.m, self.v = ([torch.zeros(n, dtype=torch.uint8, device=device) for n in sizes] for _ in range(2))
            self.m_scale, self.v_scale = ([torch.ones(-(-n // lc.ADAMW_Q8_BLOCK), **f32) for n in sizes] for _ in range(2))
            self._adam = lc.AdamWQ8Args(*lists, self.m, self.m_scale, self.v, self.v_scale, w_lowp=lowp)
        else:
            self.m, self.v = ([torch.zeros(n, **f32) for n in sizes] for _ in range(2))
            self._adam = lc.AdamWArgs(*lists, self.m, self.v, w_lowp=lowp)
        self._stream = torch.cuda.current_stream() if self.params["w"].is_cuda else None      # the last call's
        self._room: Optional[dict] = None                                   # what calls work in, for room["rows"] rows
        self._sets: Dict[Tuple[int, int], dict] = {}                        # views of it and results for (rows, top), the one used last at the end
        self._of_graphs: Dict[Tuple[int, int], dict] = {}                   # sets made while a graph recorded, which graphs alone use

    def load(self, w: torch.Tensor, gamma: torch.Tensor) -> None:
        """Sets the classifier ([vocab][width]) and the norm's scale."""
        self._follow()
        self.params["w"].zero_()
        self.params["w"][:self.vocab].copy_(w)
        self.params["gamma"].copy_(gamma)
        if self.w_lowp is not None:
            self.w_lowp.copy_(self.params["w"])

    def _check(self, rows: int, **tensors: Optional[torch.Tensor]) -> None:
        """The entry points take pointers: what a call hands over has to be contiguous, of its type and of `rows` rows (grad_scale: one float), on this object's device."""
        for name, t in tensors.items():
            if t is None:
                continue
            shape, dtype = ((rows, self.width), self.type) if name in ("x", "residual", "dtotal") else ((rows,), torch.int32 if name == "tokens" else torch.float32)
            if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device != self.params["w"].device or not t.is_contiguous() or \
                    (t.numel() != 1 if name == "grad_scale" else tuple(t.shape) != shape):
                raise ValueError(f"{name}: a contiguous {dtype} tensor of {'one element' if name == 'grad_scale' else f'shape {shape}'} on {self.params['w'].device} is needed, got " +
                                 (f"{t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}" if isinstance(t, torch.Tensor) else f"{t!r}"))

    def _follow(self) -> None:
        """Parameters, states and room are shared: the call that begins waits for the last one where that was on another stream (not while a graph records, which runs nothing)."""
        if self._stream is None or (lc._stream(None) or 0) == self._stream.cuda_stream or torch.cuda.is_current_stream_capturing():
            return
        stream = torch.cuda.current_stream()
        stream.wait_stream(self._stream)
        self._stream = stream

    def _let_go(self, b: dict) -> None:
        """Before a set is dropped: its memory is another's only when the last call's stream is done with it."""
        if self._stream is not None:
            for t in (*b.values(), *b["room"].values()):
                if isinstance(t, torch.Tensor):
                    t.record_stream(self._stream)

    def _make_set(self, rows: int, top: int, of_graphs: bool) -> dict:
        e = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=self.dev)
        norm = lc.RmsNormDesc(rows, self.width, eps=self.eps, dtype=self.dtype)
        token = lc.TokenDesc(rows, self.vocab, ld=self.padded, dtype=self.dtype, top=top)
        product = lc.ConvDesc(rows, self.width, 1, 1, self.padded, 1, 1, dtype=self.dtype)
        need = max([lc.rmsnorm_bwd_workspace_bytes(norm), lc.token_logprob_workspace_bytes(token), 256] +
                   [lc.conv2d_workspace_bytes(product, p) for p in (lc.LC_PASS_FWD, lc.LC_PASS_BWD_DATA, lc.LC_PASS_BWD_WEIGHT)])
        room = None if of_graphs else self._room
        if room is None or room["rows"] < rows or room["ws"].numel() < need:
            most = rows
            if room is not None:                                            # (freed before its successor is made, but for what graphs use)
                most, need = max(rows, room["rows"]), max(need, room["ws"].numel())
                for b in self._sets.values():
                    self._let_go(b)
                room = self._room = b = None
                self._sets = {k: b for k, b in self._sets.items() if b["in_graph"]}
            room = dict(rows=most, ws=e(need, dtype=torch.uint8), total=e(most, self.width, dtype=self.type), y=e(most, self.width, dtype=self.type),
                        rstd=e(most), logits=e(most, self.padded, dtype=self.type), lse=e(most))
            if not of_graphs:
                self._room = room
        b = dict(norm=norm, token=token, product=product, room=room, in_graph=of_graphs, ws=room["ws"], logprob=e(rows), entropy=e(rows),
                 ids=e(rows, top, dtype=torch.int32) if top else None, top=e(rows, top) if top else None)
        for name in ("total", "y", "rstd", "logits", "lse"):
            b[name] = room[name][:rows]
        return b

    def _buffers(self, rows: int, top: int, training: bool = False) -> dict:
        """What a call over `rows` tokens works in.  A set that a graph records is kept, with the room it is in; one that has to be made while a graph records is for graphs
        alone, as nothing of it is filled before one runs."""
        key, recording = (rows, top), self.params["w"].is_cuda and torch.cuda.is_current_stream_capturing()
        b = self._sets.get(key)
        of_graphs = recording and (b is None or (training and "dlogits" not in b))
        if of_graphs:
            b = self._of_graphs.get(key) or self._make_set(rows, top, True)
            self._of_graphs[key] = b
        elif b is None:
            b = self._make_set(rows, top, False)
            spare = [k for k, s in self._sets.items() if not s["in_graph"]]
            if len(spare) >= KEPT_SETS:
                self._let_go(self._sets.pop(spare[0]))
            self._sets[key] = b
        else:
            self._sets[key] = self._sets.pop(key)
            b["in_graph"] |= recording
        if training:
            if "dlogits" not in b["room"]:
                b["room"]["dlogits"] = (torch.empty_like if of_graphs else torch.zeros_like)(b["room"]["logits"])      # the pad stays zero
                b["room"]["dy"] = torch.empty_like(b["room"]["y"])
            if "dlogits" not in b:
                b["dlogits"], b["dy"], b["dx"] = b["room"]["dlogits"][:rows], b["room"]["dy"][:rows], torch.empty_like(b["y"])
            if of_graphs:
                b["dlogits"][:, self.vocab:].zero_()
        return b

    def _forward(self, b: dict, x: torch.Tensor, residual: Optional[torch.Tensor], tokens: torch.Tensor) -> None:
        if x.shape[0] == 0:                                       # (the product takes no empty batch)
            return
        w = self.params["w"] if self.w_lowp is None else self.w_lowp
        lc.rmsnorm_fwd(b["norm"], x, residual, self.params["gamma"], b["total"] if residual is not None else None, b["y"], b["rstd"])
        lc.conv2d_fwd(b["product"], b["y"], w, b["logits"], b["ws"])
        lc.token_logprob_fwd(b["token"], b["logits"], tokens, b["logprob"], b["entropy"], b["lse"], b["ids"], b["top"], b["ws"])

    def score(self, x, residual, tokens, top: int = 0):
        """Log probability and entropy of each row's token (int32; outside the vocabulary: does not count), and the `top` likeliest tokens with
        theirs.  The tensors returned are this object's buffers: the next call over as many rows writes them again.  (Before load() all logits
        are equal, and listing alternatives among them is slow.)"""
        self._check(x.shape[0], x=x, residual=residual, tokens=tokens)
        self._follow()
        b = self._buffers(x.shape[0], top)
        self._forward(b, x, residual, tokens)
        return b["logprob"], b["entropy"], b["ids"], b["top"]

    def step(self, x, residual, tokens, dlogprob, dentropy=None, dtotal=None, grad_scale=None):
        """Forward, backward and update.  dlogprob, dentropy: gradient of the loss with respect to each row's log probability and entropy (a mean
        cross-entropy: -1/rows); dtotal: gradient that reaches x + residual by another way; grad_scale: one float on the device, multiplies the
        parameters' gradients.  Returns the rows' log probabilities and entropies and the gradient with respect to x (and to residual),
        in this object's buffers.  A graph replays the step number of its recording, and with states in 8 bits the rounding of that step."""
        self._check(x.shape[0], x=x, residual=residual, tokens=tokens, dlogprob=dlogprob, dentropy=dentropy, dtotal=dtotal,
                    grad_scale=grad_scale)
        self._follow()
        b = self._buffers(x.shape[0], 0, training=True)
        self._forward(b, x, residual, tokens)
        if x.shape[0]:
            lc.token_logprob_bwd(b["token"], b["logits"], tokens, b["lse"], b["entropy"], dlogprob, dentropy, b["dlogits"], self.padded)
            w = self.params["w"] if self.w_lowp is None else self.w_lowp
            lc.conv2d_bwd_data(b["product"], b["dlogits"], w, b["dy"], b["ws"])
            lc.conv2d_bwd_weight(b["product"], b["y"], b["dlogits"], self.grads["w"], b["ws"])
            lc.rmsnorm_bwd(b["norm"], b["total"] if residual is not None else x, b["dy"], dtotal, self.params["gamma"], b["rstd"], b["dx"],
                           self.grads["gamma"], b["ws"])
        else:                                                     # gradients are sums over no rows
            for g in self.grads.values():
                g.zero_()
        self.steps += 1
        decays = [self.weight_decay, 0.0]                         # the norm's scale is not decayed
        if self.states_in_8_bits:
            lc.adamw_step_q8(self._adam, self.lr, *self.betas, self.adam_eps, self.weight_decay, self.steps, self.steps, decays, grad_scale)
        else:
            lc.adamw_step(self._adam, self.lr, *self.betas, self.adam_eps, self.weight_decay, self.steps, decays, grad_scale)
        return b["logprob"], b["entropy"], b["dx"]

    def packed(self, x, residual, group: int = 128):
        """x + residual and its norm as e4m3 codes with a scale for every `group` columns (0: one a row)."""
        rows = x.shape[0]
        self._check(rows, x=x, residual=residual)
        self._follow()
        total = torch.empty((rows, self.width), dtype=self.type, device=self.dev) if residual is not None else None
        codes = torch.empty((rows, self.width), dtype=torch.float8_e4m3fn, device=self.dev)
        scales = torch.empty((rows, -(-self.width // group) if group else 1), device=self.dev)
        if rows:
            lc.rmsnorm_fwd_q8(lc.RmsNormDesc(rows, self.width, eps=self.eps, dtype=self.dtype), x, residual, self.params["gamma"], total, codes, scales, group)
        return total, codes, scales
