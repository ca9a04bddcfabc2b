"""A whole training step of a small token model on the device: embeddings with a scale, blocks that each add a product of the stream's layer norm to the stream, and the output side of
token_head_step.py; embeddings, norms and classifier are updated by AdamW, the blocks' square matrices by the orthogonalised step.  Every operator is a call into the C library; this module only
owns parameters, states and the order of calls, and torch is used for device memory.

    model = TokenModelStep(width=1024, vocab=32000, blocks=4, dtype=lc.LC_BF16)
    logprob, entropy = model.step(tokens, targets, dlogprob)        # dlogprob: the loss's gradient with respect to each log probability
    logprob, entropy, ids, top = model.score(tokens, targets, top=5)     # one token or many, nothing is updated

stream_0 = scale * table[tokens];  stream_{l+1} = stream_l + W_l LN_l(stream_l);  the head's norm, classifier and log probabilities of the targets read the last one.  A token outside the table
enters as zeros, a target outside the vocabulary does not count.

What a call works in comes from torch's allocator on the call's stream; parameters and states are shared, so that a call on another stream than the last waits for it (a graph's replays and
other threads have to see to that themselves).  A graph replays the step number of its recording.
"""
from __future__ import annotations

import contextlib
import math
from typing import Dict, List, Optional

import torch

from . import larsconv as lc
from .token_head_step import TokenHeadStep


class TokenModelStep:
    def __init__(self, width: int, vocab: int, blocks: int, dtype: int = lc.LC_BF16, scale: Optional[float] = None, eps: float = 1e-5, lr: float = 1e-3, matrix_lr: float = 0.02,
                 momentum: float = 0.95, beta1: float = 0.9, beta2: float = 0.95, adam_eps: float = 1e-8, weight_decay: float = 0.1, device: str = "cuda:0"):
        self.head = TokenHeadStep(width, vocab, dtype, eps=eps, lr=lr, beta1=beta1, beta2=beta2, adam_eps=adam_eps, weight_decay=weight_decay, device=device)
        self.dev, self.width, self.vocab, self.blocks, self.dtype, self.eps = device, width, vocab, blocks, dtype, eps
        self.type = torch.bfloat16 if dtype == lc.LC_BF16 else torch.float32
        self.scale = math.sqrt(width) if scale is None else scale
        self.lr, self.matrix_lr, self.momentum, self.betas, self.adam_eps, self.weight_decay, self.steps = lr, matrix_lr, momentum, (beta1, beta2), adam_eps, weight_decay, 0
        f32 = dict(dtype=torch.float32, device=device)
        names = ["table"] + [f"{n}{l}" for l in range(blocks) for n in ("gamma", "beta")]
        self.params: Dict[str, torch.Tensor] = {"table": torch.zeros((vocab, width), **f32)}
        self.params |= {k: (torch.ones if k.startswith("gamma") else torch.zeros)(width, **f32) for k in names[1:]}
        self.params |= {f"w{l}": torch.zeros((width, width), **f32) for l in range(blocks)}
        self.grads = {k: torch.zeros_like(p) for k, p in self.params.items()}
        lowp = dtype == lc.LC_BF16
        self.lowp = {k: torch.zeros(self.params[k].shape, dtype=self.type, device=device) for k in ["table"] + [f"w{l}" for l in range(blocks)]} if lowp else {}
        of = lambda d, keys: [d[k] for k in keys]
        self.m, self.v = ({k: torch.zeros(self.params[k].shape, **f32) for k in names} for _ in range(2))
        self._decays = [weight_decay if k == "table" else 0.0 for k in names]                       # the norms' scales and shifts are not decayed
        self._adam = lc.AdamWArgs(of(self.params, names), of(self.grads, names), of(self.m, names), of(self.v, names),
                                  w_lowp=[self.lowp.get(k) for k in names] if lowp else None)
        matrices = [f"w{l}" for l in range(blocks)]
        self.m |= {k: torch.zeros((width, width), **f32) for k in matrices}
        self._muon = lc.MuonArgs(of(self.params, matrices), of(self.grads, matrices), of(self.m, matrices), w_lowp=of(self.lowp, matrices) if lowp else None)
        self._muon_room = torch.empty(lc.muon_workspace_bytes(self._muon), dtype=torch.uint8, device=device)
        self._cuda = self.params["table"].is_cuda
        self._stream = torch.cuda.current_stream(self.params["table"].device) if self._cuda else None      # the last call's

    def load(self, params: Dict[str, torch.Tensor], classifier: torch.Tensor, head_gamma: torch.Tensor) -> None:
        """Sets parameters by name (table [vocab][width], w0, gamma0, beta0, w1, ...) and the head's."""
        with self._call():
            for k, p in params.items():
                self.params[k].copy_(p)
                if k in self.lowp:
                    self.lowp[k].copy_(self.params[k])
            self.head.load(classifier, head_gamma)

    @contextlib.contextmanager
    def _call(self):
        """On this object's device, behind the last call where that was on another stream (not while a graph records, which runs nothing)."""
        if not self._cuda:
            yield
            return
        with torch.cuda.device(self.params["table"].device):
            stream = torch.cuda.current_stream()
            if stream != self._stream and not torch.cuda.is_current_stream_capturing():
                stream.wait_stream(self._stream)
                self._stream = stream
            yield

    def _check(self, rows: int, **tensors: Optional[torch.Tensor]) -> None:
        for name, t in tensors.items():
            dtype, shape = torch.int32 if name in ("tokens", "targets") else torch.float32, (1,) if name == "grad_scale" else (rows,)
            if t is None and name not in ("tokens", "targets", "dlogprob"):
                continue
            if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device != self.params["table"].device or not t.is_contiguous() or \
                    (t.numel() != 1 if name == "grad_scale" else tuple(t.shape) != shape):
                raise ValueError(f"{name}: a contiguous {dtype} tensor of shape {shape} on {self.params['table'].device} is needed, got " +
                                 (f"{t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}" if isinstance(t, torch.Tensor) else f"{t!r}"))

    def _weights(self, name: str) -> torch.Tensor:
        return self.lowp.get(name, self.params[name])

    def _room(self, nbytes: int) -> Optional[torch.Tensor]:
        return torch.empty(nbytes, dtype=torch.uint8, device=self.dev) if nbytes else None

    def _descs(self, rows: int):
        return (lc.EmbeddingDesc(rows, self.vocab, self.width, scale=self.scale, table_dtype=self.dtype, dtype=self.dtype),
                lc.LayerNormDesc(rows, self.width, eps=self.eps, dtype=self.dtype),
                lc.ConvDesc(rows, self.width, 1, 1, self.width, 1, 1, dtype=self.dtype))

    def _forward(self, tokens: torch.Tensor):
        """(what each block keeps for its gradient, the last product or the embeddings, the stream before it)."""
        rows = tokens.shape[0]
        embed, norm, product = self._descs(rows)
        new = lambda *shape, dtype=self.type: torch.empty(shape, dtype=dtype, device=self.dev)
        x, stream, kept = new(rows, self.width), None, []
        lc.embedding_fwd(embed, self._weights("table"), tokens, x)
        if rows == 0:                                             # (the product takes no empty batch)
            return kept, x, stream
        room = self._room(lc.conv2d_workspace_bytes(product, lc.LC_PASS_FWD))
        for l in range(self.blocks):
            total, y, mean, rstd, out = new(rows, self.width) if stream is not None else None, new(rows, self.width), new(rows, dtype=torch.float32), \
                new(rows, dtype=torch.float32), new(rows, self.width)
            lc.layernorm_fwd(norm, x, stream, self.params[f"gamma{l}"], self.params[f"beta{l}"], total, y, mean, rstd)
            stream = x if total is None else total
            kept.append((stream, y, mean, rstd))
            lc.conv2d_fwd(product, y, self._weights(f"w{l}"), out, room)
            x = out
        return kept, x, stream

    def _backward(self, kept: List[tuple], d: torch.Tensor, norm, product) -> torch.Tensor:
        """The blocks' gradients from that of the last product and of the stream before it, which are the same; returns that of the embeddings."""
        room = self._room(max([lc.layernorm_bwd_workspace_bytes(norm)] + [lc.conv2d_workspace_bytes(product, p) for p in (lc.LC_PASS_BWD_DATA, lc.LC_PASS_BWD_WEIGHT)]))
        dy = torch.empty_like(d)
        for l in reversed(range(self.blocks)):
            total, y, mean, rstd = kept[l]
            lc.conv2d_bwd_data(product, d, self._weights(f"w{l}"), dy, room)
            lc.conv2d_bwd_weight(product, y, d, self.grads[f"w{l}"], room)
            dx = torch.empty_like(d)
            lc.layernorm_bwd(norm, total, dy, d, self.params[f"gamma{l}"], mean, rstd, dx, self.grads[f"gamma{l}"], self.grads[f"beta{l}"], room)
            d = dx
        return d

    def score(self, tokens: torch.Tensor, targets: torch.Tensor, top: int = 0):
        """Log probability and entropy of each row's target (int32; outside the vocabulary: does not count), and the `top` likeliest tokens with theirs, in the head's buffers."""
        self._check(tokens.shape[0], tokens=tokens, targets=targets)
        with self._call():
            _, x, stream = self._forward(tokens)
            return self.head.score(x, stream, targets, top)

    def step(self, tokens: torch.Tensor, targets: torch.Tensor, dlogprob: torch.Tensor, dentropy: Optional[torch.Tensor] = None, grad_scale: Optional[torch.Tensor] = None):
        """Forward, backward and update.  dlogprob, dentropy: gradient of the loss with respect to each row's log probability and entropy; grad_scale: one float on the device, multiplies
        the parameters' gradients in their updates.  Returns the rows' log probabilities and entropies, in the head's buffers; gradients are in self.grads and self.head.grads."""
        rows = tokens.shape[0]
        self._check(rows, tokens=tokens, targets=targets, dlogprob=dlogprob, dentropy=dentropy, grad_scale=grad_scale)
        with self._call():
            kept, x, stream = self._forward(tokens)
            logprob, entropy, d = self.head.step(x, stream, targets, dlogprob, dentropy, None, grad_scale)
            embed, norm, product = self._descs(rows)
            if rows:
                d = self._backward(kept, d, norm, product)
            else:                                                 # gradients are sums over no rows
                for k in self.grads:
                    self.grads[k].zero_()
            lc.embedding_bwd(embed, tokens, d, self.grads["table"], self._room(lc.embedding_bwd_workspace_bytes(embed)))
            self.steps += 1
            lc.adamw_step(self._adam, self.lr, *self.betas, self.adam_eps, self.weight_decay, self.steps, self._decays, grad_scale)
            lc.muon_step(self._muon, self.matrix_lr, self.momentum, self.weight_decay, self._muon_room, grad_scale=grad_scale)
            return logprob, entropy
