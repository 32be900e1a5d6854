"""A self-attention layer served from quantized weights and a quantized key/value cache, scored under a bit configuration:
the evaluation step of the paper's searches (Alg. 1, Alg. 2) for the layers and the state of a generating model, built
from libmpq calls only.

The layer is o = W_out attention(q, k, v), (q, k, v) = W_qkv x, causal, with groups of query heads sharing key heads.
Three tensors have a width each (2..8): the weights W_qkv and W_out (Eq. 1, a step per output channel) and the cache
(Eq. 1, a step per page and head).  Inputs of the linear layers are quantized to `act_bits` with a step per token, so that
nothing has to be calibrated beforehand.  Sequences run as a serving program runs them: their prompts in one call, then
single tokens.  The accuracy handed to the searches is 1 - SSE / ||Y_ref||^2 against the layer in fp32.  torch
supplies device memory and that reference, nothing else.
"""
from __future__ import annotations

from typing import Dict, List, Sequence, Tuple

from . import mpq


class QuantAttention:
    #: what the widths of a configuration belong to, in their order
    TENSORS = ("qkv weights", "output weights", "cache")

    def __init__(self, x, lengths: Sequence[int], w_qkv, w_out, kv_heads: int, dim: int, bit_widths: Sequence[int],
                 single_tokens: int = 1, act_bits: int = 8, page: int = 16):
        """x: device tensor [sum(lengths), K] (float32, bfloat16 or float16), the sequences' tokens one after another;
        w_qkv: fp32 [(q_heads + 2 kv_heads) dim, K]; w_out: fp32 [N, q_heads dim]; bit_widths: the widths a tensor may be
        given; single_tokens: how many of a sequence's last tokens come one by one."""
        import torch
        self.torch = torch
        self.kv_heads, self.dim, self.act_bits, self.page = int(kv_heads), int(dim), int(act_bits), int(page)
        self.q_heads = w_out.shape[1] // self.dim
        if w_out.shape[1] != self.q_heads * self.dim or w_qkv.shape[0] != (self.q_heads + 2 * self.kv_heads) * self.dim:
            raise ValueError("w_qkv and w_out do not fit heads of %d channels" % self.dim)
        if w_qkv.shape[1] != x.shape[1] or x.shape[0] != sum(lengths):
            raise ValueError("x does not fit the weights or the lengths")
        self.x, self.bit_widths = x.contiguous(), [int(b) for b in bit_widths]
        self.ws = mpq.Workspace()
        self.w_qkv, self.w_out = (self._at_widths(w.contiguous()) for w in (w_qkv, w_out))

        # the calls of a run: prompts, then a token of each sequence that still has one
        lengths = [int(n) for n in lengths]
        starts = [sum(lengths[:s]) for s in range(len(lengths))]
        most = max(lengths)
        per_seq = (most + self.page - 1) // self.page
        self.pages = len(lengths) * per_seq
        table = torch.arange(self.pages, dtype=torch.int32, device=x.device).view(len(lengths), per_seq)
        self.calls = []
        for step in range(int(single_tokens) + 1):
            done = [max(n - int(single_tokens) + step, 0) for n in lengths]      # tokens of each sequence after this call
            new = done if step == 0 else [min(1, d) for d in done]
            rows = [s0 + i for s0, d, n in zip(starts, done, new) for i in range(d - n, d)]
            if not rows:
                continue
            ends = [sum(new[:s]) for s in range(len(new) + 1)]
            put = lambda a: torch.tensor(a, dtype=torch.int32, device=x.device)  # noqa: E731
            self.calls.append((torch.tensor(rows, device=x.device), mpq.KvBatch(put(ends), put(done), table, len(rows), max(new), most)))

        self.y_ref = self._reference(lengths, w_qkv, w_out)
        self.ref_norm2 = float((self.y_ref.double() ** 2).sum().item())
        self.caches: Dict[int, mpq.KvCache] = {}
        self.scored: Dict[Tuple[int, ...], float] = {}
        self.evaluations = 0

    def __len__(self):
        return len(self.TENSORS)

    def _at_widths(self, w):
        """{width: (codes or packed nibbles, steps, bits they are stored in)}"""
        absmax, out = mpq.calibrate_absmax(w, mpq.PER_ROW, ws=self.ws), {}
        for b in self.bit_widths:
            store = 4 if b <= 4 and w.shape[1] % 2 == 0 else 8
            _, codes, packed = mpq.fake_quant(w, absmax, b, mpq.PER_ROW, want_y=False, want_codes=store == 8, want_packed4=store == 4)
            out[b] = (codes if store == 8 else packed, mpq.scale_from_absmax(absmax, b), store)
        return out

    def _reference(self, lengths, w_qkv, w_out):
        torch, out, at = self.torch, [], 0
        for n in lengths:
            qkv = (self.x[at:at + n].float() @ w_qkv.t()).view(n, -1, self.dim).transpose(0, 1).contiguous()
            at += n
            q, k, v = qkv[:self.q_heads], qkv[self.q_heads:self.q_heads + self.kv_heads], qkv[self.q_heads + self.kv_heads:]
            k, v = (t.repeat_interleave(self.q_heads // self.kv_heads, 0) for t in (k, v))
            p = torch.bmm(q, k.transpose(1, 2).contiguous()) * self.dim ** -0.5
            later = torch.ones(n, n, dtype=torch.bool, device=p.device).triu(1)
            o = torch.bmm(p.masked_fill(later, -float("inf")).softmax(-1), v)
            out.append(o.transpose(0, 1).reshape(n, -1) @ w_out.t())
        return torch.cat(out).contiguous()

    def step(self, x, batch, cache, bits: Sequence[int]):
        """The layer on new tokens x [rows, K] of the batch's sequences, which go into the cache: y [rows, N] of x's type."""
        w, scale, store = self.w_qkv[int(bits[0])]
        qkv = mpq.linear_tokens(x, w, scale, store, bits=self.act_bits).view(x.shape[0], -1, self.dim)
        mpq.kv_append(cache, batch, qkv[:, self.q_heads:self.q_heads + self.kv_heads], qkv[:, self.q_heads + self.kv_heads:])
        o = mpq.kv_attention(cache, batch, qkv[:, :self.q_heads])
        w, scale, store = self.w_out[int(bits[1])]
        return mpq.linear_tokens(o.view(x.shape[0], -1), w, scale, store, bits=self.act_bits)

    def run(self, bits: Sequence[int]):
        """All tokens of all sequences, prompts first, then one by one: y [sum(lengths), N]."""
        width = int(bits[2])
        cache = self.caches.get(width)
        if cache is None:   # (never cleared: what a run reads it has written before)
            cache = self.caches[width] = mpq.KvCache.empty(self.pages, self.kv_heads, self.page, self.dim, width, self.x.device)
        y = self.x.new_empty((self.x.shape[0], self.y_ref.shape[1]))
        for rows, batch in self.calls:
            y[rows] = self.step(self.x[rows], batch, cache, bits)
        return y

    def evaluate(self, bits: Sequence[int]) -> float:
        """Accuracy 1 - SSE / ||Y_ref||^2 with W_qkv, W_out and the cache at bits[0], bits[1], bits[2]."""
        self.evaluations += 1
        sse = mpq.sse_pair(self.run(bits).float(), self.y_ref, ws=self.ws)
        return 1.0 - float(sse.item()) / self.ref_norm2

    def evaluate_once(self, bits: Sequence[int]) -> float:
        """evaluate() behind a table of the configurations already scored."""
        key = tuple(int(b) for b in bits)
        if key not in self.scored:
            self.scored[key] = self.evaluate(bits)
        return self.scored[key]

    def sensitivity(self, b: int) -> List[float]:
        """What the score loses when one tensor alone is at width b, the others at the widest."""
        top = [max(self.bit_widths)] * len(self)
        base = self.evaluate_once(top)
        return [base - self.evaluate_once(top[:i] + [b] + top[i + 1:]) for i in range(len(self))]

    def order_by(self, sensitivity: Sequence[float]) -> List[int]:
        """Tensor numbers in ascending order of sensitivity (ties: lower number first)."""
        return sorted(range(len(self)), key=lambda i: (sensitivity[i], i))

    def bisection(self, order, target):
        return mpq.search_bisection(order, sorted(self.bit_widths, reverse=True), target, self.evaluate_once, True)

    def greedy(self, order, target):
        return mpq.search_greedy(order, sorted(self.bit_widths, reverse=True), target, self.evaluate_once)
