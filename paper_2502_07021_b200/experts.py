"""A routed-expert layer on the library's router and 4-bit products.

    python -m paper_2502_07021_b200.experts        # small demonstration on cuda:0

``RoutedExperts`` is the serving form: tokens are scored, balanced against the experts' shares by Sinkhorn iterations (the
duals are added to the scores for the choice only), ordered by expert, rounded to 4 bits once each, and sent through their
experts' 4-bit matrices.  A prompt is balanced by itself; a decode step takes the duals that were kept from a batch
(``layer.duals``), since a few tokens say nothing about the experts' load.  ``route`` is the training form of the router alone: a differentiable function of the scores whose
backward pass is ``fs_router_backward``.

Everything runs on the current stream of the tensors' device; the balance, choice, ordering and products are the library's
kernels, torch does the scoring product, the activation between the two expert products and the weighted sum at the end.
"""
from __future__ import annotations

import torch

from . import binding as fs


def _launch(device, call, *args):
    """The call on the device's current stream, with the device selected: a launch goes to the current device."""
    if torch.cuda.current_device() == device.index:
        return call(*args, torch.cuda.current_stream(device))
    with torch.cuda.device(device):
        call(*args, torch.cuda.current_stream(device))


def _scratch(tokens, experts, topk, device):
    size = fs.fs_router_workspace(tokens, experts, topk)
    if size == 0:
        raise ValueError(f"unsupported router size: {tokens} tokens, {experts} experts, top {topk}")
    return torch.empty(size, dtype=torch.uint8, device=device), size


def _rows(x):
    """x itself where its rows lie one after another with their entries side by side, else a copy that does."""
    ok = (x.shape[1] < 2 or x.stride(1) == 1) and (x.shape[0] < 2 or x.stride(0) >= x.shape[1])
    return x if ok else x.contiguous()


def _scores(logits):
    if logits.dim() != 2 or not logits.is_cuda:
        raise ValueError("logits: a CUDA tensor [tokens, experts]")
    if logits.shape[1] > 1 and logits.stride(1) != 1:
        raise ValueError("logits: the experts of a token lie next to each other")
    return logits.shape[0], logits.shape[1], fs.fs_dtype(logits)


def _mask(mask, logits):
    if mask is None:
        return None
    if mask.shape != logits.shape[:1] or mask.dtype not in (torch.uint8, torch.bool):
        raise ValueError("mask: one byte or truth value per token")
    _together(logits.device, mask=mask)
    return mask.view(torch.uint8).contiguous()


def _per_expert(v, name, logits):
    if v is None:
        return None
    if v.shape != logits.shape[1:] or v.dtype != torch.float32:
        raise ValueError(f"{name}: float32 [experts]")
    _together(logits.device, **{name: v})
    return v.contiguous()


def _together(device, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != device:
            raise ValueError(f"{name}: on {t.device}, expected {device}")


def _packed(t, name, lead, need):
    """Distance in bytes between the rows of codes or scale bytes [..., >= need], rows of a stack all equally far apart."""
    if t.dtype != torch.uint8 or t.shape[:-1] != lead or t.shape[-1] < need or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name}: uint8 {[*lead]} rows of {need} bytes or more")
    if len(lead) == 2 and min(lead) > 1 and t.stride(0) != lead[1] * t.stride(1):
        raise ValueError(f"{name}: a stack whose matrices follow one another")
    apart = [d for d in range(len(lead)) if lead[d] > 1]
    return t.stride(apart[-1]) if apart else -(-need // 4) * 4      # one row: no distance


def balance(logits, eps, iters, mask=None, share=None, start=None):
    """Duals of the balanced assignment of the tokens to the experts.

    Returns (f [tokens], g [experts], err [iters]): see fs_router_duals.  g is the bias for ``choose`` and ``route``."""
    tokens, experts, dtype = _scores(logits)
    work, size = _scratch(tokens, experts, 1, logits.device)
    f, g, err = (torch.empty(n, device=logits.device) for n in (tokens, experts, iters))
    _launch(logits.device, fs.fs_router_duals, logits, dtype, logits.stride(0), tokens, experts, _mask(mask, logits),
            _per_expert(share, "share", logits), eps, iters, _per_expert(start, "start", logits), f, g, err, work, size)
    return f, g, err


def choose(logits, topk, bias=None, mask=None, normalize=True):
    """Inference form: (idx [tokens, topk] int32, gate [tokens, topk])."""
    tokens, experts, dtype = _scores(logits)
    work, size = _scratch(tokens, experts, topk, logits.device)
    idx = torch.empty(tokens, topk, dtype=torch.int32, device=logits.device)
    gate = torch.empty(tokens, topk, device=logits.device)
    _launch(logits.device, fs.fs_router_forward, logits, dtype, logits.stride(0), tokens, experts, _mask(mask, logits),
            _per_expert(bias, "bias", logits), topk, fs.FS_ROUTE_NORMALIZE if normalize else 0, idx, gate, None, None, None, None, None,
            work, size)
    return idx, gate


class _Route(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, topk, bias, mask, normalize):
        tokens, experts, dtype = _scores(logits)
        dev = logits.device
        mask, bias = _mask(mask, logits), _per_expert(bias, "bias", logits)
        work, size = _scratch(tokens, experts, topk, dev)
        idx = torch.empty(tokens, topk, dtype=torch.int32, device=dev)
        counts = torch.empty(experts + 1, dtype=torch.int32, device=dev)
        gate, lse = torch.empty(tokens, topk, device=dev), torch.empty(tokens, device=dev)
        load, prob, loss = (torch.empty(n, device=dev) for n in (experts, experts, 2))
        flags = fs.FS_ROUTE_NORMALIZE if normalize else 0
        _launch(dev, fs.fs_router_forward, logits, dtype, logits.stride(0), tokens, experts, mask, bias, topk, flags, idx, gate, lse,
                counts, load, prob, loss, work, size)
        ctx.save_for_backward(logits, idx, gate, lse, counts, load, mask)   # a mask changed in place is noticed
        ctx.flags = flags
        ctx.mark_non_differentiable(idx, counts)
        ctx.set_materialize_grads(False)
        return gate, loss, idx, counts

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_gate, d_loss, _idx, _counts):
        logits, idx, gate, lse, counts, load, mask = ctx.saved_tensors
        tokens, experts, dtype = _scores(logits)
        out = torch.empty(tokens, experts, dtype=logits.dtype, device=logits.device)
        _launch(logits.device, fs.fs_router_backward, logits, dtype, logits.stride(0), tokens, experts, mask, idx.shape[1], ctx.flags,
                idx, gate, lse, counts, load, None if d_gate is None else d_gate.float().contiguous(),
                None if d_loss is None else d_loss.float().contiguous(), out, out.stride(0))
        return out, None, None, None, None


def route(logits, topk, bias=None, mask=None, normalize=True):
    """Training form: (gate, loss, idx, counts); gate and loss = (balance, mean squared logsumexp) carry first derivatives."""
    return _Route.apply(logits, topk, bias, mask, normalize)


def quantize(x):
    """(codes, scale bytes) of a matrix or a stack [groups, rows, cols] of them, on the 4-bit microscaled grid."""
    flat = _rows(x.reshape(-1, x.shape[-1]))
    q, s = fs.mx4_empty(flat.shape[0], flat.shape[1], x.device)
    _launch(x.device, fs.fs_mx4_quantize, flat, fs.fs_dtype(flat), flat.stride(0), flat.shape[0], flat.shape[1], None, 1, flat.shape[0],
            q, q.stride(0), s, s.stride(0))
    return q.view(*x.shape[:-1], q.shape[1]), s.view(*x.shape[:-1], s.shape[1])


def product(xq, xs, weights, offsets, cols, dtype):
    """Rows ordered by group times their group's 4-bit weights (codes, scales) [groups, outs, ...].

    offsets: int32 [groups + 1], None for one group of all rows."""
    wq, ws = weights
    rows, groups, outs, nb = xq.shape[0], wq.shape[0], wq.shape[1], -(-cols // 32)
    _together(xq.device, xs=xs, wq=wq, ws=ws, offsets=offsets)
    if offsets is not None:
        if offsets.dtype != torch.int32 or offsets.shape != (groups + 1,):
            raise ValueError("offsets: int32 [groups + 1]")
        offsets = offsets.contiguous()
    pitches = [_packed(t, name, lead, need) for t, name, lead, need in (
        (xq, "xq", (rows,), 16 * nb), (xs, "xs", (rows,), nb), (wq, "wq", (groups, outs), 16 * nb), (ws, "ws", (groups, outs), nb))]
    return _product(xq, xs, wq, ws, pitches, offsets, outs, cols, dtype)


def _product(xq, xs, wq, ws, pitches, offsets, outs, cols, dtype):
    y = torch.empty(xq.shape[0], outs, dtype=dtype, device=xq.device)
    _launch(xq.device, fs.fs_mx4_product, xq, pitches[0], xs, pitches[1], xq.shape[0], wq, pitches[2], ws, pitches[3], wq.shape[0], offsets,
            outs, cols, y, fs.fs_dtype(y), y.stride(0))
    return y


class RoutedExperts:
    """y_t = sum_j gate_tj W2_e silu(W1_e x_t), e = idx_tj, with 4-bit W1 [experts, hidden, width], W2 [experts, width, hidden]."""

    def __init__(self, score, up, down, topk, eps=0.2, iters=8):
        experts, hidden, width = up.shape
        if score.shape != (experts, width) or down.shape != (experts, width, hidden):
            raise ValueError("score [experts, width], up [experts, hidden, width], down [experts, width, hidden]")
        _together(score.device, up=up, down=down)
        self.score, self.topk, self.eps, self.iters = score, topk, eps, iters
        self.width, self.hidden = width, hidden
        self.up, self.down = quantize(up), quantize(down)   # laid out once

    @staticmethod
    def _times(xq, xs, weights, offsets, outs, cols, dtype):
        packed = (xq, xs, *weights)                     # all of them made by quantize: dense rows
        return _product(*packed, [t.shape[-1] for t in packed], offsets, outs, cols, dtype)

    def duals(self, x, mask=None):
        """Duals [experts] of a batch's balance, to be kept and handed to later calls as their bias.

        Fewer tokens than experts are not balanced, the duals are then 0: with a share of less than one token per expert the
        balance spreads every token over several experts whatever its scores are; one token alone ends up indifferent."""
        x, mask = self._batch(x, mask)
        return self._duals(x @ self.score.T, mask)

    def _batch(self, x, mask):
        if x.dim() != 2 or x.shape[1] != self.width:
            raise ValueError("x: [tokens, width]")
        _together(x.device, score=self.score)
        x = _rows(x)
        return x, _mask(mask, x)

    def _duals(self, logits, mask):
        tokens, experts = logits.shape
        if tokens < experts:
            return torch.zeros(experts, device=logits.device)
        # a token whose scores are no numbers would make every dual NaN: it takes no part, and its gates are NaN
        sound = logits.amax(1) < float("inf")
        if mask is None:
            return balance(logits, self.eps, self.iters, sound)[1]
        sound &= mask != 0
        g = balance(logits, self.eps, self.iters, sound)[1]
        return torch.where(sound.sum() >= experts, g, 0.0)

    def __call__(self, x, mask=None, bias=None):
        """(y [tokens, width], idx [tokens, topk]).  mask: 0 for padding.  bias: duals [experts] for the choice, kept from an
        earlier batch (``duals``); None for those of this batch."""
        x, mask = self._batch(x, mask)
        tokens, experts = x.shape[0], self.score.shape[0]
        logits = x @ self.score.T
        if bias is None:
            bias = self._duals(logits, mask)
        idx, gate = choose(logits, self.topk, bias, mask)
        pairs = tokens * self.topk
        work, size = _scratch(tokens, experts, self.topk, x.device)
        i32 = dict(dtype=torch.int32, device=x.device)
        offsets, rows, slot = torch.empty(experts + 1, **i32), torch.empty(pairs, **i32), torch.empty(tokens, self.topk, **i32)
        _launch(x.device, fs.fs_router_dispatch, idx, tokens, self.topk, experts, offsets, rows, slot, work, size)
        xq, xs = fs.mx4_empty(pairs, self.width, x.device)
        _launch(x.device, fs.fs_mx4_quantize, x, fs.fs_dtype(x), x.stride(0), tokens, self.width, slot, self.topk, pairs, xq,
                xq.stride(0), xs, xs.stride(0))
        h = torch.nn.functional.silu(self._times(xq, xs, self.up, offsets, self.hidden, self.width, x.dtype))
        y = self._times(*quantize(h), self.down, offsets, self.width, self.hidden, x.dtype)
        # where some slot is -1 there are fewer ordered rows than slots, and the last row, which -1 names, is in no group: zeros
        picked = y[slot.view(-1)].view(tokens, self.topk, self.width)
        return torch.einsum("tkw,tk->tw", picked.float(), gate).to(x.dtype), idx


def main():
    torch.manual_seed(0)
    tokens, experts, width, hidden, topk = 4096, 32, 1024, 512, 4
    dev = "cuda:0"
    x = torch.randn(tokens, width, device=dev, dtype=torch.bfloat16)
    score = torch.randn(experts, width, device=dev, dtype=torch.bfloat16) / width ** 0.5
    x = x + 4 * score[:3].sum(0)                       # three experts that everybody likes
    layer = RoutedExperts(score, torch.randn(experts, hidden, width, device=dev, dtype=torch.bfloat16) / width ** 0.5,
                          torch.randn(experts, width, hidden, device=dev, dtype=torch.bfloat16) / hidden ** 0.5, topk)
    logits = x @ score.T
    for name, bias in (("scores alone", None), ("balanced", balance(logits, 0.2, 8)[1])):
        leaf = logits.detach().float().requires_grad_()
        gate, loss, idx, counts = route(leaf, topk, bias)
        (loss[0] + 1e-3 * loss[1] + (gate * gate).sum() / tokens).backward()
        c = counts[:experts].float()
        print(f"{name}: fullest expert {c.max() / c.mean():.2f} of the mean, balance loss {loss[0]:.3f}, "
              f"gradient norm {leaf.grad.norm():.3e}")
    y, _ = layer(x)
    print(f"layer output {tuple(y.shape)} {y.dtype}, rms {y.float().pow(2).mean().sqrt():.3f}")
    y, idx = layer(x[:1], bias=layer.duals(x))         # a decode step with the batch's duals
    print(f"one token: experts {idx[0].tolist()}, rms {y.float().pow(2).mean().sqrt():.3f}")


if __name__ == "__main__":
    main()
