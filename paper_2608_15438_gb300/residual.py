"""A residual encoder on the library's operators (ops.py), trained with L_sim.

E(x) = W_h norm(r_n) + b_h with r_0 = W_s (in_scale x) + b_s and blocks
    r_{i+1} = r_i + W_2 act(W_1 norm(r_i) + b_1) + b_2,
norm the layer norm, act GELU. The index file holds Linear-ReLU encoders only; this one's
logits go to the index build and the search as given logits
(nr_build_set_logits, nr_search_logits).

L_sim (train.lsim_loss) couples every pair of a mini-batch, so a batch cannot be
cut into smaller ones whose gradients are added, and all its activations are
held at once. With hold8 (the default) a block holds its input and its
pre-activations in 8 bits and computes the norm's output and the activation
again in the backward pass: 5.2 bytes a unit of width for an expansion of 4,
against 20 in 16 bits. Parameters are fp32, the products' operands bf16, the
logits and the loss fp32.

GatedEncoder is the same with what deeper encoders train more steadily with: a norm after a block
as well, a gate and a scale for what the block adds, all of that and the next block's norm in
one operator (ops.block_norm).

    python -m paper_2608_15438_gb300.residual --workload tiny --epochs 5 [--gate full --post rms --optimizer adamw8]
trains on a workload's first rows, builds an index from the encoder's logits
and prints Recall@10 of a search through it.
"""
from __future__ import annotations

import time

import torch

from . import ops, optim
from .train import lsim_loss

_DTYPE = torch.bfloat16


class _Once(torch.autograd.Function):
    """v, with a history (`anchor`'s) whose derivative is an error."""

    @staticmethod
    def forward(ctx, v, anchor):
        return v.view_as(v)

    @staticmethod
    def backward(ctx, dv):
        raise RuntimeError("the operators' backward passes have no derivatives: "
                           "gradients of gradients are not supported")


def _once(backward):
    """A backward pass without derivatives of its own. Under create_graph its
    outputs raise when they are differentiated: without a history a penalty on a
    gradient would vanish silently. (torch's once_differentiable does so only
    where the incoming gradient has a history itself.)"""

    def run(ctx, *dy):
        with torch.no_grad():
            out = backward(ctx, *dy)
        if not torch.is_grad_enabled():
            return out
        anchor = torch.empty(0, requires_grad=True)
        return tuple(None if v is None else _Once.apply(v, anchor) for v in out)

    return run


def _rows(v):
    """v as the operators take it, its rows contiguous: autograd brings expanded and
    transposed gradients."""
    return v if v.stride(1) == 1 else v.contiguous()


class _Linear(torch.autograd.Function):
    """x w^T + b with x [m x k] bf16, w fp32; out fp32 or bf16."""

    @staticmethod
    def forward(ctx, x, w, b, out_dtype):
        wh = w.to(_DTYPE)
        ctx.save_for_backward(x, wh)
        return ops.linear(x, wh, b, out_dtype=out_dtype)

    @staticmethod
    @_once
    def backward(ctx, dy):
        x, wh = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx, dw, db = ops.linear_backward(_rows(dy), x, wh, need=(need[0], True, True))
        return dx, dw.float(), db, None


class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, g, b):
        y, mean, rstd = ops.layer_norm(x, g, b, save=True)
        ctx.save_for_backward(x, g, mean, rstd)
        return y

    @staticmethod
    @_once
    def backward(ctx, dy):
        return ops.layer_norm_backward(_rows(dy), *ctx.saved_tensors)


class _Block(torch.autograd.Function):
    """r + W2 act(W1 norm(r) + b1) + b2, its activations held in 8 or 16 bits."""

    @staticmethod
    def forward(ctx, r, g, b, w1, b1, w2, b2, act, hold8):
        w1h, w2h = w1.to(_DTYPE), w2.to(_DTYPE)
        h, mean, rstd = ops.layer_norm(r, g, b, save=True)
        a, z = ops.linear(h, w1h, b1, act=act, save="z8" if hold8 else "z")
        ctx.act, ctx.hold8 = act, hold8
        # all of it through autograd, which frees it with the block's backward pass, notices
        # changes in place and offers it to saved-tensor hooks
        if hold8:
            r8 = ops.checkpoint8(r)
            held = (r8.codes, r8.scales, z.codes, z.scales)
        else:
            held = (r, z, h, a)
        ctx.save_for_backward(g, b, mean, rstd, w1h, w2h, *held)
        return ops.linear(a, w2h, b2, residual=r)

    @staticmethod
    @_once
    def backward(ctx, dy):
        dy = _rows(dy)
        g, b, mean, rstd, w1h, w2h, *held = ctx.saved_tensors
        if ctx.hold8:
            m = dy.shape[0]
            r = ops.Checkpoint8(held[0], held[1], (m, w1h.shape[1]), _DTYPE)
            z = ops.Checkpoint8(held[2], held[3], (m, w1h.shape[0]), _DTYPE)
            da, dw2, db2 = ops.linear_backward(dy, z, w2h, x_act=ctx.act)
            h = ops.layer_norm(r, g, b)
        else:
            r, z, h, a = held
            da, dw2, db2 = ops.linear_backward(dy, a, w2h)
        dh, dw1, db1 = ops.linear_backward(da, h, w1h, z=z, act=ctx.act)
        dr, dg, db = ops.layer_norm_backward(dh, r, g, mean, rstd, residual_grad=dy)
        return dr, dg, db, dw1.float(), db1, dw2.float(), db2, None, None


class ResidualEncoder(torch.nn.Module):
    """D -> width, `blocks` blocks of expansion `expand`, -> b logits (fp32)."""

    def __init__(self, D: int, width: int, blocks: int, b: int, expand: int = 4, act: str = "gelu",
                 hold8: bool = True, device="cuda", seed: int = 0):
        super().__init__()
        g = torch.Generator(device="cpu")
        g.manual_seed(seed)

        def matrix(n, k, scale=1.0):
            return torch.nn.Parameter((torch.randn(n, k, generator=g) * (scale / k ** 0.5)).to(device))

        def vector(n, value=0.0):
            return torch.nn.Parameter(torch.full((n,), value, device=device))

        self.act, self.hold8 = act, hold8
        self.stem = torch.nn.ParameterList([matrix(width, D), vector(width)])
        # W2's scale keeps the residual stream's variance from growing with depth
        self.blocks = torch.nn.ModuleList(
            torch.nn.ParameterList([vector(width, 1.0), vector(width), matrix(expand * width, width),
                                    vector(expand * width), matrix(width, expand * width, (2 * blocks) ** -0.5),
                                    vector(width)])
            for _ in range(blocks))
        self.head = torch.nn.ParameterList([vector(width, 1.0), vector(width), matrix(b, width), vector(b)])

    def forward(self, x):
        """Logits [m x b] fp32 of scaled rows x [m x D]."""
        r = _Linear.apply(_rows(x.to(_DTYPE)), self.stem[0], self.stem[1], _DTYPE)
        for p in self.blocks:
            r = _Block.apply(r, p[0], p[1], p[2], p[3], p[4], p[5], self.act, self.hold8)
        return _Linear.apply(_Norm.apply(r, self.head[0], self.head[1]), self.head[2], self.head[3], torch.float32)

    @torch.no_grad()
    def encode(self, rows, in_scale: float = 1.0, batch: int = 1 << 17, check: bool = True):
        """Logits of rows [n x D] (uint8 or fp32), `batch` rows at a time. check: waits
        for them and raises if a bounded wait expired on their way (ops.check); without it, and
        while a CUDA graph is captured, that is the caller's to do before the logits are used."""
        w = [p.to(_DTYPE) for p in (self.stem[0], self.head[2])]
        blocks = [(p[0], p[1], p[2].to(_DTYPE), p[3], p[4].to(_DTYPE), p[5]) for p in self.blocks]
        out = []
        for s in range(0, max(rows.shape[0], 1), batch):  # no rows: one empty batch
            r = ops.linear(_rows((rows[s:s + batch].float() * in_scale).to(_DTYPE)), w[0], self.stem[1])
            for g, b, w1, b1, w2, b2 in blocks:
                r = ops.linear(ops.linear(ops.layer_norm(r, g, b), w1, b1, act=self.act), w2, b2, residual=r)
            out.append(ops.linear(ops.layer_norm(r, self.head[0], self.head[1]), w[1], self.head[3],
                                  out_dtype=torch.float32))
        out = torch.cat(out) if len(out) != 1 else out[0]
        if check and out.is_cuda and not torch.cuda.is_current_stream_capturing():
            ops.check(out.device)
        return out


class _BlockNorm(torch.autograd.Function):
    """(y, h) of ops.block_norm; without u, y is r (its own view, so that both of r's gradients meet in one kernel)."""

    @staticmethod
    def forward(ctx, r, u, q, scale, post_weight, post_bias, weight, bias, options):
        y, h, stats = ops.block_norm(r, u, gate=q, scale=scale, post_weight=post_weight, post_bias=post_bias, weight=weight,
                                     bias=bias, save=True, **options)
        ctx.options = {k: v for k, v in options.items() if k != "out_dtype"}
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(y, u, q, scale, post_weight, post_bias, weight, bias, stats)
        return r.view_as(r) if u is None else y, h

    @staticmethod
    @_once
    def backward(ctx, dy, dh):
        y, u, q, scale, post_weight, post_bias, weight, bias, stats = ctx.saved_tensors
        if dy is None and dh is None:
            return (None,) * 9
        dh = torch.zeros_like(y, dtype=_DTYPE) if dh is None else _rows(dh)
        d = ops.block_norm_backward(dh, None if dy is None else _rows(dy), y, u, stats, gate=q, scale=scale,
                                    post_weight=post_weight, post_bias=post_bias, weight=weight, bias=bias, **ctx.options)
        return (*d, None)


class _Mlp(torch.autograd.Function):
    """W2 act(W1 h + b1) + b2, its input and pre-activations held in 8 or 16 bits."""

    @staticmethod
    def forward(ctx, h, w1, b1, w2, b2, act, hold8):
        w1h, w2h = w1.to(_DTYPE), w2.to(_DTYPE)
        a, z = ops.linear(h, w1h, b1, act=act, save="z8" if hold8 else "z")
        ctx.act, ctx.hold8 = act, hold8
        if hold8:
            h8 = ops.checkpoint8(h)
            held = (h8.codes, h8.scales, z.codes, z.scales)
        else:
            held = (h, z, a)
        ctx.save_for_backward(w1h, w2h, *held)
        return ops.linear(a, w2h, b2)

    @staticmethod
    @_once
    def backward(ctx, du):
        du = _rows(du)
        w1h, w2h, *held = ctx.saved_tensors
        if ctx.hold8:
            m = du.shape[0]
            h = ops.Checkpoint8(held[0], held[1], (m, w1h.shape[1]), _DTYPE)
            z = ops.Checkpoint8(held[2], held[3], (m, w1h.shape[0]), _DTYPE)
            da, dw2, db2 = ops.linear_backward(du, z, w2h, x_act=ctx.act)
        else:
            h, z, a = held
            da, dw2, db2 = ops.linear_backward(du, a, w2h)
        dh, dw1, db1 = ops.linear_backward(da, h, w1h, z=z, act=ctx.act)
        return dh, dw1.float(), db1, dw2.float(), db2, None, None


class GatedEncoder(torch.nn.Module):
    """D -> width, `blocks` blocks of expansion `expand`, -> b logits (fp32):
        r_0 = W_s (in_scale x) + b_s, h_0 = norm(r_0)
        u = W_2 act(W_1 h_i + b_1) + b_2, q = W_q h_i + b_q
        r_{i+1} = r_i + scale sigmoid(q) post(u), h_{i+1} = norm(r_{i+1})
        E(x) = W_h h_n + b_h.
    norm and post: "rms" or "layer" (post also "none"), with weights, layer norms with biases too. gate: "none",
    "row" (q one number a row) or "full". scale: a vector that begins with this value, or None. stream32 keeps r
    in fp32, for streams that move away from zero: gradients are made from r as stored."""

    def __init__(self, D: int, width: int, blocks: int, b: int, expand: int = 4, act: str = "gelu", norm: str = "rms",
                 post: str = "rms", gate: str = "full", scale=None, stream32: bool = False, hold8: bool = True,
                 device="cuda", seed: int = 0):
        super().__init__()
        if norm not in ("rms", "layer") or post not in ops.NORMS or gate not in ("none", "row", "full"):
            raise ValueError(f"norm, post, gate: {norm!r}, {post!r}, {gate!r}, expected 'rms' or 'layer', one of "
                             f"{', '.join(ops.NORMS)}, and 'none', 'row' or 'full'")
        g = torch.Generator(device="cpu")
        g.manual_seed(seed)

        def matrix(n, k, size=1.0):
            return torch.nn.Parameter((torch.randn(n, k, generator=g) * (size / k ** 0.5)).to(device))

        def vector(n, value=0.0):
            return torch.nn.Parameter(torch.full((n,), float(value), device=device))

        def of_norm(kind):
            return {"weight": vector(width, 1.0), **({"bias": vector(width)} if kind == "layer" else {})} if kind != "none" else {}

        self.act, self.norm, self.post, self.gate, self.stream32, self.hold8 = act, norm, post, gate, stream32, hold8
        self.stem = torch.nn.ParameterList([matrix(width, D), vector(width)])
        # norms[i] before block i, the last one before the head
        self.norms = torch.nn.ModuleList(torch.nn.ParameterDict(of_norm(norm)) for _ in range(blocks + 1))
        self.blocks = torch.nn.ModuleList()
        for _ in range(blocks):
            p = {"w1": matrix(expand * width, width), "b1": vector(expand * width),
                 "w2": matrix(width, expand * width, (2 * blocks) ** -0.5), "b2": vector(width)}
            p.update({f"post_{k}": v for k, v in of_norm(post).items()})
            if gate != "none":
                n = 1 if gate == "row" else width
                p.update(wq=matrix(n, width, 0.1), bq=vector(n))
            if scale is not None:
                p["scale"] = vector(width, scale)
            self.blocks.append(torch.nn.ParameterDict(p))
        self.head = torch.nn.ParameterList([matrix(b, width), vector(b)])

    def _options(self, first):
        post = "none" if first else self.post
        return {"post": post, "pre": self.norm, **({"out_dtype": _DTYPE} if first else {})}

    def forward(self, x):
        """Logits [m x b] fp32 of scaled rows x [m x D]."""
        r = _Linear.apply(_rows(x.to(_DTYPE)), self.stem[0], self.stem[1], torch.float32 if self.stream32 else _DTYPE)
        n = self.norms[0]
        r, h = _BlockNorm.apply(r, None, None, None, None, None, n["weight"], _of(n, "bias"), self._options(True))
        for p, n in zip(self.blocks, list(self.norms)[1:]):
            u = _Mlp.apply(h, p["w1"], p["b1"], p["w2"], p["b2"], self.act, self.hold8)
            q = _Linear.apply(h, p["wq"], p["bq"], _DTYPE) if "wq" in p else None
            r, h = _BlockNorm.apply(r, u, q, _of(p, "scale"), _of(p, "post_weight"), _of(p, "post_bias"), n["weight"],
                                    _of(n, "bias"), self._options(False))
        return _Linear.apply(h, self.head[0], self.head[1], torch.float32)

    @torch.no_grad()
    def encode(self, rows, in_scale: float = 1.0, batch: int = 1 << 17, check: bool = True):
        """As ResidualEncoder.encode."""
        stem, head = self.stem[0].to(_DTYPE), self.head[0].to(_DTYPE)
        blocks = [{k: v.to(_DTYPE) if k in ("w1", "w2", "wq") else v for k, v in p.items()} for p in self.blocks]
        norms = [{"weight": n["weight"], "bias": _of(n, "bias")} for n in self.norms]
        out = []
        for s in range(0, max(rows.shape[0], 1), batch):  # no rows: one empty batch
            r = ops.linear(_rows((rows[s:s + batch].float() * in_scale).to(_DTYPE)), stem, self.stem[1],
                           out_dtype=torch.float32 if self.stream32 else _DTYPE)
            _, h = ops.block_norm(r, **norms[0], **self._options(True))
            for p, n in zip(blocks, norms[1:]):
                u = ops.linear(ops.linear(h, p["w1"], p["b1"], act=self.act), p["w2"], p["b2"])
                q = ops.linear(h, p["wq"], p["bq"]) if "wq" in p else None
                r, h = ops.block_norm(r, u, gate=q, scale=p.get("scale"), post_weight=p.get("post_weight"),
                                      post_bias=p.get("post_bias"), **n, **self._options(False))
            out.append(ops.linear(h, head, self.head[1], out_dtype=torch.float32))
        out = torch.cat(out) if len(out) != 1 else out[0]
        if check and out.is_cuda and not torch.cuda.is_current_stream_capturing():
            ops.check(out.device)
        return out


def _of(parameters, name):
    return parameters[name] if name in parameters else None


def train_residual(x, in_scale: float, width: int, blocks: int, b: int, epochs: int = 100, batch: int = 4096,
                   lr: float = 2e-4, gamma: float = 0.6, q: float = 0.005, seed: int = 0, hold8: bool = True,
                   log=None, optimizer: str = "adam", weight_decay: float = 0.0, max_norm=None, gated=None):
    """Train on the rows x [n x D] (a device tensor, uint8 or fp32) with L_sim as
    train.train_encoder does; returns (encoder, history), history one (epoch,
    mean loss, mean tau_emb, seconds) per epoch. Raises after an epoch in which a
    bounded wait expired. optimizer, weight_decay, max_norm: as optim.of takes them. gated: options of a
    GatedEncoder (norm, post, gate, scale, stream32), which then is what is trained."""
    model = (ResidualEncoder(x.shape[1], width, blocks, b, hold8=hold8, device=x.device, seed=seed) if gated is None else
             GatedEncoder(x.shape[1], width, blocks, b, hold8=hold8, device=x.device, seed=seed, **gated))
    opt = optim.of(optimizer, model.parameters(), lr, weight_decay, max_norm)
    g = torch.Generator(device=x.device)
    g.manual_seed(seed)
    hist, t0 = [], time.time()
    for ep in range(epochs):
        perm = torch.randperm(x.shape[0], device=x.device, generator=g)
        tot, ttot, nb = torch.zeros((), device=x.device), torch.zeros((), device=x.device), 0
        for s in range(0, x.shape[0] - batch + 1, batch):
            xb = x[perm[s:s + batch]].float() * in_scale
            loss, tau, _ = lsim_loss(torch, xb, model(xb), gamma, q)
            opt.zero_grad()  # to None
            loss.backward()
            opt.step()
            tot += loss.detach()
            ttot += tau
            nb += 1
        ops.check(x.device)  # outputs after an expired wait are undefined: no further epoch on them
        hist.append((ep, float(tot) / max(nb, 1), float(ttot) / max(nb, 1), time.time() - t0))
        if log is not None:
            log(hist[-1])
    return model, hist


def main():
    import argparse
    import json
    import os
    import sys

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    if root not in sys.path:
        sys.path.insert(0, root)
    import synth

    from . import neuroute as nr
    from .builder import config

    ap = argparse.ArgumentParser()
    ap.add_argument("--workload", default="tiny")
    ap.add_argument("--rows", type=int, default=2_000_000, help="training rows (the base's first)")
    ap.add_argument("--epochs", type=int, default=5)
    ap.add_argument("--batch", type=int, default=4096)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--lr", type=float, default=1e-3)
    ap.add_argument("--probe", type=int, default=64)
    ap.add_argument("--clusters", type=int, default=64)
    ap.add_argument("--hold16", action="store_true", help="hold activations in 16 bits")
    ap.add_argument("--optimizer", choices=("adam", "adamw", "adamw8"), default="adam")
    ap.add_argument("--weight-decay", type=float, default=0.0)
    ap.add_argument("--max-norm", type=float, default=None, help="of all gradients (adamw, adamw8)")
    ap.add_argument("--gate", choices=("none", "row", "full"), help="a gated encoder; as --post and --norm")
    ap.add_argument("--post", choices=tuple(ops.NORMS))
    ap.add_argument("--norm", choices=("rms", "layer"))
    ap.add_argument("--scale", type=float, help="what the scale of a gated encoder's blocks begins with")
    a = ap.parse_args()
    gated = {k: v for k, v in (("gate", a.gate), ("post", a.post), ("norm", a.norm), ("scale", a.scale)) if v is not None}
    w = synth.WORKLOADS[a.workload]
    src = synth.DeviceRows(w, synth.SEED_DATA, device=0)
    model, _ = train_residual(src.rows(0, min(a.rows, w.n)), w.in_scale, a.width, a.blocks, w.bits, a.epochs,
                              a.batch, a.lr, hold8=not a.hold16, optimizer=a.optimizer, weight_decay=a.weight_decay,
                              max_norm=a.max_norm, gated=gated or None,
                              log=lambda h: print(json.dumps({"epoch": h[0], "loss": h[1], "s": h[3]}), flush=True))
    ops.check(0)
    bd = nr.Builder(config(w.dtype, w.dim, w.hidden, w.bits, w.k_max, w.t, mid=w.mid), w.n, synth.encoder_weights(w), 0)
    step = 1 << 20
    base = []
    for s in range(0, w.n, step):
        rows = src.rows(s, min(step, w.n - s))
        base.append(rows)
        bd.set_logits(model.encode(rows, w.in_scale), s)
    torch.cuda.synchronize()
    bd.finish()
    for i, rows in enumerate(base):
        bd.place(rows, i * step)
    ix = bd.end()
    qs = torch.from_numpy(synth.queries(w)).cuda()
    ids, _ = ix.search_logits(qs, model.encode(qs, w.in_scale), 10, a.probe, a.clusters)
    rec = recall_at_10(qs, base, ids, step)
    print(json.dumps({"workload": w.name, "width": a.width, "blocks": a.blocks, "P": a.probe, "C": a.clusters,
                      "recall_at_10": rec}))
    ix.close()


def recall_at_10(qs, base, ids, step):
    """Mean overlap of ids [nq x 10] with the exact 10 nearest rows of base (a
    list of row blocks of `step` rows), on at most 1000 queries."""
    nq = min(1000, qs.shape[0])
    q = qs[:nq].double()
    best_d = torch.full((nq, 10), float("inf"), device=q.device, dtype=torch.float64)
    best_i = torch.full((nq, 10), -1, device=q.device, dtype=torch.int64)
    for i, rows in enumerate(base):
        for s in range(0, rows.shape[0], 1 << 17):
            r = rows[s:s + (1 << 17)].double()
            d = (q * q).sum(1)[:, None] + (r * r).sum(1)[None] - 2.0 * (q @ r.T)
            d = torch.cat([best_d, d], 1)
            j = torch.cat([best_i, (torch.arange(r.shape[0], device=q.device) + i * step + s).expand(nq, -1)], 1)
            best_d, at = torch.topk(d, 10, dim=1, largest=False)
            best_i = j.gather(1, at)
    hit = (ids[:nq, :, None] == best_i[:, None, :]).any(2).double().mean()
    return float(hit)


if __name__ == "__main__":
    main()
