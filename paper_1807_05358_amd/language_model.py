"""A small language model on the training operators, and what they are for here: exeTimes measured on the device.

Three things, each in a few lines of its own:

* Decoder: a pre-norm decoder whose training step is written out, forward and backward, with layer norm, attention and the
  loss over the vocabulary from `operators` (plain matrix products are torch's);
* DeviceMeasure: the measurement that costcache.ExeTimeCache asks for (Section 5.1, task properties: a task's exeTime is
  taken from running the operation once at the task's output size), for the operations of such a model;
* graph / measured_costs: the model's training iteration as an operator graph with costs so measured, for Simulator and
  find_strategy.

  python -m paper_1807_05358_amd.language_model      trains a little, measures, and searches a strategy for 16 devices
"""
from __future__ import annotations

import numpy as np

from . import costcache, operators as O, workloads as W

# operations whose time at one output size differs; a backward op has BACKWARD added
T_QUERY, T_UP, T_DOWN = W.T_FC, W.T_FC + 32, W.T_FC + 64      # products: hidden -> hidden, hidden -> wide, wide -> hidden
T_NORM, T_LOSS = 10, 11
BACKWARD = 256


class Decoder:
    """parameters in `params` (name -> tensor); step() returns the mean loss and the gradient of every parameter"""

    def __init__(self, vocab, hidden, heads, layers, wide=None, dtype=None, seed=0, device="cuda"):
        import torch
        if hidden % heads:
            raise ValueError("heads share the hidden size evenly")
        self.vocab, self.hidden, self.heads, self.layers = vocab, hidden, heads, layers
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        dtype = torch.bfloat16 if dtype is None else dtype

        def matrix(rows, cols):
            return (torch.randn(rows, cols, generator=gen, device=device) * cols ** -0.5).to(dtype)

        wide = 4 * hidden if wide is None else wide
        self.params = {"embedding": matrix(vocab, hidden) * hidden ** 0.5, "words": matrix(vocab, hidden)}
        for n in range(layers):
            self.params.update({f"{n}.qkv": matrix(3 * hidden, hidden), f"{n}.out": matrix(hidden, hidden),
                                f"{n}.up": matrix(wide, hidden), f"{n}.down": matrix(hidden, wide)})
        for n in [f"{i}.{half}" for i in range(layers) for half in ("a", "b")] + ["last"]:
            self.params[n + ".w"] = torch.ones(hidden, device=device, dtype=dtype)
            self.params[n + ".b"] = torch.zeros(hidden, device=device, dtype=dtype)

    def step(self, tokens, targets, loss_scale=1.0):
        """tokens, targets: int32 [batch, length] (target -100: no loss).  Gradients are of loss_scale times the mean loss."""
        import torch
        p, H = self.params, self.heads
        B, S = tokens.shape
        N, D = B * S, self.hidden
        flat, targets = tokens.reshape(-1).long(), targets.reshape(-1)
        h, add, kept = p["embedding"][flat], None, []

        def norm(name):
            """of the running sum and what the last half layer adds to it"""
            x, res = (h, None) if add is None else (add, h)
            return O.layernorm_fwd(x, p[name + ".w"], p[name + ".b"], residual=res)

        for n in range(self.layers):
            y, h, *stat = norm(f"{n}.a")
            q, k, v = (y @ p[f"{n}.qkv"].t()).view(B, S, 3, H, D // H).permute(2, 0, 3, 1, 4).unbind()
            o, lse = O.attention_fwd(q, k, v, causal=True)
            mixed = o.transpose(1, 2).reshape(N, D)
            kept.append((f"{n}.a", y, h, stat, (q, k, v, o, lse, mixed)))
            add = mixed @ p[f"{n}.out"].t()
            y, h, *stat = norm(f"{n}.b")
            up = torch.relu(y @ p[f"{n}.up"].t())
            kept.append((f"{n}.b", y, h, stat, up))
            add = up @ p[f"{n}.down"].t()
        y, h, *stat = norm("last")
        loss, lse, _ = O.vocab_loss_fwd(y, p["words"], targets)
        live = (targets != -100).float()
        weight = live / live.sum().clamp_min(1)

        grads = {}
        dy, grads["words"] = O.vocab_loss_bwd(weight * loss_scale, y, p["words"], targets, lse)

        def norm_bwd(name, dy, h, stat, dh):
            dh, grads[name + ".w"], grads[name + ".b"] = O.layernorm_bwd(dy, h, p[name + ".w"], *stat, dh=dh)
            return dh

        dh = norm_bwd("last", dy, h, stat, None)       # of the sum: of what was added last, and of the sum before
        for name, y, h, stat, rest in reversed(kept):
            n, half = name.split(".")
            if half == "b":
                grads[f"{n}.down"] = dh.t() @ rest
                dup = (dh @ p[f"{n}.down"]) * (rest > 0)
                grads[f"{n}.up"] = dup.t() @ y
                dy = dup @ p[f"{n}.up"]
            else:
                q, k, v, o, lse, mixed = rest
                grads[f"{n}.out"] = dh.t() @ mixed
                do = (dh @ p[f"{n}.out"]).view(B, S, H, D // H).transpose(1, 2)
                dqkv = O.attention_bwd(do, q, k, v, o, lse, causal=True)
                dqkv = torch.stack([g.transpose(1, 2) for g in dqkv], 2).reshape(N, 3 * D)
                grads[f"{n}.qkv"] = dqkv.t() @ y
                dy = dqkv @ p[f"{n}.qkv"]
            dh = norm_bwd(name, dy, h, stat, dh)
        grads["embedding"] = torch.zeros_like(p["embedding"], dtype=torch.float32).index_add_(0, flat, dh.float()).to(dh.dtype)
        return (loss * weight).sum(), grads


class DeviceMeasure:
    """measure(op_type, shape) -> ns of one task of a decoder's operation on the current GPU; shape is the task's output, (sample, position,
    channel), for the loss (sample, position, word).  hidden, head_dim, wide and vocab (words of the embedding's table) say what the output's size does not.
    Tasks follow each other without a pause, so the time of a very small one is that of its launches."""

    def __init__(self, hidden, head_dim, wide=None, dtype=None, repeats=20, vocab=1024):
        import torch
        self.torch = torch
        self.hidden, self.head_dim, self.wide, self.repeats, self.vocab = hidden, head_dim, 4 * hidden if wide is None else wide, repeats, vocab
        self.dtype = torch.bfloat16 if dtype is None else dtype

    def _task(self, op_type, shape):
        torch, t = self.torch, self.dtype

        def normal(*size):
            return torch.randn(*size, device="cuda").to(t)

        b, s, c = shape
        rows, back, op_type = b * s, op_type >= BACKWARD, op_type % BACKWARD
        if op_type == T_NORM:             # the sum before it is an operation of its own in the graph
            x, w, bias = normal(rows, c), normal(c), normal(c)
            if not back:
                return lambda: O.layernorm_fwd(x, w, bias)
            _, h, mean, rstd = O.layernorm_fwd(x, w, bias)
            return lambda: O.layernorm_bwd(x, h, w, mean, rstd)
        if op_type == W.T_ATTN:           # a part smaller than a head takes the time of one
            q, k, v = (normal(b, s, -(-c // self.head_dim), self.head_dim).transpose(1, 2) for _ in range(3))
            if not back:
                return lambda: O.attention_fwd(q, k, v, causal=True)
            o, lse = O.attention_fwd(q, k, v, causal=True)
            return lambda: O.attention_bwd(q, q, k, v, o, lse, causal=True)
        if op_type == T_LOSS:             # a part of the vocabulary; joining the parts' sums, a few bytes a token, is not in the time
            x, w = normal(rows, self.hidden), normal(c, self.hidden) * self.hidden ** -0.5
            targets = torch.randint(0, c, (rows,), device="cuda", dtype=torch.int32)
            if not back:
                return lambda: O.vocab_loss_fwd(x, w, targets, first_word=0)
            lse = O.vocab_loss_fwd(x, w, targets, first_word=0)[1]
            dloss = torch.full((rows,), 1 / rows, device="cuda")
            return lambda: O.vocab_loss_bwd(dloss, x, w, targets, lse, first_word=0)
        if op_type in (T_QUERY, T_UP, T_DOWN):
            inputs = self.wide if op_type == T_DOWN else self.hidden
            x, w = normal(rows, inputs), normal(c, inputs)
            if not back:
                return lambda: x @ w.t()
            dy = normal(rows, c)
            return lambda: (dy @ w, dy.t() @ x)
        if op_type == W.T_EMBED:
            table, at = normal(self.vocab, c), torch.randint(0, self.vocab, (rows,), device="cuda")
            if not back:
                return lambda: table[at]
            dx = normal(rows, c)          # as Decoder.step sums it
            return lambda: torch.zeros_like(table, dtype=torch.float32).index_add_(0, at, dx.float()).to(t)
        if op_type == W.T_ELEM:           # a sum; its backward hands the gradient on, and adds where two meet
            x, y = normal(rows, c), normal(rows, c)
            return lambda: x + y
        raise ValueError(f"no task for operation type {op_type}")

    def __call__(self, op_type, shape):
        torch = self.torch
        task = self._task(op_type, shape)
        for _ in range(3):
            task()
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        for _ in range(self.repeats):
            task()
        end.record()
        end.synchronize()
        return max(1, round(start.elapsed_time(end) * 1e6 / self.repeats))


def graph(batch, length, hidden, vocab, layers, wide=None, elem_bytes=2):
    """the decoder's training iteration: (ops, edges, leader, params) as workloads.training_graph returns them, with an operation type per kind of task.
    Tensors are (sample, position, channel); the loss is (sample, position, word), its vocabulary a dim that strategies may split."""
    g = W.GraphBuilder()
    B, S, H, wide = batch, length, hidden, 4 * hidden if wide is None else wide
    owned = {}                            # op -> (elements of its parameters, the output dims they are split along, as a mask)

    def op(typ, channels, par, flops, elements=0, dims=0):
        o = g.op(typ, (B, S, channels), par, flops)
        owned[o] = (elements, dims)
        return o

    def matmul(src, typ, co):
        ci = g.extent(src)[2]
        o = op(typ, co, (0, 1, 2), 2 * B * S * ci * co, ci * co, 1 << 2)
        g.edge(src, o, [W.ident(0), W.ident(1), W.ALL])
        return o

    def norm(src):
        o = op(T_NORM, H, (0, 1), 10 * B * S * H, 2 * H)
        g.edge(src, o, [W.ident(0), W.ident(1), W.ALL])
        return o

    x = op(W.T_EMBED, H, (0, 1, 2), B * S * H, vocab * H, 1 << 2)
    for _ in range(layers):
        y = norm(x)
        qkv = [matmul(y, T_QUERY, H) for _ in range(3)]
        a = op(W.T_ATTN, H, (0, 2), 2 * B * S * S * H)
        for src in qkv:
            g.edge(src, a, [W.ident(0), W.ALL, W.ident(2)])
        x = g.elementwise([x, matmul(a, T_QUERY, H)])
        x = g.elementwise([x, matmul(matmul(norm(x), T_UP, wide), T_DOWN, H)])
    matmul(norm(x), T_LOSS, vocab)
    # (training_graph's own parameters are those of images' layers, whose channel is dim 1)
    ops, edges, _, leader, _ = W.training_graph(*g.finish())
    last = len(ops) - 1
    ops["type"][len(ops) // 2:] += BACKWARD
    params = np.zeros(len(ops), "<u4"), np.zeros(len(ops), np.uint8)
    for o, (elements, dims) in owned.items():
        params[0][last - o], params[1][last - o] = elements * elem_bytes, dims
    return ops, edges, leader, params


def measured_costs(ops, max_parts, choices, measure):
    """the cost lists of ff_sim_create_tuplecost, and the cache with what was measured"""
    cache = costcache.ExeTimeCache(measure)
    return costcache.tuple_costs(ops, max_parts, choices, cache), cache


def main():
    import torch
    from . import binding, search
    model = Decoder(vocab=1000, hidden=256, heads=4, layers=2)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    tokens = torch.randint(0, 1000, (8, 129), generator=gen, device="cuda", dtype=torch.int32)
    for i in range(31):
        loss, grads = model.step(tokens[:, :-1], tokens[:, 1:])
        for name, grad in grads.items():
            model.params[name] -= 0.5 * grad
        if i % 10 == 0:
            print(f"step {i}: loss {float(loss):.3f}")
    machine, hidden, heads, vocab, choices = W.Machine(4, 4, elem_bytes=2), 1024, 16, 32768, (1, 2, 4, 8, 16)
    ops, edges, leader, params = graph(batch=16, length=512, hidden=hidden, vocab=vocab, layers=4)
    costs, cache = measured_costs(ops, 16, choices, DeviceMeasure(hidden, hidden // heads, vocab=vocab))
    print(f"{len(ops)} ops, {cache.misses} task sizes measured on {torch.cuda.get_device_name()}, {cache.hits} taken from them")
    sim = binding.Simulator(ops, edges, machine, costs, params=params, ties=leader)
    found = search.find_strategy(sim, ops, machine, 16, choices, n_chains=64, steps=512)
    print(f"iteration on {machine.n_devices} devices: data parallelism {found.start_ns[0] / 1e6:.3f} ms, best of the search {found.best_ns / 1e6:.3f} ms")
    sim.close()


if __name__ == "__main__":
    main()
