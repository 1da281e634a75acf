"""A transformer stage of a pipeline, trained in the order that the schedule search finds for it.

`Stage` is one layer -- attention over packed sequences and a gated block inside, each between the norms around it -- whose
forward and backward passes are made of block_ops and plain matrix products.  It keeps its inputs to the products in 8 bits
(or, for comparison, everything in 16, with the gated activation by torch's own operations), which is the activation memory m of its blocks.  `plan` measures t and m of its blocks,
searches the best window under a memory cap and completes it; `run` executes the blocks of that schedule on one GPU, every
simulated device holding a stage of its own, and sums the weights' gradients over the micro-batches.

    python -m paper_2311_15269_amd.stage            (needs an MI355X)
"""
import argparse
import math
import time

from . import block_ops
from .binding import search
from .workloads import linear_placement, pipeline_problem


def _activation(kind, z):
    """an activation of 32-bit numbers and its derivative (formulas: include/tessel_block_ops.h)"""
    import torch
    if kind == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    root, cube = (2 / math.pi) ** 0.5, 0.044715
    t = torch.tanh(root * (z + cube * z * z * z))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * (1 - t * t) * z * root * (1 + 3 * cube * (z * z).clamp(max=1e6))


class Stage:
    """Weights in 16 bits, parameters of the norms and all gradients in 32.  Micro-batches are told apart by a number; what a
    forward pass keeps goes away with its backward pass.  `small`: 8-bit checkpoints."""

    def __init__(self, channels, heads, kv_heads, inner, generator, dtype, small=True, scale=1.0, act="silu"):
        import torch
        self.heads, self.kv_heads, self.dim = heads, kv_heads, channels // heads
        self.small, self.scale, self.act = small, scale, act
        wide = (heads + 2 * kv_heads) * self.dim

        def weight(rows, columns):
            return (torch.randn(rows, columns, generator=generator, device="cuda") * columns ** -0.5).to(dtype)

        def vector(value):
            return torch.full((channels,), value, device="cuda")
        self.weights = {"qkv": weight(wide, channels), "out": weight(channels, heads * self.dim), "gate": weight(inner, channels),
                        "up": weight(inner, channels), "down": weight(channels, inner)}
        # the norms behind the attention and behind the gated part: of what comes out, its gate, of what goes on
        self.norms = [{"post": vector(1.0), "gate": vector(0.5), "pre": vector(1.0)} for _ in range(2)]
        self.gradients = {k: torch.zeros(w.shape, device="cuda") for k, w in self.weights.items()}
        self.norm_gradients = [{k: torch.zeros_like(v) for k, v in n.items()} for n in self.norms]
        self.kept = {}

    # -- one product and the two of its backward pass
    def _add(self, name, dy, x):
        """the gradient of weight `name` from dy and its input, as it was kept: products of 16 bits, summed and left in 32"""
        import torch
        if isinstance(x, block_ops.Checkpoint):
            block_ops.weight_gradient(dy, x, into=self.gradients[name])
        else:
            self.gradients[name] += torch.mm(dy.t(), x, out_dtype=torch.float32)

    def _keep(self, x):
        return block_ops.checkpoint(x) if self.small else x

    def _gated(self, g, u):
        """act(g) u, and g and u as they are kept"""
        if self.small:
            return block_ops.gated(g, u, self.act)
        return (_activation(self.act, g.float())[0] * u.float()).to(g.dtype), g, u

    def _gated_backward(self, da, g, u):
        """gradients of g and u from those of act(g) u, and that once more"""
        if self.small:
            return block_ops.gated_backward(da, g, u, self.act, with_output=True)
        f, slope = _activation(self.act, g.float())
        d, w = da.float(), u.float()
        return tuple(t.to(da.dtype) for t in (d * w * slope, d * f, f * w))

    def _norm(self, i, x, y):
        n = self.norms[i]
        return block_ops.residual_norm(x, y, n["pre"], n["post"], n["gate"], self.scale)

    def _norm_backward(self, i, dr, dh, x, y, stats):
        n, g = self.norms[i], self.norm_gradients[i]
        return block_ops.residual_norm_backward(dr, dh, x, y, stats, n["pre"], n["post"], n["gate"], self.scale,
                                                into=(g["pre"], g["post"], g["gate"]))[:2]

    def forward(self, number, packing, x, h):
        """the residual stream x and its norm h [tokens, channels] -> the next stage's"""
        w, n = self.weights, x.shape[0]
        qkv = (h @ w["qkv"].t()).view(n, self.heads + 2 * self.kv_heads, self.dim)
        q, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), 1)
        o, lse = packing.attention(q, k, v)
        y = o.view(n, -1) @ w["out"].t()
        r, hr, stats = self._norm(0, x, y)
        a, g, u = self._gated(hr @ w["gate"].t(), hr @ w["up"].t())
        z = a @ w["down"].t()
        r2, h2, stats2 = self._norm(1, r, z)
        self.kept[number] = (packing, x, self._keep(h), qkv, o, lse, y, stats, r, self._keep(hr), g, u, z, stats2)
        return r2, h2

    def backward(self, number, dr, dh):
        """gradients of what forward() gave -> those of what it took"""
        packing, x, h, qkv, o, lse, y, stats, r, hr, g, u, z, stats2 = self.kept.pop(number)
        w, n = self.weights, x.shape[0]
        dr, dz = self._norm_backward(1, dr, dh, r, z, stats2)
        da = dz @ w["down"]
        dg, du, a = self._gated_backward(da, g, u)
        self._add("down", dz, a)
        self._add("gate", dg, hr)
        self._add("up", du, hr)
        dx, dy = self._norm_backward(0, dr, dg @ w["gate"] + du @ w["up"], x, y, stats)
        self._add("out", dy, o.view(n, -1))
        q, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), 1)
        import torch
        dq, dk, dv = packing.attention_backward((dy @ w["out"]).view(o.shape), q, k, v, o, lse)
        dqkv = torch.cat((dq, dk, dv), 1).view(n, -1)
        self._add("qkv", dqkv, h)
        return dx, dqkv @ w["qkv"]

    def kept_bytes(self, number):
        """what a forward pass keeps until its backward pass: m of its block.  (The residual stream that it was given too: the stage that made it does not
        keep it.)"""
        return sum(t.nbytes for t in self.kept[number] if hasattr(t, "nbytes"))


def measure(stage, packing, x, h):
    """(seconds forward, seconds backward, bytes kept) of a stage's blocks for a micro-batch"""
    import torch
    took = [0.0, 0.0]
    for turn in range(6):
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        r, hr = stage.forward(-1, packing, x, h)
        torch.cuda.synchronize()
        t1 = time.perf_counter()
        size = stage.kept_bytes(-1)
        stage.backward(-1, r, hr)
        torch.cuda.synchronize()
        if turn:                                                # (the first pass loads the kernels)
            took[0] += t1 - t0
            took[1] += time.perf_counter() - t1
    for g in list(stage.gradients.values()) + [v for n in stage.norm_gradients for v in n.values()]:
        g.zero_()
    return took[0] / 5, took[1] / 5, size


def plan(devices, seconds, kept, cap, microbatches, max_nr=4):
    """The schedule of a pipeline whose stages take seconds = (forward, backward) and keep `kept` units of memory between the two, `cap` of them
    on a device: (search result, completed schedule, operations in order).  Times go into the search in eighths of a forward pass."""
    tf, tb = 8, max(1, round(8 * seconds[1] / seconds[0]))
    # (four devices: every order, 2.9 G of them for windows of four micro-batches; more: samples)
    space, step, most = ("canonical", 0, 1 << 32) if devices <= 4 else ("sampled_repair", 12000, 1 << 26)
    problem = pipeline_problem(linear_placement(devices), [tf] * devices, [tb] * devices, devices, 1, cap, space, lead_step_q16=step, name="stage")
    problem["m"] = [kept] * devices + [-kept] * devices
    found, best = search(problem, max_nr, most)
    if best is None:
        return found, None, []
    done = best.complete_schedule(microbatches)
    return found, done, best.instantiate(microbatches, done["start"])


def run(stages, packings, xs, hs, gradient, operations):
    """Executes a schedule's operations: micro-batch mu of xs, hs through all stages, gradient(mu, r, h) -> (dr, dh) behind the last one, and
    back.  Returns the gradients of xs and hs.  (All devices share this GPU: a tensor that would be sent is there already.)"""
    n, last = len(xs), len(stages) - 1
    there, back = {}, {}
    for kind, block, *_ in operations:
        if kind != 0:
            continue
        i, mu = divmod(block, n)
        if i <= last:
            there[i, mu] = stages[i].forward(mu, packings[mu], *(there.pop((i - 1, mu)) if i else (xs[mu], hs[mu])))
        else:
            i = 2 * last + 1 - i
            back[i, mu] = stages[i].backward(mu, *(back.pop((i + 1, mu)) if i < last else gradient(mu, *there.pop((last, mu)))))
    return [back[0, mu] for mu in range(n)]


def in_turn(devices, microbatches):
    """the operations of one micro-batch after the other"""
    return [(0, i * microbatches + mu, 0, 0, 0) for mu in range(microbatches) for i in range(2 * devices)]


def make(devices, microbatches, lengths, channels, heads, kv_heads, inner, small, seed=0, dtype=None):
    """stages, packings and inputs, the same for the same seed"""
    import torch
    dtype = dtype or torch.bfloat16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    stages = [Stage(channels, heads, kv_heads, inner, gen, dtype, small) for _ in range(devices)]
    packings = [block_ops.Packing(lengths) for _ in range(microbatches)]
    xs = [torch.randn(sum(lengths), channels, generator=gen, device="cuda").to(dtype) for _ in range(microbatches)]
    one = torch.ones(channels, device="cuda")
    hs = [block_ops.residual_norm(x, torch.zeros_like(x), one)[1] for x in xs]
    return stages, packings, xs, hs


def main():
    import torch
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--devices", type=int, default=4)
    ap.add_argument("--microbatches", type=int, default=8)
    ap.add_argument("--channels", type=int, default=1024)
    ap.add_argument("--heads", type=int, default=16)
    ap.add_argument("--kv-heads", type=int, default=4)
    ap.add_argument("--lengths", default="1000,37,500,511")
    a = ap.parse_args()
    lengths = [int(n) for n in a.lengths.split(",")]
    sizes = (a.devices, a.microbatches, lengths, a.channels, a.heads, a.kv_heads, 4 * a.channels)
    unit = sum(lengths) * a.channels                            # a byte a channel
    cap = None
    for small in (False, True):
        stages, packings, xs, hs = make(*sizes, small)
        forward, backward, kept = measure(stages[0], packings[0], xs[0], hs[0])
        m = -(-kept // unit)
        if cap is None:
            cap = 3 * m                                         # what three micro-batches take in 16 bits
        found, done, operations = plan(a.devices, (forward, backward), m, cap, a.microbatches)
        print("%s: forward %.0f us, backward %.0f us, %d bytes a token and channel kept; cap %d: window of %d micro-batches, %.3f of the "
              "lower bound a micro-batch" % ("8-bit checkpoints" if small else "16 bits", forward * 1e6, backward * 1e6, m, cap, found["best_nr"],
                                             found["best_period"] / max(1, found["best_nr"]) / found["lower_bound"]))
    dr = torch.randn_like(xs[0])

    def gradient(mu, r, h):
        return dr, dr
    got = run(stages, packings, xs, hs, gradient, operations)
    again, packings, xs, hs = make(*sizes, True)
    want = run(again, packings, xs, hs, gradient, in_turn(a.devices, a.microbatches))
    same = all(torch.equal(p, q) for x, y in zip(got, want) for p, q in zip(x, y))
    same = same and all(torch.equal(s.gradients[k], t.gradients[k]) for s, t in zip(stages, again) for k in s.gradients)
    print("%d micro-batches in the order of the schedule (%d operations, makespan %d): gradients %s those of one after the other" % (
        a.microbatches, len(operations), done["makespan"], "equal" if same else "DIFFER from"))
    return 0 if same else 1


if __name__ == "__main__":
    raise SystemExit(main())
