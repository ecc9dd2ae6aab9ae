"""From a routing decision to what it chose: one GPU, one stream.

A router scores a batch of queries and picks a deployment for each.  Here the
deployments share the GPU: as experts with a weight matrix each, then as
low-rank adapters beside one shared projection.  The picks, still on the
device, are dispatched (the rows of each choice together), carried out, and a
few training steps fit experts and adapters to targets, gradients clipped to
a global norm.

    python examples/routed_layer.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_14575_gb300 as hwr  # noqa: E402
import workload  # noqa: E402


def routed_batch(Q, stream):
    """(query embeddings [Q][E] bf16, chosen deployment [Q] int32, deployments)"""
    p = workload.make_config(1, Q=Q)
    router = hwr.Router(p, stream.cuda_stream)
    il, ol = (torch.from_numpy(p[k]).cuda() for k in ("in_len", "out_len"))
    emb = torch.from_numpy(p["emb"].view("int16")).cuda().view(torch.bfloat16)
    chosen = torch.empty(Q, dtype=torch.int32, device="cuda")
    latency, utility = (torch.empty(Q, device="cuda") for _ in range(2))
    router.route_device(il, ol, emb, chosen, latency, utility, slo=p["slo"], lam=p["lam"])
    router.close()
    return emb, chosen, int(p["D"])


def fit(name, ops, weights, forward, backward, target, steps, rate, max_norm, say):
    """SGD on fp32 copies of the weights; returns the loss before each step."""
    master = [w.float() for w in weights]
    losses = []
    for step in range(steps):
        y = forward(*weights)
        diff = y.float() - target
        losses.append(float(diff.square().mean()))
        grads = backward((diff * (2.0 / y.shape[0])).to(y.dtype), *weights)
        norm = ops.clip_gradients(grads, max_norm)
        for m, w, g in zip(master, weights, grads):
            m -= rate * g.float()
            w.copy_(m)
        say(f"{name} step {step}: loss {losses[-1]:.4f}, gradient norm {float(norm):.3f}")
    return losses


def main(Q=2048, width=512, rank=16, steps=8, say=print):
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        gen = torch.Generator(device="cuda").manual_seed(1)

        def normal(*shape, std=1.0):
            return torch.empty(shape, device="cuda", dtype=torch.bfloat16).normal_(0, std, generator=gen)

        emb, chosen, D = routed_batch(Q, stream)
        x = (emb.float() * emb.shape[1] ** 0.5).to(torch.bfloat16)      # unit-variance features
        E = x.shape[1]
        ops = hwr.Operators()
        plan = ops.dispatch(chosen, D)
        used = int((plan.offsets[1:] > plan.offsets[:-1]).sum())
        say(f"{Q} queries over {used} of {D} deployments")
        target = x.float() @ normal(E, width, std=E ** -0.5).float()

        experts = [normal(D, width, E, std=0.02)]
        first = fit("experts", ops, experts,
                    lambda w: ops.grouped_forward(x, w, plan),
                    lambda dy, w: list(ops.grouped_backward(dy, x, w, plan, need_dx=False))[1:],
                    target, steps, 0.1, 40.0, say)

        shared, scale = normal(width, E, std=0.02), torch.ones(D, device="cuda")
        adapters = [normal(D, rank, E, std=E ** -0.5), torch.zeros(D, width, rank, device="cuda", dtype=torch.bfloat16)]
        second = fit("adapters", ops, adapters,
                     lambda a, b: ops.adapter_forward(x, shared, a, b, scale, plan),
                     lambda dy, a, b: list(ops.adapter_backward(dy, x, shared, a, b, scale, plan, need_dx=False))[1:],
                     target, steps, 0.2, 40.0, say)
        ops.synchronize()
        ops.close()
    return first, second


if __name__ == "__main__":
    main()
