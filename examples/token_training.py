"""Adapters trained on the tokens of given answers, and a decode step through experts.

Each query's answer token is scored under its adapter: logits of the shared projection and
the query's own low-rank terms, log probabilities of the tokens, their gradient back
through the adapters, the gradients' norm, and one optimizer's step on fp32 parameters
whose bf16 copies the products read.  Then a layer of experts takes a few rows of a decode
step, whose next tokens come with their log probabilities, alternatives and entropies.

    python examples/token_training.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_14575_gb300 as hwr  # noqa: E402


def train(ops, x, head, choice, token, groups, rank, steps, rate, bits, say):
    """Returns the mean log probability before each step, and the trained adapters."""
    def normal(*shape, std):
        return torch.empty(shape, device="cuda").normal_(0, std)

    K, V = x.shape[1], head.shape[0]
    params = [normal(groups, rank, K, std=K ** -0.5), torch.zeros(groups, V, rank, device="cuda")]
    a, b = copies = [p.to(torch.bfloat16) for p in params]
    scale = torch.ones(groups, device="cuda")
    state = ops.adamw_state(params, bits=bits, copies=copies)
    plan = ops.dispatch(choice, groups)
    weight = torch.full((x.shape[0],), -1.0 / x.shape[0], device="cuda")     # of the loss: minus the mean
    means = []
    for step in range(steps):
        logits = ops.adapter_forward(x, head, a, b, scale, plan)
        got = ops.token_logprobs(logits, token)
        means.append(got.logprob.mean())
        dlogits = ops.token_logprobs_backward(weight, logits, token, got, out=logits)
        _, da, db = ops.adapter_backward(dlogits, x, head, a, b, scale, plan, need_dx=False)
        norm = ops.clip_gradients([da, db], float("inf"))
        ops.adamw_step(state, [da, db], lr=rate, norm=norm, max_norm=1.0, seed=step)
        say(f"step {step}: log probability {float(means[-1]):.4f}, entropy {float(got.entropy.mean()):.3f}, "
            f"gradient norm {float(norm):.3f}")
    state.close()
    return [float(m) for m in means], copies


def decode(ops, x, w_in, w_out, scores, head, top):
    """Next tokens of a few rows: (token, log probability, entropy), greedily."""
    y = ops.expert_layer(x, w_in, w_out, scores=scores, top=2)
    plan = ops.dispatch(torch.zeros(x.shape[0], dtype=torch.int32, device="cuda"), 1)
    got = ops.token_logprobs(ops.grouped_forward(y, head[None], plan), top=top)
    return got.top_token[:, 0], got.top_logprob[:, 0], got.entropy


def main(rows=1024, width=256, vocab=2048, groups=6, rank=8, steps=6, bits=8, say=print):
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        torch.manual_seed(1)
        bf16 = torch.bfloat16

        def normal(*shape, std=1.0):
            return torch.empty(shape, device="cuda", dtype=bf16).normal_(0, std)

        ops = hwr.Operators()
        x, head = normal(rows, width), normal(vocab, width, std=width ** -0.5)
        choice = torch.randint(-1, groups, (rows,), device="cuda", dtype=torch.int32)
        token = torch.randint(0, vocab, (rows,), device="cuda", dtype=torch.int32)
        means, adapters = train(ops, x, head, choice, token, groups, rank, steps, 2e-3, bits, say)
        few = x[:4]
        scores = torch.randn(4, 8, device="cuda")
        tokens, logprobs, entropies = decode(ops, few, normal(8, 1024, width, std=width ** -0.5),
                                             normal(8, width, 512, std=512 ** -0.5), scores, head, 5)
        ops.synchronize()
        for t, p, h in zip(tokens.tolist(), logprobs.tolist(), entropies.tolist()):
            say(f"token {t}: log probability {p:.3f}, entropy {h:.3f}")
        ops.close()
    return means, adapters, tokens


if __name__ == "__main__":
    main()
