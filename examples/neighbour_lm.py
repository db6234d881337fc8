"""A language model and a search over its hidden states, put together from the library's calls.

    python examples/neighbour_lm.py

A small synthetic language (the next token depends on the two before it), hidden states that a frozen network makes of the
context, and an output embedding that starts at random.  The states of a training text are indexed, each with the token
that followed it.  Then, on a test text:

  1. states are quantised and multiplied with the 8-bit output embedding: logits          ivfpq_quantize_rows, ivfpq_q8_matmul
  2. the nearest stored states are found and turned into a distribution over tokens       ivfpq_search, ivfpq_neighbour_tokens
  3. the next tokens are scored under the model, and under its mixture with the neighbours    ivfpq_token_logprobs
  4. the output embedding is trained towards the neighbours' distributions                ivfpq_distill_topk_step
     and then towards the tokens that follow, with their log-probabilities' gradient       ivfpq_token_logprobs_backward

and the perplexities are printed.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2301_06672_amd as ivfpq  # noqa: E402


def language(vocab, length, gen):
    """A text in which each pair of tokens is followed by one of four."""
    pairs = 1 << 14
    follow = torch.randint(vocab, (pairs, 4), generator=gen)
    choice = torch.multinomial(torch.tensor([0.6, 0.25, 0.1, 0.05]), length, replacement=True, generator=gen).tolist()
    table = follow.tolist()
    text = [0, 1]
    for c in choice:
        text.append(table[(text[-2] % 128) * 128 + text[-1] % 128][c])
    return torch.tensor(text)


def states(text, d, gen):
    """What a frozen network makes of the two tokens before each place, and the token there."""
    vectors = torch.randn(2, 128, d, generator=gen)
    h = torch.tanh(vectors[0][text[:-2] % 128] + vectors[1][text[1:-1] % 128])
    h += 0.05 * torch.randn(h.shape, generator=gen)
    return h.float().cuda(), text[2:].int().cuda()


def head(w):
    return ivfpq.ivfpq_quantize_rows(w)


def logits_of(h, packed):
    codes, scales = ivfpq.ivfpq_quantize_rows(h)
    return ivfpq.ivfpq_q8_matmul(codes, scales, *packed, out_dtype=torch.bfloat16)


def perplexity(logprobs):
    return float(torch.exp(-logprobs.mean()))


def run(vocab=2000, d=64, train=120_000, test=4_000, k=32, steps=60, seed=1, say=print):
    gen = torch.Generator().manual_seed(seed)
    text = language(vocab, train + test, gen)
    h, after = states(text, d, gen)
    stored, tokens = h[:train].contiguous(), after[:train].contiguous()
    asked, wanted = h[train:].contiguous(), after[train:].contiguous()
    temperature = 0.3                                      # of the distances: between the noise and the distance of other contexts

    index = ivfpq.Index.ivfpq_build_device(stored, n_lists=256, pq_dim=32, pq_bits=8, kmeans_iters=8, seed=seed).ivfpq_upload()

    def neighbours(queries):
        ids, dists = index.ivfpq_search(queries, n_probes=16, k=k)
        return ivfpq.ivfpq_neighbour_tokens(ids, dists, tokens, temperature)

    near = neighbours(asked)
    w = torch.randn(vocab, d, generator=gen).cuda() * 0.02

    def score(name):
        logits = logits_of(asked, head(w))
        alone = ivfpq.ivfpq_token_logprobs(logits, wanted, top=1)
        mixed = ivfpq.ivfpq_token_logprobs(logits, wanted, top=1, neighbours=near, weight=0.5)
        got = {"model": perplexity(alone.logprobs), "mixture": perplexity(mixed.logprobs),
               "model's best right": float((alone.top_tokens[:, 0] == wanted).float().mean()),
               "mixture's best right": float((mixed.top_tokens[:, 0] == wanted).float().mean())}
        say(f"{name:28s}" + "  ".join(f"{key} {value:.3f}" for key, value in got.items()))
        return got

    result = {"before": score("before training")}
    rows = 4_096
    for step in range(steps):
        pick = torch.randint(train, (rows,), generator=gen).cuda()
        x = stored[pick]
        logits = (x @ w.t()).to(torch.bfloat16)
        weight = torch.full((rows,), 1.0 / rows, device="cuda")
        _, grad = ivfpq.ivfpq_distill_topk_step(logits, *neighbours(x), weight, out=logits)      # written over the logits
        w -= 60.0 * (grad.float().t().contiguous() @ x)
    result["distilled"] = score("trained on neighbours")
    for step in range(steps // 2):
        pick = torch.randint(train, (rows,), generator=gen).cuda()
        x, y = stored[pick], tokens[pick]
        logits = (x @ w.t()).to(torch.bfloat16)
        s = ivfpq.ivfpq_token_logprobs(logits, y)
        weight = torch.full((rows,), -1.0 / rows, device="cuda")                                 # the loss is -log p
        grad = ivfpq.ivfpq_token_logprobs_backward(logits, y, s.norms, s.entropy, weight, out=logits)
        w -= 60.0 * (grad.float().t().contiguous() @ x)
    result["trained"] = score("... and on the text")
    index.ivfpq_free()
    return result


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--vocab", type=int, default=2000)
    p.add_argument("--train", type=int, default=120_000)
    p.add_argument("--steps", type=int, default=60)
    a = p.parse_args()
    run(vocab=a.vocab, train=a.train, steps=a.steps)
