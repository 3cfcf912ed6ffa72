"""A language model of the smallest kind, trained with the library: an example of how its operators go together.

The model predicts a token from the one before it: logits = head @ (scale * embedding[token]).  One training step is

    rows            SoloEmbedding.lookup        bf16 rows of the embedding, scaled
    logits          a matrix product            (torch's)
    loss, d logits  SoloLogprob.forward_grad    the weights of a mean over tokens are known beforehand
    d head, d rows  two matrix products
    d embedding     SoloEmbedding.grad          by sorted tokens
    grad_scale      SoloGradNorm.norm           stays on the GPU
    both tables     SoloMultiTable.step         SOLO AdamW, clipped by grad_scale, bf16 copies for the next step

and after training the likeliest successors of a few tokens come from SoloLogprob.forward, as a program that answers
token by token would ask for them.  Nothing waits for the GPU but the printed losses.

    python -m paper_2505_00347_amd.bigram
"""
import math

import torch

from . import solo


class Bigram:
    def __init__(self, vocab=2000, dim=256, tokens=4096, lr=2e-2, max_norm=1.0, seed=1):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.vocab, self.tokens, self.max_norm, self.steps = vocab, tokens, max_norm, 0
        self.params = [torch.randn((vocab, dim), generator=gen, device="cuda") / math.sqrt(dim) for _ in range(2)]
        self.weights = [p.bfloat16() for p in self.params]             # embedding, head
        self.grads = [torch.empty_like(w) for w in self.weights]
        cfg = solo.make_config(4, 4, 128, solo.SOLO_GRAD_BF16, lr=lr)
        states = [solo.SoloState(p.numel(), cfg) for p in self.params]
        self.table = solo.SoloMultiTable(list(zip(self.params, self.grads, states, self.weights)), cfg)
        self.norm = solo.SoloGradNorm(self.grads)
        self.embedding = solo.SoloEmbedding(vocab, dim, tokens, scale=math.sqrt(dim))
        self.logprob = solo.SoloLogprob(tokens, vocab)
        self.weight = torch.full((tokens,), -1.0 / tokens, device="cuda")
        self.rows = torch.empty((tokens, dim), dtype=torch.bfloat16, device="cuda")
        self.logits = torch.empty((tokens, vocab), dtype=torch.bfloat16, device="cuda")

    def step(self, ids, targets):
        """One training step on tokens and their successors; the log probabilities of the successors and the gradients' norm, on the GPU."""
        embedding, head = self.weights
        self.embedding.lookup(embedding, ids, self.rows)
        torch.mm(self.rows, head.t(), out=self.logits)
        logprob, _, grad = self.logprob.forward_grad(self.logits, targets, self.weight, None, self.logits)        # (in place)
        torch.mm(grad.t(), self.rows, out=self.grads[1])
        self.embedding.grad(grad @ head, ids, self.grads[0])
        norm, grad_scale, _ = self.norm.norm(self.max_norm)
        self.steps += 1
        self.table.step(self.steps, grad_scale=grad_scale)
        return logprob, norm

    def successors(self, ids, top=3):
        """The likeliest successors of each token and their log probabilities."""
        n = ids.numel()
        rows = self.embedding.lookup(self.weights[0], ids, self.rows[:n])
        plan = solo.SoloLogprob(n, self.vocab, top=top)
        return plan.forward(rows @ self.weights[1].t(), None)[-2:]


def text(vocab, n, seed):
    """Tokens of a chain in which a successor is one function of the token four times in five, and any token otherwise."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.randint(0, vocab, (n,), generator=gen, device="cuda")
    regular = torch.rand(n, generator=gen, device="cuda") < 0.8
    return ids, torch.where(regular, follows(ids, vocab), torch.randint(0, vocab, (n,), generator=gen, device="cuda"))


def follows(ids, vocab):
    return (ids * 7 + 3) % vocab


def main(steps=200):
    model = Bigram()
    for k in range(1, steps + 1):
        logprob, norm = model.step(*text(model.vocab, model.tokens, k))
        if k == 1 or k % 20 == 0:
            print("step %3d  loss %.3f  gradient norm %.3f" % (k, -logprob.mean().item(), norm.item()), flush=True)
    best = 0.2 * math.log(5 * model.vocab) + 0.8 * math.log(1 / 0.8)
    print("a model that knows the chain: about %.3f" % best)
    ids = torch.tensor([1, 10, 100], device="cuda")
    value, token = model.successors(ids)
    for i, t, v in zip(ids.tolist(), token.tolist(), value.tolist()):
        print("after %d: %s (regular: %d)" % (i, ", ".join("%d with %.2f" % (a, math.exp(b)) for a, b in zip(t, v)), follows(i, model.vocab)))


if __name__ == "__main__":
    main()
