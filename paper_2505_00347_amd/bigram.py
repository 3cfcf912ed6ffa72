"""A language model of the smallest kind, trained with the library: an example of how its operators go together.

The model predicts a token from the one before it: logits = head @ (scale * embedding[token]), or, with norm=True,
logits = head @ layer_norm(scale * embedding[token]).  One training step is

    rows            SoloEmbedding.lookup        bf16 rows of the embedding, scaled
    hidden          SoloLayerNorm.forward       (with norm=True)
    logits          a matrix product            (torch's)
    loss, d logits  SoloLogprob.forward_grad    the weights of a mean over tokens are known beforehand
                    or SoloDistill.forward_grad from the alternatives that another model, its teacher, gives
    d head, d rows  two matrix products
    d rows, d norm  SoloLayerNorm.grad
    d embedding     SoloEmbedding.grad          by sorted tokens
    grad_scale      SoloGradNorm.norm           stays on the GPU
    all parameters  SoloMultiTable.step         SOLO AdamW, clipped by grad_scale, bf16 copies for the next step

and after training the likeliest successors of a few tokens come from SoloLogprob.forward, as a program that answers
token by token would ask for them, and a text from SoloSampler.sample.  Nothing waits for the GPU but what is printed.

    python -m paper_2505_00347_amd.bigram
"""
import math

import torch

from . import solo


class Bigram:
    def __init__(self, vocab=2000, dim=256, tokens=4096, lr=2e-2, max_norm=1.0, seed=1, norm=False):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.vocab, self.dim, self.tokens, self.max_norm, self.steps = vocab, dim, tokens, max_norm, 0
        self.params = [torch.randn((vocab, dim), generator=gen, device="cuda") / math.sqrt(dim) for _ in range(2)]
        if norm:
            self.params += [torch.ones(dim, device="cuda"), torch.zeros(dim, device="cuda")]
        self.weights = [p.bfloat16() for p in self.params]             # embedding, head, weight and bias of the norm
        self.grads = [torch.empty_like(w) for w in self.weights]
        cfg = solo.make_config(4, 4, 128, solo.SOLO_GRAD_BF16, lr=lr)
        states = [solo.SoloState(p.numel(), cfg) for p in self.params]
        self.table = solo.SoloMultiTable(list(zip(self.params, self.grads, states, self.weights)), cfg)
        self.norm = solo.SoloGradNorm(self.grads)
        self.embedding = solo.SoloEmbedding(vocab, dim, tokens, scale=math.sqrt(dim))
        self.layer = solo.SoloLayerNorm(tokens, dim) if norm else None
        self.logprob = solo.SoloLogprob(tokens, vocab)
        self.distilled = None
        self.weight = torch.full((tokens,), -1.0 / tokens, device="cuda")
        self.rows = torch.empty((tokens, dim), dtype=torch.bfloat16, device="cuda")
        self.hidden = torch.empty_like(self.rows) if norm else self.rows
        self.logits = torch.empty((tokens, vocab), dtype=torch.bfloat16, device="cuda")

    def _forward(self, ids):
        """The logits of the tokens' successors."""
        n = ids.numel()
        rows, hidden = self.rows[:n], self.hidden[:n]
        self.embedding.lookup(self.weights[0], ids, rows)
        if self.layer is not None:
            self.layer.forward(rows, self.weights[2], self.weights[3], hidden)
        return torch.mm(hidden, self.weights[1].t(), out=self.logits[:n])

    def _update(self, ids, grad):
        """The rest of a training step behind the logits' gradient; the gradients' norm."""
        head = self.weights[1]
        torch.mm(grad.t(), self.hidden, out=self.grads[1])
        grad_rows = grad @ head
        if self.layer is not None:
            self.layer.grad(grad_rows, self.rows, self.weights[2], grad_rows, self.grads[2], self.grads[3])       # (in place)
        self.embedding.grad(grad_rows, ids, self.grads[0])
        norm, grad_scale, _ = self.norm.norm(self.max_norm)
        self.steps += 1
        self.table.step(self.steps, grad_scale=grad_scale)
        return norm

    def step(self, ids, targets):
        """One training step on tokens and their successors; the log probabilities of the successors and the gradients' norm, on the GPU."""
        logits = self._forward(ids)
        logprob, _, grad = self.logprob.forward_grad(logits, targets, self.weight, None, logits)                  # (in place)
        return logprob, self._update(ids, grad)

    def learn(self, ids, value, token):
        """One training step on tokens and a teacher's alternatives of their successors (what its alternatives() returns); the rows' divergences
        and the gradients' norm, on the GPU."""
        if self.distilled is None or self.distilled.top != token.shape[1]:
            self.distilled = solo.SoloDistill(self.tokens, self.vocab, token.shape[1], rest=True)
        logits = self._forward(ids)
        loss, grad = self.distilled.forward_grad(logits, value, token, -self.weight, logits)                      # (in place)
        return loss, self._update(ids, grad)

    def alternatives(self, ids, top):
        """The likeliest successors of each token: their log probabilities and themselves."""
        return solo.SoloLogprob(ids.numel(), self.vocab, top=top).forward(self._forward(ids), None)[-2:]

    def successors(self, ids, top=3):
        """The likeliest successors of each token and their log probabilities."""
        return self.alternatives(ids, top)

    def write(self, ids, uniform, **parameters):
        """A text behind each token, drawn by the numbers uniform [length, tokens]: the tokens [length, tokens] and their log probabilities."""
        sampler = solo.SoloSampler(ids.numel(), self.vocab, **parameters)
        tokens, logprobs = torch.empty_like(uniform, dtype=torch.int64), torch.empty_like(uniform)
        for u, token, logprob in zip(uniform, tokens, logprobs):
            drawn = sampler.sample(self._forward(ids), u)
            token.copy_(drawn[0])
            logprob.copy_(drawn[1])
            ids = token
        return tokens, logprobs


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
    gen = torch.Generator(device="cuda").manual_seed(2)
    tokens, _ = model.write(ids, torch.rand((8, 3), generator=gen, device="cuda"), temperature=0.8, top_p=0.9)
    for i, t in zip(ids.tolist(), tokens.t().tolist()):
        print("a text behind %d: %s" % (i, " ".join(map(str, t))))
    student = Bigram(dim=128, norm=True, seed=3)
    for k in range(1, steps // 2 + 1):
        ids, _ = text(model.vocab, model.tokens, 1000 + k)
        loss, norm = student.learn(ids, *model.alternatives(ids, top=20))
        if k == 1 or k % 20 == 0:
            print("student, step %3d  divergence from its teacher %.3f  gradient norm %.3f" % (k, loss.mean().item(), norm.item()), flush=True)


if __name__ == "__main__":
    main()
