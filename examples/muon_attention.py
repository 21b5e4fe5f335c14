"""A small language model whose attention layers are made of the library's operators and whose weights are updated by orthogonalised momentum.

  python examples/muon_attention.py [--steps 120]

Packed documents of a toy language (each repeats a random phrase) are learned: norm and rotation of queries and keys, attention within documents with capped
scores, dropout on the residual stream, their gradients, and one grouped polar call a step for all 2-D weights of the layers.  Afterwards tokens are
generated one by one against a cache of keys and values."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2601_22137_amd import layers, optim   # noqa: E402

VOCABULARY, WIDTH, HEADS, K_HEADS, LAYERS, BATCH, LENGTH, PHRASE = 64, 256, 4, 2, 2, 16, 256, 8


class Model(torch.nn.Module):
    def __init__(self, p=0.05):
        super().__init__()
        self.embed = torch.nn.Embedding(VOCABULARY, WIDTH, device="cuda", dtype=torch.bfloat16)
        self.layers = torch.nn.ModuleList([layers.SelfAttention(WIDTH, HEADS, K_HEADS, softcap=30.0, p=p) for _ in range(LAYERS)])

    def logits(self, x):
        x = torch.nn.functional.rms_norm(x.float(), (WIDTH,))
        return x @ self.embed.weight.float().t() * WIDTH ** -0.5

    def forward(self, tokens, positions, doc, step=0):
        x = self.embed(tokens)
        for i, layer in enumerate(self.layers):
            x = layer(x, positions, doc, seed=22137, offset=step * LAYERS + i)
        return self.logits(x)


def batch(generator):
    """Sequences of documents, the last eighth padding: (tokens, positions, documents), targets -1 where there is nothing to foretell."""
    tokens = torch.zeros(BATCH, LENGTH, dtype=torch.long)
    positions, doc = torch.zeros(BATCH, LENGTH, dtype=torch.int32), torch.full((BATCH, LENGTH), -1, dtype=torch.int32)
    targets = torch.full((BATCH, LENGTH), -1)
    for b in range(BATCH):
        at, d = 0, 0
        while at < LENGTH * 7 // 8:
            n = min(int(torch.randint(3 * PHRASE, 9 * PHRASE, (1,), generator=generator)), LENGTH * 7 // 8 - at)
            phrase = torch.randint(0, VOCABULARY, (PHRASE,), generator=generator)
            text = phrase.repeat(n // PHRASE + 1)[:n]
            tokens[b, at:at + n], positions[b, at:at + n], doc[b, at:at + n] = text, torch.arange(n), d
            if n > PHRASE:
                targets[b, at + PHRASE - 1:at + n - 1] = text[PHRASE:]
            at, d = at + n, d + 1
    return [t.cuda() for t in (tokens, positions, doc)], targets.cuda()


def train(steps, say=print):
    """(model, the losses): momentum, orthogonalised for the weights of the layers, plain for the others."""
    torch.manual_seed(0)
    model = Model()
    generator = torch.Generator().manual_seed(1)
    matrices = [w for layer in model.layers for w in (layer.w_qkv, layer.w_out)]
    others = [p for p in model.parameters() if all(p is not w for w in matrices)]
    momentum = [torch.zeros_like(w) for w in matrices]
    adam = torch.optim.Adam(others, lr=3e-3)
    losses = []
    for step in range(steps):
        inputs, targets = batch(generator)
        loss = torch.nn.functional.cross_entropy(model(*inputs, step=step).flatten(0, 1), targets.flatten(), ignore_index=-1)
        model.zero_grad(set_to_none=True)
        loss.backward()
        adam.step()
        with torch.no_grad():
            for m, w in zip(momentum, matrices):
                m.mul_(0.9).add_(w.grad)
            for w, u in zip(matrices, optim.muon_orthogonalize(momentum)):
                w.add_(u, alpha=-0.02 * max(1.0, w.shape[0] / w.shape[1]) ** 0.5)
        losses.append(loss.item())
        if say and (step % 10 == 0 or step + 1 == steps):
            say("step %3d  loss %.3f" % (step, losses[-1]))
    return model, losses


@torch.no_grad()
def generate(model, prompts, count):
    """Greedy continuation of prompts [batch, token], one token at a time."""
    model.eval()
    caches = [layer.new_cache(prompts.shape[0], prompts.shape[1] + count) for layer in model.layers]
    tokens = prompts
    for at in range(prompts.shape[1] + count - 1):
        x = model.embed(tokens[:, at:at + 1])
        for layer, cache in zip(model.layers, caches):
            x = layer.step(x, cache)
        if at + 1 >= tokens.shape[1]:
            tokens = torch.cat([tokens, model.logits(x)[:, -1].argmax(-1, keepdim=True)], 1)
    return tokens


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=120)
    model, losses = train(ap.parse_args().steps)
    phrase = torch.randint(0, VOCABULARY, (4, PHRASE), device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    text = generate(model, phrase.repeat(1, 3), PHRASE)
    print("loss %.3f -> %.3f; %d of %d generated tokens repeat the phrase" % (losses[0], losses[-1], int((text[:, -PHRASE:] == phrase).sum()), phrase.numel()))


if __name__ == "__main__":
    main()
