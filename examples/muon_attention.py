"""A small language model whose attention layers are made of the library's operators and whose weights are updated by orthogonalised momentum.

  python examples/muon_attention.py [--steps 120] [--policy-steps 10]

Packed documents of a toy language (each repeats a random phrase) are learned: embedding, norm and rotation of queries and keys, attention within documents with capped
scores, dropout on the residual stream, the norm of the stream, cross entropy, their gradients, and one grouped polar call a step for all 2-D weights of the layers.  Afterwards tokens are
generated one by one against a cache of keys and values, and the model is tuned as a policy: answers are sampled and scored, and the clipped loss, with a
divergence from the model as it was, is taken on their tokens."""
import argparse
import copy
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2601_22137_amd import layers, optim, prism   # noqa: E402

VOCABULARY, WIDTH, HEADS, K_HEADS, LAYERS, BATCH, LENGTH, PHRASE = 64, 256, 4, 2, 2, 16, 256, 8
SCALE = WIDTH ** -0.5


class Model(torch.nn.Module):
    def __init__(self, p=0.05):
        super().__init__()
        self.embed = layers.Embedding(VOCABULARY, WIDTH)
        self.norm = layers.LayerNorm(WIDTH, center=False)
        self.layers = torch.nn.ModuleList([layers.SelfAttention(WIDTH, HEADS, K_HEADS, softcap=30.0, p=p) for _ in range(LAYERS)])

    def logits(self, x):
        """To be taken times SCALE."""
        return self.norm(x) @ self.embed.weight.t()

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


class Update:
    """Momentum, orthogonalised for the weights of the layers, plain for the others."""

    def __init__(self, model, rate=0.02, others_rate=3e-3):
        self.model, self.rate = model, rate
        self.matrices = [w for layer in model.layers for w in (layer.w_qkv, layer.w_out)]
        self.momentum = [torch.zeros_like(w) for w in self.matrices]
        self.adam = torch.optim.Adam([p for p in model.parameters() if all(p is not w for w in self.matrices)], lr=others_rate)

    @torch.no_grad()
    def step(self):
        self.adam.step()
        for m, w in zip(self.momentum, self.matrices):
            m.mul_(0.9).add_(w.grad)
        for w, u in zip(self.matrices, optim.muon_orthogonalize(self.momentum)):
            w.add_(u, alpha=-self.rate * max(1.0, w.shape[0] / w.shape[1]) ** 0.5)
        self.model.zero_grad(set_to_none=True)


def train(steps, say=print):
    """(model, the losses)."""
    torch.manual_seed(0)
    model = Model()
    generator = torch.Generator().manual_seed(1)
    update = Update(model)
    losses = []
    for step in range(steps):
        inputs, targets = batch(generator)
        loss, _ = layers.policy_loss(model(*inputs, step=step), targets, scale=SCALE)        # cross entropy: no ratio, no advantages
        loss.backward()
        update.step()
        losses.append(loss.item())
        if say and (step % 10 == 0 or step + 1 == steps):
            say("step %3d  loss %.3f" % (step, losses[-1]))
    return model, losses


def tune(model, steps, answers=32, length=16, say=print):
    """(mean rewards, gradient norms): answers to random phrases are sampled, the reward is the share of their tokens that repeat the phrase, and each batch of answers is taken
    twice, its own log-probabilities as they were when it was sampled."""
    model.eval()
    reference, update = copy.deepcopy(model), Update(model, 0.002, 1e-4)
    generator = torch.Generator("cuda").manual_seed(3)
    rewards, norms = [], []
    for step in range(steps):
        phrase = torch.randint(0, VOCABULARY, (answers, PHRASE), device="cuda", generator=generator)
        text = generate(model, phrase.repeat(1, 2), length, generator)
        reward = (text[:, 2 * PHRASE:] == phrase.repeat(1, length // PHRASE + 1)[:, :length]).float().mean(1)
        advantage = ((reward - reward.mean()) / (reward.std() + 1e-3)).view(-1, 1).expand(-1, text.shape[1] - 1).contiguous()
        inputs, targets = text[:, :-1], text[:, 1:].clone()
        targets[:, :2 * PHRASE - 1] = -1                                                     # the phrases were given, not answered
        positions = torch.arange(inputs.shape[1], dtype=torch.int32, device="cuda").expand(answers, -1).contiguous()
        with torch.no_grad():
            old, ref = (layers.token_logprob(m(inputs, positions, None), targets, scale=SCALE) for m in (model, reference))
        for _ in range(2):
            logits = model(inputs, positions, None)
            r = prism.policy_loss(logits.detach(), targets, advantages=advantage, old_logp=old, ref_logp=ref, kl=0.05, scale=SCALE)
            logits.backward(r.dlogits)                                                       # loss and gradient came in one pass
            norms.append(sum(float(p.grad.float().square().sum()) for p in model.parameters()) ** 0.5)
            update.step()
        rewards.append(float(reward.mean()))
        if say:
            say("policy step %2d  reward %.3f  loss %.4f" % (step, rewards[-1], float(r.loss)))
    return rewards, norms


@torch.no_grad()
def generate(model, prompts, count, sample=None):
    """Continuation of prompts [batch, token], one token at a time: the likeliest ones, or drawn by a generator."""
    model.eval()
    caches = [layer.new_cache(prompts.shape[0], prompts.shape[1] + count) for layer in model.layers]
    tokens = prompts
    for at in range(prompts.shape[1] + count - 1):
        x = model.embed(tokens[:, at:at + 1])
        for layer, cache in zip(model.layers, caches):
            x = layer.step(x, cache)
        if at + 1 >= tokens.shape[1]:
            logits = model.logits(x)[:, -1]
            taken = logits.argmax(-1, keepdim=True) if sample is None else torch.multinomial(torch.softmax(logits.float() * SCALE, -1), 1, generator=sample)
            tokens = torch.cat([tokens, taken], 1)
    return tokens


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=120)
    ap.add_argument("--policy-steps", type=int, default=10)
    args = ap.parse_args()
    model, losses = train(args.steps)
    phrase = torch.randint(0, VOCABULARY, (4, PHRASE), device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    text = generate(model, phrase.repeat(1, 3), PHRASE)
    print("loss %.3f -> %.3f; %d of %d generated tokens repeat the phrase" % (losses[0], losses[-1], int((text[:, -PHRASE:] == phrase).sum()), phrase.numel()))
    tune(model, args.policy_steps)


if __name__ == "__main__":
    main()
