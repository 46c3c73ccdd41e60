"""One Gated DeltaNet layer from training to serving, all of its sequence work through the library:

    python examples/train_and_serve.py

Training: kvb_scan forward and kvb_scan_backward, as one differentiable function over packed ragged sequences.  Serving: a batch of
prompts enters the store's states by kvb_scan; then each round drafts some tokens, kvb_verify gives the layer's outputs behind each of them, kvb_accept
says from the resulting probabilities which drafts stand and what follows them, and kvb_flush commits exactly those.

The task is recall: a sequence is a random phrase said over and over, and whoever has heard it once can go on.  The drafts are looked up in
the request's own text (what followed the last time this token was there).  The weights around the layer are torch's.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2605_19049_amd import kvb  # noqa: E402

V, Hk, Hv, D, WIDTH = 64, 2, 4, 64, 256   # vocabulary, heads, head size, model width
SCALE = D ** -0.5


class Scan(torch.autograd.Function):
    """out = kvb_scan over packed sequences that start from zero states."""

    @staticmethod
    def forward(ctx, q, k, v, g, beta, start):
        B, n = len(start) - 1, len(q)
        sh, sq = kvb.shape(B, Hk, Hv, D, D, 1, kvb.F32, scale=SCALE), kvb.seqs(start, n, B)
        out = torch.empty_like(v)
        work = torch.empty(kvb.scan_work(sh, sq), dtype=torch.uint8, device="cuda")
        kvb.kvb_scan(sh, sq, q, k, v, g, beta, None, None, out, work)
        ctx.save_for_backward(q, k, v, g, beta, start)
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, g, beta, start = ctx.saved_tensors
        B, n = len(start) - 1, len(q)
        sh, sq = kvb.shape(B, Hk, Hv, D, D, 1, kvb.F32, scale=SCALE), kvb.seqs(start, n, B)
        grads = [torch.empty_like(x) for x in (q, k, v, g, beta)]
        work = torch.empty(kvb.scan_backward_work(sh, sq), dtype=torch.uint8, device="cuda")
        kvb.kvb_scan_backward(sh, sq, q, k, v, g, beta, None, dout.contiguous(), None, *grads, None, work)
        return (*grads, None)


class Model(torch.nn.Module):
    """Embedding of a token and the one before it, one layer, logits."""

    def __init__(self):
        super().__init__()
        self.embed = torch.nn.Embedding(V, WIDTH)
        self.before = torch.nn.Embedding(V + 1, WIDTH)
        self.rows = torch.nn.Linear(WIDTH, (2 * Hk + Hv) * D + 2 * Hv)
        self.out = torch.nn.Linear(Hv * D, V)

    def inputs(self, tokens, before):
        """q, k, v, g, beta of tokens [..] that follow `before` [..] (V: nothing)"""
        x = self.rows(self.embed(tokens) + self.before(before))
        q, k, v, a, b = x.split([Hk * D, Hk * D, Hv * D, Hv, Hv], dim=-1)
        heads = lambda y, h: y.unflatten(-1, (h, D))
        unit = lambda y: torch.nn.functional.normalize(heads(y, Hk), dim=-1).contiguous()
        return unit(q), unit(k), heads(v, Hv).contiguous(), torch.nn.functional.logsigmoid(a + 4.0).contiguous(), torch.sigmoid(b).contiguous()

    def logits(self, o):
        return self.out(o.flatten(-2) * D ** 0.5)


def phrases(rng, lens):
    """Packed tokens of a random phrase each, said over and over"""
    return np.concatenate([np.resize(rng.permutation(V)[:rng.integers(5, 13)], n) for n in lens])


def before_of(tokens, start):
    b = torch.roll(tokens, 1)
    b[start[:-1][start[:-1] < len(tokens)].long()] = V
    return b


def train(model, steps, rng, log=print):
    opt = torch.optim.Adam(model.parameters(), 3e-3)
    losses = []
    for step in range(steps):
        lens = rng.integers(20, 101, 32)
        start = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
        tokens = torch.tensor(phrases(rng, lens), device="cuda")
        o = Scan.apply(*model.inputs(tokens, before_of(tokens, start)), start)
        here = torch.ones(len(tokens), dtype=torch.bool, device="cuda")
        here[start[1:].long() - 1] = False   # (nothing follows a sequence's last token)
        loss = torch.nn.functional.cross_entropy(model.logits(o)[here], tokens.roll(-1)[here])
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
        if step % 20 == 0 or step == steps - 1:
            log(f"step {step:4d}  loss {losses[-1]:.3f}")
    return losses


class Server:
    """A batch of requests: prompt, then rounds of drafting, verifying, accepting and committing."""

    def __init__(self, model, prompts, drafts):
        self.model, self.T, self.B = model, drafts, len(prompts)
        self.texts = [list(map(int, p)) for p in prompts]
        B, T, lens = self.B, drafts, [len(p) for p in prompts]
        assert min(lens) >= 2
        # row i of a verify holds the last token (not yet in the state) and the drafts behind it: T + 1 records
        self.ds = kvb.DeviceStore(B, Hk, Hv, D, D, T + 1, kvb.F32)
        self.sh = kvb.shape(B, Hk, Hv, D, D, T + 1, kvb.F32, scale=SCALE)
        self.slot = torch.arange(B, dtype=torch.int32, device="cuda")
        self.vocab = kvb.vocab(B, T, V, kvb.F32)
        self.work = torch.empty(kvb.accept_work(self.vocab) or 1, dtype=torch.uint8, device="cuda")
        # all of each prompt but its last token goes into the states
        start = torch.tensor(np.concatenate([[0], np.cumsum([n - 1 for n in lens])]), dtype=torch.int32, device="cuda")
        tokens = torch.tensor([x for t in self.texts for x in t[:-1]], device="cuda")
        ins = model.inputs(tokens, before_of(tokens, start))
        sq = kvb.seqs(start, len(tokens), B)
        work = torch.empty(kvb.scan_work(self.sh, sq), dtype=torch.uint8, device="cuda")
        kvb.kvb_scan(self.sh, sq, *ins, self.ds.state, self.ds.state, torch.empty_like(ins[2]), work)

    def draft(self, text):
        """The tokens that came the last time, behind this text's last one"""
        text = list(text)
        for _ in range(self.T):
            at = len(text) - 2
            while at >= 0 and text[at] != text[-1]:
                at -= 1
            text.append(text[at + 1] if at >= 0 else text[-1])
        return text[-self.T:]

    def round(self, temperature, gen):
        """Tokens that each request gained"""
        B, T = self.B, self.T
        drafted = [self.draft(t) for t in self.texts]
        rows = torch.tensor([t[-2:] + d for t, d in zip(self.texts, drafted)], device="cuda")   # one before, last, drafts
        q, k, v, g, beta = self.model.inputs(rows[:, 1:], rows[:, :-1])
        out = torch.empty((B, T + 1, Hv, D), device="cuda")
        kvb.kvb_verify(self.sh, self.ds.c(), self.slot, T + 1, q, k, v, g, beta, out)
        logits = self.model.logits(out)
        if temperature > 0:
            target = torch.softmax(logits / temperature, -1)
        else:
            target = torch.nn.functional.one_hot(logits.argmax(-1), V).float()
        tokens = rows[:, 2:].to(torch.int32).contiguous()
        u, s = torch.rand((B, T), generator=gen, device="cuda"), torch.rand(B, generator=gen, device="cuda")
        path = torch.empty((B, T), dtype=torch.int32, device="cuda")
        accepted, token = (torch.empty(B, dtype=torch.int32, device="cuda") for _ in range(2))
        kvb.kvb_accept(self.vocab, None, None, tokens, target.contiguous(), None, u, s, path, accepted, token, self.work)
        # the last token and the accepted drafts enter the state; the token that follows is the next round's last
        kvb.kvb_flush(self.sh, self.ds.c(), self.slot, accepted + 1, 1)
        for b, (n, t) in enumerate(zip(accepted.tolist(), token.tolist())):
            self.texts[b] += drafted[b][:n] + [t]
        return accepted + 1


@torch.no_grad()
def serve(model, prompts, drafts, rounds, temperature=0.0, seed=0):
    server = Server(model, prompts, drafts)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    gained = [server.round(temperature, gen).float().mean().item() for _ in range(rounds)]
    return server.texts, gained


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--steps", type=int, default=120)
    p.add_argument("--drafts", type=int, default=4)
    p.add_argument("--rounds", type=int, default=8)
    p.add_argument("--temperature", type=float, default=0.0)
    a = p.parse_args()
    torch.manual_seed(0)
    rng = np.random.default_rng(0)
    model = Model().cuda()
    train(model, a.steps, rng)
    prompts = [phrases(rng, [n]) for n in rng.integers(30, 200, 16)]
    texts, gained = serve(model, prompts, a.drafts, a.rounds, a.temperature)
    right = np.mean([t[i] == t[i - period(p)] for p, t in zip(prompts, texts) for i in range(len(p), len(t))])
    print(f"tokens a request gains in each round: {np.round(gained, 2).tolist()}")
    print(f"of {sum(len(t) - len(p) for p, t in zip(prompts, texts))} new tokens {100 * right:.1f} % go on as the prompt does")


def period(p):
    return next(n for n in range(1, len(p)) if p[n] == p[0])


if __name__ == "__main__":
    main()
