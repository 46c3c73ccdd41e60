"""One Gated DeltaNet layer from training to serving, all of its sequence work through the library:

    python examples/train_and_serve.py

Training: a row of the layer's projection becomes q, k, v and gates by kvb_conv, kvb_scan runs the recurrence, kvb_norm each head's norm with the output
gate; they and their backward calls are differentiable functions over packed ragged sequences, and kvb_grad_norm and kvb_clip cut the gradients.  Serving: a
batch of prompts enters the convolution's and the store's states by kvb_conv and kvb_scan; then each round drafts some tokens, kvb_conv_verify, kvb_verify and kvb_norm
give the layer's outputs behind each of them, kvb_accept says from the resulting probabilities which drafts stand and what follows them, and kvb_conv_commit and kvb_flush commit
exactly those.

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
SCALE, EPS, TAPS = D ** -0.5, 1e-6, 4
C = (2 * Hk + Hv) * D                     # channels of the convolution
ROW = C + Hv * D + 2 * Hv                 # a row of the projection: q, k and v, the output gate, what the gates are made from


def parts(row):
    """x, gate, b and a in rows [.., ROW]"""
    return row[..., :C], row[..., C:C + Hv * D], row[..., -2 * Hv:-Hv], row[..., -Hv:]


class Conv(torch.autograd.Function):
    """q, k, v, g, beta = kvb_conv over packed sequences that nothing comes before."""

    @staticmethod
    def forward(ctx, row, weight, A_log, dt_bias, start):
        B, n = len(start) - 1, len(row)
        x, _, b, a = parts(row)
        ctx.sh, ctx.sq = kvb.shape(B, Hk, Hv, D, D, 1, kvb.F32), kvb.seqs(start, n, B)
        ctx.ta = kvb.taps(weight, width=TAPS, A_log=A_log, dt_bias=dt_bias, x=x, a=a, b=b, eps=EPS)
        q, k, v = (torch.empty((n, h, D), device="cuda") for h in (Hk, Hk, Hv))
        g, beta = (torch.empty((n, Hv), device="cuda") for _ in range(2))
        kvb.kvb_conv(ctx.sh, ctx.ta, ctx.sq, x, a, b, None, None, q, k, v, g, beta)
        ctx.save_for_backward(row, weight, A_log, dt_bias, start)
        return q, k, v, g, beta

    @staticmethod
    def backward(ctx, *grads):
        row, weight, A_log, dt_bias, start = ctx.saved_tensors
        x, _, b, a = parts(row)
        drow = torch.zeros_like(row)   # (the output gate's part gets its gradient from kvb_norm)
        dx, _, db, da = parts(drow)
        dweight, dA_log, ddt_bias = (torch.empty_like(y) for y in (weight, A_log, dt_bias))
        work = torch.empty(kvb.conv_backward_work(ctx.sh, ctx.ta, ctx.sq), dtype=torch.uint8, device="cuda")
        kvb.kvb_conv_backward(ctx.sh, ctx.ta, ctx.sq, x, a, b, None, *(y.contiguous() for y in grads), None, dx, da, db, dweight, None, dA_log, ddt_bias, None, work)
        return drow, dweight, dA_log, ddt_bias, None


class Norm(torch.autograd.Function):
    """kvb_norm of each head of o [n, Hv, D] with the output gate in the rows of the projection"""

    @staticmethod
    def forward(ctx, o, row, weight):
        gate = parts(row)[1]
        ctx.ro = kvb.rows(len(o), Hv, D, kvb.F32, x=o, gate=gate, eps=EPS)
        out = torch.empty_like(o)
        kvb.kvb_norm(ctx.ro, o, None, gate, weight, None, out)
        ctx.save_for_backward(o, row, weight)
        return out

    @staticmethod
    def backward(ctx, dout):
        o, row, weight = ctx.saved_tensors
        do, drow, dweight = torch.empty_like(o), torch.zeros_like(row), torch.empty_like(weight)
        work = torch.empty(kvb.norm_backward_work(ctx.ro), dtype=torch.uint8, device="cuda")
        kvb.kvb_norm_backward(ctx.ro, o, parts(row)[1], weight, dout.contiguous(), None, do, None, parts(drow)[1], dweight, work)
        return do, drow, dweight


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
    """Embedding, one layer, logits."""

    def __init__(self):
        super().__init__()
        self.embed = torch.nn.Embedding(V, WIDTH)
        self.rows = torch.nn.Linear(WIDTH, ROW)
        with torch.no_grad():
            self.rows.bias[C:C + Hv * D] = 1.0   # the output gate starts open
        # the convolution starts as the token's own row, for keys as the row before it: what a token follows is what it is found by
        taps = 0.1 * torch.randn(C, TAPS)
        taps[:, -1] += 1.0
        taps[Hk * D:2 * Hk * D] = taps[Hk * D:2 * Hk * D].roll(-1, 1)
        self.taps = torch.nn.Parameter(taps)
        self.A_log = torch.nn.Parameter(torch.zeros(Hv))
        self.dt_bias = torch.nn.Parameter(torch.full((Hv,), -4.0))
        self.norm = torch.nn.Parameter(torch.ones(D))
        self.out = torch.nn.Linear(Hv * D, V)

    def forward(self, tokens, start):
        """Logits behind each of the packed tokens"""
        row = self.rows(self.embed(tokens))
        o = Scan.apply(*Conv.apply(row, self.taps, self.A_log, self.dt_bias, start), start)
        return self.logits(Norm.apply(o, row, self.norm))

    def logits(self, o):
        return self.out(o.flatten(-2))


def phrases(rng, lens):
    """Packed tokens of a random phrase each, said over and over"""
    return np.concatenate([np.resize(rng.permutation(V)[:rng.integers(5, 13)], n) for n in lens])


def train(model, steps, rng, log=print):
    opt = torch.optim.Adam(model.parameters(), 3e-3)
    for p in model.parameters():   # (the gradients stay where they are, so that their list is made once)
        p.grad = torch.zeros_like(p)
    grads, norm = kvb.TensorList([p.grad for p in model.parameters()]), torch.empty(1, device="cuda")
    work = torch.empty(kvb.grad_norm_work(grads.c()), dtype=torch.uint8, device="cuda")
    losses = []
    for step in range(steps):
        lens = rng.integers(20, 101, 32)
        start = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
        tokens = torch.tensor(phrases(rng, lens), device="cuda")
        here = torch.ones(len(tokens), dtype=torch.bool, device="cuda")
        here[start[1:].long() - 1] = False   # (nothing follows a sequence's last token)
        loss = torch.nn.functional.cross_entropy(model(tokens, start)[here], tokens.roll(-1)[here])
        opt.zero_grad(set_to_none=False)
        loss.backward()
        kvb.kvb_grad_norm(grads.c(), norm, work)
        kvb.kvb_clip(grads.c(), None, norm, 1.0)
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
        self.conv = torch.zeros((B, TAPS - 1, C), device="cuda")   # the convolution's states
        # all of each prompt but its last token goes into the states
        start = torch.tensor(np.concatenate([[0], np.cumsum([n - 1 for n in lens])]), dtype=torch.int32, device="cuda")
        tokens = torch.tensor([x for t in self.texts for x in t[:-1]], device="cuda")
        sq = kvb.seqs(start, len(tokens), B)
        x, _, b, a = parts(model.rows(model.embed(tokens)))
        ins = self.outputs(len(tokens))
        kvb.kvb_conv(self.sh, self.taps(x, b, a), sq, x, a, b, None, self.conv, *ins)
        work = torch.empty(kvb.scan_work(self.sh, sq), dtype=torch.uint8, device="cuda")
        kvb.kvb_scan(self.sh, sq, *ins, self.ds.state, self.ds.state, torch.empty_like(ins[2]), work)

    def taps(self, x, b, a):
        m = self.model
        return kvb.taps(m.taps, width=TAPS, A_log=m.A_log, dt_bias=m.dt_bias, x=x, a=a, b=b, eps=EPS)

    def outputs(self, *n):
        return [torch.empty(n + (h, D), device="cuda") for h in (Hk, Hk, Hv)] + [torch.empty(n + (Hv,), device="cuda") for _ in range(2)]

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
        tokens = torch.tensor([t[-1:] + d for t, d in zip(self.texts, drafted)], device="cuda")   # the last one, drafts
        row = self.model.rows(self.model.embed(tokens))
        x, gate, b, a = parts(row)
        ta, ins, out = self.taps(x, b, a), self.outputs(B, T + 1), torch.empty((B, T + 1, Hv, D), device="cuda")
        kvb.kvb_conv_verify(self.sh, ta, self.slot, B, T + 1, None, x, a, b, self.conv, *ins)
        kvb.kvb_verify(self.sh, self.ds.c(), self.slot, T + 1, *ins, out)
        ro = kvb.rows(B * (T + 1), Hv, D, kvb.F32, gate=gate.flatten(0, 1), eps=EPS)
        kvb.kvb_norm(ro, out, None, gate, self.model.norm, None, out)
        logits = self.model.logits(out)
        if temperature > 0:
            target = torch.softmax(logits / temperature, -1)
        else:
            target = torch.nn.functional.one_hot(logits.argmax(-1), V).float()
        drafts = tokens[:, 1:].to(torch.int32).contiguous()
        u, s = torch.rand((B, T), generator=gen, device="cuda"), torch.rand(B, generator=gen, device="cuda")
        path = torch.empty((B, T), dtype=torch.int32, device="cuda")
        accepted, token = (torch.empty(B, dtype=torch.int32, device="cuda") for _ in range(2))
        kvb.kvb_accept(self.vocab, None, None, drafts, target.contiguous(), None, u, s, path, accepted, token, self.work)
        # the last token and the accepted drafts enter the states; the token that follows is the next round's last
        kvb.kvb_conv_commit(self.sh, ta, self.slot, B, T + 1, None, accepted + 1, x, self.conv, self.conv)
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
