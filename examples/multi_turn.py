"""A multi-turn rollout on one GPU: prompts, a tool's answers of ragged lengths, drafts that are checked, and single tokens, all
through the paged cache.

The model is a stack of attention layers with random weights; what counts is the order of the calls, which is a serving
worker's.  Per layer of a step:

    prompts       rotate (queries and keys where the projection left them), prefill, append_chunk (keys as they are)
    any chunk     append_chunk (norm, rotation and pages in one call, queries beside them), extend
    one token     the same two calls; extend runs as a decode step

    python examples/multi_turn.py [--seqs 16] [--turns 3] [--kv e4m3]

At the end every sequence is run again from its first token as one long prompt, and the two last hidden states are compared.
"""
import argparse
import os
import sys
import time

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2507_01663_amd as ra  # noqa: E402

DEV, PAGE = "cuda:0", 16


class Model:
    """Weights of the layers: projections in bf16, norm weights and the rotation's table in float32."""

    def __init__(self, layers=2, Hq=8, Hkv=2, D=128, width=512, vocab=1000, positions=8192, seed=0):
        g = torch.Generator().manual_seed(seed)
        normal = lambda *s: torch.randn(s, generator=g)
        self.Hq, self.Hkv, self.D, self.layers, self.vocab = Hq, Hkv, D, layers, vocab
        self.embedding = normal(vocab, width).to(torch.bfloat16).to(DEV)
        self.wqkv = [(normal(width, (Hq + 2 * Hkv) * D) / width ** 0.5).to(torch.bfloat16).to(DEV) for _ in range(layers)]
        self.wo = [(normal(Hq * D, width) / (Hq * D) ** 0.5).to(torch.bfloat16).to(DEV) for _ in range(layers)]
        self.norms = [[(1 + 0.1 * normal(D)).to(DEV) for _ in "qk"] for _ in range(layers)]
        self.rope = ra.rope_table(positions, D, 1e6, DEV)

    def project(self, layer, x):
        """Views of one projection's output: q [T,Hq,D], k and v [T,Hkv,D]."""
        y = F.rms_norm(x, x.shape[-1:]) @ self.wqkv[layer]
        nq, nk = self.Hq * self.D, self.Hkv * self.D
        return (y[:, :nq].unflatten(1, (self.Hq, self.D)), y[:, nq:nq + nk].unflatten(1, (self.Hkv, self.D)),
                y[:, nq + nk:].unflatten(1, (self.Hkv, self.D)))


class Rollout:
    """Sequences of one batch: their pages in every layer's pools and their lengths."""

    def __init__(self, model, seqs, capacity, kv="bf16", dec=None):
        self.m, self.kv, self.dec, self.own = model, kv, dec or ra.Decoder(0), dec is None
        per, dtype = (capacity + PAGE - 1) // PAGE, torch.bfloat16 if kv == "bf16" else torch.uint8
        self.table = torch.randperm(seqs * per, device=DEV).to(torch.int32).view(seqs, per)
        self.lens = torch.zeros(seqs, dtype=torch.int32, device=DEV)
        shape = (seqs * per, model.Hkv, PAGE, model.D)
        self.pools = [[torch.zeros(shape, dtype=dtype, device=DEV) for _ in "kv"] for _ in range(model.layers)]
        self.scales = [[None if kv == "bf16" else torch.ones(shape[:2], device=DEV) for _ in "kv"] for _ in range(model.layers)]

    def close(self):
        torch.cuda.synchronize()
        if self.own:
            self.dec.close()

    def step(self, chunks, prompts=False):
        """chunks[b]: sequence b's new tokens.  Their keys and values enter the cache; returns the hidden state of every
        sequence's last new token.  prompts: the sequences are empty, and their tokens attend to one another alone."""
        m, most = self.m, max(map(len, chunks))
        cu = torch.tensor([0] + [len(c) for c in chunks]).cumsum(0).to(torch.int32).to(DEV)
        x = m.embedding[torch.cat([torch.as_tensor(c, dtype=torch.long) for c in chunks]).to(DEV)]
        after = self.lens + cu.diff()
        positions = None
        if prompts:
            positions = torch.cat([torch.arange(len(c), dtype=torch.int32) for c in chunks]).to(DEV)
        for i in range(m.layers):
            q, k, v = m.project(i, x)
            (kp, vp), (ks, vs), (qw, kw) = self.pools[i], self.scales[i], m.norms[i]
            out = torch.empty(q.shape, dtype=torch.bfloat16, device=DEV)
            lse = torch.empty(q.shape[:2], dtype=torch.float32, device=DEV)
            scale = m.D ** -0.5
            if prompts:
                qr, kr, vr = (torch.empty(t.shape, dtype=t.dtype, device=DEV) for t in (q, k, v))
                self.dec.rotate(ra.rotate_from_tensors(q, k, qr, kr, positions, m.rope, qw, kw))
                vr.copy_(v)
                self.dec.prefill(ra.prefill_from_tensors(qr, kr, vr, cu, most, out, lse, scale))
                self.dec.append_chunk(ra.append_chunk_from_tensors(kr, vr, cu, most, self.table, self.lens, kp, vp, ks, vs))
            else:
                self.dec.append_chunk(ra.append_chunk_from_tensors(k, v, cu, most, self.table, self.lens, kp, vp, ks, vs, q, q, None, m.rope,
                                                                   qw, kw))
                self.dec.extend(ra.extend_from_tensors(q, kp, vp, cu, most, self.table, after, out, lse, scale, ks, vs))
            x = x + out.flatten(1) @ m.wo[i]
        self.lens = after
        return x[(cu[1:] - 1).long()]

    def forget(self, counts):
        """Drops the last tokens of every sequence (a draft's that were not accepted): their slots are written again."""
        self.lens = self.lens - torch.as_tensor(counts, dtype=torch.int32, device=DEV)

    def next_tokens(self, hidden):
        return (F.rms_norm(hidden, hidden.shape[-1:]) @ self.m.embedding.T).argmax(-1)


def run(seqs=16, turns=3, kv="bf16", layers=2, prompt=(20, 400), answer=(1, 150), draft=4, singles=4, seed=0, say=print):
    """Returns the largest difference between the rollout's last hidden states and those of one pass over the whole sequences,
    relative to their norm."""
    g = torch.Generator().manual_seed(seed)
    many = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=g))
    m = Model(layers, seed=seed)
    text = [torch.randint(m.vocab, (many(*prompt),), generator=g).tolist() for _ in range(seqs)]
    room = prompt[1] + turns * (answer[1] + draft + singles) + 1
    r = Rollout(m, seqs, room, kv)
    tokens, start = 0, time.time()
    hidden = r.step(text, prompts=True)
    for turn in range(turns):
        for _ in range(singles):                             # the sequences write on their own, a token at a time
            new = r.next_tokens(hidden).tolist()
            hidden = r.step([[t] for t in new])
            text = [a + [t] for a, t in zip(text, new)]
        # a draft of a few tokens is looked at in one step; all but its first are turned down
        drafts = [torch.randint(m.vocab, (draft,), generator=g).tolist() for _ in range(seqs)]
        r.step(drafts)
        r.forget([draft - 1] * seqs)
        # a tool's answers come in; a quarter of the sequences waits for theirs and writes one token meanwhile
        new = [torch.randint(m.vocab, (many(*answer) if b % 4 else 1,), generator=g).tolist() for b in range(seqs)]
        hidden = r.step(new)
        text = [a + d[:1] + c for a, d, c in zip(text, drafts, new)]
        tokens += singles * seqs + draft * seqs + sum(map(len, new))
        torch.cuda.synchronize()
        say("turn %d: lengths %d .. %d, %d new tokens so far, %.1f ms" % (turn, min(map(len, text)), max(map(len, text)), tokens,
                                                                     1e3 * (time.time() - start)))
    assert r.lens.tolist() == [len(a) for a in text]
    whole = Rollout(m, seqs, room, kv, r.dec)
    want = whole.step(text, prompts=True)
    worst = float(((hidden - want).float().norm(dim=1) / want.float().norm(dim=1)).max())
    say("last hidden states against one pass over the whole sequences: %.4f" % worst)
    whole.close()
    r.close()
    return worst


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--seqs", type=int, default=16)
    p.add_argument("--turns", type=int, default=3)
    p.add_argument("--layers", type=int, default=2)
    p.add_argument("--kv", choices=["bf16", "e4m3"], default="bf16")
    a = p.parse_args()
    run(a.seqs, a.turns, a.kv, a.layers)
