"""A small decoder with windowed attention, trained and then asked to go on: python -m paper_2405_18047_amd.examples.long_context

What the operators for long contexts, the last stage and serving are for, next to a stage:
  training   rotary positions (scaled) and sliding-window attention with sinks, forward and backward-p1; the feed-forward halves
             as MLP-only stages with their split backward; log probabilities of the next tokens with the derivative of the logits in one
             pass; the norm of all gradients, clipped;
  answering  new tokens appended to ring caches of sinks + window rows, one token decoded over them, the most likely next tokens.

The text is synthetic: sequences that repeat a random phrase, which is shorter than the window and much shorter than the sequence, so that the
phrase has to be found again through the window.
"""
from __future__ import annotations

import argparse

import torch

import paper_2405_18047_amd as tbp

EPS = 1e-6
BASE_RATE, BETA1, BETA2 = 4e-3, 0.9, 0.99          # of the update (running means of the clipped gradients and of their squares)


class Shape:
    """Sizes of the model; the defaults train in seconds."""

    def __init__(self, layers=2, d_model=256, n_heads=4, n_kv_heads=2, head_dim=64, d_ffn=688, vocab=512, window=64, sinks=4,
                 trained_context=64, context=512):
        self.layers, self.d_model, self.n_heads, self.n_kv_heads, self.head_dim = layers, d_model, n_heads, n_kv_heads, head_dim
        self.d_ffn, self.vocab, self.window, self.sinks = d_ffn, vocab, window, sinks
        self.trained_context, self.context = trained_context, context
        self.qk_heads, self.width = n_heads + n_kv_heads, (n_heads + 2 * n_kv_heads) * head_dim


class WindowAttention:
    """x + Wo Attention(RoPE(RMSNorm(x) Wqkv)): forward, backward-p1 and backward-p2, and the form for a new token."""

    def __init__(self, c: Shape, table, params):
        self.c, self.table = c, table
        self.w_qkv, self.w_o, self.g = params

    def _heads(self):
        c = self.c
        return c.n_heads, c.n_kv_heads, c.head_dim, c.window, c.sinks

    def forward(self, x, seq):
        c = self.c
        h = tbp.tbp_rmsnorm_fwd(x, self.g, EPS)
        qkv = tbp.tbp_gemm(tbp.NN, h, self.w_qkv)
        tbp.tbp_rotary(qkv, c.qk_heads, c.head_dim, self.table, seq=seq, out=qkv)
        out, lse = tbp.tbp_window_attention_fwd(qkv, seq, *self._heads())
        self.kept = (x, h, qkv, out, lse, seq)
        return tbp.tbp_gemm(tbp.NN, out, self.w_o, R=x)

    def backward_p1(self, dy):
        c = self.c
        x, h, qkv, out, lse, seq = self.kept
        d_out = tbp.tbp_gemm(tbp.NT, dy, self.w_o)
        dqkv = tbp.tbp_window_attention_p1(qkv, out, d_out, lse, seq, *self._heads())
        tbp.tbp_rotary(dqkv, c.qk_heads, c.head_dim, self.table, seq=seq, backward=True, out=dqkv)
        dh = tbp.tbp_gemm(tbp.NT, dqkv, self.w_qkv)
        dx, self.dg = tbp.tbp_rmsnorm_p1(dh, x, self.g, EPS, resid=dy)
        self.kept = (h, dqkv, out, dy)                       # what backward-p2 contracts
        return dx

    def backward_p2(self):
        h, dqkv, out, dy = self.kept
        self.kept = None
        return [tbp.tbp_gemm(tbp.TN, h, dqkv, out_f32=True), tbp.tbp_gemm(tbp.TN, out, dy, out_f32=True), self.dg]

    def new_token(self, x, cache, workspace, lengths):
        """x [batch, d]: one new token of every sequence, `lengths` long with it (the decode answers for one at a time) -> [batch, d]."""
        c = self.c
        qkv = tbp.tbp_gemm(tbp.NN, tbp.tbp_rmsnorm_fwd(x, self.g, EPS), self.w_qkv)
        q = tbp.tbp_rotary_append(qkv, c.n_heads, c.n_kv_heads, c.head_dim, self.table, lengths, *cache, c.sinks)
        out, _ = tbp.tbp_window_decode(q, *cache, lengths, *self._heads(), workspace=workspace)
        return tbp.tbp_gemm(tbp.NN, out, self.w_o, R=x)


class Model:
    """Embedding, layers of windowed attention and MLP stage, norm and head; fp32 master weights."""

    def __init__(self, c: Shape, seq, batch, seed=1, device="cuda:0"):
        self.c, self.seq, self.batch, self.device = c, seq, batch, device
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        weight = lambda *s: torch.randn(s, generator=gen, device=device) * s[0] ** -0.5
        gain = lambda: torch.ones(c.d_model, device=device)
        d, f = c.d_model, c.d_ffn
        attn = [[weight(d, c.width), weight(c.n_heads * c.head_dim, d) * 0.5, gain()] for _ in range(c.layers)]
        mlp = [[weight(d, 2 * f), weight(f, d) * 0.5, gain()] for _ in range(c.layers)]
        ends = [torch.randn((c.vocab, d), generator=gen, device=device) * 0.5, gain(), weight(d, c.vocab)]
        self.master = [w for layer in attn for w in layer] + [w for layer in mlp for w in layer] + ends
        self.params = [w.to(torch.bfloat16) for w in self.master]
        n = 3 * c.layers
        # the context is longer than the positions are meant for: slow pairs of columns are interpolated
        self.table = tbp.tbp_rotary_table(c.context, c.head_dim, 10000.0, tbp.TBP_ROTARY_RAMP, factor=c.context / c.trained_context, low=1.0, high=8.0,
                                          original=c.trained_context)
        self.attention = [WindowAttention(c, self.table, self.params[3 * i:3 * i + 3]) for i in range(c.layers)]
        self.mlp = []
        for i in range(c.layers):
            w_gu, w_d, g2 = self.params[n + 3 * i:n + 3 * i + 3]
            cfg = tbp.tbp_config(n_layers=1, d_model=d, n_heads=0, head_dim=0, d_ffn=f, seq=seq, micro_batch=batch, max_microbatches=1, act_slots=0,
                                 causal=1, dtype=tbp.TBP_BF16, rms_eps=EPS, rope_base=10000.0, attention=tbp.TBP_ATTN_AUTO, gain_grad=tbp.TBP_GAIN_PARTIALS)
            self.mlp.append(tbp.Stage(cfg, {"w_gu": [w_gu], "w_d": [w_d], "g2": [g2]}, device))
        self.embedding, self.g_end, self.w_head = self.params[2 * n:]
        self.clipped = [torch.empty_like(w) for w in self.master]
        self.mean, self.square, self.steps = [torch.zeros_like(w) for w in self.master], [torch.zeros_like(w) for w in self.master], 0

    # ---- training ----------------------------------------------------------------------------------------------------
    def hidden(self, tokens):
        x = self.embedding[tokens.reshape(-1)]
        for a, m in zip(self.attention, self.mlp):
            x = m.forward(0, a.forward(x, self.seq))
        return x

    def logits(self, x):
        return tbp.tbp_gemm(tbp.NN, tbp.tbp_rmsnorm_fwd(x, self.g_end, EPS), self.w_head)

    def gradients(self, tokens, targets):
        """tokens, targets [batch, seq] (a target of -1 is left out) -> (mean log probability of the targets, the gradients of -mean)."""
        x = self.hidden(tokens)
        h = tbp.tbp_rmsnorm_fwd(x, self.g_end, EPS)
        logits = tbp.tbp_gemm(tbp.NN, h, self.w_head)
        t = targets.reshape(-1).to(torch.int32)
        n = int((t >= 0).sum())
        logp, _, _, d_logits = tbp.tbp_logprobs_step(logits, t, torch.full(t.shape, -1.0 / n, device=self.device), out=logits)
        d_head = tbp.tbp_gemm(tbp.TN, h, d_logits, out_f32=True)
        dx, dg_end = tbp.tbp_rmsnorm_p1(tbp.tbp_gemm(tbp.NT, d_logits, self.w_head), x, self.g_end, EPS)
        for a, m in zip(reversed(self.attention), reversed(self.mlp)):      # backward-p1 through all layers ...
            dx = a.backward_p1(m.backward_p1(0, dx))
        d_attn = [g for a in self.attention for g in a.backward_p2()]        # ... then every weight gradient
        for m in self.mlp:
            m.backward_p2([0], tbp.TBP_P2_KCONCAT, accumulate=False)
        d_mlp = [m.grads[k][0] for m in self.mlp for k in ("w_gu", "w_d", "g2")]
        d_emb = torch.zeros_like(self.master[-3]).index_add_(0, tokens.reshape(-1), dx.float())
        return logp.sum() / n, d_attn + d_mlp + [d_emb, dg_end, d_head]

    def step(self, tokens, targets, rate, max_norm=1.0):
        """One step of training at `rate` times the base rate; -> (mean log probability, norm of all gradients)."""
        mean_logp, grads = self.gradients(tokens, targets)
        norm = tbp.GradList(grads, self.clipped).clip(max_norm)
        self.steps += 1
        scale = rate * BASE_RATE * (1 - BETA2 ** self.steps) ** 0.5 / (1 - BETA1 ** self.steps)
        for w, p, g, m, v in zip(self.master, self.params, self.clipped, self.mean, self.square):
            m.lerp_(g, 1 - BETA1)
            v.mul_(BETA2).addcmul_(g, g, value=1 - BETA2)
            w.addcdiv_(m, v.sqrt().add_(1e-8), value=-scale)
            p.copy_(w)
        return mean_logp, norm

    # ---- answering ----------------------------------------------------------------------------------------------------
    def caches(self, batch):
        """Of every layer: keys and values in rings of sinks + window rows, and the decode's workspace."""
        c = self.c
        shape = (batch, c.sinks + c.window, c.n_kv_heads * c.head_dim)
        new = lambda: torch.zeros(shape, dtype=torch.bfloat16, device=self.device)
        return [((new(), new()), tbp.tbp_window_decode_workspace(batch, c.n_heads, c.n_kv_heads, c.head_dim, c.window, c.sinks, self.device))
                for _ in range(c.layers)]

    def next_logits(self, tokens, lengths, caches):
        """tokens [batch]: the last ones of sequences that are `lengths` long with them -> logits [batch, vocab]."""
        x = self.embedding[tokens]
        n = 3 * self.c.layers
        for i, (a, (cache, workspace)) in enumerate(zip(self.attention, caches)):
            x = a.new_token(x, cache, workspace, lengths)
            w_gu, w_d, g2 = self.params[n + 3 * i:n + 3 * i + 3]
            m = tbp.tbp_swiglu_fwd(tbp.tbp_gemm(tbp.NN, tbp.tbp_rmsnorm_fwd(x, g2, EPS), w_gu))
            x = tbp.tbp_gemm(tbp.NN, m, w_d, R=x)
        return self.logits(x)

    def answer(self, prompt, n_tokens, top=4):
        """prompt [batch, n] -> (the n_tokens most likely tokens one after the other [batch, n_tokens], log probabilities of the `top` candidates of
        each [batch, n_tokens, top])."""
        batch, n = prompt.shape
        caches, lengths = self.caches(batch), torch.zeros(batch, dtype=torch.int32, device=self.device)
        none = torch.full((batch,), -1, dtype=torch.int32, device=self.device)
        said, weights, tokens = [], [], None
        for i in range(n + n_tokens - 1):
            tokens = prompt[:, i] if i < n else tokens
            lengths += 1
            logits = self.next_logits(tokens, lengths, caches)
            if i >= n - 1:
                _, _, _, top_logp, top_ids = tbp.tbp_logprobs(logits, none, top=top)
                tokens = top_ids[:, 0].long()
                said.append(tokens)
                weights.append(top_logp)
        return torch.stack(said, dim=1), torch.stack(weights, dim=1)


def phrases(batch, seq, period, vocab, gen, device="cuda:0"):
    """Sequences that repeat a random phrase of `period` tokens -> (tokens, targets), the first round of each left out of the targets."""
    phrase = torch.randint(0, vocab, (batch, period), generator=gen, device=device)
    text = phrase.repeat(1, seq // period + 2)[:, :seq + 1]
    targets = text[:, 1:].clone()
    targets[:, :period - 1] = -1
    return text[:, :-1].contiguous(), targets


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=600)
    ap.add_argument("--seq", type=int, default=256)
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--period", type=int, default=24)
    ap.add_argument("--rate", type=float, default=0.5, help="times the base rate; falls to nothing over the steps")
    a = ap.parse_args()
    model = Model(Shape(), a.seq, a.batch)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(2)
    for i in range(a.steps):
        tokens, targets = phrases(a.batch, a.seq, a.period, model.c.vocab, gen)
        logp, norm = model.step(tokens, targets, a.rate * (1 - i / a.steps))
        if i % 100 == 0 or i == a.steps - 1:
            print(f"step {i}: mean log probability {float(logp):.3f}, gradient norm {float(norm):.3f}", flush=True)
    tokens, _ = phrases(2, 3 * a.period, a.period, model.c.vocab, gen)
    said, weights = model.answer(tokens, a.period)
    print(f"{float((said == tokens[:, :a.period]).float().mean()):.0%} of the next round of the phrase said as it was; "
          f"the first candidates' log probabilities: {[round(float(w), 3) for w in weights[0, 0]]}")


if __name__ == "__main__":
    main()
