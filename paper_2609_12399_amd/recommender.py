"""A generative recommender on the library's operators: item tokens in, the next tokens' log
probabilities out, and the beam search over them that the decode is made for.

The model is a stack of :class:`mixer.DeltaMixer` layers with convolution and output gates.
Between two layers one pass (``onela_block_norm``) norms a layer's output, scales it per
channel, adds it to the residual stream (fp32) and norms the sum for the next layer.  The
logits go to ``onela_token_logprobs``: for the loss and its gradient in training, for the
logarithm of the sum in the search, where ``runner.scores_for_logits`` lets
``onela_select_beams`` take the logits themselves.

    python -m paper_2609_12399_amd.recommender   # trains a small model, then searches with it
"""
from __future__ import annotations

import torch

from . import runner
from .mixer import BeamStates, BlockNormFunction, DeltaMixer, TokenLogprobsFunction
from .workload import WorkloadSpec


class Recommender:
    def __init__(self, vocab: int, width: int, num_layers: int, num_qk_heads: int,
                 num_v_heads: int, d: int, io: str = "bf16", conv_taps: int = 4,
                 rotary_dim: int = 0, max_positions: int = 0, seed: int = 0, device="cuda:0"):
        g = torch.Generator(device=device).manual_seed(seed)
        dt = {"bf16": torch.bfloat16, "f32": torch.float32}[io]
        self.vocab, self.width, self.io, self.device = vocab, width, io, device
        self.layers = [DeltaMixer(width, num_qk_heads, num_v_heads, d, d, io, rotary_dim,
                                  max_positions, seed + 1 + i, device, conv_taps, gated=True)
                       for i in range(num_layers)]

        def weight(n, m, size):
            w = torch.randn((n, m), generator=g, device=device) * size
            return w.to(dt).requires_grad_()

        def ones(n):
            return torch.ones((n, width), device=device).requires_grad_()

        self.embedding, self.head = weight(vocab, width, 1.0), weight(width, vocab, width ** -0.5)
        # before every layer and before the head; after every layer
        self.w_before, self.w_after = ones(num_layers + 1), ones(num_layers)
        self.scale = (0.5 * torch.ones((num_layers, width), device=device)).requires_grad_()

    def weights(self):
        own = [self.embedding, self.head, self.w_before, self.w_after, self.scale]
        return own + [w for layer in self.layers for w in layer.weights()]

    def _enter(self, tokens):
        """The first layer's input [tokens][width] and the residual stream."""
        x = self.embedding[tokens][:, None]
        h = x.float()
        y, _ = BlockNormFunction.apply(x, None, None, None, self.w_before[0], None, False, True,
                                       None, 1.0, 1e-6)
        return y[:, 0], h

    def _between(self, i, x, h):
        """Layer i's output x to the next layer's input (after the last one, the head's)."""
        y, h = BlockNormFunction.apply(x[:, None], h, None, self.w_after[i], self.w_before[i + 1],
                                       self.scale[i], True, True, None, 1.0, 1e-6)
        return y[:, 0], h

    def __call__(self, tokens, seq_offsets, positions=None):
        """Outputs of the last norm [tokens][width] and every layer's states, of packed sequences;
        ``outputs @ head`` are the logits.  Differentiable."""
        x, h = self._enter(tokens)
        states = []
        for i, layer in enumerate(self.layers):
            x, state = layer(x, seq_offsets, positions)
            states.append(state)
            x, h = self._between(i, x, h)
        return x, states

    def loss(self, tokens, targets, seq_offsets, positions=None):
        """The mean of minus the log probabilities of targets [tokens] (below 0: none)."""
        x, _ = self(tokens, seq_offsets, positions)
        logp = TokenLogprobsFunction.apply(x @ self.head, targets[:, None], 0, 1.0, False)[0]
        return -logp.sum() / (targets >= 0).sum()

    @torch.no_grad()
    def search(self, tokens, seq_offsets, beams: int, steps: int):
        """The ``beams`` best continuations of ``steps`` tokens after each packed prompt, best
        first: tokens [requests][beams][steps] and their log probabilities.  Prompts have one
        token at least, and at most the decode's steps (8) follow the first token."""
        R, W, V = seq_offsets.numel() - 1, beams, self.vocab
        if steps < 1 or bool((seq_offsets[1:] <= seq_offsets[:-1]).any()):
            raise ValueError("a search takes a step and prompts of one token at least")
        x, states = self(tokens, seq_offsets)
        logits = (x[seq_offsets[1:].long() - 1] @ self.head).float()
        kept = [BeamStates(conv) for _, conv in states]
        layer = self.layers[0]
        spec = WorkloadSpec("search", R, layer.HK, layer.HV, layer.dk, layer.dv, 0,
                            (W,) * max(1, steps - 1), self.io, "uniform")
        decoders = [runner.Decoder(spec, state, self.device) for state, _ in states]
        first = runner.TokenLogprobs(R, V, 0, 0, "f32", device=self.device)
        rest = runner.TokenLogprobs(R * W, V, 0, 0, "f32", device=self.device)
        choose = [runner.BeamSelector(R, n, V, W, device=self.device) for n in (1, W)]
        _, lse, *_ = first.forward(logits)
        _, token, score = choose[0](logits.unflatten(0, (R, 1)),
                                   runner.scores_for_logits(None, lse)[:, None])
        found, parents = token[..., None], None
        at = (seq_offsets[1:] - seq_offsets[:-1])[:, None].expand(R, W).flatten()
        o = torch.empty((R, W, layer.HV, layer.dv), device=self.device)
        for t in range(steps - 1):
            x, h = self._enter(token.flatten().long())
            for i, layer in enumerate(self.layers):
                step = layer.beam_step_inputs(x.unflatten(0, (R, W)), parents,
                                              at + t if layer.rotary_dim else None, kept[i])
                decoders[i].step(t, step, o, fused=True)
                x, h = self._between(i, layer.beam_outputs(o, kept[i]).flatten(0, 1), h)
            logits = (x @ self.head).float()
            _, lse, *_ = rest.forward(logits)
            parents, token, score = choose[1](
                logits.unflatten(0, (R, W)),
                runner.scores_for_logits(score, lse.unflatten(0, (R, W))))
            parents = parents.clone()  # (the selection's own; the next step reads them)
            found = torch.cat([found.gather(1, parents.long()[..., None].expand_as(found)),
                               token[..., None]], 2)
        for d in decoders:
            d.close()
        return found, score.clone()


def train(model: Recommender, tokens, targets, seq_offsets, steps: int = 30, lr: float = 3e-3):
    """Adam on the loss; the losses."""
    masters = [w.detach().float().requires_grad_() for w in model.weights()]
    opt, losses = torch.optim.Adam(masters, lr=lr), []
    for _ in range(steps):
        for w in model.weights():
            w.grad = None
        loss = model.loss(tokens, targets, seq_offsets)
        loss.backward()
        for m, w in zip(masters, model.weights()):
            m.grad = w.grad.float()
        opt.step()
        with torch.no_grad():
            for m, w in zip(masters, model.weights()):
                w.copy_(m)
        losses.append(float(loss.detach()))
    return losses


def main():
    device = "cuda:0"
    model = Recommender(256, 256, 2, 2, 4, 64, device=device)
    lengths = [120, 9, 64]
    off = torch.tensor([0, 120, 129, 193], dtype=torch.int32, device=device)
    g = torch.Generator(device=device).manual_seed(1)
    start = torch.randint(0, 256, (3,), generator=g, device=device)
    # sequences that count up by 3 from a start of their own
    tokens = torch.cat([(s + 3 * torch.arange(n, device=device)) % 256
                        for s, n in zip(start, lengths)])
    targets = ((tokens + 3) % 256).int()
    losses = train(model, tokens, targets, off)
    print(f"training: loss {losses[0]:.4f} -> {losses[-1]:.4f}")
    found, score = model.search(tokens, off, 8, 3)
    print(f"search: {found.shape[1]} beams per request, best {found[:, 0].tolist()} with log "
          f"probabilities {[round(v, 3) for v in score[:, 0].tolist()]}")


if __name__ == "__main__":
    main()
