"""A decode loop that stays on the device: from hidden states to accepted tokens, under a JSON grammar.

A step is five calls on one stream and no copy to the host: the grammar's masks from the states in device memory, logits from
hidden states with a 4-bit output projection under those masks (rows of the matrix that no request may take are not read), a
token a row under penalties, temperature, top-k, top-p and min-p, its acceptance, and the model.  The model is a stand-in with
random weights: the last token's embedding added to half of the last hidden state, normalised.

    python examples/decode.py [rows] [steps]
"""

from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2411_15100_amd as xgm  # noqa: E402
import synth_inputs as si  # noqa: E402
from paper_2411_15100_amd import workloads as wl  # noqa: E402

K, GROUP = 512, 64


class Decoder:
    def __init__(self, rows: int, steps: int, vocab_size: int = 4096, seed: int = 0):
        self.vocab = si.make_vocab("bpe", vocab_size, 0)
        self.cache = xgm.Cache(xgm.Grammar(si.JSON_GRAMMAR, "root"), wl.make_xgm_vocab(self.vocab))
        self.rows, self.V, stream = rows, vocab_size, wl.current_stream()
        self.states = xgm.DeviceBatch([xgm.Matcher(cache=self.cache) for _ in range(rows)], history=0, stream=stream)
        self.sampler = xgm.Sampler(rows, vocab_size, stream)

        g = torch.Generator(device="cuda").manual_seed(seed)
        dev = dict(generator=g, device="cuda")
        self.embedding = torch.randn((vocab_size, K), **dev)
        self.codes = torch.randint(0, 256, (vocab_size, K // 2), dtype=torch.uint8, **dev)
        self.scales = (0.02 * torch.rand((vocab_size, K // GROUP), **dev)).bfloat16()
        self.hidden = torch.randn((rows, K), **dev).bfloat16()
        self.uniform = torch.rand((steps, rows), dtype=torch.float64, **dev)

        def full(value, t=torch.float32):
            return torch.full((rows,), value, dtype=t, device="cuda")

        self.mask = torch.zeros((rows, xgm.bitmask_words(vocab_size)), dtype=torch.int32, device="cuda")
        self.logits = torch.empty((rows, vocab_size), dtype=torch.bfloat16, device="cuda")
        self.tokens = torch.zeros((rows, steps), dtype=torch.int32, device="cuda")      # the texts so far, and their lengths
        self.n_tokens = full(0, torch.int32)
        self.ended = full(False, torch.bool)
        self.stops = torch.zeros(vocab_size, dtype=torch.bool, device="cuda")
        self.stops[torch.from_numpy(np.asarray(self.vocab.stop_ids, dtype=np.int64)).cuda()] = True
        self.ids, self.logprobs = full(-1, torch.int32), full(0.0)
        self.repetition, self.frequency = full(1.1), full(0.2)
        self.temperature, self.top_p, self.min_p = full(0.8), full(0.95), full(0.01)
        self.top_k = full(100, torch.int32)
        self.rules = xgm.LogitRules(d_bitmask=self.mask.data_ptr(), v_mask=vocab_size, d_tokens=self.tokens.data_ptr(), token_stride=steps,
                                    d_n_tokens=self.n_tokens.data_ptr(), d_repetition=self.repetition.data_ptr(),
                                    d_frequency=self.frequency.data_ptr())

    def step(self, k: int):
        stream, bf16 = wl.current_stream(), xgm.DTYPE_BF16
        self.states.fill_next_token_bitmask(self.mask.data_ptr(), stream)
        xgm.q4_logits(self.hidden.data_ptr(), bf16, self.rows, K, K, self.codes.data_ptr(), self.scales.data_ptr(), 0, self.V, GROUP,
                      self.logits.data_ptr(), bf16, self.V, self.mask.data_ptr(), stream)
        draw = xgm.DrawRules(d_temperature=self.temperature.data_ptr(), d_top_k=self.top_k.data_ptr(), d_top_p=self.top_p.data_ptr(),
                             d_min_p=self.min_p.data_ptr(), d_uniform=self.uniform[k].data_ptr())
        self.sampler.sample(self.logits.data_ptr(), bf16, self.rows, self.V, self.V, self.rules, draw, self.ids.data_ptr(),
                            self.logprobs.data_ptr(), stream)
        self.ids.masked_fill_(self.ended, -1)                           # a row whose text has ended stays
        self.states.accept_tokens(self.ids.data_ptr(), stream)
        drawn = self.ids >= 0
        at = self.n_tokens.long().clamp(max=self.tokens.shape[1] - 1)[:, None]
        self.tokens.scatter_(1, at, torch.where(drawn, self.ids, self.tokens.gather(1, at)[:, 0])[:, None])
        self.n_tokens += drawn
        self.ended |= self.stops[self.ids.clamp(min=0).long()] & drawn
        h = self.embedding[self.ids.clamp(min=0).long()] + 0.5 * self.hidden.float()
        self.hidden.copy_(h * torch.rsqrt((h * h).mean(1, keepdim=True)))

    def texts(self):
        """The token ids of every row (copied to the host)."""
        tokens, n = self.tokens.cpu().numpy(), self.n_tokens.cpu().numpy()
        return [tokens[b, :n[b]].tolist() for b in range(self.rows)]


def main(rows: int = 4, steps: int = 48):
    d = Decoder(rows, steps)
    for k in range(steps):
        d.step(k)
    words = d.vocab.tokens()
    for b, ids in enumerate(d.texts()):
        print(f"{b}: {len(ids)} tokens  {b''.join(words[t] for t in ids).decode('utf-8', 'replace')!r}")


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:]))
