"""Generation with several continuations (beams) per request.

``BeamDecoder`` takes a prefilled ``RequestCache`` and goes on with K beams of
each of its B requests. Two kinds of layers can take part:

* attention layers over the cache's compressed segments. A request's prompt is
  the same for all of its beams, so its segments are copied to them once
  (uc_reorder from 1 to K); only the generated tokens follow their beams later.
* linear layers, whose past is a state of constant size per KV head
  (uc_linear_attend): the prompt goes through ``linear_prompt`` in chunks, then
  a step at a time; the states follow their beams.

A step is ``attend`` and ``linear`` for the layers, then ``advance``: the best
continuations of every request over its beams and the vocabulary
(uc_beam_select), and one uc_reorder of everything that follows the beams into
the other of two sets of segments and states. Nothing waits for the device
before ``sequences``.
"""
from __future__ import annotations

from typing import List, Optional, Sequence, Tuple

import torch

from . import api
from ._lib import KIND_EVICT, KIND_FULL
from .engine import RequestCache

MAX_SEQUENCES = 64  # UC_MAX_BATCH


class BeamDecoder:
    """K beams of every request of ``cache``, up to ``max_new`` tokens.

    ``linear_decay``: for each linear layer, its KV heads' log decay. eos: the
    end token; a beam that chose it is finished and keeps its score (-1: none).
    Sequence b * K + i of every per-beam tensor is beam i of request b."""

    def __init__(self, cache: RequestCache, n_beams: int, max_new: int,
                 linear_decay: Sequence[Sequence[float]] = (), eos: int = -1):
        if n_beams < 1 or cache.B * n_beams > MAX_SEQUENCES:
            raise ValueError(f"BeamDecoder: {cache.B} requests x {n_beams} beams, at most {MAX_SEQUENCES} sequences")
        if max_new < 1:
            raise ValueError("BeamDecoder: max_new must be at least 1")
        if cache.stream_evict:
            raise ValueError("BeamDecoder: a cache with streaming eviction keeps per-step scores of its own batch")
        self.cache, self.K, self.max_new, self.eos = cache, n_beams, max_new, eos
        self.B, self.S = cache.B, cache.B * n_beams
        self.device = cache.device
        self.decay = [[float(x) for x in d] for d in linear_decay]
        self.prompt_states: List[Optional[torch.Tensor]] = [None] * len(self.decay)
        self.ws = cache.ws
        self._prompt: List[List[api.Segment]] = []
        self._gen: List[List[api.Segment]] = [[], []]
        self._state: List[List[torch.Tensor]] = [[], []]
        self._at = 0               # which of the two sets holds the beams
        self._stepped = [0] * len(self.decay)  # tokens that each linear layer has taken behind the prompt
        self._chosen: List[Tuple[torch.Tensor, torch.Tensor]] = []
        self.n_pos = 0
        self.scores: Optional[torch.Tensor] = None
        self.finished: Optional[torch.Tensor] = None

    # ---------------------------------------------------------------- prompt
    def linear_prompt(self, layer: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                      lengths: Optional[Sequence[int]] = None) -> torch.Tensor:
        """The prompt through linear layer ``layer``: q [B, Hq, T, 128], k, v
        [B, Hkv, T, 128] -> o like q. May be called for one piece of the prompt
        after another."""
        state = self.prompt_states[layer]
        out, self.prompt_states[layer] = api.linear_attend(q, k, v, self.decay[layer], state=state, out_state=state,
                                                           lengths=lengths, ws=self.ws)
        return out

    def start(self) -> None:
        """The beams start from the prompt: every cache and state of a request
        is copied to its K beams. Only beam 0 is alive at first, the others
        would repeat it."""
        if any(not segs for segs in self.cache.layers):
            raise RuntimeError("BeamDecoder.start: prefill the cache first")
        if any(s is None for s in self.prompt_states):
            raise RuntimeError("BeamDecoder.start: a linear layer has not seen the prompt")
        c, K, dev = self.cache, self.K, self.device
        own = set(id(g) for g in c.gen if g is not None and c.gen_capacity)
        self._prompt, pairs = [], []
        for segs in c.layers:
            row = []
            for s in segs:
                if id(s) in own:
                    if max(s.n_kept()) > 0:
                        raise RuntimeError("BeamDecoder.start: the cache holds generated tokens already")
                    continue
                row.append(self._beam_segment(s))
                pairs.append((s, row[-1]))
            self._prompt.append(row)
        self._gen = [[api.Segment(KIND_EVICT, 16, self.S, c.hkv, 0, self.max_new, dev) for _ in c.layers]
                     for _ in range(2)]
        self._state = [[torch.empty((self.S,) + s.shape[1:], dtype=torch.float32, device=dev)
                        for s in self.prompt_states] for _ in range(2)]
        self._at = 0
        pairs += list(zip(self.prompt_states, self._state[0]))
        if pairs:
            api.reorder(pairs, torch.zeros((self.B, K), dtype=torch.int32, device=dev), ws=self.ws)
        self.scores = torch.full((self.B, K), float("-inf"), dtype=torch.float32, device=dev)
        self.scores[:, 0] = 0.0
        self.finished = torch.zeros((self.B, K), dtype=torch.bool, device=dev)
        self._chosen = []
        self._stepped = [0] * len(self.decay)
        self.n_pos = c.n_pos

    def _beam_segment(self, s: api.Segment) -> api.Segment:
        if s.kind == KIND_FULL:
            k = torch.empty((self.S, s.n_kv_heads, s.c.n_src, api.HEAD_DIM), dtype=torch.bfloat16, device=self.device)
            return api.Segment.view(k, torch.empty_like(k), 0, s.c.n_src)
        return api.Segment(s.kind, s.bits, self.S, s.n_kv_heads, s.c.n_src, s.cap, self.device)

    # ------------------------------------------------------------------ step
    def attend(self, layer: int, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor) -> torch.Tensor:
        """Attention layer ``layer`` for the beams' newest tokens: q [S, Hq, 1,
        128], k_new, v_new [S, Hkv, 128] -> o like q."""
        gen = self._gen[self._at][layer]
        if gen.n_kept()[0] != len(self._chosen) - 1:
            raise RuntimeError("BeamDecoder.attend: a layer attends once between two selections, the first behind one")
        api.append(gen, k_new, v_new, self.n_pos, ws=self.ws)
        return api.attend(q, self._prompt[layer] + [gen], want_lse=False, want_mass=False, ws=self.ws)[0]

    def linear(self, layer: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor) -> torch.Tensor:
        """Linear layer ``layer`` for the beams' newest tokens: q [S, Hq, 1,
        128], k, v [S, Hkv, 1, 128] -> o like q; the states advance in place."""
        if self._stepped[layer] != len(self._chosen) - 1:
            raise RuntimeError("BeamDecoder.linear: a layer steps once between two selections, the first behind one")
        self._stepped[layer] += 1
        state = self._state[self._at][layer]
        return api.linear_attend(q, k, v, self.decay[layer], state=state, out_state=state, ws=self.ws)[0]

    def advance(self, logits: torch.Tensor) -> torch.Tensor:
        """The next tokens from the beams' logits [B, K, V] (of the prompt's
        last token in every beam for the first call): selects the best K
        continuations of each request and moves caches and states to them.
        Returns the tokens, int32 [B, K]."""
        if len(self._chosen) >= self.max_new:
            raise RuntimeError(f"BeamDecoder.advance: max_new = {self.max_new} tokens are chosen")
        scores, parent, token, done = api.beam_select(
            logits, self.scores, self.K, finished=self.finished if self.eos >= 0 else None, eos=self.eos, ws=self.ws)
        if self._chosen:
            here, there = self._at, 1 - self._at
            pairs = list(zip(self._gen[here], self._gen[there])) + list(zip(self._state[here], self._state[there]))
            if pairs:
                api.reorder(pairs, parent, ws=self.ws)
            self._at = there
            self.n_pos += 1
        # (before the first selection every beam holds the prompt and nothing else)
        self.scores, self.finished = scores, done
        self._chosen.append((parent, token))
        return token

    # ---------------------------------------------------------------- result
    def sequences(self) -> Tuple[torch.Tensor, torch.Tensor]:
        """(tokens int64 [B, K, steps], scores fp32 [B, K]), best first, read
        back along the parents."""
        at = torch.arange(self.K, device=self.device).expand(self.B, self.K)
        out = []
        for parent, token in reversed(self._chosen):
            out.append(torch.gather(token.long(), 1, at))
            at = torch.gather(parent.long(), 1, at)
        return torch.stack(out[::-1], dim=2), self.scores
