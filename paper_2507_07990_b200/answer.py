"""From a video's merged tokens to answers: a small decoder that runs the merge and the cache operators
together, as a video LLM would.

    python -m paper_2507_07990_b200.answer          a synthetic video, three questions, random weights

``Answerer.watch`` merges a video and fills one cache per layer with its rows, rotated by the rows' position
ids.  ``Answerer.ask`` puts several questions to it at once: they share the video's full pages; their tokens go
through the layers one by one, collecting the attention that every slot receives; the video's rows that no
question token looks at are evicted; the answers are read from what is left.  ``Answerer.ask_together`` reads whole questions,
of any lengths, in one go and keeps nothing of the video but the one cache that they share.  Weights are random: this shows
the path, not a model.  Rotation, cache entry with its norms of queries and keys, cached attention and eviction are the library's everywhere; in
``ask_together`` the norms between blocks are too, in one pass with the residual stream and, with ``Config.int8``, the rounding to 8 bits (``watch`` and ``ask``
take them from torch).  Projections are plain matrix products, or with ``Config.int8`` the library's in 8 bits, and the video's own layers (a prefill) use torch's
attention.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Iterable, List, Optional, Sequence

import torch
import torch.nn.functional as F

from . import binding, cache, layer as decoder, prefix


@dataclass
class Config:
    width: int = 256             # channels of a token
    layers: int = 2
    q_heads: int = 7
    kv_heads: int = 1
    dim: int = 64                # channels of a head
    hidden: int = 512
    vocab: int = 512
    page: int = 16
    theta: float = 1e6
    dtype: torch.dtype = torch.bfloat16
    int8: bool = False           # the layers' projections in 8 bits (their weights stay in `dtype` beside it, to compare with)


def _rms(x: torch.Tensor, w: torch.Tensor) -> torch.Tensor:
    y = x.float()
    return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * w).to(x.dtype)


def _check_status(name: str, statuses: Iterable[torch.Tensor]) -> None:
    """Raises what any call has written into its status (waits for the calls)."""
    bits = 0
    for word in torch.cat(list(statuses)).tolist():
        bits |= word
    binding._check(binding.load_library().sttm_status_from_bits(bits), name)


class Answerer:
    def __init__(self, cfg: Config, seed: int = 0, device="cuda"):
        self.cfg, self.device = cfg, torch.device(device)
        gen = torch.Generator(device=device).manual_seed(seed)
        c, heads = cfg, cfg.q_heads + 2 * cfg.kv_heads
        mat = lambda a, b: (torch.randn((a, b), generator=gen, device=device) * a ** -0.5).to(c.dtype)
        one = lambda n: 1 + 0.1 * torch.randn(n, generator=gen, device=device)
        self.layers = [dict(norm1=one(c.width), qkv=mat(c.width, heads * c.dim), q_norm=one(c.dim), k_norm=one(c.dim),
                            out=mat(c.q_heads * c.dim, c.width), norm2=one(c.width), up=mat(c.width, 2 * c.hidden), down=mat(c.hidden, c.width))
                       for _ in range(c.layers)]
        if c.int8:                                               # every projection's output channels
            for layer in self.layers:
                layer["rows"] = {name: decoder.sttm_quantize_rows(layer[name].t().contiguous()) for name in ("qkv", "out", "up", "down")}
        self.norm, self.embed, self.head = one(c.width), mat(c.vocab, c.width) * c.vocab ** 0.5, mat(c.width, c.vocab)
        self.pools: List[cache.PagedCache] = []                  # one per layer, once a video has been watched
        self.reported: List[torch.Tensor] = []                   # statuses of the 8-bit products of the call under way
        half = c.dim // 2
        self.rotary = cache.Rotary((c.theta ** (-torch.arange(half, dtype=torch.float64) / half)).float().to(device))

    def _project(self, layer: dict, name: str, x: torch.Tensor, gated: bool = False) -> torch.Tensor:
        """``x`` (gated: ``silu(a) * b`` of rows ``[a | b]``) times one of a layer's weights."""
        if self.cfg.int8:
            rows = layer["rows"][name]
            quantize = decoder.QuantizePlan(rows.q.shape[1], self.cfg.dtype, x.shape[0], gated, self.device)
            product = decoder.MatmulPlan(rows, self.cfg.dtype, x.shape[0])
            self.reported += [quantize.status, product.status]
            return product.run(quantize.run(x))
        if gated:
            gate, up = x.chunk(2, -1)
            x = F.silu(gate) * up
        return x @ layer[name]

    def _heads(self, y: torch.Tensor):
        c = self.cfg
        y = y.view(-1, c.q_heads + 2 * c.kv_heads, c.dim)
        return y[:, :c.q_heads], y[:, c.q_heads:c.q_heads + c.kv_heads], y[:, c.q_heads + c.kv_heads:]

    def _qkv(self, layer: dict, x: torch.Tensor):
        return self._heads(self._project(layer, "qkv", _rms(x, layer["norm1"])))

    def _rest(self, layer: dict, x: torch.Tensor, attended: torch.Tensor) -> torch.Tensor:
        x = x + self._project(layer, "out", attended.reshape(x.shape[0], -1))
        return x + self._project(layer, "down", self._project(layer, "up", _rms(x, layer["norm2"])), gated=True)

    def _append_plan(self, pool: cache.PagedCache, layer: dict) -> cache.AppendPlan:
        return cache.AppendPlan(pool, self.cfg.q_heads, self.rotary, q_norm=layer["q_norm"], k_norm=layer["k_norm"])

    def watch(self, video: torch.Tensor, tau_s: float, tau_t: float) -> int:
        """Merges one video ``[T, H, W, width]`` and caches its rows; returns their number.  What a call reports in its status
        is raised (SttmError), here and in ``ask``."""
        c = self.cfg
        T, H, W, _ = video.shape
        merged = binding.sttm_merge_ex(video, tau_s, tau_t, out_dtype=c.dtype)
        n = self.rows = int(merged.out_count[0])
        self.next_position = T * H * W
        self.shared = n // c.page                                # full pages
        x, positions = merged.out_feats[:n], merged.out_pos[:n]
        offsets = torch.tensor([0, n], device=self.device)
        self.pools, pools = [], []
        statuses, self.reported = [merged.device_status], []
        for layer in self.layers:
            pool = cache.empty_cache(1, n, c.kv_heads, c.dim, c.page, c.dtype, self.device)
            q, k, v = self._qkv(layer, x)
            entered = self._append_plan(pool, layer).run(q, k, v, offsets, None, positions)
            q = entered.q
            pools.append(pool)
            statuses.append(entered.status)
            # the video's own attention, from the cache's keys and values in slot order
            ks, vs = (t.transpose(1, 2).reshape(-1, c.kv_heads, c.dim)[:n].transpose(0, 1).unsqueeze(0) for t in (pool.k, pool.v))
            att = F.scaled_dot_product_attention(q.transpose(0, 1).unsqueeze(0), ks, vs, is_causal=True, enable_gqa=True)
            x = self._rest(layer, x, att[0].transpose(0, 1))
        _check_status("Answerer.watch", statuses + self.reported)
        self.pools = pools
        return n

    def _question_caches(self, questions: int, more: int) -> List[cache.PagedCache]:
        """Per layer: the video's full pages shared by all questions, own pages for its last rows and ``more`` tokens."""
        c, full, n = self.cfg, self.shared, self.rows
        own = -(-(n - full * c.page + more) // c.page)
        out = []
        for pool in self.pools:
            k, v = (torch.cat([t, t.new_empty((questions * own, *t.shape[1:]))]) for t in (pool.k, pool.v))
            mine = pool.pages + torch.arange(questions * own, device=self.device, dtype=torch.int32).view(questions, own)
            if full < pool.pages:                                # the last page is not full: every question gets a copy
                for t in (k, v):
                    t[mine[:, 0].long()] = t[full].clone()
            table = torch.cat([pool.table[:, :full].expand(questions, full), mine], 1).contiguous()
            out.append(cache.PagedCache(k, v, table))
        return out

    def _step(self, tokens: torch.Tensor, pos: int, state: dict) -> torch.Tensor:
        """One token per question through all layers; returns logits."""
        questions = tokens.shape[0]
        positions = torch.full((questions,), pos, dtype=torch.int32, device=self.device)
        x = self.embed[tokens]
        lengths = state["lengths"]
        for i, layer in enumerate(self.layers):
            q, k, v = self._qkv(layer, x)
            a = state["append"][i].run(q, k, v, state["offsets"], lengths, positions)
            att = state["attend"][i].run(a.q, a.new_lengths, scores=None if state["scores"] is None else state["scores"][i])
            x = self._rest(layer, x, att.out)
            state["lengths"] = a.new_lengths
        return (_rms(x, self.norm) @ self.head).float()

    def _state(self, pools: List[cache.PagedCache], lengths: torch.Tensor, scored: bool) -> dict:
        questions, slots = pools[0].seqs, pools[0].width * pools[0].page
        return dict(lengths=lengths, offsets=torch.arange(questions + 1, device=self.device),
                    append=[self._append_plan(p, layer) for p, layer in zip(pools, self.layers)],
                    attend=[cache.AttendPlan(p, self.cfg.q_heads) for p in pools],
                    scores=[torch.zeros((questions, p.heads, slots), device=self.device) for p in pools] if scored else None)

    def ask_together(self, questions: Sequence[torch.Tensor], answer_tokens: int) -> torch.Tensor:
        """``questions``: token ids, one tensor a question, of any lengths.  Every question sees the video's cache, which is read once for all
        of them, and its own tokens; the questions are read in one go.  Returns greedy answers ``[questions, answer_tokens]``."""
        lengths = [int(q.numel()) for q in questions]
        if not lengths or min(lengths) < 1 or any(q.dim() != 1 for q in questions) or answer_tokens < 1:
            raise ValueError("questions must be one-dimensional, of at least one token each, answer_tokens at least 1")
        if not self.pools:
            raise ValueError("no video has been watched")
        c, n = self.cfg, len(lengths)
        own = [cache.empty_cache(n, max(lengths) + answer_tokens, c.kv_heads, c.dim, c.page, c.dtype, self.device) for _ in self.pools]
        state = Together(self, own, sum(lengths))
        ends = torch.tensor(lengths, device=self.device).cumsum(0)
        offsets = torch.cat([ends.new_zeros(1), ends])
        positions = torch.cat([self.next_position + torch.arange(m, device=self.device, dtype=torch.int32) for m in lengths])
        last = state.step(torch.cat(list(questions)), offsets, positions)[ends - 1]
        offsets, positions = torch.arange(n + 1, device=self.device), positions[ends - 1]
        answers = []
        for _ in range(answer_tokens):
            logits = (last @ self.head).float()
            tokens = logits.argmax(-1)
            answers.append(tokens)
            if len(answers) < answer_tokens:
                positions = positions + 1
                last = state.step(tokens, offsets, positions)
        self.logits = logits
        _check_status("Answerer.ask_together", state.statuses())
        return torch.stack(answers, 1)

    @staticmethod
    def _statuses(state: dict) -> List[torch.Tensor]:
        return [plan.status for plan in state["append"] + state["attend"]]

    def ask(self, questions: torch.Tensor, answer_tokens: int, keep: Optional[int] = None) -> torch.Tensor:
        """``questions`` ``[questions, length]`` token ids; ``keep``: slots that every cache keeps when the questions have
        been read (None: all).  Returns greedy answers ``[questions, answer_tokens]``."""
        if questions.dim() != 2 or 0 in questions.shape or answer_tokens < 1 or (keep is not None and keep < 1):
            raise ValueError("questions must be [questions, length] of at least one token each, answer_tokens and keep at least 1")
        if not self.pools:
            raise ValueError("no video has been watched")
        n, length = questions.shape
        pools = self._question_caches(n, length + answer_tokens)
        lengths = torch.full((n,), self.rows, dtype=torch.int32, device=self.device)
        state = self._state(pools, lengths, keep is not None)
        statuses, self.reported = self._statuses(state), []
        pos = self.next_position
        for i in range(length):
            logits = self._step(questions[:, i], pos, state)
            pos += 1
        if keep is not None:
            c = self.cfg
            kept = min(keep, self.rows + length)
            thin = [cache.empty_cache(n, kept + answer_tokens, c.kv_heads, c.dim, c.page, c.dtype, self.device) for _ in pools]
            want = torch.full((n,), kept, dtype=torch.int32, device=self.device)
            for p, t, scores in zip(pools, thin, state["scores"]):
                # the question itself stays, and the first rows, which draw attention whatever they show
                left = cache.sttm_cache_evict(p, t, state["lengths"], want, scores, kept, first=4, last=length)
                statuses.append(left.status)
            state = self._state(thin, left.new_lengths, False)
            statuses += self._statuses(state)
        answers = []
        for _ in range(answer_tokens):
            tokens = logits.argmax(-1)
            answers.append(tokens)
            if len(answers) < answer_tokens:
                logits = self._step(tokens, pos, state)
                pos += 1
        self.logits = logits
        _check_status("Answerer.ask", statuses + self.reported)
        return torch.stack(answers, 1)


class Together:
    """Several questions through the layers at once: plans of the library's calls for up to ``max_rows`` new tokens a step."""

    def __init__(self, model: Answerer, own: List[cache.PagedCache], max_rows: int):
        c = model.cfg
        self.model, self.lengths, self.seen = model, None, torch.tensor([model.rows], dtype=torch.int32, device=model.device)
        self.append = [model._append_plan(pool, layer) for pool, layer in zip(own, model.layers)]
        # (as close as token by token)
        self.attend = [prefix.PrefixPlan(video, c.q_heads, mine, max_rows, max_prefix=model.rows, fine=True) for video, mine in zip(model.pools, own)]
        # before a layer's attention and its products, and before the head, which is not in 8 bits
        norm = lambda w, int8: decoder.NormPlan(c.width, c.dtype, max_rows, pre_norm=w, eps=1e-6, quantize=int8, device=model.device)  # noqa: E731
        self.norms = [norm(layer[n], c.int8) for layer in model.layers for n in ("norm1", "norm2")] + [norm(model.norm, False)]
        self.rows, self.products = [], []
        if c.int8:
            quantize = lambda dim, gated: decoder.QuantizePlan(dim, c.dtype, max_rows, gated, model.device)  # noqa: E731
            self.rows = [(quantize(c.q_heads * c.dim, False), quantize(c.hidden, True)) for _ in model.layers]
            self.products = [{n: decoder.MatmulPlan(layer["rows"][n], c.dtype, max_rows) for n in layer["rows"]} for layer in model.layers]

    def statuses(self) -> List[torch.Tensor]:
        plans = self.append + self.attend + self.norms + [p for pair in self.rows for p in pair] + [p for layer in self.products for p in layer.values()]
        return [p.status for p in plans]

    def _project(self, i: int, name: str, x, gated: bool = False) -> torch.Tensor:
        """``x``: rows, or for what a norm leaves its output."""
        normed = isinstance(x, decoder.NormOutput)
        if not self.model.cfg.int8:
            return self.model._project(self.model.layers[i], name, x.out if normed else x, gated)
        return self.products[i][name].run(x.rows if normed else self.rows[i][1 if gated else 0].run(x))

    def step(self, tokens: torch.Tensor, offsets: torch.Tensor, positions: torch.Tensor) -> torch.Tensor:
        """New tokens of all questions (question b's are ``offsets[b]`` ... ``offsets[b + 1] - 1``) through all layers; what comes before the head."""
        model, lengths = self.model, self.lengths
        stream = self.norms[0].run(model.embed[tokens])
        for i in range(len(model.layers)):
            q, k, v = model._heads(self._project(i, "qkv", stream))
            entered = self.append[i].run(q, k, v, offsets, lengths, positions)
            attended = self.attend[i].run(entered.q, offsets, self.seen, entered.new_lengths)
            out = self._project(i, "out", attended.out.reshape(len(tokens), -1))
            stream = self.norms[2 * i + 1].run(out, stream.sum)
            stream = self.norms[2 * i + 2].run(self._project(i, "down", self._project(i, "up", stream), gated=True), stream.sum)
            self.lengths = entered.new_lengths
        return stream.out


def main() -> None:
    from . import inputs
    cfg = Config()
    spec = inputs.VideoSpec(T=16, H=13, W=13, D=cfg.width, dtype="bf16", p_static=0.8, sigma=0.05, seed=7)
    bits = inputs.make_video(spec)
    video = torch.from_numpy(bits.view("int16")).view(torch.bfloat16).cuda()
    model = Answerer(cfg)
    rows = model.watch(video, 0.97, 0.9)
    questions = torch.randint(0, cfg.vocab, (3, 12), generator=torch.Generator().manual_seed(1)).cuda()
    whole = model.ask(questions, 8)
    thin = model.ask(questions, 8, keep=rows // 2)
    print("%d tokens -> %d rows in the cache; answers from all of them %s, from half of them %s"
          % (spec.tokens, rows, whole.tolist(), thin.tolist()))
    lines = [q[:12 - 3 * i] for i, q in enumerate(questions)]
    together = model.ask_together(lines, 8)
    cfg.int8 = True
    model = Answerer(cfg)
    model.watch(video, 0.97, 0.9)
    print("questions of %s tokens read at once: answers %s, with projections in 8 bits %s"
          % ([len(q) for q in lines], together.tolist(), model.ask_together(lines, 8).tolist()))


if __name__ == "__main__":
    main()
