"""A pre-norm transformer that reads and writes token by token: linear layers with 4-bit weights, keys and values in a paged 8-bit cache.

    python -m paper_2401_10652_amd.decode [--config C2] [--batch 8] [--prompt 1024] [--stretch 512] [--steps 32] [--window 512 --sinks 4] [--beams 4 --vocab 32768]

reads a prompt for each sequence of a batch in stretches, then single tokens (each step's output is the next one's input: there is no
vocabulary here, as in the framework's other workloads), and prints one JSON line with both rates.  With a window rows see the last tokens and the first few (sinks), and pages
that no row sees any more are used again.  With beams, a beam search from each prompt over a random vocabulary is timed too.
"""
from __future__ import annotations

import argparse
import dataclasses
import json
import time

from . import binding as B
from . import inputs as I


def quantize_w4(w, group, dtype):
    """Weights [n, k] as (codes, two to a byte, [n, bytes]; scale; zero [n, ceil(k / group)] of type `dtype`): a group's numbers and 0 are spread over the codes 0..15."""
    import torch
    n, k = w.shape
    groups = -(-k // group)
    w = torch.nn.functional.pad(w.float(), (0, groups * group - k)).view(n, groups, group)
    low, high = w.amin(2).clamp(max=0), w.amax(2).clamp(min=0)
    scale = ((high - low) / 15).clamp(min=1e-30).to(dtype)
    zero = (-low / scale.float()).round().clamp(0, 15)
    codes = (w / scale.float()[..., None] + zero[..., None]).round().clamp(0, 15).to(torch.uint8).view(n, -1)[:, :k]
    codes = torch.nn.functional.pad(codes, (0, -k % 32))                # rows begin at multiples of 16 bytes
    return codes[:, 0::2] | codes[:, 1::2] << 4, scale, zero.to(dtype)


class Decoder:
    """The layers of `cfg` (weights as transformer_inputs makes them; w_qkv's rows are the queries' heads, then the keys' and the
    values', which may be fewer) and the cache of `sequences` sequences of up to `max_tokens` tokens.  `cfg` is causal: a token sees those before it and itself; and its
    queries and keys are rotated by their places, which no plan of the framework does, so that a plan's rows are not these.

    window, sinks: a token sees the last `window` ones, itself among them, and the first `sinks` ones.  pages: the cache has so many, which sequences take as they grow, give
    up as their windows leave them, and share when one goes on as several (fork); without it, and without a window, each sequence has its own, enough for max_tokens.

    `lengths`, the sequences' numbers of tokens, may be set back, whole or one of it, between calls: a sequence then goes on behind as many of its tokens; behind a fork in pages of its own, so that
    the others keep theirs, and behind a window only where what its next row sees is held still: each call gives up pages that are wholly before the first row's window, the sinks' apart."""

    window, sinks, shares = None, 0, False

    def __init__(self, cfg, layers, sequences, max_tokens, page=64, group=64, base=10000.0, window=None, sinks=0, pages=None):
        import torch
        if not cfg.causal:
            raise ValueError(f"{cfg.name} is not causal: its rows cannot be read a token at a time")
        if not (0 <= (window or 0) <= 1 << 30 and 0 <= sinks <= 1 << 30):
            raise ValueError(f"a window of {window} tokens, {sinks} sinks: 0 to 2^30 are wanted")
        self.cfg, self.group, self.max_tokens = cfg, group, max_tokens
        self.dtype = {"f32": torch.float32, "bf16": torch.bfloat16}[cfg.dtype]
        dev, d = "cuda", cfg.head_dim
        self.heads_kv = (layers[0]["w_qkv"].shape[0] // d - cfg.heads) // 2
        self.layers = []
        for w in layers:
            t = {n: torch.as_tensor(x, device=dev) for n, x in w.items()}
            self.layers.append({n: quantize_w4(x, group, self.dtype) if n.startswith("w_") else x.to(self.dtype) for n, x in t.items()})
        each = -(-max_tokens // page)
        self.window, self.sinks, self.page = window, sinks, page
        self.shares = pages is not None or window is not None
        if pages is None:
            pages = sequences * each
        if self.shares:
            self.table = torch.full((sequences, each), -1, dtype=torch.int32, device=dev)
            self.uses = torch.zeros(pages, dtype=torch.int32, device=dev)
            self.books = B.page_books(self.uses, self.table, page)
            self.next_table, self.next_uses = torch.empty_like(self.table), torch.empty_like(self.uses)      # after a fork
            self.next_books = B.page_books(self.next_uses, self.next_table, page)
            self.books_workspace = B.empty_workspace(B.ac_pages_workspace_bytes(self.books))
            self.missing = torch.zeros(1, dtype=torch.int32, device=dev)
            self.ends = [0] * sequences
            # what is asked of lengths that were set (others pay a comparison): the lengths as the calls left them; those at the last fork, whose whole pages others may have; those at the
            # begin of the last call, which tell what it gave up; and the tokens before which a call before that one may have given up pages, but for the sinks'
            self.known, self.forked, self.began, self.lost = ([0] * sequences for _ in range(4))
        else:
            self.table = torch.arange(pages, dtype=torch.int32, device=dev).view(sequences, each)
        codes = dict(dtype=torch.uint8, device=dev)
        self.caches = [B.kv_cache(torch.zeros((pages, self.heads_kv, page, d), **codes), torch.zeros((pages, self.heads_kv, page // 16, d, 16), **codes),
                                  torch.ones((pages, self.heads_kv, page // 16), device=dev), torch.ones((pages, self.heads_kv, page // 16), device=dev))
                       for _ in layers]
        self.all_caches, self.no_caches = B.kv_caches(self.caches), B.kv_caches([])
        angle = torch.arange(max_tokens, dtype=torch.float64)[:, None] * base ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))
        self.rotary = B.rotary(angle.cos().float().to(dev), angle.sin().float().to(dev))
        self.lengths = [0] * sequences
        self.workspace = B.empty_workspace(0)

    def _linear(self, w, name, x, out, **more):
        codes, scale, zero = w["w_" + name]
        B.ac_op_linear_w4(x, codes, scale, out, self.group, zero=zero, bias=w["b_" + name], **more)
        return out

    def forward(self, x, counts):
        """x [sum(counts), d_model]: the next counts[b] tokens of every sequence, one sequence after another -> the last layer's rows."""
        import torch
        cfg, n = self.cfg, sum(counts)
        if len(counts) != len(self.lengths) or min(counts) < 0 or x.shape != (n, cfg.d_model) or x.dtype is not self.dtype:
            raise ValueError(f"rows {tuple(x.shape)} of {x.dtype} for {counts} tokens of {len(self.lengths)} sequences of {cfg.d_model} x {self.dtype}")
        if n == 0:
            return x.clone()
        lengths = [a + b for a, b in zip(self.lengths, counts)]
        if max(lengths) > self.max_tokens:
            raise ValueError(f"{max(lengths)} tokens: the cache holds {self.max_tokens} of a sequence")
        was_set = self.shares and self._was_set(b for b, c in enumerate(counts) if c > 0)
        begin = [0]
        for c in counts:
            begin.append(begin[-1] + c)
        # one copy to the device for all
        seqs = len(lengths)
        where = begin + lengths
        if self.shares:
            where += self.lengths + [self.sinks] * seqs + [n - self.window + 1 if self.window is not None else 0 for n in self.lengths]
        where = torch.tensor(where, dtype=torch.int32).to("cuda")
        length = where[seqs + 1:2 * seqs + 1]
        if self.shares:
            before, drop_begin, drop_end = where[2 * seqs + 1:].view(3, seqs)
            B.ac_op_pages_update(self.books, self.books, self.books_workspace, (drop_begin, drop_end), (before, length), self.missing)
            self.ends = [max(e, -(-n // self.page)) for e, n in zip(self.ends, lengths)]
            self.began = list(self.lengths)
            self._enough(self.ends, self.lengths)
        rows = B.cache_rows(where[:seqs + 1], length, self.table, max(counts), max(lengths))
        need = self._workspace_bytes(n, rows)
        if need > self.workspace.numel():
            self.workspace = B.empty_workspace(need)
        x = self._run(x.clone(memory_format=torch.contiguous_format), rows, self.workspace)
        if self.shares:
            self._read(lengths, was_set, counts)
        self.lengths = lengths
        return x

    def _enough(self, ends, behind=None):
        """Raises where pages ran out in the last call.  ends: of each sequence, the places up to the last that may name a page (which a length that was set back does not tell);
        behind: the tokens that it had before, whose window has been left.  The device is asked only where there are fewer pages than such places."""
        most = sum(ends)
        if self.window is not None and behind is not None:
            sinks = -(-self.sinks // self.page)
            most = sum(min(e, sinks + e - max(0, n - self.window + 1) // self.page) for e, n in zip(ends, behind))
        if most > self.uses.shape[0]:
            missing = self.missing.item()
            if missing:
                raise RuntimeError(f"{missing} pages are missing: the cache has {self.uses.shape[0]}")

    def _sharing(self):
        if not self.shares:
            raise ValueError("sequences of this cache have their own pages: give it a number of `pages` to share")

    def _was_set(self, sequences):
        """Before these sequences read on, or are forked: whether lengths were set since the last call.  Refuses those that the sequences do not have (any more), and those from which a window
        reaches tokens whose pages have been given up; those that share the pages behind them go on in pages of their own."""
        if self.lengths == self.known:
            return False
        sequences = list(sequences)
        for b in sequences:
            if not 0 <= self.lengths[b] <= self.known[b]:
                raise ValueError(f"sequence {b} has {self.known[b]} tokens: it cannot go on behind {self.lengths[b]}")
        if self.window is not None:
            self.lost = [max(e, (n - self.window + 1) // self.page * self.page) for e, n in zip(self.lost, self.began)]
            sinks = -(-self.sinks // self.page) * self.page
            for b in sequences:
                n = self.lengths[b]
                if max(n - self.window + 1, sinks) < min(n, self.lost[b]):
                    raise ValueError(f"sequence {b} cannot go on behind {n} tokens: of its window of {self.window} those before {self.lost[b]} are gone")
        self._part(sequences)
        return True

    def _read(self, lengths, was_set, counts):
        """Notes that sequences have read so many tokens and are `lengths` long now.  (Tokens that were given up and are read again are there; sequences that read none stay as they were set.)"""
        if was_set:
            self.lost = [min(e, n) if c > 0 else e for e, n, c in zip(self.lost, self.lengths, counts)]
            self.known = [n if c > 0 else k for k, n, c in zip(self.known, lengths, counts)]
        else:
            self.known = list(lengths)

    def _part(self, sequences):
        """Of these sequences, those that were set back into what they have in common with others go on in pages of their own: a copy of the page that they write next, as far as they have
        it, and none behind it.  (The device is asked: where nobody else has the pages any more they stay.)"""
        import torch
        for b in sequences:
            n, page = self.lengths[b], self.page
            place, rest = divmod(n, page)
            if place >= self.forked[b] // page:
                continue
            row = self.table[b, place:]
            others = ((row >= 0) & (self.uses[row.clamp(min=0).long()] > 1)).nonzero().view(-1).tolist()
            if others:
                first, copies = place + others[0], others[0] == 0 and rest > 0
                drop, take, tokens = [0] * (2 * len(self.lengths)), [0] * (2 * len(self.lengths)), [rest]
                drop[2 * b], drop[2 * b + 1] = first * page, (1 << 31) - 1
                if copies:
                    take[2 * b], take[2 * b + 1] = place * page, n
                at = torch.tensor(drop[0::2] + drop[1::2] + take[0::2] + take[1::2] + tokens, dtype=torch.int32).to("cuda")
                ranges = at[:-1].view(4, -1)
                B.ac_op_pages_update(self.books, self.next_books, self.books_workspace, (ranges[0], ranges[1]), (ranges[2], ranges[3]), self.missing)
                if copies:
                    missing = self.missing.item()
                    if missing:
                        raise RuntimeError(f"{missing} pages are missing: the cache has {self.uses.shape[0]}")
                    B.ac_op_cache_copy_pages(self.all_caches, self.table[b, place:place + 1], self.next_table[b, place:place + 1], at[-1:])
                self.table.copy_(self.next_table)
                self.uses.copy_(self.next_uses)
                self.ends[b] = max(first, place + copies)
                self.known[b], self.began[b], self.lost[b] = n, min(n, self.began[b]), min(n, self.lost[b])        # (what lay behind is not its own any more, also where the call fails)
            self.forked[b] = n

    def release(self, sequences):
        """The sequences have no tokens any more; their pages are free, but for those that others share."""
        import torch
        self._sharing()
        n, gone = len(self.lengths), set(sequences)
        if not gone <= set(range(n)):
            raise ValueError(f"sequences {sorted(gone)} of {n}")
        ends = torch.tensor([0] * n + [(1 << 31) - 1 if b in gone else 0 for b in range(n)], dtype=torch.int32).to("cuda").view(2, n)
        B.ac_op_pages_update(self.books, self.books, self.books_workspace, drop=(ends[0], ends[1]))
        for b in gone:
            self.lengths[b] = self.ends[b] = self.known[b] = self.forked[b] = self.began[b] = self.lost[b] = 0

    def fork(self, parents, lengths=None):
        """Sequence j goes on as sequence parents[j] (or, -1, has no tokens); where pages run out all stay as they are.  parents may be on the device (int32); the caller then says the
        lengths: each its parent's, of one without a parent any."""
        import torch
        self._sharing()
        n = len(self.lengths)
        if lengths is None or not (torch.is_tensor(parents) and parents.is_cuda):
            parents = [int(p) for p in parents]
            if len(parents) != n or not all(-1 <= p < n for p in parents):
                raise ValueError(f"parents {parents} of {n} sequences")
            of = [self.lengths[p] if p >= 0 else 0 for p in parents]
            if lengths is not None and (len(lengths) != n or any(p >= 0 and t != of[j] for j, (p, t) in enumerate(zip(parents, lengths)))):
                raise ValueError(f"lengths {list(lengths)} where the parents' are {of}")
            lengths = of if lengths is None else lengths
            ends = [self.ends[p] if p >= 0 else 0 for p in parents]
        else:
            ends = [max(self.ends)] * n
        if len(lengths) != n:
            raise ValueError(f"{len(lengths)} lengths of {n} sequences")
        was_set = self._was_set(range(n) if torch.is_tensor(parents) else sorted({p for p in parents if p >= 0}))
        began, lost = self.began, self.lost
        if not torch.is_tensor(parents):
            began, lost = ([of[p] if p >= 0 else 0 for p in parents] for of in (began, lost))
        elif self.window is not None:                                   # (the most of all that are as long as the parent)
            began, lost = ([of.get(t, 0) for t in lengths] for of in (dict(sorted(zip(self.lengths, a))) for a in (began, lost)))
        if was_set:
            began, lost = ([min(e, t) for e, t in zip(a, lengths)] for a in (began, lost))
        if not torch.is_tensor(parents):
            parents = torch.tensor(parents, dtype=torch.int32).to("cuda")
        now = torch.tensor(self.lengths, dtype=torch.int32).to("cuda")
        to = (self.books, self.next_books, parents, now, torch.empty_like(now), self.books_workspace, self.missing)
        if sum(ends) > self.uses.shape[0]:                              # the books alone first: copies go into pages that a sequence may have still, if this fails
            B.ac_op_cache_fork(self.no_caches, *to)
            self._enough(ends)
        B.ac_op_cache_fork(self.all_caches, *to)
        # (the graph of a step knows the table by its address)
        self.table.copy_(self.next_table)
        self.uses.copy_(self.next_uses)
        self.lengths, self.ends, self.began, self.lost = list(lengths), ends, began, lost
        self.known, self.forked = list(lengths), list(lengths)

    def compact(self):
        """Moves the pages in use to the front of the cache; how many they are, on the device."""
        import torch
        self._sharing()
        used = torch.empty(1, dtype=torch.int32, device="cuda")
        B.ac_op_cache_compact(self.all_caches, self.books, self.books, self.books_workspace, used)
        return used

    def _heads(self, n):
        """A place for n rows' queries, keys and values, and the three as views of it."""
        import torch
        h, hk, d = self.cfg.heads, self.heads_kv, self.cfg.head_dim
        qkv = torch.empty((n, (h + 2 * hk) * d), dtype=self.dtype, device="cuda")
        return qkv, qkv[:, :h * d], qkv[:, h * d:(h + hk) * d], qkv[:, (h + hk) * d:]

    def _workspace_bytes(self, n, rows):
        import torch
        q = torch.empty((n, self.cfg.heads * self.cfg.head_dim), dtype=self.dtype, device="meta")       # (of which sizes and type are read)
        if self.window is not None:
            return B.ac_cache_attention_window_workspace_bytes(q, self.caches[0], rows, self.window, self.sinks)
        return B.ac_cache_attention_workspace_bytes(q, self.caches[0], rows)

    def _run(self, x, rows, workspace):
        """x becomes the last layer's rows."""
        import torch
        cfg, n = self.cfg, x.shape[0]
        qkv, q, k, v = self._heads(n)
        u, ctx, mid = (torch.empty((n, c), dtype=self.dtype, device="cuda") for c in (cfg.d_model, q.shape[1], cfg.d_ffn))
        act = B.ACTIVATIONS[cfg.activation]
        for w, cache in zip(self.layers, self.caches):
            B.ac_op_layernorm(x, w["ln1_g"], w["ln1_b"], u, cfg.ln_eps)
            self._linear(w, "qkv", u, qkv)
            B.ac_op_cache_append(k, v, cache, rows, q=q, q_out=q, rotary=self.rotary)
            if self.window is None:
                B.ac_op_cache_attention(q, ctx, cache, rows, workspace=workspace)
            else:
                B.ac_op_cache_attention_window(q, ctx, cache, rows, self.window, self.sinks, workspace=workspace)
            self._linear(w, "o", ctx, x, residual=x)
            B.ac_op_layernorm(x, w["ln2_g"], w["ln2_b"], u, cfg.ln_eps)
            self._linear(w, "1", u, mid, activation=act)
            self._linear(w, "2", mid, x, residual=x)
        return x

    def step_graph(self):
        """A function of x [sequences, d_model], the next token of every sequence, as forward's with counts of one, but from a graph: lengths count on the device,
        and work is laid out for max_tokens.  What it returns is overwritten by its next call.  Between calls `lengths` may be set, whole or one of it: a sequence
        then goes on behind as many of its tokens."""
        import torch
        n = len(self.lengths)
        x, begin, length = torch.zeros((n, self.cfg.d_model), dtype=self.dtype, device="cuda"), *(
            torch.arange(n + 1, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda"))
        rows = B.cache_rows(begin, length, self.table, 1, self.max_tokens)
        workspace = B.empty_workspace(self._workspace_bytes(n, rows))
        # once without a page, which leaves the cache as it is: kernels are loaded before the capture
        self._run(x.clone(), B.cache_rows(begin, length, torch.full_like(self.table, -1), 1, self.max_tokens), workspace)
        torch.cuda.synchronize()
        if self.shares:
            before, drop_begin, drop_end = torch.empty_like(length), torch.full_like(length, self.sinks), torch.zeros_like(length)
            B.ac_op_pages_update(self.books, self.books, self.books_workspace, (drop_end, drop_end), (drop_end, drop_end), self.missing)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            if self.shares:
                torch.add(length, 0, out=before)
                if self.window is not None:
                    torch.sub(length, self.window - 1, out=drop_end)
            length.add_(1)
            if self.shares:
                B.ac_op_pages_update(self.books, self.books, self.books_workspace, (drop_begin, drop_end), (before, length), self.missing)
            y = self._run(x.clone(), rows, workspace)
        on_device = None

        def step(new):
            nonlocal on_device
            if new.shape != x.shape or new.dtype is not x.dtype:
                raise ValueError(f"rows {tuple(new.shape)} of {new.dtype} for {n} sequences of {x.shape[1]} x {x.dtype}")
            if max(self.lengths) >= self.max_tokens:
                raise ValueError(f"the cache holds {self.max_tokens} tokens of a sequence")
            was_set = self.shares and self._was_set(range(n))
            if self.lengths != on_device:
                length.copy_(torch.tensor(self.lengths, dtype=torch.int32))
            x.copy_(new)
            graph.replay()
            if self.shares:
                on_device = None                                        # (where pages are missing lengths are copied again)
                self.ends = [max(e, -(-(t + 1) // self.page)) for e, t in zip(self.ends, self.lengths)]
                self.began = list(self.lengths)
                if was_set:                                             # (their next tokens are written, also where pages are missing for others)
                    self._read(self.lengths, was_set, [1] * n)
                self._enough(self.ends, self.lengths)
            lengths = [t + 1 for t in self.lengths]
            if self.shares:
                self._read(lengths, was_set, [1] * n)
            self.lengths = lengths
            on_device = list(self.lengths)                              # (the caller may change the other one in place)
            return y
        step.keep = (graph, workspace, rows, begin) + ((before, drop_begin, drop_end) if self.shares else ())
        return step


class BeamSearch:
    """Beam search with a Decoder whose sequences share pages: sequences p * beams .. (p + 1) * beams - 1 are prompt p's.  embedding [vocab, d_model] makes rows of tokens; the logits of a row y are head y (+
    bias), head [vocab, d_model] in 4 bits.  end: the token that ends a sequence (-1: none does); one that ended stays among the beams with the sum that it has."""

    def __init__(self, model, embedding, head, beams, bias=None, end=-1):
        import torch
        model._sharing()
        self.model, self.beams, self.end = model, beams, end
        self.prompts, left = divmod(len(model.lengths), beams)
        vocab, d = embedding.shape
        if left or d != model.cfg.d_model or head.shape != (vocab, d) or not -1 <= end < vocab:
            raise ValueError(f"{len(model.lengths)} sequences, {beams} beams, embedding {tuple(embedding.shape)}, head {tuple(head.shape)}, end {end}")
        dev = lambda t: torch.as_tensor(t, device="cuda")  # noqa: E731
        self.embedding, self.head = dev(embedding).to(model.dtype).contiguous(), quantize_w4(dev(head), model.group, model.dtype)
        self.bias = None if bias is None else dev(bias).to(model.dtype)
        n = len(model.lengths)
        self.logits = torch.empty((n, vocab), dtype=model.dtype, device="cuda")
        self.workspace = B.empty_workspace(B.ac_beam_select_workspace_bytes(self.logits, beams, beams))
        self._none()

    def _none(self):
        self.scores, self.ended, self.steps = None, None, []
        self.pending = None                                             # a choice behind which the sequences were forked, but whose tokens are not read

    def _logits(self, y):
        codes, scale, zero = self.head
        B.ac_op_linear_w4(y, codes, scale, self.logits, self.model.group, zero=zero, bias=self.bias)

    def start(self, prompts, stretch=512):
        """Reads the prompts, lists of tokens, each into its first beam, `stretch` tokens at a time."""
        import torch
        m, k = self.model, self.beams
        if len(prompts) != self.prompts or not all(prompts):
            raise ValueError(f"{self.prompts} prompts of one token at least are wanted")
        vocab = self.logits.shape[1]
        if min(map(min, prompts)) < 0 or max(map(max, prompts)) >= vocab:
            raise ValueError(f"tokens {min(map(min, prompts))} to {max(map(max, prompts))} of a vocabulary of {vocab}")
        self._none()
        m.release(range(len(m.lengths)))
        y = torch.zeros((self.prompts * k, m.cfg.d_model), dtype=m.dtype, device="cuda")
        for at in range(0, max(len(p) for p in prompts), stretch):
            now = [p[at:at + stretch] for p in prompts]
            rows = self.embedding[torch.tensor(sum(now, []), device="cuda")]
            out = m.forward(rows, [len(now[b // k]) if b % k == 0 else 0 for b in range(len(m.lengths))])
            row = 0
            for p, part in enumerate(now):
                row += len(part)
                if part:
                    y[p * k] = out[row - 1]
        self._logits(y)
        self.scores = torch.full((self.prompts, k), float("-inf"), device="cuda")
        self.scores[:, 0] = 0
        self.ended = None if self.end < 0 else torch.zeros((self.prompts, k), dtype=torch.int32, device="cuda")

    def step(self):
        """Chooses the beams' next tokens and reads them: (parent, token), int32 [prompts, beams] on the device.  Where that fails, as where pages run out, what was found stays, and the next
        call goes on from there."""
        m = self.model
        if self.scores is None:
            raise ValueError("no search has been started: start reads its prompts")
        if self.pending is None:
            self.pending = self._choose()
        scores, ended, parent, token = self.pending
        y = m.forward(self.embedding[token.view(-1).clamp(min=0).long()], [1] * len(m.lengths))
        self._logits(y)
        self.scores, self.ended, self.pending = scores, ended, None
        self.steps.append((parent, token))
        return parent, token

    def _choose(self):
        """The beams' next tokens, and the sequences forked by their parents."""
        import torch
        m, k = self.model, self.beams
        i32 = dict(dtype=torch.int32, device="cuda")
        scores, parent, token = torch.empty_like(self.scores), torch.empty((self.prompts, k), **i32), torch.empty((self.prompts, k), **i32)
        ended = None if self.ended is None else torch.empty_like(self.ended)
        B.ac_op_beam_select(self.logits, self.scores, scores, parent, token, self.workspace, ended=self.ended, ended_out=ended, end=self.end)
        # all beams of a prompt have its length (a beam that is none, too: what it reads has no weight)
        m.fork(parent.view(-1), [m.lengths[b // k * k] for b in range(len(m.lengths))])
        return scores, ended, parent, token

    def found(self):
        """[[(sum of logarithms, tokens)]] of each prompt, best first; tokens up to and with the end."""
        if self.scores is None:
            return [[] for _ in range(self.prompts)]
        scores = self.scores.tolist()
        steps = [(p.view(-1).tolist(), t.view(-1).tolist()) for p, t in self.steps]
        result = []
        for p in range(self.prompts):
            beams = []
            for i in range(self.beams):
                b, tokens = p * self.beams + i, []
                for parent, token in reversed(steps):
                    if b >= 0:
                        tokens.append(token[b])
                        b = parent[b]
                tokens.reverse()
                if self.end in tokens:
                    tokens = tokens[:tokens.index(self.end) + 1]
                if scores[p][i] > float("-inf"):
                    beams.append((scores[p][i], tokens))
            result.append(beams)
        return result


def main():
    import torch
    ap = argparse.ArgumentParser()
    ap.add_argument("--config", default="C2", choices=[n for n, c in I.CONFIGS.items() if isinstance(c, I.TransformerConfig) and c.causal])
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=1024)
    ap.add_argument("--stretch", type=int, default=512, help="tokens of a sequence read at once")
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--window", type=int, help="tokens that a row sees, besides the sinks")
    ap.add_argument("--sinks", type=int, default=0)
    ap.add_argument("--beams", type=int, default=0, help="time a beam search, too")
    ap.add_argument("--vocab", type=int, default=32768)
    args = ap.parse_args()
    cfg = I.CONFIGS[args.config]
    x, layers = I.transformer_inputs(dataclasses.replace(cfg, batch=1, seq=args.batch * args.prompt))
    most, page = args.prompt + args.steps + 2 * args.stretch + (0 if args.window is None else args.steps + 1), 64
    # behind a window a sequence holds its sinks, its window and a stretch
    pages = None if args.window is None else args.batch * (-(-args.sinks // page) + -(-(args.window + args.stretch) // page) + 2)
    model = Decoder(cfg, layers, args.batch, most, page, window=args.window, sinks=args.sinks, pages=pages)
    x = torch.as_tensor(x, device="cuda").to(model.dtype).view(args.batch, args.prompt, -1)

    def read(first, n):
        return model.forward(x[:, first:first + n].reshape(-1, cfg.d_model), [n] * args.batch)

    def timed(work):
        torch.cuda.synchronize()
        t = time.perf_counter()
        y = work()
        torch.cuda.synchronize()
        return y, time.perf_counter() - t

    def prompt():
        for at in range(0, args.prompt, args.stretch):
            y = read(at, min(args.stretch, args.prompt - at))
        return y.view(args.batch, -1, cfg.d_model)[:, -1].contiguous()

    def steps(y, step):
        for _ in range(args.steps):
            y = step(y)
        return y

    def anew(lengths):
        if model.shares and not any(lengths):
            model.release(range(args.batch))
        model.lengths = lengths

    read(0, min(args.stretch, args.prompt))                             # code and clocks
    anew([0] * args.batch)
    y, reading = timed(prompt)
    y, writing = timed(lambda: steps(y, lambda x: model.forward(x, [1] * args.batch)))
    step = model.step_graph()
    step(y)
    if not model.shares:
        anew([args.prompt] * args.batch)
    y, replaying = timed(lambda: steps(y, step))
    found = {}
    if args.beams:
        each = -(-(args.prompt + args.steps) // page)
        shared = Decoder(cfg, layers, args.batch * args.beams, args.prompt + args.steps, page, window=args.window, sinks=args.sinks,
                         pages=args.batch * (each + 2 * args.beams * (2 + args.steps // page)))
        g = torch.Generator(device="cuda")
        g.manual_seed(1)
        embedding, head = (torch.randn((args.vocab, cfg.d_model), generator=g, device="cuda") * s for s in (1.0, cfg.d_model ** -0.5))
        search = BeamSearch(shared, embedding, head, args.beams)
        prompts = torch.randint(0, args.vocab, (args.batch, args.prompt), generator=g, device="cuda").tolist()
        search.start(prompts, args.stretch)
        search.step()
        _, searching = timed(lambda: [search.step() for _ in range(args.steps - 1)])
        best = search.found()
        found = {"beams": args.beams, "vocab": args.vocab, "beam_ms_per_step": round(searching / max(1, args.steps - 1) * 1e3, 3),
                 "beam_tokens": [len(best[0][0][1]), min(len(b) for b in best)]}
    print(json.dumps(found | {"config": cfg.name, "layers": cfg.layers, "dtype": cfg.dtype, "weights": "4 bits", "cache": "8 bits", "batch": args.batch,
                      "prompt": args.prompt, "prompt_tokens_per_s": round(args.batch * args.prompt / reading, 1), "steps": args.steps,
                      "tokens_per_s": round(args.batch * args.steps / writing, 1), "ms_per_step": round(writing / args.steps * 1e3, 3),
                      "graph_tokens_per_s": round(args.batch * args.steps / replaying, 1), "graph_ms_per_step": round(replaying / args.steps * 1e3, 3),
                      "finite": bool(torch.isfinite(y).all())}))


if __name__ == "__main__":
    main()
