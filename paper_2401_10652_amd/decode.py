"""A pre-norm transformer that reads and writes token by token: linear layers with 4-bit weights, keys and values in a paged 8-bit cache.

    python -m paper_2401_10652_amd.decode [--config C2] [--batch 8] [--prompt 1024] [--stretch 512] [--steps 32]

reads a prompt for each sequence of a batch in stretches, then single tokens (each step's output is the next one's input: there is no
vocabulary here, as in the framework's other workloads), and prints one JSON line with both rates.
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
    queries and keys are rotated by their places, which no plan of the framework does, so that a plan's rows are not these."""

    def __init__(self, cfg, layers, sequences, max_tokens, page=64, group=64, base=10000.0):
        import torch
        if not cfg.causal:
            raise ValueError(f"{cfg.name} is not causal: its rows cannot be read a token at a time")
        self.cfg, self.group, self.max_tokens = cfg, group, max_tokens
        self.dtype = {"f32": torch.float32, "bf16": torch.bfloat16}[cfg.dtype]
        dev, d = "cuda", cfg.head_dim
        self.heads_kv = (layers[0]["w_qkv"].shape[0] // d - cfg.heads) // 2
        self.layers = []
        for w in layers:
            t = {n: torch.as_tensor(x, device=dev) for n, x in w.items()}
            self.layers.append({n: quantize_w4(x, group, self.dtype) if n.startswith("w_") else x.to(self.dtype) for n, x in t.items()})
        each = -(-max_tokens // page)
        pages = sequences * each
        self.table = torch.arange(pages, dtype=torch.int32, device=dev).view(sequences, each)
        codes = dict(dtype=torch.uint8, device=dev)
        self.caches = [B.kv_cache(torch.zeros((pages, self.heads_kv, page, d), **codes), torch.zeros((pages, self.heads_kv, page // 16, d, 16), **codes),
                                  torch.ones((pages, self.heads_kv, page // 16), device=dev), torch.ones((pages, self.heads_kv, page // 16), device=dev))
                       for _ in layers]
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
        begin = [0]
        for c in counts:
            begin.append(begin[-1] + c)
        # one copy to the device for both
        where = torch.tensor(begin + lengths, dtype=torch.int32).to("cuda")
        rows = B.cache_rows(where[:len(begin)], where[len(begin):], self.table, max(counts), max(lengths))
        need = self._workspace_bytes(n, rows)
        if need > self.workspace.numel():
            self.workspace = B.empty_workspace(need)
        x = self._run(x.clone(memory_format=torch.contiguous_format), rows, self.workspace)
        self.lengths = lengths
        return x

    def _heads(self, n):
        """A place for n rows' queries, keys and values, and the three as views of it."""
        import torch
        h, hk, d = self.cfg.heads, self.heads_kv, self.cfg.head_dim
        qkv = torch.empty((n, (h + 2 * hk) * d), dtype=self.dtype, device="cuda")
        return qkv, qkv[:, :h * d], qkv[:, h * d:(h + hk) * d], qkv[:, (h + hk) * d:]

    def _workspace_bytes(self, n, rows):
        import torch
        q = torch.empty((n, self.cfg.heads * self.cfg.head_dim), dtype=self.dtype, device="meta")       # (of which sizes and type are read)
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
            B.ac_op_cache_attention(q, ctx, cache, rows, workspace=workspace)
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
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            length.add_(1)
            y = self._run(x.clone(), rows, workspace)
        on_device = None

        def step(new):
            nonlocal on_device
            if new.shape != x.shape or new.dtype is not x.dtype:
                raise ValueError(f"rows {tuple(new.shape)} of {new.dtype} for {n} sequences of {x.shape[1]} x {x.dtype}")
            if max(self.lengths) >= self.max_tokens:
                raise ValueError(f"the cache holds {self.max_tokens} tokens of a sequence")
            if self.lengths != on_device:
                length.copy_(torch.tensor(self.lengths, dtype=torch.int32))
            x.copy_(new)
            graph.replay()
            self.lengths = [t + 1 for t in self.lengths]
            on_device = list(self.lengths)                              # (the caller may change the other one in place)
            return y
        step.keep = (graph, workspace, rows, begin)
        return step


def main():
    import torch
    ap = argparse.ArgumentParser()
    ap.add_argument("--config", default="C2", choices=[n for n, c in I.CONFIGS.items() if isinstance(c, I.TransformerConfig) and c.causal])
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=1024)
    ap.add_argument("--stretch", type=int, default=512, help="tokens of a sequence read at once")
    ap.add_argument("--steps", type=int, default=32)
    args = ap.parse_args()
    cfg = I.CONFIGS[args.config]
    x, layers = I.transformer_inputs(dataclasses.replace(cfg, batch=1, seq=args.batch * args.prompt))
    model = Decoder(cfg, layers, args.batch, args.prompt + args.steps + 2 * args.stretch)
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

    read(0, min(args.stretch, args.prompt))                             # code and clocks
    model.lengths = [0] * args.batch
    y, reading = timed(prompt)
    y, writing = timed(lambda: steps(y, lambda x: model.forward(x, [1] * args.batch)))
    step = model.step_graph()
    step(y)
    model.lengths = [args.prompt] * args.batch
    y, replaying = timed(lambda: steps(y, step))
    print(json.dumps({"config": cfg.name, "layers": cfg.layers, "dtype": cfg.dtype, "weights": "4 bits", "cache": "8 bits", "batch": args.batch,
                      "prompt": args.prompt, "prompt_tokens_per_s": round(args.batch * args.prompt / reading, 1), "steps": args.steps,
                      "tokens_per_s": round(args.batch * args.steps / writing, 1), "ms_per_step": round(writing / args.steps * 1e3, 3),
                      "graph_tokens_per_s": round(args.batch * args.steps / replaying, 1), "graph_ms_per_step": round(replaying / args.steps * 1e3, 3),
                      "finite": bool(torch.isfinite(y).all())}))


if __name__ == "__main__":
    main()
