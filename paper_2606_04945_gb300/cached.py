"""Block-wise denoising behind a cached prefix, with 4-bit weights.

A stack of pre-norm blocks (by default Dream-7B-shaped: hidden 3584, 28 query
heads over 4 key/value heads of 128, FFN 18944, bf16), random-init weights.
The answer is generated block by block: a block's positions start masked, each
step runs the stack over the block alone and unmasks its most confident
positions, and the prompt and the finished blocks are in the cache. A step
rewrites the block's own rows of the cache behind the same prefix; when the
block is finished, a last pass leaves the rows of its final tokens there. (Where the
prefix ends inside a page, its rows there share their scale with the block's:
a step that makes the scale grow rounds them again, and it stays grown. A
prompt that fills its pages avoids that.) Per layer:

    h = RMSNorm(x)                              glue_add_rmsnorm
    q, k, v = h Wqkv^T + b                      w4g_linear
    q, k = rotary positions; k, v to the cache  kv_cache_append
    a = softmax(q K^T / sqrt 128) V             kv_cache_attention, over prefix and block
    x = x + a Wo^T; h = RMSNorm(x)              w4g_linear, glue_add_rmsnorm
    x = x + (silu(g) u) Wdown^T, g, u = h Wgu^T w4g_linear twice, glue_add_rmsnorm

and the logits are one more w4g_linear of the last norm, in float32. The
weights carry one scale per group of input channels, the cache 8-bit codes;
activations stay 16-bit. The rotary table is filled once (glue_rope_table);
torch holds the buffers, multiplies silu(g) u and picks the tokens.

`python -m paper_2606_04945_gb300.cached` generates and prints the time of a
step. A linear takes at most 32 rows a call: a prompt goes through it in
slices, so a long prompt is not this module's strength. Attention is given
the capacity as the bound of the lengths, since one recorded pass serves every
block: with up to 64 rows of a key/value head a short prefix in a large cache
takes the kernel for long ones.
"""

from dataclasses import dataclass

import torch

from . import abi

EPS = 1e-6
ROWS = 32                                   # of one w4g_linear call


@dataclass
class CachedConfig:
    hidden: int = 3584
    ffn: int = 18944
    heads: int = 28
    kv_heads: int = 4
    dim: int = 128
    layers: int = 4
    vocab: int = 8192
    batch: int = 1
    block: int = 32                         # positions denoised together
    unmask_per_step: int = 4
    capacity: int = 1024                    # tokens of a sequence
    page: int = 64
    group: int = 64                         # input channels that share a weight's scale
    theta: float = 1e6
    scaling: str = "none"                   # of the rotary table
    factor: float = 1.0
    original: float = 0.0
    dtype: torch.dtype = torch.bfloat16
    seed: int = 0


class GroupLinear:
    """A linear with packed 4-bit weights and one scale per group of input
    channels."""

    def __init__(self, W16, group, bias=None):
        self.N, self.K = W16.shape
        dev = W16.device
        self.Wq = torch.empty(self.N, self.K // 2, dtype=torch.uint8, device=dev)
        self.scales = torch.empty(self.N, self.K // group, dtype=torch.float32, device=dev)
        self.bias = bias
        # a group is a row of its own: per-row quantisation without a transform
        abi.sgat_prepare_weight(W16.view(-1, group), None, 1, self.Wq.view(-1, group // 2), self.scales.view(-1))

    def run(self, X, Y):
        for r in range(0, X.shape[0], ROWS):
            abi.w4g_linear(X[r:r + ROWS], self.Wq, self.scales, Y[r:r + ROWS], bias=self.bias)


class CachedStack:
    def __init__(self, cfg: CachedConfig, device="cuda"):
        c = self.cfg = cfg
        self.device = device
        g = torch.Generator(device=device).manual_seed(c.seed)
        w = lambda n, k: (torch.randn(n, k, generator=g, device=device) * k ** -0.5).to(c.dtype)
        lin = lambda n, k, bias=None: GroupLinear(w(n, k), c.group, bias)
        self.width = (c.heads + 2 * c.kv_heads) * c.dim
        self.embed = torch.randn(c.vocab, c.hidden, generator=g, device=device).to(c.dtype)
        self.mask_id = 0
        self.layers = [dict(qkv=lin(self.width, c.hidden, torch.randn(self.width, generator=g, device=device) * 0.1),
                            o=lin(c.hidden, c.heads * c.dim), gu=lin(2 * c.ffn, c.hidden), down=lin(c.hidden, c.ffn))
                       for _ in range(c.layers)]
        self.head = lin(c.vocab, c.hidden)
        self.gain = torch.ones(c.hidden, dtype=torch.float32, device=device)
        self.rope = torch.empty(c.capacity, c.dim // 2, 2, dtype=torch.float32, device=device)
        abi.rope_table(self.rope, c.theta, c.scaling, c.factor, c.original)
        # a sequence's pages are its own, one cache a layer, one page table for all of them
        pages = (c.capacity + c.page - 1) // c.page
        self.caches = [abi.KVCache.empty(c.batch * pages, c.kv_heads, c.page, c.dim, device) for _ in range(c.layers)]
        self.page_table = torch.arange(c.batch * pages, dtype=torch.int32, device=device).view(c.batch, pages)
        self.past = torch.zeros(c.batch, dtype=torch.int32, device=device)
        self.held = 0                       # past, on the host
        self.buffers = {}

    def _buffers(self, n):
        """Buffers and index vectors of a pass over n positions a sequence."""
        if n not in self.buffers:
            c, T, dev = self.cfg, self.cfg.batch * n, self.device
            t = lambda *s: torch.empty(*s, dtype=c.dtype, device=dev)
            self.buffers[n] = dict(
                x=t(T, c.hidden), h=t(T, c.hidden), qkv=t(T, self.width), q=t(T, c.heads * c.dim),
                attn=t(T, c.heads * c.dim), o=t(T, c.hidden), gu=t(T, 2 * c.ffn), act=t(T, c.ffn), down=t(T, c.hidden),
                logits=torch.empty(T, c.vocab, dtype=torch.float32, device=dev),
                start=torch.arange(c.batch + 1, dtype=torch.int32, device=dev) * n,
                step=torch.arange(n, dtype=torch.int32, device=dev),
                workspace=torch.empty(abi.kv_cache_attention_workspace_size(c.batch, n, c.heads, c.kv_heads, c.dim),
                                      dtype=torch.uint8, device=dev))
        return self.buffers[n]

    def forward(self, tok, hook=None):
        """One pass over tok [batch][n], the n positions behind each
        sequence's past tokens: their keys and values go into the cache, and
        the logits [batch n][vocab] are returned. hook(layer, name, values)
        sees what each operator read and wrote (for tests)."""
        c = self.cfg
        n = tok.shape[1]
        if self.held + n > c.capacity:
            raise ValueError(f"{self.held} cached and {n} new positions are more than the cache's {c.capacity} tokens")
        b = self._buffers(n)
        hk = hook or (lambda layer, name, values: None)
        kq, kv = c.heads * c.dim, c.kv_heads * c.dim
        pos = (self.past[:, None] + b["step"][None]).view(-1)
        held = self.past + n
        x, h, qkv = b["x"], b["h"], b["qkv"]
        x.copy_(self.embed[tok.reshape(-1)])
        abi.add_rmsnorm(x, self.gain, h, eps=EPS)
        for i, (m, cache) in enumerate(zip(self.layers, self.caches)):
            m["qkv"].run(h, qkv)
            hk(i, "qkv", (m["qkv"], h, qkv))
            abi.kv_cache_append(cache, qkv[:, kq:kq + kv], qkv[:, kq + kv:], b["start"], self.past, self.page_table, pos,
                                self.rope, max_new=n, Q=qkv[:, :kq], Q_out=b["q"])
            hk(i, "append", (cache, qkv, b["q"], pos))
            abi.kv_cache_attention(b["q"], cache, self.page_table, held, b["start"], b["attn"], max_new=n,
                                   max_len=c.capacity, workspace=b["workspace"])
            hk(i, "attention", (cache, b["q"], held, b["attn"]))
            m["o"].run(b["attn"], b["o"])
            hk(i, "o", (m["o"], b["attn"], b["o"]))
            abi.add_rmsnorm(b["o"], self.gain, h, R=x, h_out=x, eps=EPS)
            m["gu"].run(h, b["gu"])
            hk(i, "gu", (m["gu"], h, b["gu"]))
            torch.mul(torch.nn.functional.silu(b["gu"][:, :c.ffn]), b["gu"][:, c.ffn:], out=b["act"])
            m["down"].run(b["act"], b["down"])
            hk(i, "down", (m["down"], b["act"], b["down"]))
            abi.add_rmsnorm(b["down"], self.gain, h, R=x, h_out=x, eps=EPS)
        self.head.run(h, b["logits"])
        hk(c.layers, "head", (self.head, h, b["logits"]))
        return b["logits"]

    def prefill(self, prompt):
        """The prompt [batch][P] begins the sequences: its tokens see one
        another and stay in the cache."""
        if prompt.shape[1] > self.cfg.capacity:
            raise ValueError(f"the prompt is longer than the cache's {self.cfg.capacity} tokens")
        self.past.zero_()
        self.held = 0
        if prompt.shape[1] > 0:
            self.forward(prompt)
            self.keep(prompt.shape[1])

    def keep(self, n):
        """The last pass's n positions become part of the prefix."""
        self.past += n
        self.held += n

    def capture(self):
        """Records a pass over a block in a CUDA graph; returns (graph, token
        buffer [batch][block], logits). It reads `past` where it is, so one
        graph serves every block. (The recording itself is a pass over masked
        positions behind the prefix, which has to leave them room.)"""
        c = self.cfg
        tok = torch.full((c.batch, c.block), self.mask_id, dtype=torch.long, device=self.device)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.forward(tok)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            logits = self.forward(tok)
        return graph, tok, logits

    def generate(self, prompt, blocks, captured=None):
        """Prompt [batch][P], then `blocks` blocks of new tokens; returns
        [batch][blocks x block]. captured: capture()'s result."""
        c = self.cfg
        if prompt.shape[1] + blocks * c.block > c.capacity:
            raise ValueError(f"prompt and answer are longer than the cache's {c.capacity} tokens")
        self.prefill(prompt)
        graph, tok, logits = captured or (None, torch.empty(c.batch, c.block, dtype=torch.long, device=self.device), None)
        out = []
        for _ in range(blocks):
            tok.fill_(self.mask_id)
            masked = torch.ones(c.batch, c.block, dtype=torch.bool, device=self.device)
            for left in range(c.block, 0, -c.unmask_per_step):
                if graph is None:
                    logits = self.forward(tok)
                else:
                    graph.replay()
                logits[:, self.mask_id] = float("-inf")                # a position never becomes masked again
                best, new = torch.softmax(logits, -1).view(c.batch, c.block, -1).max(-1)
                pick = best.masked_fill(~masked, -1.0).topk(min(c.unmask_per_step, left), dim=1).indices
                tok.scatter_(1, pick, new.gather(1, pick))
                masked.scatter_(1, pick, False)
            if graph is None:
                self.forward(tok)
            else:
                graph.replay()
            self.keep(c.block)
            out.append(tok.clone())
        return torch.cat(out, 1) if out else tok[:, :0].clone()


def main():
    cfg = CachedConfig()
    stack = CachedStack(cfg)
    prompt = torch.randint(1, cfg.vocab, (cfg.batch, 512), device="cuda")
    stack.prefill(prompt)
    captured = stack.capture()
    tokens = stack.generate(prompt, 4, captured)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    passes = 20
    torch.cuda.synchronize()
    start.record()
    for _ in range(passes):
        captured[0].replay()
    end.record()
    torch.cuda.synchronize()
    abi.check_status()
    print(f"{tokens.shape[1]} tokens behind {prompt.shape[1]}: {tokens[0, :8].tolist()} ...; {cfg.layers} layers over "
          f"{cfg.block} positions and {stack.held} cached tokens: {start.elapsed_time(end) / passes:.3f} ms a step")


if __name__ == "__main__":
    main()
