"""A decoder's attention block served in 8 and 4 bits, put together from the operators of ``binding``:

    x [tokens, E] --linear--> queries, keys, values --kv4_write--> paged cache, of 4 bits (kv8_write: of 8)
                                      \\--------------kv4_attend----------/--linear--> y [tokens, E]

``AttentionBlock`` holds the weights (one factor per output channel), the cache with its block table and free pages, and
the workspaces; ``step`` takes the new tokens of any of its requests, a prompt's or a decoding step's, and ``select`` lets
requests go on several times (beams, samples of one prompt) or not at all, ``compact`` moves the pages in use to the front of
the pool.  Host code orders
the launches and counts pages; every piece of arithmetic is the library's.  Run as a program, it serves a few requests
and reports how far 8 and 4 bits are from the same block in fp32.
"""
import torch

from . import binding as B


class Linear8:
    """Weights of an 8-bit linear layer: fp32 [N, K] -> int8 with a factor per row, packed; ``bias`` fp32 [N] or None."""

    def __init__(self, weight, bias=None):
        self.N, self.K = weight.shape
        self.q_w, z_w = B.quantize_weights_per_channel(weight.contiguous())
        self.packed = B.linear_pack(z_w)
        self.bias = bias

    def __call__(self, x, out=None, workspace=None):
        return B.linear(x, self.packed, self.q_w, self.bias, out=out, workspace=workspace)


class AttentionBlock:
    """``w_qkv`` fp32 [(heads (ratio + 2)) D, E]: queries of all query heads (``ratio`` to a key head), keys, values;
    ``w_out`` fp32 [E, heads ratio D].  ``n_pages`` pages of ``page`` tokens are shared by ``requests`` requests of up to
    ``longest`` tokens each; a step has ``most`` new tokens at most; ``bits``: 4 or 8, of the cache."""

    def __init__(self, w_qkv, w_out, heads, ratio, D, n_pages, page, requests, longest, most, b_qkv=None, b_out=None,
                 window=0, dtype=torch.bfloat16, bits=4):
        dev, i32 = w_qkv.device, torch.int32
        assert w_qkv.shape[0] == heads * (ratio + 2) * D and w_out.shape[1] == heads * ratio * D
        self.heads, self.ratio, self.D, self.page, self.window, self.dtype = heads, ratio, D, page, window, dtype
        self.qkv, self.out = Linear8(w_qkv, b_qkv), Linear8(w_out, b_out)
        assert bits in (4, 8), bits
        self.bits, self._write, self._attend = (4, B.kv4_write, B.kv4_attend) if bits == 4 else (8, B.kv8_write, B.kv8_attend)
        self.cache = (B.kv4_cache if bits == 4 else B.kv8_cache)(n_pages, heads, page, D, dev)
        self.table = torch.full((requests, -(-longest // page)), -1, dtype=i32, device=dev)
        self.lengths = [0] * requests                                  # tokens in the cache, as the host counts them
        self.free = torch.arange(n_pages, dtype=i32, device=dev)       # of which the first `taken` are in use
        self.taken = 0
        self._shared = False                                           # whether requests have pages in common
        self._lengths = torch.zeros(requests, dtype=i32, device=dev)
        self._grown = torch.empty_like(self._lengths)
        self._starts = torch.empty(requests + 1, dtype=i32, device=dev)
        self._counts = torch.empty(3, dtype=i32, device=dev)
        self._slots = torch.empty(most, dtype=torch.int64, device=dev)
        self._positions = torch.empty(most, dtype=i32, device=dev)
        q = torch.empty((most, heads * ratio, D), dtype=dtype, device=dev)
        self._attend_ws = (B.kv4_attend_workspace if bits == 4 else B.kv8_attend_workspace)(q, self.cache, requests, longest, dev)
        sizes = [B.lib.q8_linear_workspace_bytes(most, w.N, w.K) for w in (self.qkv, self.out)]
        self._linear_ws = torch.empty(max(sizes), dtype=torch.uint8, device=dev)

    def pages_needed(self, added):
        """Pages that these new tokens (a number for each request) take."""
        return sum(-(-(n + a) // self.page) - -(-n // self.page) for n, a in zip(self.lengths, added))

    def step(self, x, added):
        """x [T, E], fp16 or bf16: the new tokens of request 0, then those of request 1, ...; ``added``: how many each request has.
        -> [T, E], the block's output for them.  Raises MemoryError if they do not fit (nothing is done then)."""
        T, need = x.shape[0], self.pages_needed(added)
        assert len(added) == len(self.lengths) and sum(added) == T and all(a >= 0 for a in added)
        assert x.dim() == 2 and x.shape[1] == self.qkv.K and x.dtype in (torch.float16, torch.bfloat16), (x.shape, x.dtype)
        longest = self.table.shape[1] * self.page
        if need > self.free.numel() - self.taken or T > self._slots.numel() or \
                any(n + a > longest for n, a in zip(self.lengths, added)):
            raise MemoryError(f"{need} pages, {T} tokens")
        more = torch.tensor(added, dtype=torch.int32).to(x.device)
        y = self.launch(x, more, self.free[self.taken:], self._slots[:T], self._positions[:T])
        self._lengths, self._grown = self._grown, self._lengths
        self.lengths = [n + a for n, a in zip(self.lengths, added)]
        self.taken += need
        return y

    def launch(self, x, added, free, slots, positions, out=None):
        """The launches of a step (all on the current stream; nothing is waited for): also inside a stream capture.
        They leave the requests' new lengths in the block's other buffer: ``step`` moves on to it."""
        H, D = self.heads, self.D
        B.page_tables(self._lengths, added, self.page, free, self.table, slots, positions, self._starts, self._grown,
                      self._counts)
        joint = self.qkv(x, workspace=self._linear_ws).view(x.shape[0], H * (self.ratio + 2), D)
        q, k, v = joint[:, :H * self.ratio], joint[:, -2 * H:-H], joint[:, -H:]
        self._write(self.cache, k, v, slots)
        o = self._attend(q, self.cache, self.table, self._grown, self._starts, window=self.window,
                         workspace=self._attend_ws)
        return self.out(o.view(x.shape[0], H * self.ratio * D), out=out, workspace=self._linear_ws)

    def select(self, parents):
        """Request c goes on as request parents[c] was, -1: as none, one without tokens; for every request of the block.  Several
        of one parent share its full pages, and each has a last page of its own.  Waits for the number of pages in use.
        Raises MemoryError if there are no pages for that (nothing is done then)."""
        n = len(self.lengths)
        assert len(parents) == n and all(-1 <= c < n for c in parents), parents
        kept = B.page_select(torch.tensor(parents, dtype=torch.int32).to(self.table.device), self._lengths, self.table, self.page,
                             self.cache.shape[0])
        free, copies, empty, used = kept["counts"].tolist()
        if empty:
            raise MemoryError(f"{copies + empty} pages to copy, {copies} free")
        if copies:
            B.page_copy(self.cache, kept["copies"])
        self.table.copy_(kept["table"])
        self._lengths.copy_(kept["lengths"])
        self.free[used:] = kept["free_pages"][:free]
        self.taken = used
        going = [c for c in parents if c >= 0 and self.lengths[c] > 0]
        self._shared = len(set(going)) < len(going) or (self._shared and len(going) > 0)
        self.lengths = [self.lengths[c] if c >= 0 else 0 for c in parents]

    def compact(self):
        """The pages in use move to the front of the pool; returns how many there are (waits for their number)."""
        moved = B.page_compact(self._lengths, self.table, self.page, self.cache.shape[0], table=self.table)
        free, copies, _, used = moved["counts"].tolist()
        if copies:
            B.page_copy(self.cache, moved["copies"])
        self.free[used:] = moved["free_pages"][:free]
        self.taken = used
        return used

    def release(self, request):
        """A request has ended: its pages are free again, but those that others share."""
        if self._shared:
            return self.select([c if c != request else -1 for c in range(len(self.lengths))])
        held = -(-self.lengths[request] // self.page)
        pages = self.table[request, :held].clone()
        self.taken -= held
        self.free[self.taken:self.taken + held] = pages
        self.lengths[request] = 0
        self._lengths[request] = 0


def _plain(w_qkv, w_out, xs, heads, ratio, D):
    """The block in fp32 on whole requests: xs, a tensor [tokens, E] each."""
    out = []
    for x in xs:
        T = x.shape[0]
        joint = (x @ w_qkv.t()).view(T, -1, D)
        q = joint[:, :heads * ratio].view(T, heads, ratio, D).permute(1, 2, 0, 3)
        k, v = [joint[:, a:a + heads].permute(1, 0, 2)[:, None] for a in (heads * ratio, heads * (ratio + 1))]
        score = (q @ k.transpose(-1, -2).contiguous()) * D ** -0.5
        score = score.masked_fill(torch.ones(T, T, dtype=torch.bool, device=x.device).triu(1), float("-inf"))
        o = torch.softmax(score, -1) @ v
        out.append(o.permute(2, 0, 1, 3).reshape(T, -1) @ w_out.t())
    return out


def main():
    torch.manual_seed(1)
    E, heads, ratio, D, prompts, steps = 1024, 4, 4, 64, (100, 37, 260), 8
    dev = torch.device("cuda")
    w_qkv = torch.randn(heads * (ratio + 2) * D, E, device=dev) / E ** 0.5
    w_out = torch.randn(E, heads * ratio * D, device=dev) / (heads * ratio * D) ** 0.5
    xs = [torch.randn(n + steps, E, device=dev) for n in prompts]
    want = _plain(w_qkv, w_out, xs, heads, ratio, D)
    for bits in (4, 8):
        # (a place for a second copy of the last request)
        block = AttentionBlock(w_qkv, w_out, heads, ratio, D, n_pages=64, page=16, requests=len(prompts) + 1, longest=512, most=512,
                               bits=bits)
        half = [x.to(block.dtype) for x in xs]
        got = block.step(torch.cat([h[:n] for h, n in zip(half, prompts)]), list(prompts) + [0]).split(prompts)
        block.select([*range(len(prompts)), len(prompts) - 1])
        got = [[g] for g in got]
        for i in range(steps):
            rows = [h[n + i] for h, n in zip(half, prompts)]
            y = block.step(torch.stack(rows + rows[-1:]), [1] * (len(prompts) + 1))
            assert torch.equal(y[-1], y[-2])                 # (both copies go the same way here)
            for g, row in zip(got, y.split(1)):
                g.append(row)
        for b, (g, w) in enumerate(zip(got, want)):
            off = (torch.cat(g).float() - w).norm() / w.norm()
            print(f"{bits} bits, request {b}: {len(w)} tokens, {block.taken} pages in use, {off:.3f} of the fp32 block's output away from it")
        block.release(0)
        print(f"{bits} bits: {block.compact()} pages in use at the front of the pool without request 0")
        for b in range(1, len(prompts) + 1):
            block.release(b)
        assert block.taken == 0


if __name__ == "__main__":
    main()
