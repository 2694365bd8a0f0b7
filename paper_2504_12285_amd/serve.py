"""A batch of requests served through the 2B-style layers with their attention: block tables, the rotary append into an
8-bit key/value cache and the attention over it stand where the chain (chain.py) has its context-length-1 stand-in.

    layers = CachedLayers(weights, gains, requests=8, rows=8, max_blocks=64, n_blocks=512, device="cuda:0")
    y = layers.step(x, new_len)          # x fp32 [rows][2560]: the new tokens' hidden states, request after request
    tokens = TokenLayers(layers, vocabulary)
    ids = tokens.step(ids, new_len)      # int32 [rows] in, the next id of each request out

Layer, per token: qkv = BL_qkv(norm(x)); Q, K (normed where the layer has gains for it) turned, K and V into the cache; a = attention; o = BL_o(norm(a)); h1 = x + o;
gu = BL_gu(norm(h1)); x' = h1 + BL_down(norm(relu(g)^2 * u)).  Orchestration only: every arithmetic step runs inside the HIP
kernels reached through the C-ABI; what is done here is that rows without a slot are cleared, and that of the logits the largest is taken.  A step reads nothing back and allocates
nothing that it keeps, so that it may be captured in a HIP graph.

Requests may share a prefix (groups=): a prompt that one place has taken in is given to a group, other places begin behind it, and each layer's attention reads it once for all.

`python -m paper_2504_12285_amd.serve` runs prompts and decode steps on random weights and prints their times.
"""
import time

import torch

from . import binding as bl
from .chain import HEAD_DIM, N_KV, N_Q, SHAPES, ChainBuffers

# Rows up to which a product takes its producer along (a layer of one row 34 us, 43 with the quantiser apart; of two 55.6 and 52.3,
# of four 82 and 53), and up to which it streams the weights once (of four 53 us, 63 with the prefill product; of eight 55 and 64).
FUSED_ROWS, GROUP_ROWS = 1, 64


def rotary_angles(n_pos, device, base=500000.0, dim=HEAD_DIM):
    """cos and sin fp32 [n_pos][dim / 2] of position * base^(-2i / dim), from angles in 64 bits."""
    angle = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * \
        base ** (-torch.arange(dim // 2, dtype=torch.float64, device=device) * 2 / dim)
    return angle.cos().float(), angle.sin().float()


class CachedLayers:
    """Layers, their caches and the buffers of a step.  weights: per layer a dict name -> (packed, beta); gains: per layer a
    dict name -> fp32 [K] or None.  requests: places in the batch; rows: new tokens of a step at most; max_new: of one
    request (one that brings more is refused: tables.bad counts it, tables.start is -1); max_blocks: blocks of one request; n_blocks: of the pool (each layer has a cache of that many).
    qk_gains: per layer the fp32 [128] gains of the norms of Q and K heads (a pair, either may be None), or None: no such norms.
    groups: prefixes that may be shared at a time (share, join, release)."""

    def __init__(self, weights, gains, requests, rows, max_blocks, n_blocks, device, layout=bl.BL_LAYOUT_K16, block=64,
                 kind=bl.BL_KV_INT8, max_new=None, window=0, eps=1e-5, qk_gains=None, groups=0):
        i32 = dict(dtype=torch.int32, device=device)
        max_new = max_new or None                # (0: no limit)
        self.weights, self.gains, self.layout, self.rows, self.eps = weights, gains, layout, rows, eps
        self.buffers = ChainBuffers(rows, device)
        self.x = torch.zeros((rows, SHAPES["down"][0]), dtype=torch.float32, device=device)
        self.new_len = torch.zeros(requests, **i32)
        self.seq_len = torch.zeros(requests, **i32)
        self.table = torch.full((requests, max_blocks), -1, **i32)
        self.free_list = torch.arange(n_blocks - 1, -1, -1, **i32)
        self.free_count = torch.full((1,), n_blocks, **i32)
        self.block, self.groups = block, groups
        self.held = None
        if groups:
            self.held, self.group = torch.zeros(requests, **i32), torch.full((requests,), -1, **i32)
            self.shared_table, self.shared_blocks = torch.full((groups, max_blocks), -1, **i32), torch.zeros(groups, **i32)
            self.ended = torch.zeros(requests, dtype=torch.bool, device=device)
            self.prefix = [0] * groups           # blocks of each group's prefix, as the host knows them
        self.tables = bl.KVTables(self.seq_len, self.new_len, self.table, self.free_list, self.free_count, block, rows, in_place=True,
                                  max_new=max_new, held=self.held)
        self.nowhere = torch.zeros(rows, dtype=torch.bool, device=device)
        cos, sin = rotary_angles(max_blocks * block, device)
        self.bad = torch.zeros(1, **i32)
        q = torch.empty((rows, N_Q * HEAD_DIM), dtype=torch.bfloat16, device=device)
        out = torch.zeros_like(q)               # (rows of no request stay as they are)
        self.caches = [bl.KVCache.empty(n_blocks, N_KV, block, HEAD_DIM, device, kind) for _ in weights]
        self.append = []
        for i, c in enumerate(self.caches):
            args = (c, self.buffers.qkv, N_Q, self.tables.slots, self.tables.positions, cos, sin, q, self.bad)
            self.append.append(bl.KVAppend(*args) if qk_gains is None else
                               bl.KVNormAppend(*args, q_gain=qk_gains[i][0], k_gain=qk_gains[i][1], eps=eps))
        space = None
        self.attend = []
        for c in self.caches:
            more = dict(n_q=N_Q, max_q=rows if max_new is None else max_new, window=window, out=out, workspace=space)
            if groups:
                a = bl.KVSharedAttention(c, q, self.tables.q_start, self.seq_len, self.table, self.group, self.shared_table, self.shared_blocks, **more)
            else:
                a = bl.KVAttention(c, q, self.tables.q_start, self.seq_len, self.table, **more)
            space = a.workspace
            self.attend.append(a)

    def _norm(self, layer, name):
        return dict(norm=True, gain=self.gains[layer].get(name), eps=self.eps)

    def _product(self, layer, name, prod, out, residual=None):
        """out = [residual +] BL_name(prod), with the producer's rows quantised on the way."""
        (N, K), (packed, beta), B = SHAPES[name], self.weights[layer][name], self.buffers
        item = dict(packed=packed, beta=beta, N=N, K=K, y=out, residual=residual)
        if self.rows <= FUSED_ROWS:
            bl.bl_bitlinear_decode_group(bl.make_decode_descs([dict(item, prod=prod)]), self.layout, self.rows)
            return
        q = B.q["f" if K == SHAPES["down"][1] else "h"]
        bl.bl_quant_act_ex(prod, self.rows, K, B.device, q=q, scale=B.scale, rowsum=B.rowsum)
        if self.rows <= GROUP_ROWS:
            bl.bl_bitlinear_decode_group(bl.make_decode_descs([dict(item, q=q, scale=B.scale, rowsum=B.rowsum)]), self.layout, self.rows)
        else:
            bl.bl_gemm_w158a8_res(packed, beta, self.layout, q, B.scale, B.rowsum, N, residual, want_acc=False, y=out)

    def run(self):
        """One step over what x and new_len hold; the result is in buffers.x_next.  Rows whose token has no slot (of a refused request,
        padding) went through the products and an attention that knows nothing of them: they are zeros at the end."""
        B = self.buffers
        self.tables.run()
        if self.groups:                         # an ended request leaves its group
            torch.lt(self.new_len, 0, out=self.ended)
            self.group.masked_fill_(self.ended, -1)
            self.held.masked_fill_(self.ended, 0)
        x, y = self.x, B.x_next
        for i in range(len(self.weights)):
            self._product(i, "qkv", bl.make_producer(bl.BL_PROD_F32, x, **self._norm(i, "qkv")), B.qkv)
            self.append[i].run()
            self.attend[i].run()
            self._product(i, "o", bl.make_producer(bl.BL_PROD_BF16, self.attend[i].out, **self._norm(i, "o")), B.o)
            self._product(i, "gate_up", bl.make_producer(bl.BL_PROD_RESIDUAL, x, B.o, B.h1, **self._norm(i, "gate_up")), B.gu)
            self._product(i, "down", bl.make_producer(bl.BL_PROD_RELU2_GATE, B.gu, **self._norm(i, "down")), y, residual=B.h1)
            x = y                               # (the layer has read x when its last product writes)
        torch.lt(self.tables.slots, 0, out=self.nowhere)
        return y.masked_fill_(self.nowhere[:, None], 0.0)

    def step(self, x, new_len):
        """x: fp32 [rows][2560], the rows of the requests' new tokens in order (rows behind them are padding); new_len: int32
        [requests], tokens that each brings, -1: it ends.  Returns the rows' hidden states (a buffer of the next step); those of a refused
        request (tables.bad of them, tables.start is -1) and of padding are zeros."""
        for t, own, name in ((x, self.x, "x"), (new_len, self.new_len, "new_len")):
            if t.shape != own.shape:             # (a copy would repeat a single row for all)
                raise ValueError("%s must have the shape %s, has %s" % (name, tuple(own.shape), tuple(t.shape)))
        self.x.copy_(x)
        self.new_len.copy_(new_len)
        return self.run()


    # These three stand between steps and read back what they check.

    def _within(self, group, place=0):
        """A negative number would be that of another group or place, and as a request's group that of none."""
        if not 0 <= group < self.groups:
            raise ValueError("group %d of %d" % (group, self.groups))
        if not 0 <= place < self.seq_len.shape[0]:
            raise ValueError("place %d of %d" % (place, self.seq_len.shape[0]))

    def share(self, group, place, blocks):
        """The first `blocks` blocks of the request at `place`, whole ones, become the group's prefix.  They belong to the group from now on: the request
        may go on or end, and release gives them back.  The request is in no group so far."""
        self._within(group, place)
        if self.prefix[group]:
            raise ValueError("group %d has a prefix" % group)
        if not 0 < blocks <= int(self.seq_len[place]) // self.block:
            raise ValueError("a prefix has 1 to %d of the blocks at place %d, not %d" % (int(self.seq_len[place]) // self.block, place, blocks))
        if int(self.group[place]) >= 0:
            raise ValueError("the request at place %d is in group %d" % (place, int(self.group[place])))
        self.shared_table[group, :blocks] = self.table[place, :blocks]
        self.shared_blocks[group], self.prefix[group] = blocks, blocks
        self.held[place] = blocks
        self.group[place] = group

    def join(self, place, group):
        """The next request at `place`, which is empty, begins behind the group's prefix."""
        self._within(group, place)
        n = self.prefix[group]
        if not n:
            raise ValueError("group %d has no prefix" % group)
        if int(self.seq_len[place]):
            raise ValueError("place %d has a request" % place)
        self.table[place, :n] = self.shared_table[group, :n]
        self.held[place], self.group[place] = n, group
        self.seq_len[place] = n * self.block

    def release(self, group):
        """Gives the group's blocks back, once no request is in it any more."""
        self._within(group)
        n = self.prefix[group]
        if bool((self.group == group).any()):
            raise ValueError("group %d has requests" % group)
        at = self.free_count.long() + torch.arange(n, device=self.table.device)
        self.free_list.scatter_(0, at, self.shared_table[group, :n])
        self.free_count += n
        self.shared_blocks[group], self.prefix[group] = 0, 0


class TokenLayers:
    """CachedLayers from token ids to token ids.  vocabulary: F8Matrix [tokens][2560], whose rows are the embeddings (times `multiplier`) and whose product
    with the normed hidden states (gain fp32 [2560] or None) are the logits, or head: another one for the logits."""

    def __init__(self, layers, vocabulary, head=None, gain=None, multiplier=1.0):
        dev, requests = layers.x.device, layers.new_len.shape[0]
        self.layers = layers
        self.ids = torch.full((layers.rows,), -1, dtype=torch.int32, device=dev)
        self.bad = torch.zeros(1, dtype=torch.int32, device=dev)
        self.embed = bl.F8Embedding(vocabulary, self.ids, out=layers.x, multiplier=multiplier, bad=self.bad)
        self.hidden = torch.zeros((requests, layers.x.shape[1]), dtype=torch.float32, device=dev)
        self.head = bl.F8Linear(vocabulary if head is None else head, self.hidden, norm=True, gain=gain, eps=layers.eps)
        self.logits = self.head.y
        self.next = torch.full((requests,), -1, dtype=torch.int32, device=dev)

    def run(self):
        """One step over what ids and layers.new_len hold.  next: the id of each request's largest logit (the first of several), -1 for one that brought no
        token or was refused.  bad counts ids that name no row, but for -1 (padding); such rows are zeros."""
        L = self.layers
        self.embed.run()
        y = L.run()
        last = (L.tables.q_start[1:] - 1).clamp_(min=0)
        torch.index_select(y, 0, last, out=self.hidden)
        self.head.run()
        best = torch.argmax(self.logits, 1).to(torch.int32)
        self.next.copy_(torch.where((L.new_len > 0) & (L.tables.start >= 0), best, -1))
        return self.next

    def step(self, ids, new_len):
        """ids: int32 [rows], the requests' new tokens in order (-1 behind them); new_len as in CachedLayers.step."""
        for t, own, name in ((ids, self.ids, "ids"), (new_len, self.layers.new_len, "new_len")):
            if t.shape != own.shape:
                raise ValueError("%s must have the shape %s, has %s" % (name, tuple(own.shape), tuple(t.shape)))
        self.ids.copy_(ids)
        self.layers.new_len.copy_(new_len)
        return self.run()


def random_layers(n, device, seed=0, layout=bl.BL_LAYOUT_K16):
    """Packed random weights and unit gains of n layers."""
    g = torch.Generator(device=device).manual_seed(seed)
    weights = [{name: bl.bl_pack_ternary(torch.randn(N, K, generator=g, device=device) * 0.02, layout) for name, (N, K) in SHAPES.items()}
               for _ in range(n)]
    return weights, [{name: None for name in SHAPES} for _ in range(n)]


def time_prompts(layers, x, lens):
    """Seconds of the step that brings prompts of `lens` tokens to places that are all empty at its start (whatever they hold now ends first)."""
    layers.step(x, torch.full_like(lens, -1))
    torch.cuda.synchronize()
    t = time.perf_counter()
    y = layers.step(x, lens)
    torch.cuda.synchronize()
    return time.perf_counter() - t, y


def main(layers=4, requests=8, prompt=1000, steps=64):
    dev = torch.device("cuda:0")
    weights, gains = random_layers(layers, dev)
    blocks = (prompt + steps) // 64 + 2
    g = torch.Generator(device=dev).manual_seed(1)
    lens = torch.tensor([prompt - 37 * b for b in range(requests)], dtype=torch.int32, device=dev)
    rows = int(lens.sum())
    fill = CachedLayers(weights, gains, requests, rows, blocks, requests * blocks, dev, max_new=prompt)
    x = torch.randn(rows, SHAPES["down"][0], generator=g, device=dev)
    fill.step(x, lens)
    t, y = time_prompts(fill, x, lens)
    print("%d prompts, %d tokens, %d layers: %.2f ms" % (requests, rows, layers, t * 1e3))
    # decode: the same state with a row for each request, captured once and replayed
    decode = CachedLayers(weights, gains, requests, requests, blocks, requests * blocks, dev, max_new=1)
    for name in ("seq_len", "table", "free_list", "free_count"):
        getattr(decode, name).copy_(getattr(fill, name))
    for a, b in zip(decode.caches, fill.caches):
        for name in ("k", "v", "k_scale", "v_scale"):
            getattr(a, name).copy_(getattr(b, name))
    last = torch.cumsum(lens, 0) - 1
    decode.step(y[last.long()], torch.ones_like(lens))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        decode.x.copy_(decode.run())                     # a stand-in for sampling and embedding the next token
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(steps - 2):
        graph.replay()
    torch.cuda.synchronize()
    print("decode of %d requests, %d layers: %.1f us a step; lengths now %s, refused %d" % (
        requests, layers, (time.perf_counter() - t) * 1e6 / (steps - 2), decode.seq_len.tolist(), int(decode.tables.bad)))


def main_shared(layers=4, requests=16, prompt=4096, steps=64, vocabulary=128256):
    """A system prompt, taken in once, and requests behind it that answer token by token: from ids to ids."""
    dev = torch.device("cuda:0")
    weights, gains = random_layers(layers, dev)
    g = torch.Generator(device=dev).manual_seed(2)
    words = bl.F8Matrix.quantise(torch.randn(vocabulary, SHAPES["down"][0], generator=g, device=dev, dtype=torch.bfloat16) * 0.02)
    ones = torch.ones(HEAD_DIM, device=dev)
    blocks, shared = (prompt + steps) // 64 + 2, prompt // 64
    more = dict(n_blocks=shared + requests * (steps // 64 + 2), device=dev, qk_gains=[(ones, ones)] * layers, groups=1)
    fill = CachedLayers(weights, gains, requests, prompt, blocks, max_new=prompt, **more)
    new = torch.zeros(requests, dtype=torch.int32, device=dev)
    new[0] = prompt
    TokenLayers(fill, words, multiplier=50.0).step(torch.randint(0, vocabulary, (prompt,), generator=g, device=dev, dtype=torch.int32), new)
    decode = CachedLayers(weights, gains, requests, requests, blocks, max_new=1, **more)
    for name in ("seq_len", "table", "free_list", "free_count"):
        getattr(decode, name).copy_(getattr(fill, name))
    for a, b in zip(decode.caches, fill.caches):
        for name in ("k", "v", "k_scale", "v_scale"):
            getattr(a, name).copy_(getattr(b, name))
    decode.share(0, 0, shared)
    for place in range(1, requests):
        decode.join(place, 0)
    tokens = TokenLayers(decode, words, multiplier=50.0)
    tokens.step(torch.randint(0, vocabulary, (requests,), generator=g, device=dev, dtype=torch.int32), torch.ones_like(new))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tokens.ids.copy_(tokens.run())
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(steps - 2):
        graph.replay()
    torch.cuda.synchronize()
    print("decode of %d requests behind one prompt of %d tokens, %d layers and a vocabulary of %d: %.1f us a step; lengths now %s, refused %d" % (
        requests, prompt, layers, vocabulary, (time.perf_counter() - t) * 1e6 / (steps - 2), decode.seq_len.tolist(), int(decode.tables.bad)))


if __name__ == "__main__":
    main()
    main_shared()
