"""Attention layers that serve several streams at once: each stream has its own
K/V history in pages of one pool and its own low-rank adapter, and a pass takes a
chunk of new tokens of any of them, packed behind one another.

``begin`` opens a pass: it finds pages for the new tokens and hands their places
to the device.  Then every layer runs ``layer_pass``, on the caller's stream:

1. ``mssa_adapter_project``: q, k, v of all tokens, each stream with its adapter;
2. ``mssa_paged_append``: queries and keys rotated, keys and values stored;
3. ``mssa_paged_attention``: each stream's new tokens over its pages, if wanted
   joined with an attention over other keys (a window's, a sink's).

All layers share one page table: a page holds a stream's tokens in every layer.
They also share buffers and a workspace: passes on several HIP streams have to
wait for one another.  An adapter is one pair of factors over q, k and v together;
where those have first factors of their own, they are stacked behind one another
(three times the rank), with zeros in b where a feature does not take a factor.
This module only keeps the table and sequences library calls (torch owns the
buffers); all arithmetic runs in the library.
"""

from . import mssa


class PagedStreams:
    def __init__(self, layers, hidden, q_heads, kv_heads, head_dim, pages, page_tokens, max_stream_pages, max_tokens,
                 max_batch, adapters=0, rank=0, freqs=None, rotate_dims=None, halves=True, axis_pairs=None, mask_block=1,
                 softmax_scale=0.0, device="cuda"):
        """pages of page_tokens tokens each, at most max_stream_pages a stream; a pass takes at most max_tokens tokens
        of max_batch streams.  freqs [rotate_dims / 2] fp32: radians a position (None: no rotation).  mask_block as in
        mssa_paged_attention (1: causal, 0: a chunk sees all of itself)."""
        import torch

        self.layers, self.hidden, self.device = int(layers), int(hidden), device
        self.q_heads, self.kv_heads, self.head_dim = int(q_heads), int(kv_heads), int(head_dim)
        self.pages, self.page_tokens, self.max_stream_pages = int(pages), int(page_tokens), int(max_stream_pages)
        self.max_tokens, self.max_batch = int(max_tokens), int(max_batch)
        self.adapters, self.rank, self.mask_block, self.scale = int(adapters), int(rank), int(mask_block), float(softmax_scale)
        self.q_width, self.kv_width = self.q_heads * self.head_dim, self.kv_heads * self.head_dim
        self.width = self.q_width + 2 * self.kv_width
        self.freqs, self.halves, self.axis_pairs = freqs, bool(halves), axis_pairs
        self.rotate_dims = 0 if freqs is None else (self.head_dim if rotate_dims is None else int(rotate_dims))
        if freqs is not None and (freqs.dtype != torch.float32 or not freqs.is_contiguous() or freqs.numel() != self.rotate_dims // 2):
            raise ValueError(f"freqs must be contiguous fp32 [{self.rotate_dims // 2}], not {freqs.dtype} {tuple(freqs.shape)}")
        if freqs is None:
            self.axis_pairs = None

        def buf(*shape, dtype=torch.bfloat16):
            return torch.empty(shape, dtype=dtype, device=device)

        pool = (self.pages, self.page_tokens, self.kv_heads, self.head_dim)
        self.k_pages, self.v_pages = ([torch.zeros(pool, dtype=torch.bfloat16, device=device) for _ in range(self.layers)]
                                      for _ in range(2))
        self.qkv, self.q = buf(self.max_tokens, self.width), buf(self.max_tokens, self.q_heads, self.head_dim)
        self.new = self.qkv, self.qkv[:, self.q_width:], self.qkv[:, self.q_width + self.kv_width:]  # q, k, v of new tokens
        self.free = list(range(self.pages))[::-1]
        self.streams = {}  # id -> [pages, tokens held, tokens dropped before them, adapter]
        self.weights = [None] * self.layers
        self.used = set()  # (HIP stream, layer): what those passes read and write is held for the stream
        self.batch = None
        self.workspace = buf(256, dtype=torch.uint8)
        if freqs is not None:
            self._here("freqs", freqs)

    def _here(self, name, t):
        if t.device != self.qkv.device:
            raise ValueError(f"{name} must be on {self.qkv.device}, not on {t.device}")

    def init_layer(self, layer, w_qkv, b_qkv=None, a=None, b=None, scale=None):
        """w_qkv [q_width + 2 kv_width, hidden] and b_qkv bf16; a [adapters, rank, hidden], b [adapters, width, rank] bf16,
        scale [adapters] fp32."""
        import torch

        want = dict(w_qkv=(w_qkv, (self.width, self.hidden)), b_qkv=(b_qkv, (self.width,)))
        if self.adapters:
            want.update(a=(a, (self.adapters, self.rank, self.hidden)), b=(b, (self.adapters, self.width, self.rank)))
        for name, (t, shape) in want.items():
            if t is None and name == "b_qkv":
                continue
            if t is None or t.dtype != torch.bfloat16 or not t.is_contiguous() or tuple(t.shape) != shape:
                raise ValueError(f"{name} must be contiguous bf16 {shape}")
            self._here(name, t)
        if scale is not None and (scale.dtype != torch.float32 or not scale.is_contiguous() or scale.numel() != self.adapters):
            raise ValueError(f"scale must be contiguous fp32 [{self.adapters}]")
        if scale is not None:
            self._here("scale", scale)
        self.weights[layer] = (w_qkv, b_qkv, a, b, scale)
        self.used = {u for u in self.used if u[1] != layer}

    def open(self, stream, adapter=-1):
        """A new stream without tokens; adapter: its low-rank adapter, -1 for none."""
        if stream in self.streams:
            raise ValueError(f"stream {stream!r} is open")
        if not -1 <= adapter < self.adapters:
            raise ValueError(f"there is no adapter {adapter}")
        self.streams[stream] = [[], 0, 0, int(adapter)]

    def close(self, stream):
        """Its pages are free again, once the work enqueued so far is done: passes of one program follow one another on
        one HIP stream."""
        self.free.extend(reversed(self.streams.pop(stream)[0]))

    def drop(self, stream, tokens):
        """Forget the oldest `tokens` tokens, whole pages of them; positions go on counting."""
        state = self.streams[stream]
        n = int(tokens) // self.page_tokens
        if n * self.page_tokens != tokens or tokens > state[1] or n < 0:
            raise ValueError("whole pages that the stream holds can be dropped")
        self.free.extend(reversed(state[0][:n]))
        del state[0][:n]
        state[1] -= int(tokens)
        state[2] += int(tokens)

    def begin(self, chunks):
        """Opens a pass: chunks is a list of (stream, new tokens), in the order of the packed rows."""
        import torch

        if not 1 <= len(chunks) <= self.max_batch:
            raise ValueError(f"a pass takes 1..{self.max_batch} streams")
        names = [s for s, _ in chunks]
        if len(set(names)) != len(names):
            raise ValueError("a stream can be in a pass once")
        if any(s not in self.streams for s in names):
            raise ValueError("a stream of the pass is not open")
        news = [int(n) for _, n in chunks]
        if min(news) < 0 or sum(news) > self.max_tokens:
            raise ValueError(f"a pass takes at most {self.max_tokens} tokens")
        want = []
        for s, n in zip(names, news):
            held, have = self.streams[s][1] + n, len(self.streams[s][0])
            need = -(-held // self.page_tokens)
            if need > self.max_stream_pages:
                raise ValueError(f"stream {s!r} would hold more than {self.max_stream_pages} pages")
            want.append(need - have)
        if sum(want) > len(self.free):
            raise RuntimeError(f"{sum(want)} pages are needed and {len(self.free)} are free")
        # what can be refused or raise comes before anything changes
        b, t, m = len(chunks), sum(news), self.max_stream_pages
        project = mssa.adapter_project_desc(t, self.hidden, self.width, b if self.adapters else 0, self.adapters, self.rank)
        append, check = (mssa.paged_append_desc(n, b, self.q_heads, self.kv_heads, self.head_dim, self.page_tokens, self.pages,
                                                m, rotate_dims=self.rotate_dims, halves=self.halves,
                                                axis_pairs=self.axis_pairs, q_stride=self.width, k_stride=self.width,
                                                v_stride=self.width) for n in (t, 0))
        mssa.mssa_paged_append(check, *[None] * 11, stream=0)  # checks the sizes; without tokens nothing is enqueued
        attend = mssa.paged_attention_desc(t, b, max(1, *news), self.q_heads, self.kv_heads, self.head_dim, self.page_tokens,
                                           self.pages, m, mask_block=self.mask_block, softmax_scale=self.scale)
        size = max(mssa.mssa_adapter_project_workspace_size(project), mssa.mssa_paged_attention_workspace_size(attend))
        spare, begin, lens, which, table, positions, held = len(self.free), [0], [], [], [], [], []
        for s, n, w in zip(names, news, want):
            pages, had, dropped, adapter = self.streams[s]
            pages, spare = pages + self.free[spare - w:spare][::-1], spare - w
            positions.extend(range(dropped + had, dropped + had + n))
            held.append([pages, had + n, dropped, adapter])
            begin.append(begin[-1] + n)
            lens.append(had + n)
            which.append(adapter)
            table.extend(pages + [-1] * (m - len(pages)))
        # one copy for all of it
        host = torch.tensor(begin + lens + which + table + positions, dtype=torch.int32)
        workspace = self.workspace
        if workspace.numel() < size:
            workspace = torch.empty(size, dtype=torch.uint8, device=self.device)
        dev = host.to(self.device)
        # nothing raises from here on: the pass is open
        self.streams.update(zip(names, held))
        del self.free[spare:]
        cut = lambda at, n: dev[at:at + n]  # noqa: E731
        self.chunk_begin, self.kv_len, self.adapter = cut(0, b + 1), cut(b + 1, b), cut(2 * b + 1, b)
        self.table, self.positions = cut(3 * b + 1, b * m), cut(3 * b + 1 + b * m, t)
        self.places, self.workspace = dev, workspace
        self.tokens, self.project, self.append, self.attend = t, project, append, attend
        self.batch = b

    def layer_pass(self, layer, x, out, lse=None, positions=None, prior_out=None, prior_lse=None, stream=None):
        """x [tokens, hidden], out [tokens, q_heads, head_dim] bf16, lse [q_heads, tokens] fp32 or None, of the pass that
        is open.  positions [axes, tokens] int32 (None: tokens of the stream before, one axis); prior_out and prior_lse: an
        attention of the same queries over other keys, joined with this one (they may be out and lse).  Captured into a
        graph it serves the pass that is open, until the next begin."""
        import torch

        if self.batch is None:
            raise ValueError("no pass is open")
        t = self.tokens
        want = [("x", x, (t, self.hidden), torch.bfloat16), ("out", out, (t, self.q_heads, self.head_dim), torch.bfloat16)]
        if prior_out is not None:
            want.append(("prior_out", prior_out, (t, self.q_heads, self.head_dim), torch.bfloat16))
        for name, v in (("lse", lse), ("prior_lse", prior_lse)):
            if v is not None:
                want.append((name, v, (self.q_heads, t), torch.float32))
        if positions is not None:
            want.append(("positions", positions, (len(self.axis_pairs or [0]), t), torch.int32))
        elif self.axis_pairs is not None and len(self.axis_pairs) > 1:
            raise ValueError("several axes need positions")
        for name, v, shape, dtype in want:
            if v.dtype != dtype or not v.is_contiguous() or tuple(v.shape) != shape:
                raise ValueError(f"{name} must be contiguous {dtype} {shape}, not {v.dtype} {tuple(v.shape)}")
            self._here(name, v)
            if dtype == torch.bfloat16 and v.data_ptr() % 16:
                raise ValueError(f"{name} must be 16-byte aligned")
        if self.weights[layer] is None:
            raise ValueError(f"layer {layer} has no weights")
        # what a later one of the calls would refuse is refused before the first
        if (prior_out is None) != (prior_lse is None):
            raise ValueError("prior_out and prior_lse come together")
        if any(out.data_ptr() == b.data_ptr() for b in (self.q, self.k_pages[layer], self.v_pages[layer])):
            raise ValueError("out must not be a buffer of the layers")
        w, bias, a, b, scale = self.weights[layer]
        qkv = self.qkv
        if x.is_cuda:
            if torch.cuda.current_device() != x.device.index:
                raise ValueError(f"the current device must be the layers', {x.device}")
            # begin replaces the first two, while this stream may still be reading them; the others go with the object
            handle = mssa._stream(stream)
            used, held = torch.cuda.ExternalStream(handle, device=x.device), [self.places, self.workspace]
            if (handle, layer) not in self.used:
                held += [qkv, self.q, self.freqs, self.k_pages[layer], self.v_pages[layer], w, bias, a, b, scale]
                self.used.add((handle, layer))
            for v in held:
                if v is not None:
                    v.record_stream(used)
        mssa.mssa_adapter_project(self.project, x, w, bias, self.chunk_begin, self.adapter, a, b, scale, self.workspace, [qkv],
                                  stream=stream)
        mssa.mssa_paged_append(self.append, *self.new, self.chunk_begin, self.kv_len, self.table,
                               self.positions if positions is None else positions, self.freqs, self.q, self.k_pages[layer],
                               self.v_pages[layer], stream=stream)
        mssa.mssa_paged_attention(self.attend, self.q, self.k_pages[layer], self.v_pages[layer], self.chunk_begin, self.kv_len,
                                  self.table, prior_out, prior_lse, self.workspace, out, lse, stream=stream)
