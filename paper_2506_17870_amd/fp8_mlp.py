"""The MLP blocks of a transformer on the fp8 operators, from one token to a long prompt; calls only the C ABI.

A block is norm -> first layer -> activation -> second layer, and its output is the branch that the next norm adds to the
residual stream.  Between two matrix products stands one launch each: nq_block_norm (norm of the last branch, gate, residual sum,
norm, e4m3 codes) before the first layer, nq_quantize_fp8 (activation, product with the gated half, codes) before the second.
Everything a forward pass writes is allocated by allocate(), so that it can be captured into a HIP graph.
"""
from __future__ import annotations

import contextlib

import torch

import paper_2506_17870_amd as nq

_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}       # nq_dtype


class Fp8Mlp:
    """layers: sequence of dicts of float tensors on the device,
        up      [F][D], or [2 F][D]: the rows that go through the activation first, then those it is multiplied with
        down    [D][F]
        pre     fp32 [D], weight of the RMS norm before the block
        post    fp32 [D] or absent, weight of the RMS norm after it
        gate    dtype [D] or absent, factors of the branch per channel
    dtype: of branches and activations (the residual stream has h_dtype).

    A pass runs on the stream it is given, else on the current one, where its input has to be ready.  It comes after all that this object
    has on other streams (the weights' quantiser, the buffers' fills, the last pass), and what it uses is not given away before
    that stream is done.  Of a stream given as a raw handle, which need not outlive its work, torch cannot know that once the object or
    the input is gone: keep both until then.

    A graph captured from run() or forward() holds this object's addresses: it needs the object as long as it is replayed.  The buffers of
    a token count that was captured stay as they are, and allocate() or forward() with that count come back to them."""

    _STATE = ("tokens", "x", "h", "branch", "mid", "a", "norms", "_buffers", "_home", "_recorded")        # what allocate() makes

    def __init__(self, layers, act=nq.NQ_ACT_SILU, dtype=torch.bfloat16, h_dtype=None, eps=1e-5, residual_scale=1.0, branch_scale=1.0):
        self.act, self.dtype, self.h_dtype, self.eps = act, dtype, h_dtype or dtype, eps
        self.residual_scale, self.branch_scale = residual_scale, branch_scale
        self.layers = []
        for L in layers:
            D, F = L["down"].shape
            if L["up"].shape[1] != D or L["up"].shape[0] not in (F, 2 * F):
                raise ValueError(f"up {tuple(L['up'].shape)} does not fit down {tuple(L['down'].shape)}")
            for name, want in (("pre", torch.float32), ("post", torch.float32), ("gate", dtype)):
                t = L.get(name)
                if t is not None and (t.dtype != want or tuple(t.shape) != (D,)):
                    raise ValueError(f"{name} must be {want} [{D}], got {t.dtype} {tuple(t.shape)}")
            self.layers.append(dict(D=D, F=F, gated=L["up"].shape[0] == 2 * F, up=nq.Fp8Matrix.from_float(L["up"].contiguous()),
                                    down=nq.Fp8Matrix.from_float(L["down"].contiguous()), pre=L["pre"], post=L.get("post"), gate=L.get("gate")))
        if len({L["D"] for L in self.layers}) > 1:
            raise ValueError("the layers differ in width")
        self.tokens = None
        self._weights = [t for L in self.layers for t in (L["up"].q, L["up"].scale, L["down"].q, L["down"].scale, L["pre"], L["post"], L["gate"])
                         if t is not None]
        self._device, self._buffers, self._recorded = self._weights[0].device, [], set()
        self._captured = {}                  # by token count: the state whose addresses are in a graph
        # by handle: the streams that the next pass has to come after, those that came as handles with an event behind the last pass
        self._home = torch.cuda.current_stream(self._device)
        self._after = {self._home.cuda_stream: (self._home, None)}

    def _wait(self, stream):
        for handle, (other, event) in self._after.items():
            if handle != stream.cuda_stream:
                stream.wait_event(event or other.record_event())

    @contextlib.contextmanager
    def _on(self, stream):
        """The stream as the current one, behind what _after names.  A stream that is captured cannot wait for work outside its graph:
        torch waits for the device before a capture begins, and the order of replays and other passes is the caller's."""
        with torch.cuda.stream(nq.torch_stream(stream, self._device)) if stream is not None else contextlib.nullcontext():
            now = torch.cuda.current_stream(self._device)
            if torch.cuda.is_current_stream_capturing():
                self._captured[self.tokens] = {name: getattr(self, name) for name in self._STATE}
                yield now
                return
            self._wait(now)
            if not isinstance(stream, int) and now.cuda_stream not in self._recorded:
                self._recorded.add(now.cuda_stream)
                for t in self._weights + self._buffers:
                    t.record_stream(now)
            try:
                yield now
            finally:
                self._after = {now.cuda_stream: (now, now.record_event() if isinstance(stream, int) else None)}

    def _settled(self, stream):
        """Whether the pass goes where the last one went, with nothing left to order: the usual case, in a microsecond instead of four."""
        if stream is not None or len(self._after) != 1:
            return False
        handle = nq.current_raw_stream(self._device.index)
        return (self._after.get(handle, (None, True))[1] is None and handle in self._recorded
                and not torch.cuda.is_current_stream_capturing())

    def allocate(self, tokens: int):
        """Buffers and descriptors for `tokens` tokens, made on the current stream."""
        if tokens in self._captured:
            self.__dict__.update(self._captured[tokens])
            return self
        now = torch.cuda.current_stream(self._device)
        if not torch.cuda.is_current_stream_capturing():
            self._wait(self._home)                        # the old buffers go back to the stream they were made on
        self._home, self._recorded = now, set()
        self._after.setdefault(now.cuda_stream, (now, None))
        self.tokens, self.D = tokens, self.layers[0]["D"]
        dev = self._device
        self.x = nq.Fp8Matrix(tokens, self.D, device=dev)
        self.h = torch.empty(tokens, self.D, dtype=self.h_dtype, device=dev)
        self.branch = torch.empty(tokens, self.D, dtype=self.dtype, device=dev)
        most = max(L["up"].rows for L in self.layers)
        self.mid = torch.empty(tokens * most, dtype=self.dtype, device=dev)
        self.a = {F: nq.Fp8Matrix(tokens, F, device=dev) for F in {L["F"] for L in self.layers}}
        dt, hdt = _DTYPES[self.dtype], _DTYPES[self.h_dtype]
        none = nq.make_norm(nq.NQ_NORM_NONE)
        # norm i stands before layer i: it ends what layer i - 1 began
        self.norms = []
        for i, L in enumerate(self.layers + [None]):
            last = self.layers[i - 1] if i else None
            post = nq.make_norm(nq.NQ_NORM_RMS, self.eps, last["post"]) if last and last["post"] is not None else none
            pre = nq.make_norm(nq.NQ_NORM_RMS, self.eps, L["pre"]) if L else none
            gate = last["gate"] if last else None
            self.norms.append(nq.make_block_norm(
                self.h, hdt, self.D, self.branch if last else None, dt, self.D, gate, self.D, tokens if gate is not None else 0,
                self.residual_scale if last else 1.0, self.branch_scale, post, pre, self.h if last else None, self.D, None, 0,
                self.x.desc if L else None))
        self._buffers = [self.h, self.branch, self.mid] + [t for m in (self.x, *self.a.values()) for t in (m.q, m.scale)]
        return self

    def forward(self, h, stream=None):
        """h: [tokens][D] of h_dtype.  stream: a stream or its raw handle, as for every call.  Returns the stream behind the last block
        (a buffer of this object: the next forward overwrites it)."""
        if h.dim() != 2 or h.shape[1] != self.layers[0]["D"]:
            raise ValueError(f"the stream must be [tokens][{self.layers[0]['D']}], got {tuple(h.shape)}")
        if self.tokens != h.shape[0]:                     # (memory belongs to streams that torch knows)
            with torch.cuda.stream(None if isinstance(stream, int) else stream):
                self.allocate(h.shape[0])
        if self._settled(stream):
            self.h.copy_(h)
            return self._pass(None)
        with self._on(stream) as now:
            self.h.copy_(h)
            if stream is not None and not isinstance(stream, int):
                h.record_stream(now)
            return self._pass(stream)

    def run(self, stream=None):
        """The same on the stream that lies in self.h already."""
        if self._settled(stream):
            return self._pass(None)
        with self._on(stream):
            return self._pass(stream)

    def _pass(self, stream):
        dt, es = _DTYPES[self.dtype], self.mid.element_size()
        for L, norm in zip(self.layers, self.norms):
            F, rows, a = L["F"], L["up"].rows, self.a[L["F"]]
            nq.nq_block_norm(norm, self.tokens, self.D, stream)
            nq.nq_gemm_fp8(self.x.desc, L["up"].desc, None, self.mid, dt, rows, stream)
            mul = self.mid.data_ptr() + F * es if L["gated"] else None
            nq.nq_quantize_fp8(self.mid, dt, rows, mul, rows, self.act, a.desc, stream)
            nq.nq_gemm_fp8(a.desc, L["down"].desc, None, self.branch, dt, self.D, stream)
        nq.nq_block_norm(self.norms[-1], self.tokens, self.D, stream)
        return self.h
