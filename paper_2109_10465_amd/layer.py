"""Buffer owner and call sequence for one MoE layer step on one GPU.

Holds the device buffers (torch tensors used as raw memory) and makes the two
C-ABI calls of a step: moe_layer_fwd (gate -> capacity/RTS -> dispatch -> experts
-> combine) and moe_layer_bwd, its reverse.  No arithmetic happens here.
"""
import torch

from . import binding as B

_TORCH_DT = {B.F32: torch.float32, B.BF16: torch.bfloat16}


class MoELayer:
    def __init__(self, T, d_model, d_ff, E, k, capacity, dtype, act, device="cuda:0", aux_coef=0.0,
                 forward_only=False, groups=1, jitter_eps=0.0, drop_p=0.0):
        if not torch.cuda.is_available():
            raise B.MoeError("MoELayer needs a GPU; there is no CPU fallback")
        B.lib()
        self.shape = B.make_shape(T, d_model, d_ff, E, k, capacity, dtype, act)
        self.T, self.d, self.f, self.E, self.k, self.C = T, d_model, d_ff, E, k, capacity
        self.device = torch.device(device)
        self.aux_coef = float(aux_coef)     # weight of the balancing loss in the objective (0 = off)
        self.jitter_eps = float(jitter_eps)  # gate jitter (training); the seed is given per step
        self.drop_p = float(drop_p)          # expert dropout on the hidden activation (training)
        self.seed = 0
        self.groups = int(groups)           # > 1: token selection inside groups of T/groups consecutive tokens
        self.forward_only = bool(forward_only)   # evaluation: no saved derivative, no backward buffers
        adt = _TORCH_DT[dtype]
        dev = self.device

        def buf(shape, dt):
            return torch.empty(shape, dtype=dt, device=dev)

        i32, f32 = torch.int32, torch.float32
        self.logits = buf((T, E), f32)
        self.probs = buf((T, E), f32)
        self.expert_idx = buf((T, k), i32)
        self.gate_w = buf((T, k), f32)
        self.slot = buf((T, k), i32)
        self.expert_count = buf((E,), i32)
        self.expert_demand = buf((E,), i32)
        self.slot_src = buf((E, capacity), i32)
        self.first_frac = buf((E,), f32)     # balancing loss: first-choice share, mean probability, value
        self.mean_prob = buf((E,), f32)
        self.aux_loss = buf((1,), f32)
        self.xd = buf((E, capacity, d_model), adt)
        self.h = buf((E, capacity, d_ff), adt)       # act(z)
        self.dact = None if forward_only else buf((E, capacity, d_ff), adt)    # act'(z)
        self.yd = buf((E, capacity, d_model), adt)
        self.y = buf((T, d_model), adt)
        self.utilisation = torch.zeros((E,), dtype=torch.int64, device=dev)   # tokens routed to each expert so far
        nbytes = B.moe_workspace_bytes(self.shape)
        if nbytes == 0:
            raise B.MoeError("unsupported shape")
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        if forward_only:
            return
        # backward
        self.dyd = buf((E, capacity, d_model), adt)
        self.dgate_w = buf((T, k), f32)
        self.dxd = buf((E, capacity, d_model), adt)
        self.dW1 = buf((E, d_model, d_ff), f32)
        self.dW2 = buf((E, d_ff, d_model), f32)
        self.dlogits = buf((T, E), f32)
        self.dWg = buf((d_model, E), f32)
        self.dx = buf((T, d_model), adt)

    # what moe_layer_fwd and moe_layer_bwd take, in the order of B.LayerBuffers; a forward-only layer has no
    # derivative and no backward buffers
    _FWD = ("logits", "probs", "expert_idx", "gate_w", "slot", "expert_count", "expert_demand", "slot_src",
            "utilisation", "first_frac", "mean_prob", "aux_loss", "xd", "h", "dact", "yd", "y")
    _BWD = ("dyd", "dgate_w", "dxd", "dW1", "dW2", "dlogits", "dWg", "dx")

    def _call_args(self, logits_given=False):
        """Options and buffers of one call, from the layer's attributes as they are now."""
        at = self.__dict__
        ptrs = [None if at[n] is None else at[n].data_ptr() for n in self._FWD]
        ptrs += [None] * len(self._BWD) if self.forward_only else [None if at[n] is None else at[n].data_ptr() for n in self._BWD]
        # attributes may have been set anew since: whatever is a number, and fewer than two groups is plain routing
        return (B.LayerOptions(max(1, int(self.groups)), bool(self.forward_only), logits_given, self.aux_coef,
                               self.jitter_eps, self.drop_p, int(self.seed) & 0xFFFFFFFFFFFFFFFF),
                B.LayerBuffers(*ptrs, self.ws.data_ptr(), self.ws.numel() * self.ws.element_size()))

    def forward(self, x, Wg, bias, W1, W2, rts_keys, logits=None, seed=0):
        """logits: optional precomputed [T,E] fp32 gate logits; the projection call is
        then skipped and routing runs on exactly these values."""
        self._saved = (x, Wg, W1, W2)
        self.seed = int(seed)     # of this step's jitter and dropout draws
        if logits is not None:
            self.logits.copy_(logits)
        B.moe_layer_fwd(self.shape, *self._call_args(logits is not None), x, Wg, bias, W1, W2, rts_keys)
        return self.y

    def backward(self, dy):
        if self.forward_only:
            raise B.MoeError("this layer was built forward-only")
        x, Wg, W1, W2 = self._saved
        B.moe_layer_bwd(self.shape, *self._call_args(), x, Wg, W1, W2, dy)
        return self.dx, self.dWg, self.dW1, self.dW2

    def step(self, x, Wg, bias, W1, W2, rts_keys, dy, logits=None, seed=0):
        self.forward(x, Wg, bias, W1, W2, rts_keys, logits, seed)
        return self.backward(dy)

    def capture_step(self, x, Wg, bias, W1, W2, rts_keys, dy, seed=0):
        """Records one forward+backward step into a HIP graph and returns it (`.replay()` runs the step again on
        the same tensors: refill x, dy, the weights and the keys in place between replays).  The library
        allocates nothing and clears nothing with memset, so every call of the step is a plain kernel node.
        Replay takes the host out of the loop (18 us of host time instead of 44 for a 256-token step); the time of a
        step stays about the same, since the chain of dependent kernels sets it, not their launch (256 tokens, fp32:
        51 us eager; 55 eager and 57 replayed when its expert products took 1-2 us longer each).
        The seed of the step's noise draws is a host value and is recorded with the graph."""
        if self.forward_only:
            raise B.MoeError("this layer was built forward-only")
        self.step(x, Wg, bias, W1, W2, rts_keys, dy, seed=seed)       # first use of every kernel happens eagerly
        torch.cuda.synchronize(self.device)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.step(x, Wg, bias, W1, W2, rts_keys, dy, seed=seed)
        return graph

    def clip_gradients(self, max_norm, others=()):
        """Clips the last backward pass's dWg, dW1 and dW2 together with `others` (gradients of the rest of the model: float32
        or bfloat16, contiguous) to the global norm max_norm, in place, and returns that norm (a device tensor of one float)."""
        if self.forward_only:
            raise B.MoeError("this layer was built forward-only")
        others, dev = list(others), self.dWg.device
        for g in others:
            if g.device != dev:
                raise B.MoeError(f"a gradient on {g.device}, not {dev}")
        grads = B.make_grads([(g, g) for g in (self.dWg, self.dW1, self.dW2, *others)])
        # of this call alone: a captured call keeps its own, whatever is clipped later
        norm = torch.empty(1, dtype=torch.float32, device=dev)
        ws = torch.empty(B.moe_grad_workspace_bytes(grads), dtype=torch.uint8, device=dev)
        with torch.cuda.device(dev):
            B.moe_clip_grads(grads, max_norm, norm, ws)
        return norm


class Fp8MoELayer:
    """Forward-only layer with a wide gate and experts on 8-bit operands: gate projection -> router -> rows expert by
    expert -> 8-bit dispatch -> experts -> mixture, as one native call.  Nothing is dropped: every choice has a row.

    W1, W2: pairs (q, b) of 8-bit weights and their exponent bytes, as quantise_weights() makes them from W1 [E, d_model, d_ff]
    and W2 [E, d_ff, d_model]."""

    _NAMES = ("logits", "expert_idx", "gate_w", "row_of", "expert_start", "xq", "xb", "hq", "hb", "yd", "y", "ws")

    def __init__(self, T, d_model, d_ff, E, k, dtype, act, W1, W2, score=B.SOFTMAX, n_groups=1, top_groups=1, group_best=1,
                 renormalise=True, scale=1.0, device="cuda:0"):
        if not torch.cuda.is_available():
            raise B.MoeError("Fp8MoELayer needs a GPU; there is no CPU fallback")
        B.lib()
        self.shape = B.make_fp8_shape(T, d_model, d_ff, E, k, dtype, act)
        self.router = B.make_router(T, E, k, score, n_groups, top_groups, group_best, renormalise, scale)
        nbytes = B.moe_sort_workspace_bytes(self.router)
        if nbytes == 0:
            raise B.MoeError("unsupported router")
        for (q, b), (K, N) in ((W1, (d_model, d_ff)), (W2, (d_ff, d_model))):
            want = (E, B.fp8_padded(N), B.fp8_padded(K)), (E, B.fp8_padded(N) // 128, B.fp8_scale_bytes(K))
            if (tuple(q.shape), tuple(b.shape)) != want or q.dtype not in (torch.float8_e4m3fn, torch.uint8) or b.dtype != torch.uint8:
                raise B.MoeError(f"8-bit weights (float8_e4m3fn or its bytes, and uint8 exponents) of shapes {want} expected, not "
                                 f"{q.dtype} of {tuple(q.shape)}, {b.dtype} of {tuple(b.shape)}")
            if not (q.is_contiguous() and b.is_contiguous()):
                raise B.MoeError("8-bit weights must be contiguous")
        self.W1, self.W2 = W1, W2
        self.device = torch.device(device)
        B.moe_fp8_kernels(self.shape)           # (refuses what the experts' block refuses)
        R = T * k

        def buf(shape, dt):
            return torch.empty(shape, dtype=dt, device=self.device)

        u8 = torch.uint8
        self.logits, self.gate_w = buf((T, E), torch.float32), buf((T, k), torch.float32)
        self.expert_idx, self.row_of = buf((T, k), torch.int32), buf((T, k), torch.int32)
        self.expert_start = buf((E + 1,), torch.int32)
        self.xq, self.xb = buf((R, B.fp8_padded(d_model)), u8), buf((R, B.fp8_scale_bytes(d_model)), u8)
        self.hq, self.hb = buf((R, B.fp8_padded(d_ff)), u8), buf((R, B.fp8_scale_bytes(d_ff)), u8)
        self.yd, self.y = buf((R, d_model), torch.float32), buf((T, d_model), _TORCH_DT[dtype])
        self.ws = buf((nbytes,), u8)
        self.device = self.y.device
        for t in (*W1, *W2):
            if t.device != self.y.device:
                raise B.MoeError(f"8-bit weights on {t.device}, not {self.y.device}")
        # what forward() takes: shape and type
        f32 = torch.float32
        self._takes = {"x": ((T, d_model), self.y.dtype), "Wg": ((d_model, E), f32), "logits": ((T, E), f32),
                       "select_bias": ((E,), f32), "token_mask": ((T,), u8)}

    def _check(self, name, t):
        shape, dt = self._takes[name]
        if t is not None and (tuple(t.shape) != shape or t.dtype != dt or t.device != self.y.device or not t.is_contiguous()):
            raise B.MoeError(f"{name}: contiguous {dt} of {shape} on {self.y.device} expected, not {t.dtype} of {tuple(t.shape)} "
                             f"with strides {t.stride()} on {t.device}")

    @staticmethod
    def quantise_weights(W):
        """W [E, K, N] (float32 or bfloat16, on the GPU) -> (q, b) as the experts take them."""
        E, K, N = W.shape
        if not (W.is_contiguous() and W.is_cuda):
            raise B.MoeError("weights must be contiguous and on a GPU")
        q = torch.empty((E, B.fp8_padded(N), B.fp8_padded(K)), dtype=torch.float8_e4m3fn, device=W.device)
        b = torch.empty((E, B.fp8_padded(N) // 128, B.fp8_scale_bytes(K)), dtype=torch.uint8, device=W.device)
        with torch.cuda.device(W.device):
            B.moe_quantise_weights_fp8(E, K, N, W, q, b)
        return q, b

    def forward(self, x, Wg=None, logits=None, select_bias=None, token_mask=None):
        """x [T, d_model]; Wg [d_model, E] fp32, or logits [T, E] fp32 in its place; select_bias [E] fp32; token_mask [T]
        uint8 or bool, 0 for padding (its rows of y are 0)."""
        if (Wg is None) == (logits is None):
            raise B.MoeError("either Wg or logits")
        if token_mask is not None and token_mask.dtype == torch.bool:
            token_mask = token_mask.view(torch.uint8)
        for name, t in (("x", x), ("Wg", Wg), ("logits", logits), ("select_bias", select_bias), ("token_mask", token_mask)):
            self._check(name, t)
        ptrs = [(logits if n == "logits" and logits is not None else getattr(self, n)).data_ptr() for n in self._NAMES]
        with torch.cuda.device(self.device):
            B.moe_layer_fwd_fp8(self.shape, self.router, logits is not None, B.Fp8Buffers(*ptrs, self.ws.numel()), x, Wg,
                                select_bias, token_mask, *self.W1, *self.W2)
        return self.y

    def update_select_bias(self, select_bias, rate):
        """After a forward pass: raises the bias of experts with fewer choices than the mean by rate, lowers the others'."""
        self._check("select_bias", select_bias)
        with torch.cuda.device(self.device):
            B.moe_router_bias_update(self.router, self.expert_start, rate, select_bias)
