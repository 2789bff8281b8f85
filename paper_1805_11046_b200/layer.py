"""Device-memory bookkeeping for one quantised layer: owns the buffers that
qbp_layer_fwd / qbp_layer_bwd need (codes, parameters, saved statistics,
gradient copies, workspace) as torch tensors and passes their addresses
through the C ABI.  No arithmetic happens here."""
from __future__ import annotations

import threading

import torch

from . import binding as B


class QuantizedLayer:
    """conv: a binding.ConvDesc for a convolution layer (x NHWC, w KRSC), or None for a linear
    layer y = x w with x [batch, in_features], w [in_features, out_features]."""

    def __init__(self, conv=None, batch=0, in_features=0, out_features=0, relu=False, seed=0,
                 tensor_id8=1, tensor_id16=2, device="cuda", input_from: "QuantizedLayer | None" = None,
                 emit_codes=False, keep_y=True, keep_z=True, keep_g=True):
        """input_from: the layer whose output feeds this one already quantised (it must have been built with
        emit_codes=True): this layer then owns no input codes of its own and its forward takes no fp32 input.
        emit_codes: the forward also writes the 8-bit codes of the output (and each row's code sum) for the next
        layer; keep_y=False then leaves the fp32 output unwritten.  keep_z=False (forward only, with emit_codes and
        keep_y=False): the fp32 output of the product is not kept either -- the convolution is run twice instead.
        keep_g=False: the backward pass does not write the fp32 gradient arriving at the product (only its 8-bit and
        16-bit copies); for shapes the library quantises as it computes the gradient (it says so otherwise)."""
        self.device = torch.device(device)
        d = B.LayerDesc()
        if conv is not None:
            d.conv = conv
            self.rows, self.cin, self.cout = conv.N * conv.H * conv.W, conv.C, conv.K
            self.x_shape = (conv.N, conv.H, conv.W, conv.C)
            self.w_shape = (conv.K, conv.R, conv.S, conv.C)
            self.z_shape = (conv.N, conv.H, conv.W, conv.K)
        else:
            d.batch, d.in_features, d.out_features = batch, in_features, out_features
            self.rows, self.cin, self.cout = batch, in_features, out_features
            self.x_shape, self.w_shape, self.z_shape = (batch, in_features), (in_features, out_features), (batch, out_features)
        d.relu, d.seed, d.tensor_id8, d.tensor_id16 = int(relu), seed, tensor_id8, tensor_id16
        self.desc = d
        dev = self.device
        e = lambda shape, dt: torch.empty(shape, dtype=dt, device=dev)
        self.w_codes = e(self.w_shape, torch.int8)
        self.qw, self.qg8, self.qg16 = (B.new_qparams(1, dev) for _ in range(3))
        self.rq_in = None
        if input_from is not None:
            assert input_from.rq_out is not None and input_from.z_shape == self.x_shape
            self.x_codes, self.qx = input_from.out_codes, input_from.q_out
            self.rq_in = input_from.rq_out
            self.x_chan_sums = input_from.out_chan_sums
        else:
            self.x_codes, self.qx = e(self.x_shape, torch.int8), B.new_qparams(1, dev)
            self.x_chan_sums = e((self.cin,), torch.int64) if conv is not None and self.rows < (1 << 22) else None
        self.rq_out = None
        if emit_codes:
            self.out_codes, self.q_out = e(self.z_shape, torch.int8), B.new_qparams(1, dev)
            self.out_row_sums = e((self.rows,), torch.int32)
            self.out_chan_sums = e((self.cout,), torch.int64) if conv is not None and self.rows < (1 << 22) else None
            self.rq_out = B.requant(self.out_codes, self.q_out, self.out_row_sums, self.out_chan_sums)
        assert keep_z or (emit_codes and not keep_y)
        self.z = e(self.z_shape, torch.float32) if keep_z else None
        self.g = e(self.z_shape, torch.float32) if (keep_z and keep_g) else None
        self.save_mean, self.save_min, self.save_max = (e((self.cout,), torch.float32) for _ in range(3))
        bshape = self.z_shape if keep_z else (0,)          # (no backward pass without z)
        self.g8, self.ghi, self.glo = e(bshape, torch.int8), e(bshape, torch.int8), e(bshape, torch.uint8)
        assert keep_y or emit_codes
        self.y = e(self.z_shape, torch.float32) if keep_y else None
        self.dx, self.dw = e(self.x_shape, torch.float32), e(self.w_shape, torch.float32)
        self.dgamma, self.dbeta = e((self.cout,), torch.float32), e((self.cout,), torch.float32)
        self.ws = torch.empty(max(B.qbp_layer_workspace_bytes(d), 256), dtype=torch.uint8, device=dev)
        c = B.LayerCtx()
        for name, t in (("x_codes", self.x_codes), ("qx", self.qx), ("w_codes", self.w_codes), ("qw", self.qw),
                        ("z", self.z), ("save_mean", self.save_mean), ("save_min", self.save_min),
                        ("save_max", self.save_max), ("g", self.g), ("g8", self.g8), ("qg8", self.qg8),
                        ("g_hi", self.ghi), ("g_lo", self.glo), ("qg16", self.qg16), ("x_chan_sums", self.x_chan_sums)):
            setattr(c, name, t.data_ptr() if t is not None and t.numel() else None)
        self.ctx = c
        self.gamma = self.beta = None

    def forward(self, x, w, gamma=None, beta=None):
        """x: the fp32 input, or None for a layer built with input_from (its input codes are already there)."""
        self.gamma, self.beta = gamma, beta
        assert (x is None) == (self.rq_in is not None)
        if self.rq_in is None and self.rq_out is None:
            return B.qbp_layer_fwd(self.desc, x, w, gamma, beta, self.y, self.ctx, self.ws)
        return B.qbp_layer_fwd_chained(self.desc, x, self.rq_in, w, gamma, beta, self.y, self.rq_out, self.ctx, self.ws)

    def backward(self, dy):
        return B.qbp_layer_bwd(self.desc, self.ctx, dy, self.gamma, self.beta, self.dx, self.dw, self.dgamma,
                               self.dbeta, self.ws)

    def status(self) -> int:
        return B.status_word(self.ws)


class QuantizedStack:
    """A chain of quantised convolution layers, each followed by Range BN + ReLU, trained as the method prescribes
    (Sections 4 and 6): every inner activation is handed on as the 8-bit codes its Range BN wrote (no range scan and
    no quantisation pass between layers), gradients flow back through qbp_layer_bwd, and the fp32 master weights,
    gamma and beta are updated once per minibatch by qbp_sgd_update.  Buffer bookkeeping and call order only."""

    def __init__(self, convs, weights, seed=0, chained=True, keep_y=False, lr=0.1, momentum=0.9, weight_decay=1e-4,
                 device="cuda"):
        """convs: binding.ConvDesc per layer (layer i's output shape = layer i+1's input shape); weights: the fp32
        master weights (KRSC device tensors, updated in place).  chained=False runs every layer from the fp32
        activation of the one before (range scan + quantiser per layer) -- the unfused composition, for comparison."""
        self.chained, self.lr, self.momentum, self.weight_decay = chained, lr, momentum, weight_decay
        self.w = list(weights)
        self.layers = []
        n = len(convs)
        for i, conv in enumerate(convs):
            last = i == n - 1
            prev = self.layers[-1] if (self.layers and chained) else None
            self.layers.append(QuantizedLayer(conv=conv, relu=True, seed=seed, tensor_id8=i + 1, tensor_id16=i + 1, device=device,
                                              input_from=prev, emit_codes=chained and not last,
                                              keep_y=(not chained) or last or keep_y))
        dev = torch.device(device)
        self.gamma = [torch.ones(L.cout, dtype=torch.float32, device=dev) for L in self.layers]
        self.beta = [torch.zeros(L.cout, dtype=torch.float32, device=dev) for L in self.layers]
        mk = lambda ts: [torch.zeros_like(t) for t in ts] if momentum else [None] * len(ts)
        self.vw, self.vg, self.vb = mk(self.w), mk(self.gamma), mk(self.beta)

    def forward(self, x):
        a = x
        for L, w, g, b in zip(self.layers, self.w, self.gamma, self.beta):
            y = L.forward(a if L.rq_in is None else None, w, g, b)
            a = y
        return self.layers[-1].y

    def backward(self, dy):
        d = dy
        for L in reversed(self.layers):
            d, _, _, _ = L.backward(d)         # dx of a layer is the gradient at the previous layer's output
        return d

    def update(self):
        tensors = []
        for L, w, g, b, vw, vg, vb in zip(self.layers, self.w, self.gamma, self.beta, self.vw, self.vg, self.vb):
            tensors += [(w, L.dw, vw, self.weight_decay), (g, L.dgamma, vg, 0.0), (b, L.dbeta, vb, 0.0)]
        B.qbp_sgd_update_many(tensors, self.lr, self.momentum)

    def train_step(self, x, dy):
        self.forward(x)
        dx = self.backward(dy)
        self.update()
        return dx

    def status(self) -> int:
        return min(L.status() for L in self.layers)


class TernarizedLayer:
    """The low-bit form of the quantised layer (Appendix C, Ternarized Back-Propagation): 1-bit weights and activations,
    a ternary gradient for the layer-gradient product, and Algorithm 1 (the mean over `samples` ternarisations) for the
    weight gradient; Range BN after the product as in the 8-bit layer.  Call order and buffers only: binarise x and w
    -> product (the +-1 dot product of XNOR + popcount, on the int8 tensor cores) -> Range BN; backwards Range BN ->
    ternarise the gradient -> layer-gradient product; ternarise `samples` times -> weight-gradient product."""

    def __init__(self, conv=None, relu=False, seed=0, tensor_id=1, samples=1):
        self.conv, self.relu, self.seed, self.tensor_id, self.samples = conv, relu, seed, tensor_id, samples
        self.saved = None

    def forward(self, x, w, gamma=None, beta=None):
        a, qa = B.qbp_binarize_s8(x)
        wb, qw = B.qbp_binarize_s8(w)
        if self.conv is not None:
            _, z, _ = B.qbp_conv_s8_implicit(B.QBP_CONV_FPROP, self.conv, a, qa, wb, qw)
        else:
            _, z, _ = B.qbp_gemm_s8(a, qa, wb, qw)                     # x [batch x in] . w [in x out]
        y, mean, vmin, vmax, _ = B.qbp_rangebn_fwd(z, gamma, beta, relu=self.relu)
        self.saved = dict(a=a, qa=qa, wb=wb, qw=qw, z=z, mean=mean, vmin=vmin, vmax=vmax, gamma=gamma, beta=beta)
        return y

    def backward(self, dy):
        s = self.saved
        g, dgamma, dbeta = B.qbp_rangebn_bwd(dy, s["z"], s["mean"], s["vmin"], s["vmax"], s["gamma"], s["beta"], relu=self.relu)
        # sample 0 of the gradient's stream serves the layer gradient; the weight gradient draws its own samples
        t, qt = B.qbp_stc_ternarize_s8(g, samples=1, seed=self.seed, tensor_id=self.tensor_id)
        if self.conv is not None:
            _, dx, _ = B.qbp_conv_s8_implicit(B.QBP_CONV_DGRAD, self.conv, t, qt, s["wb"], s["qw"])
        else:
            _, dx, _ = B.qbp_gemm_s8(t, qt, s["wb"], s["qw"], transB=True)
        _, dw, _, _, _ = B.qbp_tbp_weight_gradient(s["a"], s["qa"], g, self.samples, seed=self.seed, tensor_id=self.tensor_id + 1,
                                                   d=self.conv)
        self.g, self.t, self.qt = g, t, qt
        return dx, dw, dgamma, dbeta


class _F8Space:
    """A layer's own workspaces: `words` of 256 bytes, each a call's status word (cleared), and the calls' scratch behind them.
    Outgrown ones are kept, because a captured graph keeps the addresses of its calls (each is twice the last one at least, so that they
    add up to no more than the newest)."""

    def __init__(self, words, device):
        self.words, self.device, self.kept = words, torch.device(device), []

    def get(self, scratch=0):
        """The workspace, with at least so many bytes behind its words."""
        need = 256 * self.words + scratch
        if not self.kept or self.kept[-1].numel() < need:
            size = max(need, 2 * self.kept[-1].numel() if self.kept else 0)
            # (one that is first asked for within a capture is not cleared: the graph would clear it in every replay, other calls' words too)
            captured = self.device.type == "cuda" and torch.cuda.is_current_stream_capturing()
            self.kept.append((torch.empty if captured else torch.zeros)(-(-size // 256) * 256, dtype=torch.uint8, device=self.device))
        return self.kept[-1]

    def at(self, word, scratch=0):
        """For a call that takes its status word and scratch in one piece: the workspace from a word on.  The call's scratch lies
        over the words behind it, whose calls have to follow this one."""
        return self.get(scratch)[256 * word:]

    def status(self) -> int:
        """0, or the status of a call that failed (synchronises the current stream).  The kernels raise one status alone; anything else is
        what a captured call that has not been replayed found in its memory."""
        failed = any(bool((t[:256 * self.words].view(torch.int32)[::64] == B.QBP_ERR_TIMEOUT).any()) for t in self.kept)
        return B.QBP_ERR_TIMEOUT if failed else 0


class F8Linear:
    """A linear layer y = x w^T in 8-bit floating point with a scale for each block of 128: the activation and the gradient are
    quantised along their rows for y and dx and along their columns for dw, the fp32 master weights w [out_features,
    in_features] in 128 x 128 blocks, once per forward.  Call order and buffers only.  grad_format: B.QBP_E5M2 gives the gradient
    the wider range.  A layer's training calls follow one another (their workspace, the codes, saved tensors and dw are its own, and the next
    step's calls write them again); serve() may be called from several streams and host threads at a time.  In a captured graph
    the calls keep their addresses: the codes are written again in place, so that a captured serve()
    answers with the weights as the last quantise() or forward() found them."""

    def __init__(self, w, grad_format=B.QBP_E4M3):
        self.w, self.grad_format = w, grad_format
        self.space = _F8Space(3, w.device)                                      # dw, dx, y
        self.serving = {}                                                       # serve()'s, by (stream, host thread)
        self.codes = self.saved = self.dw = None

    def quantise(self):
        """The weights' codes and scales, as a layer that serves keeps them until its weights change."""
        self.codes = B.qbp_quantize_f8_square(self.w, out=self.codes)
        return self.codes

    def serve(self, x, ws=None):
        """y for an activation of any number of rows, from the codes that quantise() or forward() left, outside of a capture for one (a stream
        that serves has to wait for the one that made them).  The workspace is the stream's and the host thread's own, kept with the layer; a captured graph
        whose replays may overlap other calls on the stream it was captured on takes a `ws` (qbp_linear_f8_workspace_bytes,
        its first four bytes the status word)."""
        q, s, _ = self.codes or self.quantise()
        if ws is None:
            key = B._stream_handle(self.w.get_device()), threading.get_ident()
            space = self.serving.get(key)
            if space is None: space = self.serving[key] = _F8Space(1, self.w.device)
            ws = space.get(B.qbp_linear_f8_workspace_bytes(x.numel() // max(x.shape[-1], 1), *q.shape) - 256)
        return B.qbp_linear_f8(x, q, s, ws=ws)

    def forward(self, x):
        q, s, _ = self.quantise()
        xq, sx, xqt, sxt = B.qbp_quantize_f8(x, cols=True)
        self.saved = (xqt, sxt)
        return B.qbp_gemm_f8(xq, sx, q, s, transB=True, out_dtype=x.dtype, ws=self.space.at(2))

    def backward(self, g):
        """dx in g's type; the weights' gradient is left in dw (fp32)."""
        q, _, st = self.codes
        xqt, sxt = self.saved
        gq, sg, gqt, sgt = B.qbp_quantize_f8(g, format=self.grad_format, cols=True)
        dx = B.qbp_gemm_f8(gq, sg, q, st, formatA=self.grad_format, out_dtype=g.dtype, ws=self.space.at(1))
        self.dw = B.qbp_gemm_f8(gqt, sgt, xqt, sxt, transA=True, formatA=self.grad_format, out=self.dw, ws=self.space.at(0))
        return dx

    def status(self) -> int:
        """The worst status of the layer's calls that the current stream has waited for, on whichever streams they were."""
        return min(space.status() for space in [self.space, *self.serving.values()])


class F8ResidualStack:
    """Residual blocks of one linear layer each: h = norm(x) w_pre, and for every block b = linear(h), r = alpha x + gate *
    dropout(norm(b) w_post), the next block's h = norm(r) w_pre, with the join after a block and before the next one as one pass.
    Master weights, norms and gates are fp32 and updated by qbp_sgd_update_many.  Call order and buffers only.  A captured step
    repeats its draws of the dropout: their number is an argument of its calls."""

    def __init__(self, weights, alpha=1.0, eps=1e-6, p=0.0, seed=0, lr=0.1, momentum=0.9, weight_decay=0.0, grad_format=B.QBP_E5M2):
        """weights: [C, C] fp32 device tensors, one for each block, updated in place, and so no two of them in the same memory."""
        spans = sorted((w.data_ptr(), w.data_ptr() + w.numel() * w.element_size()) for w in weights)
        if any(end > start for (_, end), (start, _) in zip(spans, spans[1:])): raise ValueError("two blocks' weights share memory: each would be updated by both gradients at once")
        self.linears = [F8Linear(w, grad_format) for w in weights]
        C, dev = weights[0].shape[0], weights[0].device
        ones = lambda: torch.ones(C, dtype=torch.float32, device=dev)
        self.w_first = ones()                                              # the norm before the first block
        self.w_post, self.w_pre, self.gate = ([ones() for _ in weights] for _ in range(3))
        self.alpha, self.eps, self.p, self.seed, self.lr, self.momentum, self.weight_decay = alpha, eps, p, seed, lr, momentum, weight_decay
        self.step = 0
        self.velocity = None
        self.saved = self.grads = None
        self.space = _F8Space(2 * (len(weights) + 1), dev)                      # the joins forward, then backward in their order

    def forward(self, x, h_dtype=torch.bfloat16):
        """x [rows, C]: the residual stream, of its own type.  Returns the last block's h (h_dtype)."""
        n = len(self.linears)
        first = B.resnorm_desc(x, eps=self.eps, h_dtype=h_dtype)
        _, h, _, q = B.qbp_resnorm_fwd(first, x, w_pre=self.w_first, ws=self.space.at(0))
        joins, r = [], x
        for i, lin in enumerate(self.linears):
            b = lin.forward(h)
            # (a stream of draws for each block and step)
            d = B.resnorm_desc(r, b, alpha=self.alpha, eps=self.eps, p=self.p, seed=self.seed, tensor_id=self.step * n + i)
            r, h, q1, q2 = B.qbp_resnorm_fwd(d, r, b, self.w_post[i], self.gate[i], self.w_pre[i], ws=self.space.at(1 + i))
            joins.append((d, b, r, q1, q2))
        self.saved = (first, x, q, joins)
        return h

    def backward(self, dh):
        """dh: the gradient at forward's result.  Returns the gradient at x; the parameters' are left in grads."""
        first, x, q, joins = self.saved
        dr, grads = None, []
        n, need = len(joins), B.qbp_resnorm_bwd_workspace_bytes(first)
        for i in reversed(range(len(joins))):
            d, b, r, q1, q2 = joins[i]
            dr, db, dw1, dg, dw2 = B.qbp_resnorm_bwd(d, dr, dh, b, r, q1, q2, self.w_post[i], self.gate[i], self.w_pre[i], ws=self.space.at(2 * n - i, need))
            dh = self.linears[i].backward(db)
            grads.append((self.linears[i].dw, dw1, dg.view(-1), dw2))
        dx, _, _, _, dw = B.qbp_resnorm_bwd(first, dr, dh, None, x, None, q, w_pre=self.w_first, ws=self.space.at(2 * n + 1, need))
        self.grads = (grads[::-1], dw)
        return dx

    def update(self):
        blocks, dw_first = self.grads
        ws = [self.w_first] + [t for i, lin in enumerate(self.linears) for t in (lin.w, self.w_post[i], self.gate[i], self.w_pre[i])]
        gs = [dw_first] + [t for g in blocks for t in g]
        if self.momentum and self.velocity is None: self.velocity = [torch.zeros_like(w) for w in ws]
        vs = self.velocity or [None] * len(ws)
        B.qbp_sgd_update_many([(w, g, v, self.weight_decay if w.dim() == 2 else 0.0) for w, g, v in zip(ws, gs, vs)], self.lr, self.momentum)
        self.step += 1

    def status(self) -> int:
        return min([self.space.status()] + [lin.status() for lin in self.linears])
