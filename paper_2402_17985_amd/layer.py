"""Buffer bookkeeping for one quantized linear layer (FqLinear) and for one with group-scaled 4-bit weights (FqGroupLinear): owns the
device buffers the C ABI wants (map, quantized weights, scales, workspace) and forwards to the fq_* calls.  No arithmetic."""
import numpy as np

from . import binding as B


class FqLinear:
    """Offline: plan from (chmax, T) and quantize/repeat W.  Online: forward(X) -> Y."""

    def __init__(self, W, chmax: np.ndarray, T: float, bits: int, device="cuda:0", align: int = 0):
        """align = 0 picks the flattened-width padding that makes every quantized row start on a
        128-byte boundary (128 channels for INT8, 256 for packed INT4; E3M2 storage is blocked by 128), which the
        GEMM's direct global-to-LDS copies want; any multiple of 32 (the paper's padding) is accepted
        (128 for E3M2 storage).  bits = 8, 4, or binding.FQ_BITS_I4_E3M2 (4-bit values held as 6-bit codes
        for the 6-bit matrix pipe)."""
        import torch
        self.torch = torch
        self.bits = bits
        self.N, self.K = W.shape
        if align == 0:
            align = {8: 128, 4: 256, B.FQ_BITS_I4_E3M2: 128}[bits]
        src, rep, self.Kprime, self.Kpad = B.fq_flatten_plan(chmax, T, align)
        self.src_host, self.rep_host = src, rep
        self.src = torch.from_numpy(src).to(device)
        self.rep = torch.from_numpy(rep).to(device)
        if bits == B.FQ_BITS_I4_E3M2:
            self.Wq = torch.empty((self.Kpad // 128, self.N, 96), dtype=torch.uint8, device=device)
        else:
            cols = self.Kpad if bits == 8 else self.Kpad // 2
            self.Wq = torch.empty((self.N, cols), dtype=torch.int8 if bits == 8 else torch.uint8, device=device)
        self.s_w = torch.empty(1, dtype=torch.float32, device=device)
        ws = torch.empty(B.fq_weights_workspace_bytes(self.K, self.Kpad), dtype=torch.uint8, device=device)
        B.fq_flatten_weights(W, self.src, bits, self.Wq, self.s_w, ws)
        self.device = device
        self._ws = None
        self._ws_M = 0

    def workspace(self, M: int):
        if self._ws is None or self._ws_M < M:
            nbytes = B.fq_linear_workspace_bytes(M, self.K, self.Kpad, self.bits)
            self._ws = self.torch.empty(nbytes, dtype=self.torch.uint8, device=self.device)
            self._ws_M = M
        return self._ws

    def forward(self, X, Y=None, out_dtype=None, absmax_in=None):
        M = X.shape[0]
        if Y is None:
            Y = self.torch.empty((M, self.N), dtype=out_dtype or self.torch.bfloat16, device=X.device)
        B.fq_linear(X, self.src, self.rep, self.Wq, self.s_w, self.bits, Y, self.workspace(M), absmax_in=absmax_in)
        return Y

    def forward_norm(self, X, gamma, eps: float, R=None, R_out=None, Y=None, out_dtype=None, absmax_in=None):
        """The layer on the root-mean-square norm of X (plus the residual R, whose sum goes to R_out; R_out=None: into R itself): the norm's result goes
        to the product as codes.  See fq_rms_norm_quant; absmax_in bounds the norm's result, after gamma."""
        M = X.shape[0]
        t = self.torch
        if Y is None:
            Y = t.empty((M, self.N), dtype=out_dtype or t.bfloat16, device=X.device)
        if R is not None and R_out is None:
            R_out = R
        # of this call: torch's allocator gives them to no other stream before the kernels are through
        if self.bits == B.FQ_BITS_I4_E3M2:
            Xq = t.empty((self.Kpad // 128, M, 96), dtype=t.uint8, device=X.device)
        else:
            Xq = t.empty((M, self.Kpad if self.bits == 8 else self.Kpad // 2), dtype=t.int8 if self.bits == 8 else t.uint8, device=X.device)
        s_x = t.empty(1, dtype=t.float32, device=X.device)
        ws = None if absmax_in is not None else t.empty(B.fq_rms_norm_workspace_bytes(M, self.K, self.Kpad), dtype=t.uint8, device=X.device)
        B.fq_rms_norm_quant(X, gamma, eps, R=R, R_out=R_out, src_idx=self.src, rep=self.rep, bits=self.bits, Xq_out=Xq, s_x_out=s_x, workspace=ws, absmax_in=absmax_in)
        if self.bits == B.FQ_BITS_I4_E3M2:
            B.fq_gemm_i4_e3m2(Xq, self.Wq, s_x, self.s_w, None, Y)
        else:
            (B.fq_gemm_i8 if self.bits == 8 else B.fq_gemm_i4)(Xq, self.Wq, s_x, self.s_w, Y)
        return Y


class FqGroupLinear:
    """A linear layer with 4-bit weights and a scale (and offset) for each row and group of columns; activations stay 16-bit."""

    def __init__(self, W, group: int = 128, offsets: bool = False, scale_dtype=None, bias=None, device="cuda:0"):
        """W [N, K], K a multiple of 32; group 32, 64 or 128; scale_dtype: of scales and offsets (W's type); bias fp32 [N]."""
        import torch
        self.torch = torch
        self.N, self.K = W.shape
        self.group, self.bias = group, bias
        if group not in (32, 64, 128):
            raise ValueError(f"groups of {group} columns: 32, 64 or 128")
        shape = (self.N, -(-self.K // group))
        self.Wq = torch.empty((self.N, self.K // 2), dtype=torch.uint8, device=device)
        self.S = torch.empty(shape, dtype=scale_dtype or W.dtype, device=device)
        self.B = torch.empty_like(self.S) if offsets else None
        B.fq_group_weights_i4(W, group, self.Wq, self.S, B_out=self.B)

    def forward(self, X, Y=None, out_dtype=None):
        if Y is None:
            Y = self.torch.empty((X.shape[0], self.N), dtype=out_dtype or X.dtype, device=X.device)
        B.fq_linear_group_i4(X, self.Wq, self.S, self.group, Y, B=self.B, bias=self.bias)
        return Y
