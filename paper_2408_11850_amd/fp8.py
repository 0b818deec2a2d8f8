"""8-bit operands: rows and weights in e4m3 with a scale per block of 128, and their products (see include/spec.h).

Argument marshalling only.  Every call runs on the current stream of the tensors' device; the results are that device's.
"""
from __future__ import annotations

from typing import List, Optional, Tuple

import torch

from . import EPI_STORE, EPI_SWIGLU, FP8_BLOCK, SPEC_BF16, SPEC_F32, load_library
from .binding import call_on, need as _need

_TYPES = {torch.float32: SPEC_F32, torch.bfloat16: SPEC_BF16}
E4M3 = torch.float8_e4m3fn


def _blocks(k: int) -> int:
    return -(-k // FP8_BLOCK)


def _rows(x: torch.Tensor, name: str) -> int:
    """Row stride of a matrix of rows in fp32 or bf16."""
    if not (x.is_cuda and x.dtype in _TYPES and x.dim() == 2 and (x.stride(1) == 1 or x.shape[1] == 1)):
        raise ValueError(f"{name}: rows in float32 or bfloat16 on a GPU, their elements neighbours, are wanted")
    if x.shape[0] >> 31 or x.shape[1] >> 31:           # ctypes would keep the low 32 bits
        raise ValueError(f"{name}: rows and columns below 2^31 are wanted")
    return x.stride(0) if x.shape[0] > 1 else x.shape[1]


def add_norm_fp8(h: torch.Tensor, delta: Optional[torch.Tensor], gain: torch.Tensor,
                 eps: float) -> Tuple[torch.Tensor, torch.Tensor]:
    """h += delta in place (None: nothing is added), then (q, scale) of the RMS norm of h times gain.

    h [M][d] and delta [M][d] fp32 or bf16, rows at any stride (delta's may be 0: the same row for all; it is h itself
    or shares no element with it); gain bf16 [d].
    q e4m3 [M][d], scale fp32 [ceil(d / 128)][M]."""
    ldh, (M, d), dev = _rows(h, "h"), h.shape, h.get_device()
    if not (gain.dtype is torch.bfloat16 and gain.get_device() == dev and gain.shape == (d,) and gain.is_contiguous()):
        raise ValueError("gain: bfloat16 [d] on the device of h is wanted")
    dp, dt, ldd = None, 0, 0
    if delta is not None:
        ldd = _rows(delta, "delta")
        if delta.get_device() != dev or delta.shape != h.shape:
            raise ValueError("delta: the shape and device of h are wanted")
        dp, dt = delta.data_ptr(), _TYPES[delta.dtype]
    q = h.new_empty((M, d), dtype=E4M3)
    scale = h.new_empty((_blocks(d), M), dtype=torch.float32)
    call_on(dev, load_library().spec_add_norm_quant, h.data_ptr(), _TYPES[h.dtype], ldh, dp, dt, ldd, gain.data_ptr(), eps, M, d,
            q.data_ptr(), scale.data_ptr())
    return q, scale


def quant_fp8(x: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """(q, scale) of rows x [M][K] in fp32 or bf16 at any row stride: q e4m3 [M][K], scale fp32 [ceil(K / 128)][M]."""
    ldx, (M, K) = _rows(x, "x"), x.shape
    q = x.new_empty((M, K), dtype=E4M3)
    scale = x.new_empty((_blocks(K), M), dtype=torch.float32)
    call_on(x.get_device(), load_library().spec_quant_rows, x.data_ptr(), _TYPES[x.dtype], ldx, M, K, q.data_ptr(),
            scale.data_ptr())
    return q, scale


def quant_weight_fp8(w: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """(q, scale) of a bf16 matrix [N][K]: q e4m3 [N][K], scale fp32 [ceil(N / 128)][ceil(K / 128)]."""
    _need(w.is_cuda and w.dim() == 2 and w.dtype == torch.bfloat16 and w.is_contiguous(),
          "w: a contiguous bfloat16 matrix on a GPU is wanted")
    N, K = w.shape
    _need(not (N >> 31 or K >> 31), "w: rows and columns below 2^31 are wanted")
    lib = load_library()
    q = torch.empty((N, K), dtype=E4M3, device=w.device)
    scale = torch.empty((_blocks(N), _blocks(K)), dtype=torch.float32, device=w.device)
    call_on(w.get_device(), lib.spec_quant_weight, w.data_ptr(), N, K, q.data_ptr(), scale.data_ptr())
    return q, scale


class Fp8Weight:
    """Packed e4m3 weights [N][K] and the scales of their panels."""

    __slots__ = ("data", "scale", "N", "K", "interleaved")

    def __init__(self, data: torch.Tensor, scale: torch.Tensor, N: int, K: int, interleaved: bool):
        _need(N > 0 and N % 16 == 0 and K > 0 and K % 16 == 0, "need N % 16 == 0 and K % 16 == 0")
        _need(not (N >> 31 or K >> 31), "need N and K below 2^31")
        _need(data.is_cuda and data.dtype == torch.uint8 and data.is_contiguous() and
              data.numel() == N // 16 * _blocks(K) * 2048, "data: 2048 bytes per panel of 16 rows and block of 128 are wanted")
        _need(scale.dtype == torch.float32 and scale.is_contiguous() and scale.device == data.device and
              tuple(scale.shape) == (N // 16, _blocks(K)), "scale: float32 [N / 16][ceil(K / 128)] is wanted")
        self.data, self.scale, self.N, self.K, self.interleaved = data, scale, N, K, interleaved


def pack_weights_fp8(mats: List[Tuple[torch.Tensor, torch.Tensor]], interleave: bool = False) -> Fp8Weight:
    """Packs e4m3 matrices [N_i][K] with scales [ceil(N_i / 128)][ceil(K / 128)] one behind the other, or (gate and up) with
    their panels of 16 rows interleaved."""
    _need(len(mats) > 0, "no matrices")
    K, device = mats[0][0].shape[1], mats[0][0].device
    for q, s in mats:
        _need(q.is_cuda and q.dim() == 2 and q.dtype == E4M3 and q.is_contiguous() and q.shape[1] == K and q.device == device,
              "e4m3 matrices of one width on one GPU are wanted")
        _need(s.dtype == torch.float32 and s.is_contiguous() and s.device == device and
              tuple(s.shape) == (_blocks(q.shape[0]), _blocks(K)), "scales: float32 [ceil(N / 128)][ceil(K / 128)] are wanted")
        _need(not interleave or q.shape == mats[0][0].shape, "only matrices of one shape can be interleaved")
    lib = load_library()
    N = sum(q.shape[0] for q, _ in mats)
    _need(not (N >> 31 or K >> 31), "rows, of all matrices together, and columns below 2^31 are wanted")
    _need(all(lib.spec_packed_quant_bytes(q.shape[0], K) > 0 for q, _ in mats), "need N % 16 == 0 and K % 16 == 0")
    data = torch.empty(sum(lib.spec_packed_quant_bytes(q.shape[0], K) for q, _ in mats), dtype=torch.uint8, device=device)
    scale = torch.empty((N // 16, _blocks(K)), dtype=torch.float32, device=device)
    start = 0
    for i, (q, s) in enumerate(mats):
        call_on(data.get_device(), lib.spec_pack_quant, data.data_ptr(), scale.data_ptr(), q.data_ptr(), s.data_ptr(), q.shape[0], K,
                i if interleave else start, len(mats) if interleave else 1)
        start += q.shape[0] // 16
    return Fp8Weight(data, scale, N, K, interleave and len(mats) == 2)


def gemm_fp8(x: torch.Tensor, x_scale: torch.Tensor, w: Fp8Weight, epilogue: int = EPI_STORE,
             dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """x W^T of e4m3 rows [M][K] with scales [ceil(K / 128)][M].

    epilogue 0: returns y [M][N] in bfloat16 or float32; 2: z [M][N / 2] bf16 = silu(gate) * up of weights packed with
    interleave=True."""
    (M, K), dev, N = x.shape, x.get_device(), w.N
    if not (x.is_cuda and x.dtype is E4M3 and x.is_contiguous() and not M >> 31 and K == w.K and w.data.get_device() == dev):
        raise ValueError("x: contiguous e4m3 rows of the weights' width on their device are wanted")
    if not (x_scale.dtype is torch.float32 and x_scale.is_contiguous() and x_scale.get_device() == dev and
            x_scale.shape == (_blocks(K), M)):
        raise ValueError("x_scale: float32 [ceil(K / 128)][M] is wanted")
    if dtype not in _TYPES:
        raise ValueError("results in bfloat16 or float32")
    if epilogue == EPI_SWIGLU and not w.interleaved:
        raise ValueError("epilogue 2 wants a gate and an up matrix packed with interleave=True")
    out = x.new_empty((M, N // 2 if epilogue == EPI_SWIGLU else N), dtype=dtype)
    call_on(dev, load_library().spec_gemm_quant, out.data_ptr(), _TYPES[dtype], x.data_ptr(), x_scale.data_ptr(),
            w.data.data_ptr(), w.scale.data_ptr(), M, N, K, epilogue)
    return out
