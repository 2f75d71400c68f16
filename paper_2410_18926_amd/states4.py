"""Binding of the 4-bit state store (include/lorann_states4.h): the 8-bit store's calls (states.py) over a store that takes little more than half the memory."""
from __future__ import annotations

import torch

from .states import CStates4, States, _array

EXPORTS = ["lorann_states4_write", "lorann_states4_read", "lorann_attend4_chunk", "lorann_attend4_passages", "lorann_attend4_workspace"]


class States4(States):
    """Keys and values of tokens in 4 bits with one step per token and head and a factor for each 32 values, in pages.

    k_codes    [pages, heads, page_size, dim / 2] uint8     v_codes    [pages, heads, dim / 2, page_size] uint8 (transposed inside a page)
    k_factors  [pages, heads, page_size, 4] uint8           v_factors  the same
    k_scales   [pages, heads, page_size] float32            v_scales   the same
    The tensors stay the caller's; slot = page * page_size + place in the page.  Calls and arguments are those of States."""

    _write, _read, _chunk, _passages, _attend_room = "lorann_states4_write", "lorann_states4_read", "lorann_attend4_chunk", "lorann_attend4_passages", "lorann_attend4_workspace"
    _weights, _weights_room, _evict = "lorann_attend4_weights", "lorann_attend4_weights_workspace", "lorann_states4_evict"

    def __init__(self, k_codes, v_codes, k_factors, v_factors, k_scales, v_scales):
        self.k_codes, self.v_codes, self.k_factors, self.v_factors, self.k_scales, self.v_scales = k_codes, v_codes, k_factors, v_factors, k_scales, v_scales
        if k_codes.dim() != 4:
            raise ValueError(f"k_codes must be [pages, heads, page_size, dim / 2], got {tuple(k_codes.shape)}")
        n, h, p, half = k_codes.shape
        self.pages, self.heads, self.page_size, self.dim = n, h, p, 2 * half
        self._gpu = k_codes.device.index if k_codes.is_cuda else None
        steps, factors = (n, h, p), (n, h, p, 4)
        if not (k_codes.dtype is v_codes.dtype is k_factors.dtype is v_factors.dtype is torch.uint8 and k_scales.dtype is v_scales.dtype is torch.float32
                and v_codes.shape == (n, h, half, p) and k_factors.shape == factors and v_factors.shape == factors and k_scales.shape == steps and v_scales.shape == steps
                and k_codes.is_contiguous() and v_codes.is_contiguous() and k_factors.is_contiguous() and v_factors.is_contiguous() and k_scales.is_contiguous() and v_scales.is_contiguous()):
            for t, dtype, shape, what in ((k_codes, torch.uint8, (n, h, p, half), "k_codes"), (v_codes, torch.uint8, (n, h, half, p), "v_codes"),
                                          (k_factors, torch.uint8, factors, "k_factors"), (v_factors, torch.uint8, factors, "v_factors"),
                                          (k_scales, torch.float32, steps, "k_scales"), (v_scales, torch.float32, steps, "v_scales")):
                _array(t, dtype, shape, what)          # (says which)
        self._st = CStates4(k_codes.data_ptr(), v_codes.data_ptr(), k_factors.data_ptr(), v_factors.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(), n, h, p, 2 * half)

    @classmethod
    def empty(cls, pages: int, heads: int, page_size: int, dim: int, device="cuda") -> "States4":
        """A store of zeros."""
        if dim % 2:
            raise ValueError(f"two values share a byte: dim {dim} is odd")
        z = lambda *shape, t=torch.uint8: torch.zeros(shape, dtype=t, device=device)  # noqa: E731
        return cls(z(pages, heads, page_size, dim // 2), z(pages, heads, dim // 2, page_size), z(pages, heads, page_size, 4), z(pages, heads, page_size, 4),
                   z(pages, heads, page_size, t=torch.float32), z(pages, heads, page_size, t=torch.float32))
