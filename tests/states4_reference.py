"""The 4-bit state store from its definition, in 64 bits on the CPU (numpy).  The attention over it is states_reference's: what a row is held as, r_g * code, takes the place of the 8-bit
codes (its products with 16-bit queries and weights are exact in the same way), the steps are steps."""
import types

import numpy as np
import torch

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def factor_of(byte):
    """The number that a byte of the factors stands for."""
    b = np.asarray(byte, np.uint16)
    return (b << 7).view(np.float16).astype(np.float64)


FACTORS = factor_of(np.arange(0x10, 0x79))          # 2^-13 .. 1


def quantise(x):
    """(codes 0 .. 15 [..., dim], bytes [..., dim / 32], steps [...]) of rows [..., dim] float32.  Every product and comparison here is exact in 64 bits."""
    x = np.asarray(x, np.float32)
    bad = ~np.isfinite(x).all(-1)
    size = np.abs(np.where(bad[..., None], 0, x)).astype(np.float64)
    groups = size.reshape(*size.shape[:-1], -1, 32)
    top = size.max(-1)
    zero = bad | (top < 2.0 ** -100)
    a = np.where(zero, 1.0, top)
    group = np.where(zero[..., None], 0.0, groups.max(-1))
    index = (FACTORS * a[..., None, None] < group[..., None]).sum(-1)          # the first that reaches the group's largest
    unit = FACTORS[index] * a[..., None]
    t, n = (24 * groups)[..., None], unit[..., None, None]          # 4 * 6 |x| against 4 times the halfway points
    borders = np.array([1, 3, 5, 7, 10, 14, 20]) * n
    up = np.array([False, True, False, True, False, True, False])              # halfway: to the even code
    code = ((t > borders) | ((t == borders) & up)).sum(-1).reshape(x.shape)
    code = np.where(zero[..., None], 0, code + 8 * np.signbit(x))
    step = np.where(bad, np.float32(np.nan), np.where(zero, np.float32(0), top.astype(np.float32) / np.float32(6))).astype(np.float32)
    return code.astype(np.uint8), (index + 0x10).astype(np.uint8), step


def values(code, byte, step):
    """What codes, bytes and steps read back as, in float."""
    c = np.where(code & 8, -LEVELS[code & 7], LEVELS[code & 7])
    held = (c.reshape(*c.shape[:-1], -1, 32) * factor_of(byte)[..., None]).reshape(c.shape)
    return held.astype(np.float32) * step[..., None]


def pack_keys(code):
    return (code[..., 0::2] | code[..., 1::2] << 4).astype(np.uint8)


def pack_values(code):
    c = code.reshape(*code.shape[:-1], -1, 2, 16)
    return (c[..., 0, :] | c[..., 1, :] << 4).astype(np.uint8).reshape(*code.shape[:-1], -1)


NAMES = ("k_codes", "v_codes", "k_factors", "v_factors", "k_scales", "v_scales")


def arrays(st):
    return {n: getattr(st, n).cpu().numpy() for n in NAMES}


def held(st):
    """The store with r_g * code in the place of codes, as the 8-bit store has them (k_codes [pages, heads, page, dim], v_codes [pages, heads, dim, page])."""
    table = torch.tensor(np.concatenate([LEVELS, -LEVELS]), dtype=torch.float64, device=st.k_codes.device)
    factor = torch.tensor(np.concatenate([np.zeros(0x10), FACTORS, np.zeros(256 - 0x79)]), dtype=torch.float64, device=st.k_codes.device)
    groups = st.dim // 32
    k = table[torch.stack([st.k_codes & 15, st.k_codes >> 4], -1).flatten(-2).long()]
    v = st.v_codes.unflatten(2, (groups, 1, 16))
    v = table[torch.cat([v & 15, v >> 4], 3).flatten(2, 4).long()]
    kf, vf = (factor[f[..., :groups].long()].repeat_interleave(32, -1) for f in (st.k_factors, st.v_factors))
    return types.SimpleNamespace(pages=st.pages, heads=st.heads, page_size=st.page_size, dim=st.dim, k_codes=k * kf, v_codes=v * vf.transpose(2, 3), k_scales=st.k_scales,
                                 v_scales=st.v_scales)
