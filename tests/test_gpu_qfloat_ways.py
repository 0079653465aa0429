"""Products in 8-bit floating point by groups through every tile, and the layer element by element.

The layer's tolerance.  x and W_gate are small whole numbers (over 16): the gate product's products are multiples of 1 / 16 up to 1, of which the instruction cuts nothing, and its
fp32 sums are exact.  So hidden values are off by SiLU's arithmetic alone: the exponential's argument by half a unit of z log2(e) and of its product, 2^-23 |z| together, its result and the
reciprocal by a unit or two each, three products by half a unit each: at most (2 |z| + 16) 2^-24 of the value.  The 8 bits of a value between these ends may be those of either end, for the block's
exponent of either end of its magnitude; what an output may move by for it is the largest of these steps times the weight, summed.  Behind that the down product's cut
sums and bf16's rounding, as in test_gpu_qfloat.py."""
import numpy as np
import pytest
import torch

from oracle import qfloat_oracle as Q
from paper_2601_10639_amd import stemlib as L
from tests.test_gpu_qfloat import DEV, bf, check_linear, cut, dev, draw, i32, make_ctx, num, offsets_of, wide

pytestmark = pytest.mark.gpu

# (T, N, K, groups), (T, d, F, groups): the tiles that they reach are held in test_qfloat_ways_cpu.py
TILES = {"ring": [(4200, 2100, 4200, 2), (4500, 2304, 4096, 3), (8000, 1025, 4097, 5)], "pair": [(3000, 1500, 300, 3)], "128x128": [(2000, 1100, 520, 3)],
         "128x64": [(900, 600, 300, 3)]}
GATES = {"64x128": [(100, 128, 320, 3), (60, 64, 448, 1)], "128x128": [(1500, 192, 1600, 3), (1200, 192, 1600, 4), (1500, 192, 1600, 1)],
         "pair": [(4400, 128, 2240, 3), (4400, 128, 2240, 1)], "few": [(1, 256, 1024, 1), (7, 128, 320, 3), (8, 128, 4160, 1), (16, 192, 2112, 1)]}
flat = lambda table: [shape for shapes in table.values() for shape in shapes]


@pytest.mark.parametrize("T,N,K,groups", flat(TILES))
def test_tiles_by_groups(T, N, K, groups):
    ctx = make_ctx(T, 64, wide(K), groups=groups)
    check_linear(ctx, T, N, K, groups, offsets_of(T, T, groups, 5, T - 77), residual=True)
    check_linear(ctx, T, N, K, groups, np.array([0] + [T - 300] * (groups - 1) + [T], np.int32))     # one has nearly all rows


def ends(h, off):
    """The largest step from Q(h) to 8 bits that a value within `off` may have instead, in blocks of a row."""
    step = np.zeros_like(h)
    for lo in range(0, h.shape[1], 128):
        v, d = h[:, lo:lo + 128], off[:, lo:lo + 128]
        q = Q.blocks(v, 1)
        for top in (Q.magnitude(np.abs(v) - d, 1), Q.magnitude(np.abs(v) + d, 1)):
            s = np.ldexp(1.0, Q.exponent(top))
            for u in (v - d, v, v + d):
                other = Q.e4m3(u / s) * s                    # (a magnitude beyond the smaller exponent's largest value is none: it goes with the larger one)
                step[:, lo:lo + 128] = np.fmax(step[:, lo:lo + 128], np.abs(other - q))
    return step


@pytest.mark.parametrize("T,d,F,groups", flat(GATES))
def test_layer_element_by_element(T, d, F, groups):
    ctx, V = make_ctx(T, d, F, groups=groups), 60
    whole = lambda seed, *s: torch.randint(-4, 5, s, generator=torch.Generator().manual_seed(seed)).to(bf).to(DEV)
    x, Wg, ids = whole(1, T, d), whole(2, groups, F, d) / 16, torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(3)).to(i32).to(DEV)
    Wd, E, res = draw(4, groups, d, F, std=0.04), draw(5, V, F), draw(6, T, d)
    offsets = None if groups == 1 else offsets_of(T, T, groups, T // 9, T - T // 7)
    gate, down, y = L.stem_qfloat_weights(ctx, Wg), L.stem_qfloat_weights(ctx, Wd), torch.full((T, d), 7.0, dtype=bf, device=DEV)
    L.stem_qfloat_ffn_forward(ctx, x, ids, gate, down, E, y, residual=res, offsets=dev(offsets))
    z, _ = Q.linear(num(x), num(Wg), offsets)
    h = Q.hidden(num(x), ids.cpu().numpy(), num(Wg), num(E), offsets)
    none = np.isnan(h).any(1)
    z, h = np.where(none[:, None], 0.0, z), np.where(none[:, None], 0.0, h)
    step = ends(h, np.abs(h) * (2 * np.abs(z) + 16) * 2.0 ** -24)
    assert (step > 0).mean() < 1e-3                          # (nearly all hidden values are what they are)
    out, size = Q.linear(h, num(Wd), offsets)
    bound = np.zeros((T, d))
    for g, (lo, hi) in enumerate(Q.bounds(offsets, T, groups)):
        w = Q.squares(num(Wd[g]))
        bound[lo:hi] = step[lo:hi] @ np.abs(w).T + cut(Q.blocks(h[lo:hi], 1), w, size[lo:hi])
    want = out + num(res)
    off = np.abs(num(y) - want)
    assert (none[:, None] | (off <= np.abs(want) * (2.0 ** -8 * (1 + 2 ** -7) + 2.0 ** -22) + bound)).all(), np.nanmax(off)
    assert (num(y)[none] == 7.0).all()
