"""Distillation where one logit has nearly all of the row's probability, at every place of a row in turn: an element that is left out
of a sum, counted twice or not written shows in its row, however long that is."""
import math

import pytest
import torch

import paper_2002_09539_b200 as lib

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]
HIGH = 30.0   # of that logit; all others are 0


def _check(V, heavy, dtype, offset, pitch, pairs):
    """Rows whose logit heavy[r] is HIGH; the teacher's one token lies half a row further (and `pairs` - 1 ids are none)."""
    N, ld = heavy.numel(), V + pitch
    x = torch.zeros(offset + N * ld, dtype=dtype, device="cuda")[offset:].view(N, ld)[:, :V]
    r = torch.arange(N, device="cuda")
    x[r, heavy] = HIGH
    token = (heavy + V // 2) % V
    ids = torch.full((N, pairs), -1, dtype=torch.int32, device="cuda")
    ids[:, pairs - 1] = token
    z, w = torch.zeros((N, pairs), device="cuda"), 0.5 + (r % 7).float() / 8
    # p: (s, 1, .. 1) / (s + V - 1) with s = e^HIGH; loss = log(s + V - 1), q = 1
    s = math.exp(HIGH)
    loss, light = math.log(s + V - 1), 1.0 / (s + V - 1)
    # the exponent -HIGH log2 e is below 64: one rounding of the product and one of the constant are 2^-19 each at most (times ln 2), the
    # exponential is off by 2 steps; taken twice, for a gradient that is the product of two of them.  The sum is 1 and V such
    # terms, and the heavy element is exact: V terms of 1e-13, in whatever order, move it by less than V 1e-13.
    rel = 2 * (2 * 2.0 ** -19 * math.log(2.0) + 4 * U)
    tol = 8 * U * loss + V * light * (1 + rel)
    plain, both = lib.distill_loss(x, ids, z), lib.distill_loss(x, ids, z, d_loss=w)
    for got in (plain, both):
        assert float((got.loss.double() - loss).abs().max()) <= tol
    i = torch.finfo(dtype)
    for d in (both.d_logits, lib.distill_backward(w, x, ids, z, plain.stats)):
        at = w.double() * (1 - (V - 1) * light)
        for place, want in ((heavy, at), (token, w.double() * (light - 1))):
            err = (d[r, place].double() - want).abs()
            assert bool((err <= want.abs() * (i.eps / 2 + 8 * U) + V * light * 2).all())
        # the other places: put the first of them there, then look at whole rows
        want = w.double() * light
        first = torch.where((heavy != 0) & (token != 0), 0, torch.where((heavy != 1) & (token != 1), 1, 2))
        if V > 2:
            d[r, heavy] = d[r, first]
            d[r, token] = d[r, first]
            tiny = want * (rel + 8 * U + i.eps / 2) + i.smallest_normal * i.eps
            assert bool(((d.amax(dim=1).double() - want) <= tiny).all()) and bool(((want - d.amin(dim=1).double()) <= tiny).all())
        del d


# rows that a warp has, that a CTA holds by 32 and by 40 elements a thread (to the last that it does), that take two passes; multiples of
# 16 bytes and not, so that rows start everywhere
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,offset,pitch,pairs", [(37, 0, 0, 1), (256, 0, 0, 1), (1001, 3, 0, 2), (1024, 0, 0, 1), (1031, 0, 0, 1), (2056, 0, 0, 3), (4096, 0, 0, 100), (4095, 1, 0, 70),
                                                  (8192, 0, 0, 1), (8199, 2, 0, 1), (16384, 0, 0, 40), (16385, 5, 0, 1), (24317, 0, 0, 1)])
def test_every_element_of_a_row_counts_once(dtype, V, offset, pitch, pairs):
    _check(V, torch.arange(V, device="cuda"), dtype, offset, pitch, pairs)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V,offset,pitch", [(39673, 0, 0), (39680, 0, 0), (39689, 3, 0), (65536, 0, 8), (50257, 1, 0)])
def test_every_element_of_a_long_row_counts_once(dtype, V, offset, pitch):
    for first in range(0, V, 8192):
        _check(V, torch.arange(first, min(V, first + 8192), device="cuda"), dtype, offset, pitch, 2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [1, 2, 5])
@pytest.mark.parametrize("V,offset,pitch", [(20000, 0, 0), (50257, 0, 0), (131072, 0, 0), (200003, 5, 0), (1000003, 1, 2)])
def test_elements_at_the_ends_of_parts_and_segments_count_once(dtype, N, V, offset, pitch):
    """Few rows: their sums go by parts, their gradients by segments.  Whatever the sizes of these, they end at multiples of
    256 elements behind the boundary at or before the row."""
    g = torch.Generator(device="cuda")
    g.manual_seed(V + N)
    ends = torch.arange(0, V + 256, 256, device="cuda")[:, None] + torch.tensor([-9, -8, -7, -1, 0, 1], device="cuda")
    places = torch.cat([ends.flatten(), torch.tensor([0, 1, V - 1, V - 2, V - 7, V - 8, V - 9], device="cuda")])
    places = places[(places >= 0) & (places < V)].unique()
    chosen = places[torch.randperm(places.numel(), generator=g, device="cuda")[:60 * N]]
    chosen = torch.cat([chosen, torch.tensor([0, V - 1, V - 8] + [V - 9] * (2 * N - 3 if N > 1 else 0), device="cuda")])
    for heavy in chosen[:chosen.numel() // N * N].view(-1, N):
        _check(V, heavy, dtype, offset, pitch, 1)
