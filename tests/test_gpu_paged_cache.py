"""The paged cache on the GPU: appending, attention of one new token with the weights of the cached tokens, eviction; each against
plain 64-bit loops, at the sizes and masks where it can go wrong, and all of them as a decoding loop runs them."""
import os

import numpy as np
import pytest
import torch

from paper_2605_13915_b200 import binding, inputs
from paged_reference import attention, evicted, make_cache, sequence

pytestmark = pytest.mark.gpu

HALF_BF16 = torch.finfo(torch.bfloat16).eps / 2      # 2^-8: one rounding to BF16
FP32 = 2.0 ** -23                                     # one FP32 operation, rounded or cut


def _args(c):
    return c["k"], c["v"], c["k_scale"], c["v_scale"], c["table"], c["seqlens"]


def _check_attention(q, c, scale, got, lse=None, before=None, weights=None):
    """What the arithmetic allows: a score is a sum of D products in FP32, then scaled (and for INT8 scaled again): off by at most
    d = (D + 8) 2^-23 sum |q k| scale; the softmax of scores that are off by d has probabilities off by a factor e^(2d), and exp2, the
    sums and the division add a few FP32 roundings (16 are granted).  P goes into the product as two BF16 values, which leave out
    2^-16 of it (INT8: P times the value's scale, relative to the largest scale, as one FP16 value: 2^-11); the result is rounded to BF16."""
    want, want_lse, want_w, mass, reach = attention(q, c, scale)
    D = q.shape[2]
    d = (D + 8) * FP32 * reach
    rel = torch.expm1(2 * d) + 16 * FP32
    # sums over the tokens: FP32 additions in chains of at most (length / 64 + 64)
    longest = int(c["seqlens"].max()) if len(c["seqlens"]) else 0
    rel = rel + (longest / 64 + 64) * FP32
    p_rounding = 2.0 ** -16 if c["k_scale"] is None else 2.0 ** -11
    bound = HALF_BF16 * want.abs() + (p_rounding + rel[..., None]) * mass * (1 + 2 * HALF_BF16)
    assert torch.isfinite(got.float()).all()
    assert ((got.double() - want).abs() <= bound + 1e-38).all(), ((got.double() - want).abs() - bound).max()
    if lse is not None:
        empty = want_lse == float("-inf")
        assert torch.equal(lse == float("-inf"), empty)
        diff = torch.where(empty, 0.0, (lse.double() - torch.where(empty, 0.0, want_lse)).abs())
        assert (diff <= d + rel + 4 * FP32 * torch.where(empty, 0.0, want_lse.abs())).all()
    if weights is not None:
        G = q.shape[1] // c["k"].shape[2]
        for b, w in enumerate(want_w):
            n = w.shape[1]
            assert torch.equal(weights[b, :, n:], before[b, :, n:]), "weights past the last token were touched"
            r = rel[b].view(-1, G).amax(-1)[:, None] if n else 0.0
            total = before[b, :, :n].double() + w
            assert ((weights[b, :, :n].double() - total).abs() <= w * (r + G * FP32) + total * FP32 + 1e-38).all()


# (lengths, Hq, Hkv, D, Dv, page, layout): a tile is 64 or 128 tokens
SHAPES = [
    ([1], 4, 1, 64, 64, 16, "tokens"),
    ([0], 4, 1, 128, 128, 16, "tokens"),
    ([5, 0, 64, 63, 65, 0, 127, 128, 129, 1], 8, 2, 128, 128, 16, "tokens"),
    ([300, 17, 1000], 12, 12, 64, 64, 8, "heads"),
    ([700, 33], 32, 4, 128, 128, 64, "joint"),
    ([257, 600], 32, 2, 128, 128, 20, "heads"),             # 16 query heads to a KV head, pages of 20
    ([450, 31], 40, 2, 96, 96, 1, "tokens"),                # 20: a second group of heads; a page a token
    ([513, 90], 7, 1, 80, 64, 32, "tokens"),
    ([200, 1030], 10, 2, 64, 128, 128, "joint"),
    ([333, 64], 8, 1, 256, 256, 16, "heads"),
    ([129, 500], 6, 3, 192, 240, 48, "tokens"),
    ([77], 17, 1, 16, 16, 16, "tokens"),
    ([9000, 3, 0, 2500], 16, 4, 128, 128, 64, "tokens"),    # cut over many CTAs
    ([20000], 8, 1, 64, 64, 100, "tokens"),
]


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("lengths,Hq,Hkv,D,Dv,page,layout", SHAPES)
def test_attention(lengths, Hq, Hkv, D, Dv, page, layout, int8):
    c = make_cache(lengths, Hkv, D, Dv, page, int8, seed=len(lengths) + D, layout=layout)
    g = torch.Generator(device="cuda").manual_seed(5)
    q = torch.randn(len(lengths), Hq, D, generator=g, device="cuda").to(torch.bfloat16)
    before = torch.rand(len(lengths), Hkv, max(lengths) + 3, generator=g, device="cuda")
    weights = before.clone()
    out, lse = binding.attn_decode_paged(q, *_args(c), D ** -0.5, weights=weights, want_lse=True)
    binding.last_device_status()
    _check_attention(q, c, D ** -0.5, out, lse, before, weights)
    # without weights the result is the same, bit for bit
    assert torch.equal(binding.attn_decode_paged(q, *_args(c), D ** -0.5), out)
    binding.last_device_status()


@pytest.mark.parametrize("int8", [False, True])
def test_attention_of_many_short_sequences(int8):
    """More sequences than the threads that cut the list of tiles, empty ones among them."""
    g = torch.Generator().manual_seed(1)
    lengths = torch.randint(0, 90, (700,), generator=g).tolist()
    lengths[3] = lengths[698] = lengths[699] = 0
    c = make_cache(lengths, 2, 64, 64, 16, int8, seed=4)
    q = torch.randn(700, 4, 64, generator=g).to(torch.bfloat16).cuda()
    before = torch.rand(700, 2, 90, generator=g).cuda()
    weights = before.clone()
    out, lse = binding.attn_decode_paged(q, *_args(c), 0.125, weights=weights, want_lse=True)
    binding.last_device_status()
    _check_attention(q, c, 0.125, out, lse, before, weights)


@pytest.mark.parametrize("D,Dv", [(8, 24), (40, 8), (72, 136), (136, 200)])
def test_attention_with_odd_head_sizes(D, Dv):
    """BF16 heads need whole 16 bytes only."""
    c = make_cache([70, 300], 2, D, Dv, 24, seed=D)
    q = torch.randn(2, 6, D, generator=torch.Generator().manual_seed(D)).to(torch.bfloat16).cuda()
    before = torch.zeros(2, 2, 300, device="cuda")
    weights = before.clone()
    out, lse = binding.attn_decode_paged(q, *_args(c), D ** -0.5, weights=weights, want_lse=True)
    binding.last_device_status()
    _check_attention(q, c, D ** -0.5, out, lse, before, weights)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("G", [2, 11])
@pytest.mark.parametrize("D,Dv", [(80, 96), (96, 80), (160, 64), (128, 192), (192, 144), (208, 256)])
def test_attention_with_every_width_of_a_row(D, Dv, G, int8):
    """Rows are laid out in shared memory by the wider of a key and a value, rounded up to 64, 96, 128, 192 or 256."""
    c = make_cache([333, 0, 64, 700, 17], 2, D, Dv, 16, int8, seed=D + G, layout="heads")
    q = torch.randn(5, 2 * G, D, generator=torch.Generator().manual_seed(D)).to(torch.bfloat16).cuda()
    before = torch.rand(5, 2, 700, generator=torch.Generator().manual_seed(G)).cuda()
    weights = before.clone()
    out, lse = binding.attn_decode_paged(q, *_args(c), D ** -0.5, weights=weights, want_lse=True)
    binding.last_device_status()
    _check_attention(q, c, D ** -0.5, out, lse, before, weights)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("D,Dv", [(64, 64), (80, 96), (128, 112), (128, 192), (256, 64)])
@pytest.mark.parametrize("G", [17, 20, 24, 25, 40])
def test_attention_with_many_heads_to_a_kv_head(G, D, Dv, int8):
    """17 to 24 heads are one group of a CTA's slots, 33 to 48 two, where rows are not wider than 192."""
    c = make_cache([450, 0, 31, 129], 2, D, Dv, 16, int8, seed=G)
    q = torch.randn(4, 2 * G, D, generator=torch.Generator().manual_seed(G)).to(torch.bfloat16).cuda()
    before = torch.rand(4, 2, 450, generator=torch.Generator().manual_seed(D)).cuda()
    weights = before.clone()
    out, lse = binding.attn_decode_paged(q, *_args(c), D ** -0.5, weights=weights, want_lse=True)
    binding.last_device_status()
    _check_attention(q, c, D ** -0.5, out, lse, before, weights)
    assert torch.equal(binding.attn_decode_paged(q, *_args(c), D ** -0.5), out)


# calls with so few tiles that one kernel does everything, and their neighbours: (lengths, Hq, Hkv, D, Dv)
FEW = [([4000], 32, 8, 128, 128), ([4200], 32, 8, 128, 128), ([2049], 7, 1, 64, 64), ([65], 16, 16, 80, 80), ([1500], 4, 2, 256, 192), ([129], 3, 1, 192, 192),
       ([100, 0, 64, 17, 128], 10, 2, 128, 128), ([0, 1, 2, 3, 70, 5, 0, 40], 24, 8, 64, 64), ([33, 250], 32, 32, 128, 64), ([0, 0], 4, 4, 64, 64),
       ([1] * 16, 8, 8, 128, 128), ([1800], 32, 2, 128, 128), ([70, 3], 9, 1, 256, 256), ([500], 24, 2, 80, 192), ([0, 64, 200], 26, 2, 64, 64), ([(7 * i) % 61 for i in range(40)], 54, 27, 64, 64)]


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("lengths,Hq,Hkv,D,Dv", FEW)
def test_attention_over_few_tiles(lengths, Hq, Hkv, D, Dv, int8):
    B, ld = len(lengths), max(max(lengths), 1)
    c = make_cache(lengths, Hkv, D, Dv, 16, int8, seed=sum(lengths))
    q = torch.randn(B, Hq, D, generator=torch.Generator().manual_seed(D)).to(torch.bfloat16).cuda()
    before = torch.rand(B, Hkv, ld, generator=torch.Generator().manual_seed(B)).cuda()
    got = []
    for no_pdl in (-1, 1):
        binding.debug_set_option("MSD_NO_PDL", no_pdl)
        ws = binding.workspace(binding.attn_decode_paged_workspace_bytes(B, Hq, Hkv, Dv, ld))
        for _ in range(2):
            ws.fill_(255)
            weights = before.clone()
            got.append(binding.attn_decode_paged(q, *_args(c), D ** -0.5, weights=weights, want_lse=True, ws=ws) + (weights,))
    binding.last_device_status()
    _check_attention(q, c, D ** -0.5, *got[0][:2], before, got[0][2])
    for other in got[1:]:
        for x, y in zip(got[0], other):
            assert torch.equal(x, y)
    assert torch.equal(binding.attn_decode_paged(q, *_args(c), D ** -0.5), got[0][0])


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("lengths,Hq,Hkv,D,Dv", FEW)
def test_attention_over_few_tiles_where_a_cluster_is_refused(lengths, Hq, Hkv, D, Dv, int8):
    """The call goes on with two kernels, in the same workspace."""
    B, ld = len(lengths), max(max(lengths), 1)
    c = make_cache(lengths, Hkv, D, Dv, 16, int8, seed=sum(lengths))
    q = torch.randn(B, Hq, D, generator=torch.Generator().manual_seed(D)).to(torch.bfloat16).cuda()
    before = torch.rand(B, Hkv, ld, generator=torch.Generator().manual_seed(B)).cuda()
    weights = before.clone()
    binding.debug_set_option("MSD_ATTN_CLUSTER", 0)
    out, lse = binding.attn_decode_paged(q, *_args(c), D ** -0.5, weights=weights, want_lse=True)
    binding.last_device_status()
    _check_attention(q, c, D ** -0.5, out, lse, before, weights)
    assert torch.equal(binding.attn_decode_paged(q, *_args(c), D ** -0.5), out)


def test_attention_with_more_heads_than_places_on_the_machine():
    """Every CTA walks all sequences of its KV head; one query head each, and 8 groups of 16 for the others."""
    for Hq, Hkv in ((900, 900), (640, 5)):
        c = make_cache([70, 0, 33, 130], Hkv, 16, 16, 16, int8=True, seed=2)
        q = torch.randn(4, Hq, 16, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
        before = torch.rand(4, Hkv, 130, generator=torch.Generator().manual_seed(3)).cuda()
        weights = before.clone()
        out, lse = binding.attn_decode_paged(q, *_args(c), 0.25, weights=weights, want_lse=True)
        binding.last_device_status()
        _check_attention(q, c, 0.25, out, lse, before, weights)
        assert torch.equal(binding.attn_decode_paged(q, *_args(c), 0.25), out)


def test_attention_over_a_cache_in_one_piece():
    """A page that holds everything: the contiguous cache of one sequence, and one page of two that share it as a prefix."""
    c = make_cache([3000], 2, 64, 64, 5000, seed=14)
    q = torch.randn(1, 8, 64, generator=torch.Generator().manual_seed(14)).to(torch.bfloat16).cuda()
    _check_attention(q, c, 0.125, binding.attn_decode_paged(q, *_args(c), 0.125))
    c["table"], c["seqlens"] = c["table"].expand(2, 1).contiguous(), torch.tensor([3000, 1700], dtype=torch.int32, device="cuda")
    q = q.expand(2, 8, 64).contiguous()
    before = torch.zeros(2, 2, 3000, device="cuda")
    weights = before.clone()
    out = binding.attn_decode_paged(q, *_args(c), 0.125, weights=weights)
    binding.last_device_status()
    _check_attention(q, c, 0.125, out, None, before, weights)


@pytest.mark.parametrize("int8", [False, True])
def test_attention_does_not_look_at_other_places(int8):
    """What lies behind the last token, in pages of nobody and in the workspace, is poison in the other tests; here the table's unused
    entries point at pages that do not exist, and values of one sequence are huge."""
    c = make_cache([50, 77], 2, 64, 64, 16, int8, seed=15)
    wide = torch.full((2, 9), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    wide[:, :5] = torch.where(c["table"] >= 0, c["table"], 2 ** 31 - 1)
    q = torch.randn(2, 4, 64, generator=torch.Generator().manual_seed(15)).to(torch.bfloat16).cuda()
    q[1] *= 1e30
    want = binding.attn_decode_paged(q[:1], c["k"], c["v"], c["k_scale"], c["v_scale"], c["table"][:1], c["seqlens"][:1], 0.125)
    got = binding.attn_decode_paged(q, c["k"], c["v"], c["k_scale"], c["v_scale"], wide, c["seqlens"], 0.125)
    binding.last_device_status()
    assert torch.equal(got[:1], want)


def test_attention_of_nothing_but_empty_sequences():
    c = make_cache([0, 0, 0], 2, 128, 128, 16)
    q = torch.ones(3, 8, 128, dtype=torch.bfloat16, device="cuda")
    weights = torch.full((3, 2, 7), 0.5, device="cuda")
    out, lse = binding.attn_decode_paged(q, *_args(c), 0.1, weights=weights, want_lse=True)
    binding.last_device_status()
    assert (out == 0).all() and (lse == float("-inf")).all() and (weights == 0.5).all()


@pytest.mark.parametrize("int8", [False, True])
def test_attention_with_scores_far_apart(int8):
    """Scores of hundreds: the running maximum moves and most probabilities vanish."""
    c = make_cache([900, 140], 2, 128, 128, 16, int8, seed=9, scale_of_k=30.0)
    q = torch.randn(2, 8, 128, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    before = torch.zeros(2, 2, 900, device="cuda")
    weights = before.clone()
    out, lse = binding.attn_decode_paged(q, *_args(c), 1.0, weights=weights, want_lse=True)
    binding.last_device_status()
    _check_attention(q, c, 1.0, out, lse, before, weights)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("length,first,last", [(33, 32, 33), (200, 0, 200), (40000, 0, 2048), (40000, 38016, 40000), (40000, 20000, 20001)])
def test_attention_passes_nan_on(length, first, last, int8):
    """Keys that are no numbers, where a warp, a CTA or several of them see nothing else: their KV head's results are none either, and
    the other head's are what they were."""
    c = make_cache([length, 50], 2, 64, 64, 16, int8, seed=25)
    q = torch.randn(2, 8, 64, generator=torch.Generator().manual_seed(25)).to(torch.bfloat16).cuda()
    weights = [torch.zeros(2, 2, max(length, 50), device="cuda") for _ in range(2)]
    want, want_lse = binding.attn_decode_paged(q, *_args(c), 0.125, weights=weights[0], want_lse=True)
    pos = torch.arange(first, last, device="cuda")
    (c["k_scale"] if int8 else c["k"])[c["table"][0, pos // 16].long(), pos % 16, 1] = float("nan")
    out, lse = binding.attn_decode_paged(q, *_args(c), 0.125, weights=weights[1], want_lse=True)
    binding.last_device_status()
    for got, ref in ((out, want), (lse, want_lse)):
        assert got[0, 4:].isnan().all() and torch.equal(got[0, :4], ref[0, :4]) and torch.equal(got[1], ref[1])
    assert weights[1][0, 1, :length].isnan().all() and (weights[1][0, 1, length:] == 0).all() and torch.equal(weights[1][0, 0], weights[0][0, 0])
    assert torch.equal(weights[1][1], weights[0][1])


@pytest.mark.parametrize("lengths,Hq,Hkv,D", [([1, 33], 4, 2, 64), ([200], 32, 8, 128), ([9000, 700], 16, 4, 128), ([40000], 20, 1, 64), ([450], 40, 2, 192),
                                              ([3000], 2, 2, 256)])
def test_attention_of_infinite_values(lengths, Hq, Hkv, D):
    """An infinity among the values of a token comes out as one, whatever the bits of the token's probability are: of every head that reads
    it, and the rest of the results is what it was.  (Probabilities are above 2^-40 here.)"""
    c = make_cache(lengths, Hkv, D, D, 16, seed=33)
    g = torch.Generator().manual_seed(33)
    q = torch.randn(len(lengths), Hq, D, generator=g).to(torch.bfloat16).cuda()
    want, want_lse = binding.attn_decode_paged(q, *_args(c), D ** -0.5, want_lse=True)
    G = Hq // Hkv
    there = torch.zeros(want.shape, device="cuda")
    for b, n in enumerate(lengths):
        for d in range(1, D - 1):
            j, h, sign = int(torch.randint(n, (1,), generator=g)), d % Hkv, 1 - 2 * (d // Hkv % 2)
            c["v"][c["table"][b, j // 16], j % 16, h, d] = sign * float("inf")
            there[b, h * G:(h + 1) * G, d] = sign
    out, lse = binding.attn_decode_paged(q, *_args(c), D ** -0.5, want_lse=True)
    binding.last_device_status()
    assert torch.equal(out, torch.where(there == 0, want, (there * float("inf")).to(torch.bfloat16))) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("factor", [1e38, -1e38, 1e-24])
@pytest.mark.parametrize("lengths,Hq,Hkv,D", [([1, 33], 4, 2, 64), ([200], 32, 8, 128), ([9000, 700], 16, 4, 128), ([40000], 20, 1, 64), ([3000], 2, 2, 256)])
def test_attention_of_values_at_the_ends_of_their_range(lengths, Hq, Hkv, D, factor, int8):
    """Values of 1e38 to 3e38, whose sum over the tokens no FP32 number holds, and of 1e-24: their mean is a number of that size."""
    c = make_cache(lengths, Hkv, D, D, 16, int8, seed=34, poison=False)
    g = torch.Generator().manual_seed(34)
    if int8:
        c["v"].copy_(torch.randint(1, 128, c["v"].shape, generator=g))
        c["v_scale"].copy_((torch.rand(c["v_scale"].shape, generator=g) + 1.25) * abs(factor) / 127)
        if factor < 0:
            c["v"].neg_()
    else:
        c["v"].copy_(((torch.rand(c["v"].shape, generator=g) * 2 + 1) * factor).to(torch.bfloat16))
    q = torch.randn(len(lengths), Hq, D, generator=g).to(torch.bfloat16).cuda()
    before = torch.zeros(len(lengths), Hkv, max(lengths), device="cuda")
    weights = before.clone()
    out, lse = binding.attn_decode_paged(q, *_args(c), D ** -0.5, weights=weights, want_lse=True)
    binding.last_device_status()
    _check_attention(q, c, D ** -0.5, out, lse, before, weights)


def test_attention_with_unequal_scales():
    """Values whose scales are a million times apart.  P times the scale is FP16 in units of the largest scale: below 2^-21 of it the
    error is 2^-32 of that scale (rounded up to a power of two) for each token, times its code."""
    c = make_cache([700, 90], 2, 64, 64, 16, int8=True, seed=16, poison=False)
    g = torch.Generator().manual_seed(16)
    c["v_scale"] *= torch.exp2(torch.randint(-10, 11, c["v_scale"].shape, generator=g)).cuda()
    c["k_scale"] *= torch.exp2(torch.randint(-4, 1, c["k_scale"].shape, generator=g)).cuda()
    q = torch.randn(2, 8, 64, generator=g).to(torch.bfloat16).cuda()
    out = binding.attn_decode_paged(q, *_args(c), 0.125)
    binding.last_device_status()
    want, _, _, mass, reach = attention(q, c, 0.125)
    rel = torch.expm1(2 * (64 + 8) * FP32 * reach) + (16 + 700 / 64 + 64) * FP32
    small = 2.0 ** -32 * 2 * float(c["v_scale"].max()) * 127 * 700
    bound = HALF_BF16 * want.abs() + (2.0 ** -11 + rel[..., None]) * mass * (1 + 2 * HALF_BF16) + small
    assert ((out.double() - want).abs() <= bound).all()


def test_attention_takes_slices_of_a_projection():
    """q as a slice of a fused projection's result, on another stream than the default one."""
    c = make_cache([130, 40], 2, 64, 64, 16, seed=3)
    qkv = torch.randn(2, 8 + 4, 64, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    q = qkv[:, :8]
    want = binding.attn_decode_paged(q.contiguous(), *_args(c), 0.125)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = binding.attn_decode_paged(q, *_args(c), 0.125)
    s.synchronize()
    assert torch.equal(got, want)
    _check_attention(q, c, 0.125, got)


@pytest.mark.parametrize("int8", [False, True])
def test_attention_gives_equal_bits_and_replays(int8):
    """Equal inputs give equal bits, captured or not; a workspace full of rubbish does no harm; lengths may change between replays."""
    c = make_cache([5000, 700, 64], 4, 128, 128, 16, int8, seed=6)
    q = torch.randn(3, 16, 128, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16).cuda()
    weights = torch.zeros(3, 4, 5000, device="cuda")
    ws = binding.workspace(binding.attn_decode_paged_workspace_bytes(3, 16, 4, 128, 5000))
    ws.fill_(0xFF)
    out = torch.empty(3, 16, 128, dtype=torch.bfloat16, device="cuda")
    call = lambda: binding.attn_decode_paged(q, *_args(c), 0.1, weights=weights, ws=ws, out=out)
    call()
    want, want_w = out.clone(), weights.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        call()
        with torch.cuda.graph(graph, stream=side):
            call()
    torch.cuda.synchronize()
    for _ in range(2):
        weights.zero_()
        out.zero_()
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(weights, want_w)
    c["seqlens"].copy_(torch.tensor([17, 0, 40], dtype=torch.int32))
    weights.zero_()
    graph.replay()
    torch.cuda.synchronize()
    binding.last_device_status()
    _check_attention(q, c, 0.1, out, None, torch.zeros_like(weights), weights)


def test_launches_without_overlap_give_the_same():
    """Kernels that may start before their predecessors end (and wait for them) against kernels that may not."""
    c = make_cache([900, 100], 2, 64, 64, 16, int8=True, seed=24)
    q = torch.randn(2, 8, 64, generator=torch.Generator().manual_seed(24)).to(torch.bfloat16).cuda()
    got = []
    for off in (-1, 1):
        binding.debug_set_option("MSD_NO_PDL", off)
        w = torch.zeros(2, 2, 900, device="cuda")
        for _ in range(3):
            out = binding.attn_decode_paged(q, *_args(c), 0.125, weights=w)
        got.append((out, w))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_attention_reports_pages_and_lengths_that_do_not_exist():
    c = make_cache([100, 100], 1, 64, 64, 16, seed=2)
    q = torch.ones(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    want = binding.attn_decode_paged(q, *_args(c), 0.1)
    binding.last_device_status()
    for bad in (-1, c["k"].shape[0], 2 ** 31 - 1):
        t = c["table"].clone()
        t[0, 2] = bad
        got = binding.attn_decode_paged(q, c["k"], c["v"], None, None, t, c["seqlens"], 0.1)
        with pytest.raises(binding.MsdError, match="BAD_SHAPE"):
            binding.last_device_status()
        assert torch.equal(got[1], want[1])
    for bad in (-5, 113):
        got = binding.attn_decode_paged(q, c["k"], c["v"], None, None, c["table"], torch.tensor([bad, 100], dtype=torch.int32, device="cuda"), 0.1)
        with pytest.raises(binding.MsdError, match="BAD_SHAPE"):
            binding.last_device_status()
        assert torch.equal(got[1], want[1])
    # weights with room for fewer positions than a sequence has
    weights = torch.zeros(2, 1, 50, device="cuda")
    binding.attn_decode_paged(q, *_args(c), 0.1, weights=weights)
    with pytest.raises(binding.MsdError, match="BAD_SHAPE"):
        binding.last_device_status()


def test_attention_past_32_bit_offsets():
    """A cache of more than 4 GB whose last pages are in use."""
    page, Hkv, D = 64, 8, 128
    blocks = (5 << 30) // (page * Hkv * D * 2)
    small = make_cache([300, 150], Hkv, D, D, page, seed=8, spare=0)
    k = torch.zeros(blocks, page, Hkv, D, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    n = small["k"].shape[0]
    k[-n:], v[-n:] = small["k"], small["v"]
    table = torch.where(small["table"] >= 0, small["table"] + (blocks - n), -1).int()
    q = torch.randn(2, 16, D, generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).cuda()
    got = binding.attn_decode_paged(q, k, v, None, None, table, small["seqlens"], 0.1)
    binding.last_device_status()
    assert torch.equal(got, binding.attn_decode_paged(q, *_args(small), 0.1))
    _check_attention(q, small, 0.1, got)


# ---- append ----------------------------------------------------------------------------------------------------------------
def _append_reference(c, k_new, v_new, cu):
    """The cache after the append, on the host; INT8 codes by the numpy quantizer that the tests of the other kernels use."""
    k, v = c["k"].cpu().clone(), c["v"].cpu().clone()
    ks, vs = (None, None) if c["k_scale"] is None else (c["k_scale"].cpu().clone(), c["v_scale"].cpu().clone())
    table, lengths, page = c["table"].cpu(), c["seqlens"].tolist(), c["k"].shape[1]
    for b, n in enumerate(lengths):
        m = cu[b + 1] - cu[b]
        for i in range(m):
            pos = n - m + i
            blk, slot = int(table[b, pos // page]), pos % page
            for pool, scale, new in ((k, ks, k_new), (v, vs, v_new)):
                row = new[cu[b] + i].cpu()
                if scale is None:
                    pool[blk, slot] = row
                else:
                    codes, s = inputs.quantize_rows_int8(row.contiguous().view(torch.int16).numpy().view(np.uint16))
                    pool[blk, slot], scale[blk, slot] = torch.from_numpy(codes), torch.from_numpy(s)
    return k, v, ks, vs


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("lengths,new,Hkv,D,Dv,page,layout", [
    ([1], [1], 1, 64, 64, 16, "tokens"),
    ([40, 0, 7, 129], [1, 0, 7, 30], 8, 128, 128, 16, "tokens"),
    ([300, 20], [300, 0], 3, 80, 96, 20, "heads"),
    ([65, 64, 63], [65, 1, 2], 5, 256, 144, 1, "joint"),
    ([33] * 70, [1] * 70, 2, 128, 64, 32, "tokens"),
])
def test_append(lengths, new, Hkv, D, Dv, page, layout, int8):
    c = make_cache(lengths, Hkv, D, Dv, page, int8, seed=D, layout=layout, poison=False)
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    g = torch.Generator().manual_seed(7)
    pad = 3                                               # rows behind the last sequence's, as in a padded batch
    kv = torch.randn(cu[-1] + pad, Hkv * (D + Dv), generator=g).to(torch.bfloat16)
    # short integers times a power of two: quotients that lie on or near a half; and rows of zeros, tiny and huge values
    kv[:: 2] = (torch.randint(-127, 128, kv[::2].shape, generator=g).float() * 0.5).to(torch.bfloat16)
    kv[0, :D] = 0
    kv[-pad - 1] *= 2.0 ** -120
    kv[cu[-1] // 2] *= 2.0 ** 118
    kv = kv.cuda()
    k_new, v_new = kv[:, :Hkv * D].unflatten(1, (Hkv, D)), kv[:, Hkv * D:].unflatten(1, (Hkv, Dv))      # slices: rows with a stride
    weights = torch.full((len(lengths), Hkv, max(lengths) + 2), 0.25, device="cuda")
    want = _append_reference(c, k_new, v_new, cu)
    binding.kv_append_paged(k_new, v_new, *_args(c), torch.tensor(cu, dtype=torch.int32, device="cuda"), weights=weights)
    binding.last_device_status()
    for got, ref in zip((c["k"], c["v"], c["k_scale"], c["v_scale"]), want):
        if ref is not None:
            bits = {1: torch.int8, 2: torch.int16, 4: torch.int32}[ref.element_size()]
            assert torch.equal(got.cpu().contiguous().view(bits), ref.contiguous().view(bits))
    for b, n in enumerate(lengths):
        m = new[b]
        assert (weights[b, :, n - m:n] == 0).all() and (weights[b, :, :n - m] == 0.25).all() and (weights[b, :, n:] == 0.25).all()


def test_append_quantises_every_largest_value():
    """Each positive finite BF16 number as the largest of a row, the others at or next to halves of a step."""
    top = torch.arange(1, 0x7F80, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    n = top.numel()
    step = torch.arange(15).float() * 9 - 60.5
    rows = torch.cat([top[:, None], (top.float()[:, None] / 127 * step).to(torch.bfloat16)], 1).view(n, 1, 16)
    c = make_cache([n], 1, 16, 16, 64, int8=True, poison=False)
    want = _append_reference(c, rows, rows.flip(2), [0, n])
    binding.kv_append_paged(rows.cuda(), rows.flip(2).contiguous().cuda(), *_args(c), torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    binding.last_device_status()
    for got, ref in zip((c["k"], c["v"], c["k_scale"].view(torch.int32), c["v_scale"].view(torch.int32)),
                        (want[0], want[1], want[2].view(torch.int32), want[3].view(torch.int32))):
        assert torch.equal(got.cpu(), ref)


def test_append_quantises_every_pair_of_significands():
    """Each significand of a row's largest value m with each of x, |x| <= m, at every difference of their exponents that gives a
    quotient of at least a quarter, both signs: the codes are those of IEEE divisions."""
    sig = torch.arange(128, 256).float()
    x = (sig[:, None] * torch.exp2(-torch.arange(10).float())).flatten()          # 1280 values from 255 down to 128 / 512
    rows = []
    for m in sig:
        v = x[x <= m]
        v = torch.cat([v, -v])
        v = torch.cat([v, torch.zeros(-len(v) % 127)]).view(-1, 127)
        rows.append(torch.cat([torch.full((len(v), 1), float(m)), v], 1))
    rows = torch.cat(rows).to(torch.bfloat16)[:, None]                            # [n, 1, 128], a power of two times small integers: exact
    n = len(rows)
    other = (rows.float() * 2.0 ** 60).to(torch.bfloat16)
    c = make_cache([n], 1, 128, 128, 64, int8=True, poison=False)
    want = _append_reference(c, rows, other, [0, n])
    binding.kv_append_paged(rows.cuda(), other.cuda(), *_args(c), torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    binding.last_device_status()
    for got, ref in zip((c["k"], c["v"], c["k_scale"].view(torch.int32), c["v_scale"].view(torch.int32)),
                        (want[0], want[1], want[2].view(torch.int32), want[3].view(torch.int32))):
        assert torch.equal(got.cpu(), ref)


@pytest.mark.parametrize("what", ["nan", "inf", "-inf", "nan and inf", "only nan"])
@pytest.mark.parametrize("D,Dv", [(64, 64), (128, 112), (256, 144)])
def test_append_passes_on_what_is_no_finite_number(D, Dv, what):
    """A NaN or an infinity in a row of an INT8 cache: alone in its 16 bytes, beside the row's largest finite value, in the last piece of
    the row (the second one of its lane where rows are wide), in a key or in a value.  The row's scale tells of it and its codes are 0;
    all other rows are what they would be."""
    g = torch.Generator().manual_seed(D)
    n, Hkv = 24, 3
    new = {"k": torch.randn(n, Hkv, D, generator=g).to(torch.bfloat16), "v": torch.randn(n, Hkv, Dv, generator=g).to(torch.bfloat16)}
    bad = {x: torch.zeros(n, Hkv, dtype=torch.bool) for x in new}
    for i in range(0, n, 2):
        x, h = "kv"[i // 2 % 2], i // 4 % Hkv
        row = new[x][i, h]
        at = (0, 9, len(row) - 8, len(row) - 1, len(row) // 2)[i // 2 % 5]
        if i % 3 == 0:
            row[at ^ 1] = 300.0                                   # in the same 16 bytes
        if what == "only nan":
            row[:] = float("nan")
        else:
            row[at] = float(what.split()[0])
            if what == "nan and inf":
                row[(at + 16) % len(row)] = float("inf")
        bad[x][i, h] = True
    c = make_cache([n], Hkv, D, Dv, 16, int8=True, poison=False)
    finite = {x: torch.where(bad[x][..., None], torch.zeros_like(new[x]), new[x]) for x in new}
    want = _append_reference(c, finite["k"], finite["v"], [0, n])
    binding.kv_append_paged(new["k"].cuda(), new["v"].cuda(), *_args(c), torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    binding.last_device_status()
    pos, table = torch.arange(n), c["table"].cpu()
    for x, codes, scales, ref_codes, ref_scales in (("k", c["k"], c["k_scale"], want[0], want[2]), ("v", c["v"], c["v_scale"], want[1], want[3])):
        assert torch.equal(codes.cpu(), ref_codes), x             # (zeros in the rows that are no numbers)
        scales, ref_scales = (s.cpu()[table[0, pos // 16].long(), pos % 16] for s in (scales, ref_scales))
        assert torch.equal(scales[~bad[x]].view(torch.int32), ref_scales[~bad[x]].view(torch.int32)), x
        none = scales[bad[x]]
        assert (none.isnan() if "nan" in what else none == float("inf")).all(), x


def test_attention_over_appended_rows_that_are_no_numbers():
    """What an INT8 cache was given as NaN comes out as NaN, as from a BF16 cache, and only from the KV head that was given it."""
    new = torch.randn(2, 40, 2, 64, generator=torch.Generator().manual_seed(31)).to(torch.bfloat16).cuda()
    new[0, 7, 1, 3] = new[1, 30, 0, 60] = float("nan")
    cu = torch.tensor([0, 40], dtype=torch.int32, device="cuda")
    q = torch.randn(1, 4, 64, generator=torch.Generator().manual_seed(32)).to(torch.bfloat16).cuda()
    for int8 in (False, True):
        c = make_cache([40], 2, 64, 64, 16, int8, poison=False)
        binding.kv_append_paged(new[0], new[1], *_args(c), cu)
        out, lse = binding.attn_decode_paged(q, *_args(c), 0.125, want_lse=True)
        binding.last_device_status()
        assert lse[0, :2].isfinite().all() and lse[0, 2:].isnan().all()
        assert out[0, 2:].isnan().all() and out[0, :2, 60].isnan().all() and (int8 or out[0, :2, :60].isfinite().all())


def test_append_reports_what_does_not_fit():
    c = make_cache([20, 20], 2, 64, 64, 16, seed=1, poison=False)
    new = torch.ones(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    cu = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    before = c["k"].clone()

    def reported(table, lengths, cu=cu):
        binding.kv_append_paged(new, new, c["k"], c["v"], None, None, table, lengths, cu)
        with pytest.raises(binding.MsdError, match="BAD_SHAPE"):
            binding.last_device_status()

    off = torch.full_like(c["table"], -1)
    reported(off, c["seqlens"])
    reported(torch.full_like(off, c["k"].shape[0]), c["seqlens"])
    reported(c["table"], torch.tensor([33, 400], dtype=torch.int32, device="cuda"))       # no room in the table
    reported(c["table"], torch.tensor([1, -3], dtype=torch.int32, device="cuda"))         # more new tokens than tokens
    assert torch.equal(c["k"], before)


@pytest.mark.parametrize("int8", [False, True])
def test_append_reports_lengths_and_rows_that_no_new_row_points_at(int8):
    """Lengths of sequences without new tokens, more new tokens than rows, and offsets that fall are reported too; rows before the first
    sequence and behind the last one are left out, and are no fault."""
    c = make_cache([20, 20, 20], 2, 64, 64, 16, int8, seed=1, poison=False)
    new = torch.ones(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    room = c["table"].shape[1] * 16

    def append(lengths, cu, weights=None):
        binding.kv_append_paged(new, new, c["k"], c["v"], c["k_scale"], c["v_scale"], c["table"], i32(*lengths), i32(*cu), weights=weights)
        binding.last_device_status()

    for lengths, cu in (((20, 20, 20), (0, 2, 2, 4)), ((20, 0, room), (0, 0, 0, 4)), ((20, 20, 20), (1, 2, 2, 3)), ((0, 0, 0), (0, 0, 0, 0))):
        append(lengths, cu)
    append((20, 20, 20), (0, 1, 1, 2), torch.zeros(3, 2, 20, device="cuda"))
    for lengths, cu in (((20, -1, 20), (0, 2, 2, 4)), ((20, room + 1, 20), (0, 2, 2, 4)), ((2 ** 31 - 1, 20, 20), (0, 0, 0, 4)),
                        ((20, 20, 20), (0, 2, 2, 5)), ((20, 20, 20), (0, 2, 1, 4)), ((20, 20, 20), (0, 4, 5, 4)), ((20, 20, 20), (-1, 2, 2, 4)),
                        ((20, 20, 3), (0, 0, 0, 4)), ((-2, -2, -2), (0, 0, 0, 0))):
        with pytest.raises(binding.MsdError, match="BAD_SHAPE"):
            append(lengths, cu)
    with pytest.raises(binding.MsdError, match="BAD_SHAPE"):
        append((20, 21, 20), (0, 2, 2, 4), torch.zeros(3, 2, 20, device="cuda"))        # weights of fewer positions


def test_append_looks_at_every_sequence_of_a_large_batch():
    B = 5000
    c = make_cache([4] * B, 1, 16, 16, 4, seed=1, poison=False)
    new = torch.ones(3, 1, 16, dtype=torch.bfloat16, device="cuda")
    cu = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    cu[1:] = 3
    binding.kv_append_paged(new, new, *_args(c), cu)
    binding.last_device_status()
    for b in (0, 1, 127, 128, 1023, 1024, 4096, B - 1):
        lengths = c["seqlens"].clone()
        lengths[b] = -1
        binding.kv_append_paged(new, new, c["k"], c["v"], None, None, c["table"], lengths, cu)
        with pytest.raises(binding.MsdError, match="BAD_SHAPE"):
            binding.last_device_status()


# ---- eviction ----------------------------------------------------------------------------------------------------------------
def _evict_case(lengths, Hkv, D, Dv, page, budget, int8, seed, layout="tokens"):
    """A cache with pages left for what is kept; the destination pages are in random order too."""
    kept = [min(n, budget) for n in lengths]
    need = [(n + page - 1) // page for n in kept]
    c = make_cache(lengths, Hkv, D, Dv, page, int8, seed=seed, layout=layout, spare=sum(need) + 2)
    blocks = c["k"].shape[0]
    used = set(c["table"][c["table"] >= 0].tolist())
    free = [p for p in range(blocks) if p not in used]
    g = torch.Generator().manual_seed(seed + 1)
    free = [free[i] for i in torch.randperm(len(free), generator=g).tolist()]
    dst = torch.full((len(lengths), max([1] + need)), -1, dtype=torch.int32)
    for b, n in enumerate(need):
        for j in range(n):
            dst[b, j] = free.pop()
    return c, dst.cuda()


def _check_evicted(c, dst, weights, got, budget, recent, sinks, pools):
    new_seqlens, new_weights, kept = (t.cpu() for t in got)
    table, to, w = c["table"].cpu(), dst.cpu(), weights.cpu()
    page = c["k"].shape[1]
    for b, n in enumerate(c["seqlens"].tolist()):
        m = min(n, budget)
        assert int(new_seqlens[b]) == m
        for h in range(c["k"].shape[2]):
            stay = evicted(w[b, h].tolist(), n, budget, recent, sinks)
            assert kept[b, h, :m].tolist() == stay
            if not m:
                continue
            src, at = torch.tensor(stay), torch.arange(m)
            assert torch.equal(new_weights[b, h, :m].view(torch.int32), w[b, h, src].view(torch.int32))
            for pool, before in pools:
                if pool is None:
                    continue
                a = pool.cpu()[to[b, at // page].long(), at % page, h]
                r = before[table[b, src // page].long(), src % page, h]
                bits = {1: torch.int8, 2: torch.int16, 4: torch.int32}[a.element_size()]
                assert torch.equal(a.contiguous().view(bits), r.contiguous().view(bits))


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("lengths,Hkv,D,Dv,page,budget,recent,sinks,layout", [
    ([1, 0, 5], 1, 64, 64, 16, 3, 1, 1, "tokens"),
    ([700, 90, 512, 0, 64], 4, 128, 128, 16, 64, 10, 4, "tokens"),
    ([300, 1000], 2, 80, 96, 20, 257, 0, 0, "heads"),
    ([3000, 2100], 2, 128, 64, 64, 2048, 0, 2048, "tokens"),     # nothing but the first ones
    ([777], 3, 256, 144, 32, 500, 500, 0, "joint"),               # nothing but the last ones
    ([40], 1, 16, 16, 1, 1, 0, 0, "tokens"),
    ([100, 100], 2, 64, 64, 16, 5000, 3, 3, "tokens"),            # room for everything
])
def test_eviction(lengths, Hkv, D, Dv, page, budget, recent, sinks, layout, int8):
    c, dst = _evict_case(lengths, Hkv, D, Dv, page, budget, int8, seed=D + budget, layout=layout)
    g = torch.Generator(device="cuda").manual_seed(3)
    weights = torch.rand(len(lengths), Hkv, max(lengths) + 1, generator=g, device="cuda").mul_(8).round_().div_(8)      # ties
    pools = [(c[x], None if c[x] is None else c[x].cpu().clone()) for x in ("k", "v", "k_scale", "v_scale")]
    got = binding.kv_evict_paged(*_args(c), weights, budget, dst, recent=recent, sinks=sinks)
    binding.last_device_status()
    _check_evicted(c, dst, weights, got, budget, recent, sinks, pools)
    # nothing but the destination rows was written
    written = torch.zeros(c["k"].shape[:2], dtype=torch.bool)
    for b, n in enumerate(lengths):
        at = torch.arange(min(n, budget))
        written[dst.cpu()[b, at // page].long(), at % page] = True
    for pool, before in pools:
        if pool is not None:
            bits = {1: torch.int8, 2: torch.int16, 4: torch.int32}[pool.element_size()]
            assert torch.equal(pool.cpu()[~written].contiguous().view(bits), before[~written].contiguous().view(bits))


@pytest.mark.parametrize("values", ["equal", "negative", "infinite", "nan", "tiny", "zeros"])
def test_eviction_orders_every_kind_of_weight(values):
    n, budget = 1500, 700
    c, dst = _evict_case([n, n - 1], 2, 16, 16, 16, budget, True, seed=4)
    w = torch.randn(2, 2, n, generator=torch.Generator().manual_seed(4))
    w = {"equal": torch.full_like(w, 0.75), "negative": -w.abs(), "infinite": torch.where(w > 1, float("inf"), torch.where(w < -1, float("-inf"), w)),
         "nan": torch.where(w > 0.2, float("nan"), w), "tiny": w * 1e-40, "zeros": torch.where(w > 0, 0.0, -0.0)}[values].cuda()
    pools = [(c[x], c[x].cpu().clone()) for x in ("k", "v", "k_scale", "v_scale")]
    got = binding.kv_evict_paged(*_args(c), w, budget, dst, recent=100, sinks=7)
    binding.last_device_status()
    _check_evicted(c, dst, w, got, budget, 100, 7, pools)


@pytest.mark.parametrize("n,room", [(2048, 2048), (2049, 2049), (9000, 9000), (16385, 16385), (70000, 70000), (140000, 140000), (3000, 140000)])
def test_eviction_of_long_sequences(n, room):
    """Rows that a CTA holds, rows for clusters of two to eight, and rows that are read again in every round; and a short sequence
    whose buffers have room for a long one."""
    budget = n // 3
    c, dst = _evict_case([n], 1, 16, 16, 64, budget, True, seed=5)
    w = torch.randn(1, 1, room, generator=torch.Generator().manual_seed(5)).mul_(3).exp_()
    w[..., ::3] = 1.0
    w = w.cuda()
    table = torch.full((1, (room + 63) // 64), -1, dtype=torch.int32, device="cuda")
    table[:, :c["table"].shape[1]] = c["table"]
    pools = [(c[x], c[x].cpu().clone()) for x in ("k", "v", "k_scale", "v_scale")]
    got = binding.kv_evict_paged(c["k"], c["v"], c["k_scale"], c["v_scale"], table, c["seqlens"], w, budget, dst, recent=50, sinks=4)
    binding.last_device_status()
    _check_evicted(c, dst, w, got, budget, 50, 4, pools)


def test_eviction_reports_what_does_not_fit():
    c, dst = _evict_case([100, 100], 1, 64, 64, 16, 40, False, seed=2)
    w = torch.rand(2, 1, 100, device="cuda")

    def reported(table, lengths, to, weights=w):
        binding.kv_evict_paged(c["k"], c["v"], None, None, table, lengths, weights, 40, to)
        with pytest.raises(binding.MsdError, match="BAD_SHAPE"):
            binding.last_device_status()

    reported(torch.full_like(c["table"], -1), c["seqlens"], dst)
    reported(c["table"], c["seqlens"], torch.full_like(dst, c["k"].shape[0]))
    reported(c["table"], torch.tensor([100, 113], dtype=torch.int32, device="cuda"), dst, torch.rand(2, 1, 200, device="cuda"))
    reported(c["table"], c["seqlens"], dst[:, :1].contiguous())                # no room for 40 tokens
    reported(c["table"], c["seqlens"], dst, w[..., :50].contiguous())          # weights of fewer positions


# ---- what the wrappers refuse ------------------------------------------------------------------------------------------------
def test_wrappers_refuse_tensors_that_do_not_fit():
    c = make_cache([40, 9], 2, 64, 64, 16, seed=1, poison=False)
    i = make_cache([40, 9], 2, 64, 64, 16, int8=True, seed=1, poison=False)
    k, v, _, _, table, n = _args(c)
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda")
    q, cu, new = z(2, 4, 64), torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), z(2, 2, 64)
    w = z(2, 2, 64, dtype=torch.float32)
    attend = lambda q=q, k=k, v=v, ks=None, vs=None, t=table, n=n, **more: binding.attn_decode_paged(q, k, v, ks, vs, t, n, 0.1, **more)
    append = lambda a=new, b=new, t=table, n=n, cu=cu, w=None: binding.kv_append_paged(a, b, k, v, None, None, t, n, cu, weights=w)
    dst = z(2, 1, dtype=torch.int32)
    evict = lambda w=w, budget=8, dst=dst, **more: binding.kv_evict_paged(k, v, None, None, table, n, w, budget, dst, **more)
    for call in (lambda: attend(q=q.float()), lambda: attend(k=k.half(), v=v.half()), lambda: attend(n=n.long()), lambda: attend(t=table.long()),
                 lambda: attend(v=i["v"]), lambda: attend(weights=w.double()), lambda: append(a=new.float()), lambda: append(cu=cu.float()),
                 lambda: evict(w=w.to(torch.bfloat16)), lambda: evict(kept=z(2, 2, 8, dtype=torch.int64))):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: attend(q=z(2, 4, 128)), lambda: attend(q=z(3, 4, 64)), lambda: attend(q=q.transpose(1, 2).contiguous().transpose(1, 2)),
                 lambda: attend(k=k.flatten(0, 1)), lambda: attend(v=v[:, :8]), lambda: attend(k=k.transpose(2, 3), v=v.transpose(2, 3)),
                 lambda: attend(ks=i["k_scale"], vs=i["v_scale"]), lambda: attend(k=i["k"], v=i["v"]), lambda: attend(k=i["k"], v=i["v"], ks=i["k_scale"]),
                 lambda: attend(t=table[:1]), lambda: attend(n=n[:1]), lambda: attend(t=table.t().contiguous().t()), lambda: attend(weights=z(2, 4, 64, dtype=torch.float32)),
                 lambda: attend(out=z(2, 4, 32)), lambda: attend(n=n.cpu()), lambda: append(a=z(3, 2, 64)), lambda: append(b=z(2, 2, 32)),
                 lambda: append(cu=cu[:2]), lambda: append(w=z(2, 1, 64, dtype=torch.float32)), lambda: evict(budget=0), lambda: evict(recent=9),
                 lambda: evict(sinks=-1), lambda: evict(dst=z(1, 1, dtype=torch.int32)), lambda: evict(kept=z(2, 2, 9, dtype=torch.int32)),
                 lambda: evict(new_weights=z(2, 1, 64, dtype=torch.float32))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: attend(q=z(2, 3, 64)), lambda: attend(ws=z(4096, dtype=torch.uint8)), lambda: attend(q=z(1, 4, 64).expand(2, 4, 64)),
                 lambda: evict(recent=5, sinks=4), lambda: evict(dst=table), lambda: evict(new_weights=z(2, 2, 7, dtype=torch.float32))):
        with pytest.raises(binding.MsdError):
            call()
    binding.last_device_status()


def test_results_in_the_place_of_inputs_are_refused():
    """Attention whose results would overwrite queries that other CTAs still read, and an eviction that writes into what it reads; buffers
    that only touch are taken."""
    c = make_cache([5000, 40], 2, 64, 64, 16, seed=35, poison=False)
    g = torch.Generator().manual_seed(35)
    q = torch.randn(2, 8, 64, generator=g).to(torch.bfloat16).cuda()
    want = binding.attn_decode_paged(q, *_args(c), 0.125)
    room = torch.zeros(4 * 8 * 64 + 8, dtype=torch.bfloat16, device="cuda")
    room[:1024] = q.flatten()
    at = lambda first: room[first:first + 1024].view(2, 8, 64)
    for first in (0, 8, 1016):
        with pytest.raises(binding.MsdError, match="UNSUPPORTED"):
            binding.attn_decode_paged(at(0), *_args(c), 0.125, out=at(first))
    assert torch.equal(binding.attn_decode_paged(at(0), *_args(c), 0.125, out=at(1024)), want)
    # between the rows of a slice
    wide = torch.zeros(2, 2048, dtype=torch.bfloat16, device="cuda")
    wide[:, :512] = q.flatten(1)
    rows = wide[:, :512].unflatten(1, (8, 64))
    assert torch.equal(binding.attn_decode_paged(rows, *_args(c), 0.125, out=wide[0, 512:1536].view(2, 8, 64)), want)
    with pytest.raises(binding.MsdError, match="UNSUPPORTED"):
        binding.attn_decode_paged(rows, *_args(c), 0.125, out=wide.flatten()[1032:2056].view(2, 8, 64))
    dst = torch.arange(2, dtype=torch.int32, device="cuda")[:, None].contiguous()
    arena = torch.zeros(100000, device="cuda")
    w = arena[:2 * 2 * 5000].view(2, 2, 5000)
    for changes in ({"new_weights": arena[19999:19999 + 64].view(2, 2, 16)}, {"new_weights": arena[:64].view(2, 2, 16)},
                    {"kept": arena[19990:19990 + 64].view(torch.int32).view(2, 2, 16)}, {"new_seqlens": c["seqlens"]}, {"new_seqlens": dst.flatten()}):
        with pytest.raises(binding.MsdError, match="UNSUPPORTED"):
            binding.kv_evict_paged(*_args(c), w, 16, dst, **changes)
    binding.last_device_status()


def test_weights_without_a_position_are_refused():
    c = make_cache([5], 2, 64, 64, 16, poison=False)
    q, none = torch.ones(1, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 2, 0, device="cuda")
    with pytest.raises(ValueError):
        binding.attn_decode_paged(q, *_args(c), 0.1, weights=none)
    with pytest.raises(ValueError):
        binding.kv_append_paged(q[:, :2], q[:, :2], *_args(c), torch.tensor([0, 1], dtype=torch.int32, device="cuda"), weights=none)


# ---- together ------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("int8", [False, True])
def test_decoding_loop(int8):
    """Prompts go in, tokens are decoded, the cache is shortened and decoding goes on: the whole run against one that keeps its rows in
    plain lists."""
    Hq, Hkv, D, page, budget = 8, 2, 64, 16, 48
    prompts, steps = [50, 7, 64], 12
    B, ld, width = len(prompts), 96, 6
    g = torch.Generator().manual_seed(11)
    blocks = 2 * B * width
    k = torch.zeros(blocks, page, Hkv, D, dtype=torch.int8 if int8 else torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    ks, vs = (torch.zeros(blocks, page, Hkv, device="cuda"), torch.zeros(blocks, page, Hkv, device="cuda")) if int8 else (None, None)
    tables = torch.randperm(blocks, generator=g).int().view(2, B, width).cuda()
    weights = torch.full((B, Hkv, ld), float("nan"), device="cuda")               # nothing of it may show
    lengths = list(prompts)
    rows = [{"k": [[] for _ in range(Hkv)], "v": [[] for _ in range(Hkv)], "w": [[] for _ in range(Hkv)]} for _ in range(B)]

    def stored(x):                                        # what the cache holds for a row, 64 bits
        if not int8:
            return x.double()
        codes, s = inputs.quantize_rows_int8(x.contiguous().view(torch.int16).numpy().view(np.uint16))
        return torch.from_numpy(codes).double() * torch.from_numpy(np.asarray(s)).double()[..., None]

    def append(new_counts, table):
        cu = [0]
        for n in new_counts:
            cu.append(cu[-1] + n)
        kn, vn = (torch.randn(cu[-1], Hkv, D, generator=g).to(torch.bfloat16) for _ in range(2))
        binding.kv_append_paged(kn.cuda(), vn.cuda(), k, v, ks, vs, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"),
                                torch.tensor(cu, dtype=torch.int32, device="cuda"), weights=weights)
        for b in range(B):
            for i in range(cu[b], cu[b + 1]):
                sk, sv = stored(kn[i]), stored(vn[i])
                for h in range(Hkv):
                    rows[b]["k"][h].append(sk[h])
                    rows[b]["v"][h].append(sv[h])
                    rows[b]["w"][h].append(0.0)

    at = 0
    append(prompts, tables[at])
    for step in range(steps):
        for b in range(B):
            lengths[b] += 1
        append([1] * B, tables[at])
        q = torch.randn(B, Hq, D, generator=g).to(torch.bfloat16)
        got = binding.attn_decode_paged(q.cuda(), k, v, ks, vs, tables[at], torch.tensor(lengths, dtype=torch.int32, device="cuda"), 0.125,
                                        weights=weights)
        for b in range(B):
            for h in range(Hkv):
                K, V = torch.stack(rows[b]["k"][h]), torch.stack(rows[b]["v"][h])
                heads = slice(h * Hq // Hkv, (h + 1) * Hq // Hkv)
                p = torch.softmax(q[b, heads].double() @ K.T * 0.125, -1)
                want, mass = p @ V, p @ V.abs()
                # two roundings to BF16; the FP32 part (about (D + 8) 2^-23 sum |q k| scale, twice) stays below 2^-12 here
                bound = HALF_BF16 * want.abs() + (HALF_BF16 + 2.0 ** -12) * mass
                assert ((got[b, heads].double().cpu() - want).abs() <= bound).all()
                rows[b]["w"][h] = [x + y for x, y in zip(rows[b]["w"][h], p.sum(0).tolist())]
                now = weights[b, h, :lengths[b]].double().cpu()
                ref = torch.tensor(rows[b]["w"][h])
                assert ((now - ref).abs() <= 2.0 ** -12 * ref.abs() + 1e-12).all()
        if step % 4 == 3:
            old = torch.tensor(lengths, dtype=torch.int32, device="cuda")
            new_seqlens, new_weights, kept = binding.kv_evict_paged(k, v, ks, vs, tables[at], old, weights, budget, tables[1 - at], recent=8, sinks=2)
            # which tokens stay goes by the weights as they are: compared exactly, from the same numbers
            for b in range(B):
                for h in range(Hkv):
                    stay = evicted(weights[b, h].tolist(), lengths[b], budget, 8, 2)
                    assert kept[b, h, :len(stay)].tolist() == stay
                    for x in ("k", "v", "w"):
                        rows[b][x][h] = [rows[b][x][h][j] for j in stay]
            lengths = new_seqlens.tolist()
            assert lengths == [len(rows[b]["k"][0]) for b in range(B)]
            weights, at = new_weights, 1 - at
            # the pages that were left are anybody's again
            for pool in (k, v):
                pool[tables[1 - at].flatten().long()] = 127 if int8 else float("nan")
    binding.last_device_status()


def test_the_loop_of_the_readme_goes_on_after_an_eviction():
    """README's lines, run as they stand for three steps, an eviction in each: the attention reads the tokens that were kept, on the pages
    they went to, and the new one."""
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")) as f:
        text = f.read().split("### A decoding loop around a paged cache")[1].split("\n## ")[0]
    lines = "\n".join(line[4:] for line in text.splitlines() if line.startswith("    "))
    Hkv, D, page, width, B, budget = 2, 64, 16, 20, 2, 280
    g = torch.Generator().manual_seed(36)
    c = make_cache([300, 290], Hkv, D, D, page, int8=True, seed=36, poison=False, spare=2 * B * width)
    used = set(c["table"][c["table"] >= 0].tolist())
    free = torch.tensor([x for x in range(c["k"].shape[0]) if x not in used], dtype=torch.int32)
    tables = [torch.full((B, width), -1, dtype=torch.int32, device="cuda"), free[:B * width].view(B, width).cuda()]
    tables[0][:, :c["table"].shape[1]] = c["table"]
    names = {"k": c["k"], "v": c["v"], "ks": c["k_scale"], "vs": c["v_scale"], "block_table": tables[0], "seqlens": c["seqlens"],
             "weights": torch.rand(B, Hkv, page * width, generator=g).cuda(), "cu_new": torch.arange(B + 1, dtype=torch.int32, device="cuda"),
             "scale": 0.125, "budget": budget, "ws": binding.workspace(binding.attn_decode_paged_workspace_bytes(B, 8, Hkv, D, page * width))}
    held = {x: [[list(sequence(c, b, x)[:, h].cpu()) for h in range(Hkv)] for b in range(B)] for x in ("k", "v")}      # rows of each head, in order
    spare = free[B * width:2 * B * width].view(B, width).cuda()
    for step in range(3):
        names["seqlens"] = names["seqlens"] + 1
        names["new_block_table"] = (tables[1], spare)[step % 2]
        for x in ("k", "v"):
            new = torch.randn(B, Hkv, D, generator=g).to(torch.bfloat16)
            names[x + "_new"] = new.cuda()
            codes, s = inputs.quantize_rows_int8(new.view(torch.int16).numpy().view(np.uint16))
            rows = torch.from_numpy(codes).double() * torch.from_numpy(np.asarray(s)).double()[..., None]
            for b in range(B):
                for h in range(Hkv):
                    held[x][b][h].append(rows[b, h])
        names["q"] = torch.randn(B, 8, D, generator=g).to(torch.bfloat16).cuda()
        exec(lines, names)
        binding.last_device_status()
        for b in range(B):
            for h in range(Hkv):
                K, V = torch.stack(held["k"][b][h]), torch.stack(held["v"][b][h])
                p = torch.softmax(names["q"][b, 4 * h:4 * h + 4].double().cpu() @ K.T * 0.125, -1)
                # two roundings to 8 bits or more, and the FP32 part, which stays below 2^-12 here
                bound = HALF_BF16 * (p @ V).abs() + (HALF_BF16 + 2.0 ** -12) * (p @ V.abs())
                assert ((names["out"][b, 4 * h:4 * h + 4].double().cpu() - p @ V).abs() <= bound).all(), step
                for x in ("k", "v"):
                    held[x][b][h] = [held[x][b][h][j] for j in names["kept"][b, h].tolist()]
        assert names["seqlens"].tolist() == [budget, budget]


@pytest.mark.parametrize("int8", [False, True])
def test_a_captured_step_decodes_on(int8):
    """The new token's rows go in and its query attends, in one graph that is replayed with longer sequences each time: every step as
    the eager calls on a copy of the cache."""
    Hq, Hkv, D, page, B, width = 8, 2, 128, 16, 3, 5
    g = torch.Generator().manual_seed(21)
    c = make_cache([40, 0, 13], Hkv, D, D, page, int8, seed=21, poison=False, spare=B * width)
    blocks = c["k"].shape[0]
    tables = torch.randperm(blocks, generator=g)[:B * width].view(B, width).int().cuda()
    n = torch.zeros(B, dtype=torch.int32, device="cuda")
    cu = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    kn, vn = (torch.zeros(B, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros(B, Hq, D, dtype=torch.bfloat16, device="cuda")
    pools = [c["k"], c["v"], c["k_scale"], c["v_scale"]]
    weights, out = torch.zeros(B, Hkv, page * width, device="cuda"), torch.zeros(B, Hq, D, dtype=torch.bfloat16, device="cuda")
    ws = binding.workspace(binding.attn_decode_paged_workspace_bytes(B, Hq, Hkv, D, page * width))

    def step(pools, n, weights, out):
        n += 1
        binding.kv_append_paged(kn, vn, *pools, tables, n, cu, weights=weights)
        binding.attn_decode_paged(q, *pools, tables, n, 0.1, weights=weights, ws=ws, out=out)

    eager = [None if p is None else p.clone() for p in pools]
    n2, weights2, out2 = n.clone(), weights.clone(), out.clone()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step(pools, n, weights, out)
    n.copy_(torch.tensor([37, 0, 12], dtype=torch.int32))
    n2.copy_(n)
    for _ in range(20):
        for t in (kn, vn, q):
            t.copy_(torch.randn(t.shape, generator=g))
        graph.replay()
        step(eager, n2, weights2, out2)
        torch.cuda.synchronize()
        assert torch.equal(out, out2) and torch.equal(weights, weights2) and torch.equal(n, n2)
    binding.last_device_status()
    for a, b in zip(pools, eager):
        assert a is None or torch.equal(a, b)


def test_calls_on_two_streams_at_once():
    """Workspaces of their own, work that overlaps on the GPU: the results are those of the calls alone."""
    cases = [make_cache([3000, 1200], 4, 128, 128, 16, int8, seed=22 + int8) for int8 in (False, True)]
    q = torch.randn(2, 16, 128, generator=torch.Generator().manual_seed(22)).to(torch.bfloat16).cuda()
    want = []
    for c in cases:
        w = torch.zeros(2, 4, 3000, device="cuda")
        want.append((binding.attn_decode_paged(q, *_args(c), 0.1, weights=w), w))
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        got = []
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                w = torch.zeros(2, 4, 3000, device="cuda")
                got.append((binding.attn_decode_paged(q, *_args(c), 0.1, weights=w), w))
        torch.cuda.synchronize()
        for (a, b), (x, y) in zip(want, got):
            assert torch.equal(a, x) and torch.equal(b, y)
    binding.last_device_status()


def test_append_and_eviction_past_32_bit_offsets():
    """The last pages of a cache of more than 4 GB."""
    page, Hkv, D = 64, 8, 128
    blocks = (5 << 30) // (page * Hkv * D * 2)
    k = torch.zeros(blocks, page, Hkv, D, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    table = torch.arange(blocks - 3, blocks, dtype=torch.int32, device="cuda")[None]
    dst = torch.tensor([[blocks - 4]], dtype=torch.int32, device="cuda")
    n, cu = torch.tensor([150], dtype=torch.int32, device="cuda"), torch.tensor([0, 150], dtype=torch.int32, device="cuda")
    new = torch.randn(2, 150, Hkv, D, generator=torch.Generator().manual_seed(23)).to(torch.bfloat16).cuda()
    w = torch.zeros(1, Hkv, 150, device="cuda")
    binding.kv_append_paged(new[0], new[1], k, v, None, None, table, n, cu, weights=w)
    w[:, :, 60:100] = 1.0
    _, _, kept = binding.kv_evict_paged(k, v, None, None, table, n, w, 50, dst, recent=7, sinks=3)
    binding.last_device_status()
    stay = [0, 1, 2] + list(range(60, 100)) + list(range(143, 150))
    assert kept[0, 0].tolist() == stay
    assert torch.equal(k[-3:].flatten(0, 1)[:150], new[0]) and torch.equal(v[-3:].flatten(0, 1)[:150], new[1])
    assert torch.equal(k[-4, :50], new[0, stay]) and torch.equal(v[-4, :50], new[1, stay])
    assert not k[:-4].any() and not k[-4, 50:].any()


def test_eviction_replays_from_a_graph():
    c, dst = _evict_case([600, 130], 2, 64, 64, 16, 100, True, seed=12)
    w = torch.rand(2, 2, 600, generator=torch.Generator().manual_seed(12)).cuda()
    pools = [(c[x], c[x].cpu().clone()) for x in ("k", "v", "k_scale", "v_scale")]
    got = binding.kv_evict_paged(*_args(c), w, 100, dst, recent=9, sinks=1)
    new_seqlens, new_weights, kept = got
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        binding.kv_evict_paged(*_args(c), w, 100, dst, recent=9, sinks=1, new_seqlens=new_seqlens, new_weights=new_weights, kept=kept)
    w.copy_(torch.rand(2, 2, 600, generator=torch.Generator().manual_seed(13)))
    graph.replay()
    binding.last_device_status()
    _check_evicted(c, dst, w, got, 100, 9, 1, pools)
