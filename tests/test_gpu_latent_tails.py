"""GPU: the absorbed form where weights differ much: one token with most of the weight before thousands of small ones, weights all
alike, against oracle/latent.py in 64 bits.

Tolerance of an output, beside its own rounding (half an ulp) and the scores', exponentials' and sums' as in test_gpu_latent.py: a
weight is off by 2^-9 (bf16, two terms of four bits) or 2^-14 (fp16, three) of itself, or by 2^-21 or 2^-25 of the largest
weight of its 64 tokens (`tiles`), which is in [2^7, 2^8) where the last term's half step is 2^-14 or 2^-18; of eight products side by
side what lies 2^-13 below the largest is dropped: 2^-10 of the sum of magnitudes of these eight.  Nothing in it grows with the number of tokens but the
sums' own 2^-24 of each addition.
"""
import numpy as np
import pytest
import torch

from oracle import latent as ref
from oracle.kv import encode

from test_gpu_latent import dev, ints, np_of
from test_gpu_rotary import LEAST, TYPES, U_OUT

pytestmark = pytest.mark.gpu

U_W = {"bf16": 2.0 ** -9, "fp16": 2.0 ** -14}
TILE = {"bf16": 2.0 ** -21, "fp16": 2.0 ** -25}


@pytest.fixture(scope="module")
def uz():
    import paper_2604_17172_amd as m
    return m


def check_weights(got, want, kind, products, tokens, dropped):
    """products: of a score, those that are not zero; dropped: of each output, the sum of magnitudes of groups of eight whose
    products differ by more than 2^6, in p |c|."""
    out, lse = got
    out, lse = np_of(out), lse.cpu().numpy().astype(np.float64)
    score = (products * 2.0 ** -24 + 2.0 ** -22) * want["size"] + 2.0 ** -21 + 2.0 ** -23 * want["shift"]
    eps = 2 * (score + tokens * 2.0 ** -24)
    assert eps.max() < 2.0 ** -6                                          # else nothing is tested
    tol = U_OUT[kind] * np.abs(want["out"]) + (U_W[kind] + 2.0 ** -14 + eps)[..., None] * want["spread"] + TILE[kind] * want["tiles"]
    tol = tol + 2.0 ** -10 * dropped + LEAST[kind]
    off = np.abs(out - want["out"])
    assert (off <= tol).all(), (np.argwhere(~(off <= tol))[:4].tolist(), np.nanmax(off / tol))
    assert (np.abs(lse - want["lse"]) <= eps + 2.0 ** -22 * np.abs(want["lse"])).all()


def attend(uz, codes, exps, rot, q, tokens, requests, scale, fmt="e4m3fn"):
    """`requests` requests of the same pages and queries [heads, width], one new token each."""
    page = codes.shape[1]
    cache = uz.LatentCache(dev(codes), dev(exps), rot, fmt)
    table = np.tile(np.arange(codes.shape[0], dtype=np.int32), (requests, 1))
    rows = q[None].expand(requests, -1, -1).contiguous()
    got = uz.latent_attend(rows, cache, ints(table), ints([tokens] * requests), ints(np.arange(requests + 1)), 1, scale)
    torch.cuda.synchronize()
    latent = codes.shape[2] - rot
    want = ref.attend(np_of(rows[:1]), codes, exps, latent, fmt, table[:1], [tokens], [0, 1], page, scale)
    return got, want


def first_token_case(kind, latent, heads, tokens, share, g):
    """Codes and exponents, and queries whose rotary part gives token 0 that share of the weight; its magnitude is in four channels, the other
    tokens' latents point one way."""
    rot, page, scale = 64, 64, 0.0625
    pages = -(-tokens // page)
    codes = g.integers(0x30, 0x41, (pages, page, latent + rot)).astype(np.uint8)  # 0.5 to 2.25
    codes[..., :latent] |= (g.integers(0, 2, latent) << 7).astype(np.uint8)
    codes[..., latent:] |= (g.integers(0, 2, (pages, page, rot)) << 7).astype(np.uint8)
    codes[..., latent] = 0
    exps = g.integers([117, 121], [120, 124], (pages, page, 2)).astype(np.uint8)
    codes[0, 0] = 0
    codes[0, 0, [3, 70, 130, 255]] = [0x70, 0xF1, 0x72, 0x73]
    codes[0, 0, latent], exps[0, 0] = 0x38, [122, 127]                    # a rotary key of 1 in its first channel
    q = np.zeros((heads, latent + rot))
    q[:, latent + 1:] = g.standard_normal((heads, rot - 1)) * 8          # scores that differ by about 0.2
    q[:, latent] = np.log(share * tokens / (1 - share)) / scale
    return codes, exps, torch.from_numpy(q.astype(np.float32)).to(TYPES[kind]).cuda(), scale


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("tokens,share", [(8190, 0.7), (8190, 0.9), (16383, 0.5), (16383, 0.7), (60000, 0.5), (60000, 0.9)])
@pytest.mark.parametrize("latent,heads,requests", [(512, 16, 256), (256, 64, 256), (512, 40, 3)])
def test_small_weights_beside_a_large_one(uz, kind, tokens, share, latent, heads, requests):
    """256 requests: a workgroup takes all of a request's tokens; 3: each is cut into pieces."""
    print("[tail]", kind, tokens, share, latent, heads, requests, flush=True)
    codes, exps, q, scale = first_token_case(kind, latent, heads, tokens, share, np.random.default_rng(61))
    got, want = attend(uz, codes, exps, 64, q, tokens, requests, scale)
    weight = np.exp(scale * np_of(q) @ np.eye(1, q.shape[1], latent)[0] - want["lse"][0])
    assert (abs(weight - share) < 0.15).all()
    sink = np.abs(ref.code_values("e4m3fn")[codes[0, 0, :latent]]) * 2.0 ** (122 - 127)
    check_weights(got, want, kind, 63, tokens, weight[:, None] * sink)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("fmt", ["e4m3fn", "e5m2"])
@pytest.mark.parametrize("latent", [256, 512])
def test_weights_that_are_alike_keep_their_bits(uz, kind, fmt, latent):
    """All of a row's weights the same, 32 fractions of an octave over the heads: what a weight loses they lose alike."""
    g, rot, heads, tokens, scale = np.random.default_rng(62), 64, 32, 640, 2.0 ** -7
    one, least, most = {"e4m3fn": (0x38, 0x30, 0x41), "e5m2": (0x3C, 0x38, 0x41)}[fmt]
    codes = g.integers(least, most, (10, 64, latent + rot)).astype(np.uint8)
    codes[..., latent:] = 0
    codes[..., latent] = one
    exps = np.full((10, 64, 2), 127, np.uint8)
    q = torch.zeros(heads, latent + rot, dtype=TYPES[kind], device="cuda")
    q[:, latent] = torch.arange(heads) / 32 * np.log(2) / scale
    got, want = attend(uz, codes, exps, rot, q, tokens, 1, scale, fmt)
    check_weights(got, want, kind, 1, tokens, 0.0)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("fmt", ["e4m3fn", "e5m2"])
@pytest.mark.parametrize("latent", [256, 512])
@pytest.mark.parametrize("least,most,tokens", [(78, 163, 200), (27, 246, 64), (27, 246, 1000), (27, 80, 700), (110, 246, 130)])
def test_scales_that_are_far_apart(uz, kind, fmt, latent, least, most, tokens):
    """Latents of all sizes side by side, their scores alike: every token counts in the divisor, those of the largest scales make the
    output."""
    top = {"bf16": 246 if fmt == "e4m3fn" else 239, "fp16": 132 if fmt == "e4m3fn" else 125}[kind]  # outputs are within the type
    most = min(most, top)
    g, rot, page, scale = np.random.default_rng(63), 64, 16, 0.05
    pages = -(-tokens // page)
    codes = (g.integers(0, 256, (pages, page, latent + rot)) & 0xBB).astype(np.uint8)
    exps = g.integers(least, most + 1, (pages, page, 2)).astype(np.uint8)
    exps[..., 1] = {"e4m3fn": 125, "e5m2": 118}[fmt]
    q = torch.zeros(24, latent + rot, dtype=TYPES[kind], device="cuda")
    q[:, latent:] = torch.from_numpy(g.standard_normal((24, rot)).astype(np.float32))
    for requests in (1, 300):
        got, want = attend(uz, codes, exps, rot, q, tokens, requests, scale, fmt)
        check_weights(got, want, kind, rot, tokens, want["spread"])


@pytest.mark.parametrize("heads", [1, 40])
def test_latents_of_zero(uz, heads):
    """The least scale, in millions of tokens: the divisor is their number, of whose logarithm 22 rounding to 24 bits takes 2^-20 each time."""
    page, latent, rot, pages = 256, 512, 64, 1 << 14
    codes, exps = torch.zeros(1, page, latent + rot, dtype=torch.uint8, device="cuda"), torch.full((1, page, 2), 27, dtype=torch.uint8, device="cuda")
    q = torch.randn(1, heads, latent + rot, device="cuda").to(torch.bfloat16)
    out, lse = uz.latent_attend(q, uz.LatentCache(codes, exps, rot), ints(np.zeros((1, pages))), ints([pages * page]), ints([0, 1]), 1, 0.05)
    assert (out == 0).all() and (lse.double() - np.log(pages * page)).abs().max() < 2.0 ** -18


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("latent,rot", [(256, 32), (512, 32), (512, 64)])
def test_an_infinite_rotary_key_counts_by_its_score(uz, kind, latent, rot):
    """Minus infinity: as if the token were not there; plus infinity, or none since a query's channel is 0: no number."""
    g, page, tokens, scale = np.random.default_rng(64), 16, 75, 0.05
    codes = (g.integers(0, 256, (5, page, latent + rot)) & 0xBB).astype(np.uint8)
    codes[..., latent:] &= 0xB7
    exps = np.full((5, page, 2), 118, np.uint8)
    codes[4, 10, latent + 9] = 0x7C                                       # the last token's
    q = torch.from_numpy(g.standard_normal((40, latent + rot)).astype(np.float32)).to(TYPES[kind]).cuda()
    q[20:, latent + 9] = q[20:, latent + 9].abs()
    q[:20, latent + 9] = -q[:20, latent + 9].abs()
    q[39, latent + 9] = 0
    got, _ = attend(uz, codes, exps, rot, q, tokens, 2, scale, "e5m2")
    codes[4, 10, latent + 9] = 0
    _, want = attend(uz, codes, exps, rot, q[:20], tokens - 1, 1, scale, "e5m2")
    check_weights((got[0][:, :20], got[1][:, :20]), want, kind, latent + rot, tokens, want["spread"])
    assert torch.isnan(got[0][:, 20:]).all() and torch.isnan(got[1][:, 20:]).all()


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("fmt", ["e4m3fn", "e5m2"])
@pytest.mark.parametrize("latent,heads", [(256, 24), (512, 64)])
@pytest.mark.parametrize("of_latent,of_rot", [(-18, 2), (-19, 7), (2, -18), (9, -17)])
def test_scores_of_latents_and_rotary_keys_of_unlike_sizes(uz, kind, fmt, latent, heads, of_latent, of_rot):
    """Latents of 2^20 to 2^26 times the rotary keys' size or the other way round, queries so that both parts of a score are alike: a
    score is a sum of exact products in 32 bits."""
    g, rot, page, tokens, scale = np.random.default_rng(65), 64, 16, 130, 4.0
    codes = g.integers(0, 256, (9, page, latent + rot)) & 0xBF        # magnitudes below 2
    exps = np.full((9, page, 2), [127 + of_latent, 127 + of_rot], np.uint8)
    part = np.repeat([2.0 ** -(6 + of_latent + (latent == 512) / 2), 2.0 ** -(5 + of_rot)], [latent, rot])  # within fp16
    q = torch.from_numpy((g.standard_normal((heads, latent + rot)) * part).astype(np.float32)).to(TYPES[kind]).cuda()
    got, want = attend(uz, codes.astype(np.uint8), exps.astype(np.uint8), rot, q, tokens, 2, scale, fmt)
    check_weights(got, want, kind, latent + rot, tokens, want["spread"])


@pytest.mark.parametrize("nope,rot,value,heads,tokens", [(128, 64, 128, 3, 60000), (64, 32, 64, 200, 3000), (64, 32, 64, 70, 9000), (64, 64, 64, 2, 200000)])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_expanded_small_weights_beside_a_large_one(uz, kind, nope, rot, value, heads, tokens):
    """Keys after the first that weigh 2^-25.5 of it: a weight is a number of the type, in fp16 with 11 bits down to 2^-21 of the largest, and
    off by at most 2^-32 of it below."""
    g, scale, rows = np.random.default_rng(66), 2.0 ** -5, 65
    k = torch.zeros(tokens, heads, nope, dtype=TYPES[kind], device="cuda")
    k[0, :, 0] = 16
    v = torch.rand(tokens, heads, value, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).add_(0.5).to(TYPES[kind])
    v[0] = 0                                                              # what there is comes from the others
    q = torch.zeros(rows, heads, nope + rot, dtype=TYPES[kind], device="cuda")
    q[..., 0] = torch.from_numpy(25.5 * np.log(2) / 16 / scale + g.standard_normal((rows, heads)) * 0.1).cuda()
    r = torch.zeros(tokens, rot, dtype=TYPES[kind], device="cuda")
    out, lse = uz.latent_attend_expanded(q, k, r, v, ints([0, rows]), ints([0, tokens]), rows, scale=scale)
    torch.cuda.synchronize()
    first = np_of(q[..., 0]) * 16 * scale                                 # the others' scores are 0
    seen = (tokens - rows + 1 + np.arange(rows))[:, None]
    total = np.exp(first) + seen - 1
    sums = v.double().cumsum(0)[tokens - rows:].cpu().numpy()
    want = sums / total[..., None]
    # beside the rounding of an output: a weight's, the exponential's and the score's, the sums'
    eps = 2.0 ** -21 + 2.0 ** -22 * first.max() + 2 * tokens * 2.0 ** -24
    tol = U_OUT[kind] * want + ({"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}[kind] + 2 * eps) * want + LEAST[kind]
    if kind == "fp16":
        tol = tol + 2.0 ** -32 * sums
    assert (np.abs(np_of(out) - want) <= tol).all(), np.nanmax(np.abs(np_of(out) - want) / tol)
    assert (np.abs(lse.cpu().numpy() - np.log(total)) <= 2 * eps + 2.0 ** -22 * np.log(total)).all()


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("power", [12, 16, 18, 20, 22, 23, 24, 26, 30])
def test_scores_past_what_32_bits_tell_apart(uz, kind, power):
    """Scores of up to 2^34, where a reference some powers of two from them is rounded, and up to 2^24 for the expanded form: outputs are
    means of what a row sees."""
    g, scale, tokens = np.random.default_rng(67), 2.0 ** power, 300
    x = lambda *s: torch.from_numpy(g.standard_normal(s).astype(np.float32)).to(TYPES[kind]).cuda()  # noqa: E731
    codes = (g.integers(0, 256, (20, 16, 288)) & 0xBB).astype(np.uint8)
    exps = g.integers(118, 124, (20, 16, 2)).astype(np.uint8)
    got, want = attend(uz, codes, exps, 32, x(40, 288), 310, 2, scale)
    values = np.abs(ref.code_values("e4m3fn")[codes[..., :256]] * 2.0 ** (exps[..., :1].astype(np.float64) - 127)).reshape(-1, 256)[:310]
    assert (np.abs(np_of(got[0])) <= values.max(axis=0) * (1 + 2.0 ** -7)).all() and torch.isfinite(got[1]).all()
    k, v, r, q = x(tokens, 100, 64), x(tokens, 100, 64), x(tokens, 32), x(tokens, 100, 96)
    out, lse = uz.latent_attend_expanded(q, k, r, v, ints([0, tokens]), ints([0, tokens]), tokens, scale=min(scale, 2.0 ** 18))
    most = v.float().abs().cummax(0).values
    assert (out.float().abs() <= most * (1 + 2.0 ** -7)).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("heads", [3, 16, 40])
def test_what_a_workspace_held_changes_no_bit(uz, kind, heads):
    g, latent, rot, tokens = np.random.default_rng(68), 512, 64, 3000
    codes = (g.integers(0, 256, (47, 64, latent + rot)) & 0xBB).astype(np.uint8)
    exps = g.integers(110, 124, (47, 64, 2)).astype(np.uint8)
    codes[..., latent], exps[..., 1] = encode(np.arange(47) / 8, "e4m3fn")[:, None], 127  # weights that grow from piece to piece
    cache = uz.LatentCache(dev(codes), dev(exps), rot)
    q = torch.from_numpy(g.standard_normal((2, heads, latent + rot)).astype(np.float32)).to(TYPES[kind]).cuda()
    q[..., latent:] = 0
    q[..., latent] = 500
    table, lens, q_start = ints(np.tile(np.arange(47), (2, 1))), ints([tokens, 70]), ints([0, 1, 2])
    ws = uz.latent_attend_workspace(q, cache, 2, 1)
    first = None
    for fill in (0, 0x01, 0x3F, 0x7F, 0x80, 0xC2, 0xFF):
        ws.fill_(fill)
        got = uz.latent_attend(q, cache, table, lens, q_start, 1, 0.004, ws=ws)
        first = first or got
        assert torch.equal(got[0], first[0]) and torch.equal(got[1], first[1]), fill
