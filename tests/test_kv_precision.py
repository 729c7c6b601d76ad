"""The 24 bits that fp32 attention over the 8-bit cache keeps of queries and probabilities, each as three bf16 terms.

The bound of the other tests is a worst case over many roundings, far above 2^-24.  Here two tokens share nearly all of a
row's weight and no channel holds values of both, so that an output of the lighter token is w v / (w + 1) and its error
relative to itself is what w's own roundings are.  Scores lie between 6 and 7.  What is rounded, as shares of the output,
root mean square: scores times the scale in a step that is masked, half an ulp of [8, 16) each, 2^-21.8 in the exponent for
one and 2^-21.3 for both, times ln 2 and the other token's share of about 0.6: 2^-22.5; the exponential, up to one ulp: 2^-24;
sums, the reciprocal and the last product, up to an ulp: 2^-23.  Together 2^-22; the bound is twice that.  Without the third
term of a probability, 2^-18 of it at most, errors are near 2^-19, without that of a query, 2^-18 of 6 to 7, near 2^-17: the
kernel's arithmetic with fewer terms, done here in numpy, is shown not to pass."""
import numpy as np
import pytest

BOUND, LSE_BOUND = 2.0 ** -21, 2.0 ** -22
f32 = np.float32


def problem(dim, rows, seed):
    """Queries [rows, dim] and the two tokens' keys and values [2, dim]; every number of the tokens is a code."""
    g = np.random.default_rng(seed)
    at = g.choice(dim, 2, replace=False)
    q = g.standard_normal((rows, dim)).astype(f32)
    q[:, at] = 6 + g.random((rows, 2)).astype(f32)
    k, v = np.zeros((2, dim), f32), np.zeros((2, dim), f32)
    k[0, at[0]] = k[1, at[1]] = 1
    v[0, 0::2], v[1, 1::2] = 1.5, 1.75
    return q, k, v, at


def errors(out, lse, q, k, v):
    """Root mean squares of the relative errors of the lighter token's outputs and of lse, against 64 bits."""
    z = q.astype(np.float64) @ k.T.astype(np.float64)
    top = z.max(axis=1, keepdims=True)
    w = np.exp(z - top)
    want = (w / w.sum(axis=1, keepdims=True)) @ v.astype(np.float64)
    light = z.argmin(axis=1)
    rel = np.concatenate([(out[r, t::2] - want[r, t::2]) / want[r, t::2] for r, t in enumerate(light)])
    sums = (top + np.log(w.sum(axis=1, keepdims=True)))[:, 0]
    return np.sqrt((rel ** 2).mean()), np.sqrt((((lse - sums) / sums) ** 2).mean())


def bf16(x):
    u = np.asarray(x, f32).view(np.uint32).astype(np.uint64)
    return (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(f32)


def terms(x, n):
    out = []
    for _ in range(n):
        out.append(bf16(x))
        x = x - out[-1]
    return out


def arithmetic(q, k, v, q_terms, p_terms, masked):
    """The kernel's roundings in numpy: sums in 32 bits, smaller terms first."""
    s = np.zeros((len(q), len(k)), f32)
    for t in reversed(terms(q, q_terms)):
        for d in np.flatnonzero(k.any(axis=0)):
            s = s + t[:, d:d + 1] * k[:, d]
    c = f32(1.4426950408889634)
    if masked:
        s = s * c
        top = s.max(axis=1, keepdims=True)
        arg = s - top
    else:
        top = s.max(axis=1, keepdims=True) * c
        arg = (s.astype(np.float64) * np.float64(c) - top).astype(f32)
    p = np.exp2(arg.astype(np.float64)).astype(f32)
    total = p[:, :1] + p[:, 1:]
    acc = np.zeros((len(q), v.shape[1]), f32)
    for t in reversed(terms(p, p_terms)):
        for n in range(2):
            acc = acc + t[:, n:n + 1] * v[n]
    lse = (top + np.log2(total.astype(np.float64)).astype(f32)) * f32(0.6931471805599453)
    return (acc * (f32(1) / total)).astype(np.float64), lse[:, 0].astype(np.float64)


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
def test_the_bound_tells_three_terms_from_two(dim, masked):
    for seed in range(4):
        q, k, v, _ = problem(dim, 80, seed)
        out, lse = errors(*arithmetic(q, k, v, 3, 3, masked), q, k, v)
        assert out < BOUND and lse < LSE_BOUND
        out, lse = errors(*arithmetic(q, k, v, 2, 3, masked), q, k, v)
        assert out > 4 * BOUND and lse > 2 * LSE_BOUND
        out, _ = errors(*arithmetic(q, k, v, 3, 2, masked), q, k, v)
        assert out > 2 * BOUND


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["e4m3fn", "e5m2"])
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
def test_fp32_attention_keeps_24_bits(dim, fmt):
    import torch

    import paper_2604_17172_amd as uz
    from oracle import kv as ref
    page, new, group = 16, 40, 2
    for seed, (total, two) in enumerate([(42, (0, 1)), (150, (3, 90)), (150, (100, 109)), (3000, (5, 2900)), (3000, (2957, 700))]):
        print("[kv] 24 bits", dim, fmt, total, two, flush=True)
        q, k2, v2, at = problem(dim, new * group, seed)
        k, v = np.zeros((total, dim), f32), np.zeros((total, dim), f32)
        k[:, at] = -8                                                     # scores near -100: no weight
        k[list(two)], v[list(two)] = k2, v2
        pages = -(-total // page)
        room = pages * page - total
        code = [np.pad(ref.encode(x, fmt), ((0, room), (0, 0))).reshape(pages, 1, page, dim) for x in (k, v)]
        code[1] = np.ascontiguousarray(code[1].transpose(0, 1, 3, 2))
        one = torch.full((pages, 1), 127, dtype=torch.uint8, device="cuda")
        cache = uz.KVCache(torch.from_numpy(code[0]).cuda(), one, torch.from_numpy(code[1]).cuda(), one.clone(), fmt)
        table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
        lens, starts = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([total], [0, new]))
        out, lse = uz.kv_attend(torch.from_numpy(q).cuda().view(new, group, dim), cache, table, lens, starts, new, scale=1.0)
        got = errors(out.view(-1, dim).double().cpu().numpy(), lse.view(-1).double().cpu().numpy(), q, k2, v2)
        print("[kv]   errors of 2 to the", np.log2(got).round(2), flush=True)
        assert got[0] < BOUND and got[1] < LSE_BOUND, (total, two)
