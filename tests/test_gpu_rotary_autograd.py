"""GPU: rotary positions and latent attention among autograd's tensors: outputs that the caller gave, tangents, gradients that no call
gives."""
import numpy as np
import pytest
import torch

from test_gpu_rotary import TYPES, dev, freq_of, ints, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def uz():
    import paper_2604_17172_amd as m
    return m


def test_what_autograd_saved_is_not_changed_unseen(uz):
    x, freq = torch.randn(3, 2, 32, device="cuda", requires_grad=True), dev(freq_of(32))
    lens, q_start, places = ints([10]), ints([0, 3]), ints([0, 0, 0])
    uz.kv_positions(lens, q_start, 3, out=places)
    y = uz.rotate(x, places, freq)
    uz.kv_positions(ints([20]), q_start, 3, out=places)                   # the next step's
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    w = x * 2
    z = (w * w).sum()
    with torch.no_grad():
        uz.rotate(w, places, freq, out=w)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.backward()


def test_versions_of_given_outputs(uz):
    g = np.random.default_rng(0)
    h = lambda *s: rows_of(s, "bf16", g)  # noqa: E731
    freq, places, slots = dev(freq_of(32)), ints([0, 1]), torch.tensor([0, 1], device="cuda")
    cache, pages = uz.LatentCache.empty(1, 256, 32, 16), uz.KVCache.empty(1, 1, 64, 16)
    cache.codes.zero_()
    cache.exps.fill_(127)
    table, lens, q_start = ints([[0]]), ints([2]), ints([0, 2])
    out, lse, wide, q_out = h(2, 3, 256), torch.zeros(2, 3, device="cuda"), h(2, 3, 64), h(2, 3, 32)
    calls = [
        ((q_out,), lambda: uz.rotate(h(2, 3, 32), places, freq, out=q_out)),
        ((places,), lambda: uz.kv_positions(lens, q_start, 2, out=places)),
        ((wide,), lambda: uz.kv_rotate_store(pages, h(2, 1, 64), h(2, 1, 64), places, freq, slots, ints([[0, 2]]), ints([1, 1]), q=h(2, 3, 64), q_out=wide)),
        ((q_out,), lambda: uz.latent_store(cache, h(2, 1, 256)[:, 0], h(2, 1, 32)[:, 0], places, freq, slots, q=h(2, 3, 32), q_out=q_out)),
        ((out, lse), lambda: uz.latent_attend(h(2, 3, 288), cache, table, lens, q_start, 2, 0.1, out=out, lse=lse)),
        ((wide, lse), lambda: uz.latent_attend_expanded(h(2, 3, 96), h(2, 3, 64), h(2, 1, 32)[:, 0], h(2, 3, 64), q_start, q_start, 2, out=wide, lse=lse)),
    ]
    for given, call in calls:
        before = [x._version for x in given]
        call()
        assert all(x._version > v for x, v in zip(given, before))
        with torch.inference_mode():
            call()
    torch.cuda.synchronize()


def test_tangents(uz):
    """Forward derivatives: the operator of the tangent, also of a gradient; calls that serve refuse dual tensors."""
    import torch.autograd.forward_ad as fw
    g = np.random.default_rng(1)
    x, t, up = (rows_of((4, 3, 40), "fp32", g) for _ in range(3))
    places, freq = ints([3, 70, 9, 1]), dev(freq_of(32))
    how = dict(interleaved=True, first=4, magnitude=1.5)
    with fw.dual_level():
        for tangent in (t, t[:, :1].expand(-1, 3, -1), t.transpose(0, 2).contiguous().transpose(0, 2)):
            y = uz.rotate(fw.make_dual(x, tangent), places, freq, **how)
            assert torch.equal(fw.unpack_dual(y).tangent, uz.rotate(tangent.contiguous(), places, freq, **how))
            assert torch.equal(fw.unpack_dual(y).primal, uz.rotate(x, places, freq, **how))
        with torch.no_grad():
            assert fw.unpack_dual(uz.rotate(fw.make_dual(x, t), places, freq, **how)).tangent is not None
        w = x.clone().requires_grad_(True)
        y = uz.rotate(fw.make_dual(w, t), places, freq, **how)
        grad, = torch.autograd.grad(y, w, fw.make_dual(up, t))
        assert torch.equal(fw.unpack_dual(grad).tangent, uz.rotate(t, places, freq, inverse=True, **how))
        dual = fw.make_dual(x, t)
        with pytest.raises(ValueError):
            uz.rotate(dual, places, freq, out=torch.empty_like(x))
        h = lambda *s: rows_of(s, "bf16", g)  # noqa: E731
        d = lambda *s: fw.make_dual(h(*s), h(*s))  # noqa: E731
        pages, cache, slots, q_start = uz.KVCache.empty(1, 1, 64, 16), uz.LatentCache.empty(1, 256, 32, 16), torch.tensor([0, 1], device="cuda"), ints([0, 2])
        two = ints([0, 1])
        for call in (
                lambda: uz.kv_rotate_store(pages, d(2, 1, 64), h(2, 1, 64), two, freq, slots, ints([[0, 2]]), ints([1, 1])),
                lambda: uz.kv_rotate_store(pages, h(2, 1, 64), h(2, 1, 64), two, freq, slots, ints([[0, 2]]), ints([1, 1]), q=d(2, 3, 64)),
                lambda: uz.latent_store(cache, d(2, 1, 256)[:, 0], h(2, 1, 32)[:, 0], two, freq, slots),
                lambda: uz.latent_attend(d(2, 3, 288), cache, ints([[0]]), ints([2]), q_start, 2, 0.1),
                lambda: uz.latent_attend_expanded(h(2, 3, 96), h(2, 3, 64), h(2, 1, 32)[:, 0], d(2, 3, 64), q_start, q_start, 2)):
            with pytest.raises(ValueError, match="no gradient"):
                call()


def test_frequencies_that_are_learned_and_outputs_that_are_followed(uz):
    """Their gradient would be lost: refused, and taken under no_grad."""
    g = np.random.default_rng(2)
    h = lambda *s: rows_of(s, "bf16", g)  # noqa: E731
    freq, places, slots, q_start = dev(freq_of(32)).requires_grad_(True), ints([0, 1]), torch.tensor([0, 1], device="cuda"), ints([0, 2])
    pages, cache, lse = uz.KVCache.empty(1, 1, 64, 16), uz.LatentCache.empty(1, 256, 32, 16), torch.zeros(2, 3, device="cuda", requires_grad=True)
    cache.codes.zero_()
    cache.exps.fill_(127)
    calls = [lambda: uz.rotate(h(2, 3, 32), places, freq),
             lambda: uz.kv_rotate_store(pages, h(2, 1, 64), h(2, 1, 64), places, freq, slots, ints([[0, 2]]), ints([1, 1])),
             lambda: uz.latent_store(cache, h(2, 1, 256)[:, 0], h(2, 1, 32)[:, 0], places, freq, slots),
             lambda: uz.latent_attend(h(2, 3, 288), cache, ints([[0]]), ints([2]), q_start, 2, 0.1, lse=lse),
             lambda: uz.latent_attend_expanded(h(2, 3, 96), h(2, 3, 64), h(2, 1, 32)[:, 0], h(2, 3, 64), q_start, q_start, 2, lse=lse)]
    for call in calls:
        with pytest.raises(ValueError):
            call()
        with torch.no_grad():
            call()
    torch.cuda.synchronize()


def test_outputs_whose_rows_share_memory_are_refused(uz):
    """One rotary key for all heads, turned where it is, would be turned once for each."""
    g = np.random.default_rng(4)
    h = lambda *s: rows_of(s, "bf16", g)  # noqa: E731
    freq, places, slots, q_start = dev(freq_of(32)), ints([0, 1]), torch.tensor([0, 1], device="cuda"), ints([0, 2])
    pages, cache = uz.KVCache.empty(1, 1, 64, 16), uz.LatentCache.empty(1, 256, 32, 16)
    key = h(2, 1, 32).expand(2, 3, 32)
    calls = [lambda: uz.rotate(key, places, freq, out=key),
             lambda: uz.kv_rotate_store(pages, h(2, 1, 64), h(2, 1, 64), places, freq, slots, ints([[0, 2]]), ints([1, 1]), q=h(2, 3, 64),
                                        q_out=h(1, 3, 64).expand(2, 3, 64)),
             lambda: uz.latent_store(cache, h(2, 1, 256)[:, 0], h(2, 1, 32)[:, 0], places, freq, slots, q=h(2, 3, 32), q_out=key),
             lambda: uz.latent_attend(h(2, 3, 288), cache, ints([[0]]), ints([2]), q_start, 2, 0.1, out=h(2, 1, 256).expand(2, 3, 256)),
             lambda: uz.latent_attend_expanded(h(2, 3, 96), h(2, 3, 64), h(2, 1, 32)[:, 0], h(2, 3, 64), q_start, q_start, 2, out=h(1, 3, 64).expand(2, 3, 64))]
    for call in calls:
        with pytest.raises(ValueError, match="lie on one another"):
            call()
    turned = uz.rotate(key, places, freq)                                 # read, they may
    assert torch.equal(turned, uz.rotate(key.contiguous(), places, freq))
