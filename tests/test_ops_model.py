"""The plain 64-bit operators that the GPU tests compare with, pinned on the
CPU: the generator against published outputs of Philox4x32-10, gradients
against differences."""
import torch

import ops_model as m


def test_generator_known_answers():
    # the known answers that Salmon et al. publish with the method
    assert m.philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 0xFFFFFFFF
    assert m.philox((ones,) * 4, (ones,) * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert m.philox((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == \
        [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_masks_keep_the_expected_share_and_differ_by_step():
    n, p = 1 << 14, 0.1
    a, b = m.keep_mask(n, p, 11, 0), m.keep_mask(n, p, 11, 1)
    for k in (a, b):
        # six deviations of a binomial count
        assert abs(int(k.sum()) - n * (1 - p)) < 6 * (n * p * (1 - p)) ** 0.5 + 1
    both = int((a & b).sum())
    q = (1 - p) ** 2
    assert abs(both - n * q) < 6 * (n * q * (1 - q)) ** 0.5 + 1
    assert m.keep_mask(10, 0.0, 3, 3).all() and not m.keep_mask(10, 1.0, 3, 3).any()


def test_embedding_gradient_is_the_transpose_of_the_lookup():
    g = torch.Generator().manual_seed(1)
    tokens = torch.randint(0, 7, (3, 5), generator=g)
    table, dy = m.normal(g, 7, 4), m.normal(g, 3, 5, 4)
    table.requires_grad_()
    m.embedding(tokens, table, 1.5).backward(dy)
    assert torch.allclose(table.grad, m.embedding_grad(tokens, dy, 7, 1.5)[0], rtol=1e-14, atol=1e-14)


def test_norm_gradients_against_differences():
    g = torch.Generator().manual_seed(2)
    x, z = m.normal(g, 6, 5), m.normal(g, 6, 5)
    w = [m.normal(g, 5) for _ in range(4)]
    gate = m.normal(g, 2, 5)

    def f(x, z, w1, b1, w2, b2, gate):
        return m.residual_norm(x, z, "layer", w1, b1, gate, 0.7, "rms", w2, b2, 1e-3)

    args = [t.requires_grad_() for t in (x, z, *w, gate)]
    assert torch.autograd.gradcheck(f, args, eps=1e-6, atol=1e-7, rtol=1e-5)


def test_cross_entropy_gradients_against_differences():
    g = torch.Generator().manual_seed(3)
    h, w = m.normal(g, 5, 4).requires_grad_(), m.normal(g, 7, 4).requires_grad_()
    targets = torch.tensor([0, 6, -100, 3, 3])
    assert torch.autograd.gradcheck(lambda h, w: m.cross_entropy(h, w, targets, -100)[0], (h, w), eps=1e-6, atol=1e-8,
                                    rtol=1e-6)
    gl = m.normal(g, 5)
    dh, dw = torch.autograd.grad(m.cross_entropy(h, w, targets, -100)[0], (h, w), gl)
    p = m.cross_entropy_grad(h.detach(), w.detach(), targets, gl, -100)
    assert torch.allclose(p @ w.detach(), dh, rtol=1e-12, atol=1e-13)
    assert torch.allclose(p.t() @ h.detach(), dw, rtol=1e-12, atol=1e-13)
