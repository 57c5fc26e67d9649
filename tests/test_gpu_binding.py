"""Tensors whose values are not what their memory holds, and arguments at the ends of their types, through the binding."""
import pytest

from paper_1908_04172_amd import workloads as wl

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def he():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1908_04172_amd import he as he_mod
    he_mod.lib()
    return he_mod


def test_conjugated_and_negated_tensors(he):
    """A conjugate that torch has not carried out is refused by every call that reads slots; carried out, its values count."""
    ctx = he.Context(10, wl.modulus_chain([40, 40], 1 << 10))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    parts = torch.randn((20, 512, 2), dtype=torch.float64, device="cuda", generator=gen)
    u = torch.rand(1024, dtype=torch.float64, device="cuda", generator=gen)
    slots = torch.view_as_complex(parts)
    lazy = slots.conj()
    assert lazy.is_conj() and lazy.is_contiguous()
    with pytest.raises(TypeError):
        ctx.sample_slots(lazy, u, parts=he.SLOTS_COMPLEX)
    with pytest.raises(TypeError):
        ctx.encode_vector(lazy, 2.0**20)
    with pytest.raises(TypeError):
        ctx.sample_slots(slots, torch._neg_view(u), parts=he.SLOTS_COMPLEX)
    flipped = torch.view_as_complex(parts * torch.tensor([1.0, -1.0], dtype=torch.float64, device="cuda"))
    got = ctx.sample_slots(lazy.resolve_conj(), u, parts=he.SLOTS_COMPLEX)
    want = ctx.sample_slots(flipped, u, parts=he.SLOTS_COMPLEX)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(ctx.encode_vector(lazy.resolve_conj(), 2.0**20), ctx.encode_vector(flipped, 2.0**20))


def test_top_k_is_unsigned(he):
    """Numbers of 2^31 and more, which an int32 tensor holds as negative ones, are more than any row has: off, as 0 is."""
    ctx = he.Context(10, wl.modulus_chain([40], 1 << 10))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    for n in (50, 1000):                                            # (rows that are ranked at once, and rows with histograms)
        slots = torch.view_as_complex(torch.randn((n, 512, 2), dtype=torch.float64, device="cuda", generator=gen))
        u = torch.rand(512, dtype=torch.float64, device="cuda", generator=gen)
        p = torch.full((512,), 0.9, dtype=torch.float64, device="cuda")
        want, filtered = ctx.sample_slots(slots, u), ctx.sample_slots(slots, u, top_p=p)
        for k in (-1, -2**31, 2**31 - 1, n, 0):
            top_k = torch.full((512,), k, dtype=torch.int32, device="cuda")
            for got, expect in ((ctx.sample_slots(slots, u, top_k=top_k), want), (ctx.sample_slots(slots, u, top_k=top_k, top_p=p), filtered)):
                assert all(torch.equal(a, b) for a, b in zip(got, expect)), (n, k)


def test_rows_per_slot_are_one_or_two(he):
    ctx = he.Context(10, wl.modulus_chain([40], 1 << 10))
    slots = torch.zeros((4, 512), dtype=torch.complex128, device="cuda")
    for parts in (0, 3, -1):
        with pytest.raises(he.HeError) as e:
            ctx.sample_slots(slots, torch.zeros(6, dtype=torch.float64, device="cuda"), parts=parts)
        assert e.value.status == -1, parts
