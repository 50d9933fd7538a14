"""What the binding refuses before it calls the library."""
import pytest


def test_sizes_beyond_32_bits_are_refused():
    # The C structures hold them in 32 bits: 2^32 + 8 columns would have been 8, and the rest of the result left as it was
    import torch
    from paper_2510_23498_b200 import binding as b

    def of(*shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="meta")           # sizes and strides without memory

    words = of(2, dtype=torch.int64)
    for n in ((1 << 31), (1 << 32) + 8):
        calls = [lambda: b.dropout(of(n), 0.5, words), lambda: b.dropout(of(3, n), 0.5, words),
                 lambda: b.ResidualStep(8).forward(of(n, 8, dtype=torch.float32)), lambda: b.ResidualStep(8).backward(of(n, 8, dtype=torch.float32)),
                 lambda: b.ResidualStep(n), lambda: b.ResidualStep(8).backward(of(3, 8, dtype=torch.float32), scale_exp=n)]
        for shape in ((n, 1, 1), (1, n, 1), (1, 1, n)):
            calls += [lambda s=shape: b.recurrence_forward(of(*s), of(*s)), lambda s=shape: b.recurrence_backward(of(*s), of(*s), of(*s), None)]
        for i, f in enumerate(calls):
            with pytest.raises(b.MpodeError) as e:
                f()
            assert e.value.status == b.ERR_UNSUPPORTED and "32 bits" in str(e.value), (i, str(e.value))


def test_a_site_beyond_32_bits_is_refused():
    # 0 and 2^32 would have drawn the same masks
    import torch
    from paper_2510_23498_b200 import binding as b
    x, words = torch.zeros(4, 8), torch.zeros(2, dtype=torch.int64)
    for site in (1 << 32, -(1 << 31) - 1):
        for f in (lambda: b.dropout(x, 0.5, words, site=site), lambda: b.ResidualStep(8, site=site)):
            with pytest.raises(b.MpodeError, match="site"):
                f()
