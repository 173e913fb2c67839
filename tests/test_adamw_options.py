"""What nomad_adamw_step takes for its options: checked before any device is asked for (no GPU needed)."""
import struct

import pytest

from paper_2505_15511_amd import _build, binding

INVALID = -1


@pytest.fixture(scope="module")
def lib():
    if _build.is_stale():
        _build.build_library()
    return binding.load_library()


def _step(lib, bits=8, dither=0, size=None, whole=True, **more):
    fields = dict(step=1, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.0)
    fields.update(more)
    packed = binding.ADAMW_OPTIONS.pack(binding.ADAMW_OPTIONS.size if size is None else size, bits, *fields.values(), 0, 0, 0, dither)
    return lib.nomad_adamw_step(None, 0, packed if whole else packed[:size])


def test_dither_is_0_or_1_and_for_8_bits(lib):
    for bits, dither in ((8, 0), (8, 1), (32, 0)):
        assert _step(lib, bits, dither) != INVALID
    for bits, dither in ((8, 2), (8, -1), (8, 1 << 32), (32, 1)):
        assert _step(lib, bits, dither) == INVALID


def test_options_that_end_before_dither(lib):
    shorter = struct.calcsize("@Iiq5dPPi4x")
    assert shorter == binding.ADAMW_OPTIONS.size - 8
    assert _step(lib, size=shorter, whole=False) != INVALID
    assert _step(lib, size=shorter, dither=77) != INVALID              # (not looked at)
    for size in (0, shorter - 8, shorter + 4, shorter + 16):
        assert _step(lib, size=size) == INVALID


def test_numbers_that_are_refused(lib):
    for more in (dict(step=0), dict(lr=float("nan")), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(eps=float("inf")), dict(decay=float("inf"))):
        assert _step(lib, **more) == INVALID
    assert _step(lib, bits=16) == INVALID
