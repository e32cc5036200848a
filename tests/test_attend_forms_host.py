"""The lengths that tests use for each way of running attention do lead there, and its records fit.  No GPU needed."""
import pytest

from attend_forms import FORMS, blocks_per_range, launch_form
from helpers import ensure_lib


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("form", FORMS)
def test_forms(form, fmt):
    P = ensure_lib()
    hkv, lens, max_length, each = FORMS[form]
    name, parts = launch_form(fmt, 128, 3 * hkv, hkv, lens, max_length)
    assert name == form.split("-")[0]
    assert each is None or blocks_per_range(fmt, 128, 3 * hkv, hkv, lens) in (each, 2 * each if each > 2 else each)
    size = P.pallas_attend_workspace_size(len(lens), 3 * hkv, hkv, 128, max_length)
    for s, part in enumerate(parts):
        if part is not None:      # record numbers: the row's first, plus the row
            assert size >= 8 * len(lens) + (part[0] + s + part[1]) * 3 * hkv * (128 + 2) * 4
