"""qk_norm_rope_append_scaled at the row counts where its work is split another way: one row to a search for runs below
512 rows, four below 4,096, sixteen from there on."""
import numpy as np
import pytest

from test_gpu_scaled_append import check, note, sequences

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [511, 512, 4095, 4096])
@pytest.mark.parametrize("most", [1, 7, 40])
def test_lines(gpu_lib, rows, most):
    """Sequences of up to `most` rows, begun anywhere in a block: their runs cross the searches' four or sixteen rows."""
    note(f"scaled append {rows} rows, runs of sequences of up to {most}")
    rng = np.random.default_rng(rows + most)
    new = rng.integers(1, most + 1, rows)
    new = new[:int(np.searchsorted(np.cumsum(new), rows))]
    new = np.append(new, rows - new.sum())
    specs = [(int(c), int(n)) for c, n in zip(rng.integers(0, 40, len(new)), new)]
    nb = sum(-(-(c + n) // 16) for c, n in specs) + 3
    slots, pos = sequences(rng, specs, nb, 500)
    assert len(slots) == rows
    check(gpu_lib, rng, slots, pos, hq=1, hkv=1, nb=nb, paired=rows % 2 == 0)
