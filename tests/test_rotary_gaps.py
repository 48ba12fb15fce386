"""Which rows and keys of a batch take part, against the definition's mask (no GPU)."""
import numpy as np
import pytest

import window_util
from paper_2510_18121_amd.autograd import rows_in_use


@pytest.mark.parametrize("seed", range(40))
def test_rows_in_use(seed):
    rng = np.random.default_rng(seed)
    lens = rng.integers(1, 90, int(rng.integers(1, 5))).tolist()
    tasks = []
    for _ in range(int(rng.integers(0, 6))):
        doc = int(rng.integers(len(lens)))
        a = int(rng.integers(lens[doc]))
        tasks.append((doc, a, int(rng.integers(1, lens[doc] - a + 1))))
    b = window_util.batch(lens, tasks, 2, 1, 64)
    for i in range(len(tasks)):
        if rng.random() < 0.3:
            b.task_kv_len[i] = int(rng.integers(1, lens[tasks[i][0]] + 1))
    b.total_q, b.total_kv = b.total_q + int(rng.integers(0, 5)), b.total_kv + int(rng.integers(0, 5))
    for window, sinks in ((None, 0), (1, 0), (1, 3), (7, 0), (40, 2), (200, 90)):
        q, kv = rows_in_use(b, window, sinks)
        see = window_util.visible(b, 10 ** 9 if window is None else window, sinks)
        has_task = np.zeros(b.total_q, bool)
        for a, n in zip(b.task_q_start, b.task_q_len):
            has_task[a:a + n] = True
        assert np.array_equal(kv, see.any(0)) and np.array_equal(q, has_task)
