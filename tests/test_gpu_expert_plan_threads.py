"""Plans of different numbers of experts from two threads at once: one's shared memory
does not depend on the other's."""
import threading

import pytest
import torch

from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu


def test_two_threads():
    ids = {E: torch.randint(0, E, (8, 4), device="cuda", dtype=torch.int32) for E in (1024, 700)}
    want = {E: api.expert_plan(ids[E], E=E).row_of.clone() for E in ids}
    torch.cuda.synchronize()
    errors = []

    def plans(E):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                plan = api.ExpertPlan(8, E, 4, 32, ids[E].device)
                for _ in range(3000):
                    api.expert_plan(ids[E], E=E, plan=plan)
                same = torch.equal(plan.row_of, want[E])
            if not same:
                errors.append((E, "another plan"))
        except Exception as e:
            errors.append((E, e))
    threads = [threading.Thread(target=plans, args=(E,)) for E in ids]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
