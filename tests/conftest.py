import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built HIP library")


@pytest.fixture(scope="session", autouse=True)
def _oracle_built():
    from oracle.build import LIB, build

    src = os.path.join(ROOT, "oracle", "oracle.c")
    if not os.path.exists(LIB) or os.path.getmtime(LIB) < os.path.getmtime(src):
        build()
    yield


# GPU tests that need the stream they take to run beside the default one
BESIDE = {"test_plan_runs_beside_a_merge"}


@pytest.fixture(autouse=True)
def _side_streams(request):
    if getattr(request.node, "originalname", "") in BESIDE:
        import torch

        if torch.cuda.is_available():
            from tests.gpu_util import side_streams_from_the_first_beside

            side_streams_from_the_first_beside()
    yield
