import os
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (runs the HIP library)")


def pytest_terminal_summary(terminalreporter):
    """How many float comparisons of the GPU parity tests passed only through the absolute floor."""
    pu = sys.modules.get("parity_util")
    if pu is not None and pu.STATS.compared:
        terminalreporter.write_line("parity tolerance (1e-4 relative + floor): " + pu.STATS.summary())


class LibraryWithoutGpu:
    """The compiled library with GPU -1 in every call (the last argument but one): arguments are checked as ever, and a call that passes the
    checks ends there, before anything could be launched on the addresses that it was given."""

    def __init__(self, lib):
        self._lib = lib

    def __getattr__(self, name):
        fn = getattr(self._lib, name)
        return fn if name.endswith("_workspace") or name == "pqt_last_error" else lambda *args: fn(*args[:-2], -1, args[-1])


@pytest.fixture
def library_without_gpu(monkeypatch):
    import paper_1702_05911_amd.binding as binding
    monkeypatch.setattr(binding, "_lib", LibraryWithoutGpu(binding._lib))
    return binding._lib


@pytest.fixture(autouse=True)
def made_up_addresses_stay_off_the_gpu(request):
    """Refusals are tested with addresses that nobody may read.  Where a GPU is there, a check that is missing must not run a kernel on them."""
    if request.node.name == "test_refusals_of_the_library":
        request.getfixturevalue("library_without_gpu")


@pytest.fixture(scope="session")
def tiny():
    """Tiny workload: vectors, queries and an oracle-built index."""
    from workloads import CONFIGS, tiny_mixture
    from oracle import pqt_build
    cfg = CONFIGS["tiny"]
    X = tiny_mixture(cfg.N, d=cfg.D, seed=cfg.data_seed)
    Y = tiny_mixture(cfg.nq, d=cfg.D, seed=cfg.query_seed)
    ix = pqt_build.build_index(X, cfg.P, cfg.k1, cfg.k2, cfg.M, H=cfg.H, T=cfg.T, C=cfg.C)
    return cfg, X, Y, ix


@pytest.fixture(scope="session")
def tiny_pair(tiny):
    """The tiny index with its codes stored as (centroid pair, lambda level) per sub-part."""
    import dataclasses
    from oracle import pqt_build
    cfg, X, Y, ix = tiny
    codes = pqt_build.encode_pair_lambda(X, ix.C1, ix.M)[ix.ids]
    return cfg, X, Y, dataclasses.replace(ix, codes=np.ascontiguousarray(codes), code_format=1)


@pytest.fixture(scope="session")
def rng():
    return np.random.default_rng(12345)
