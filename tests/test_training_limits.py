"""Numbers beyond what the library's arguments hold are refused by the torch
forms before anything is allocated, not cut to 32 bits."""

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture
def host(libpgc, monkeypatch):
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    return libpgc


@pytest.mark.parametrize("k", [-1, 65, 1 << 31, (1 << 32) + 5, -(1 << 32) + 5])
def test_numbers_of_alternatives(host, k):
    from paper_2607_20739_gb300 import losses
    with pytest.raises(host.PGCError) as e:
        losses.token_scores(torch.zeros(1, 8), None, k)
    assert e.value.code == (host.EINVAL if k < 0 else host.ENOTSUP)


@pytest.mark.parametrize("n", [-1, 0, 1025, 1 << 31, (1 << 32) + 8, -(1 << 32) + 8])
def test_numbers_of_experts(host, n):
    from paper_2607_20739_gb300 import experts
    with pytest.raises(host.PGCError) as e:
        experts.route(torch.zeros(4, 2, dtype=torch.int32), n)
    assert e.value.code == (host.EINVAL if n < 1 else host.ENOTSUP)
