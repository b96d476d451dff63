"""What the paged cache's calls owe beside their values: reports that are neither lost nor given twice, whatever the streams."""
import pytest
import torch

import test_paged_gpu as T

pytestmark = pytest.mark.gpu

RANGE = 5                                                  # FK_ERR_RANGE


def _busy(ms=60):
    """Keep the current stream busy for a while."""
    torch.cuda._sleep(int(ms * 2e6))


def test_a_report_is_cleared_on_its_own_stream():
    """A report read on a side stream is cleared there and then: not when the legacy stream, busy with other work, comes to it, which
    would give it twice and take a later one with it."""
    side = torch.cuda.Stream()
    good = torch.ones((3, 2, 128), dtype=torch.bfloat16, device="cuda")
    bad = torch.full((3, 2, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    with T._cache() as cache, torch.cuda.stream(side):
        cache.step([0], [3])
        cache.append(0, bad, good)
        side.synchronize()
        with torch.cuda.stream(torch.cuda.default_stream()):
            _busy()
        assert cache.sync_status() == RANGE
        assert cache.sync_status() == 0                    # (while the default stream is still busy)
        cache.append(0, good, bad)
        side.synchronize()
        torch.cuda.default_stream().synchronize()
        assert cache.sync_status() == RANGE and cache.sync_status() == 0


def test_reports_of_two_streams():
    """What one stream reports and clears leaves what another sets afterwards."""
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    good = torch.ones((3, 2, 128), dtype=torch.bfloat16, device="cuda")
    bad = torch.full((3, 2, 128), float("inf"), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    with T._cache() as cache:
        cache.step([0], [3], stream=one)
        cache.append(0, good, bad, stream=one)
        assert cache.sync_status(stream=one) == RANGE
        cache.append(0, bad, good, stream=two)
        assert cache.sync_status(stream=two) == RANGE and cache.sync_status(stream=one) == 0
        cache.append(0, good, good, stream=two)
        assert cache.sync_status(stream=two) == 0


@pytest.mark.parametrize("call", ["append", "attend", "read"])
def test_outputs_made_for_another_stream(call):
    """A tensor that the current stream has given back while its work on it is still queued is not written by another one."""
    side, n = torch.cuda.Stream(), 64
    kv = torch.ones((n, 4, 128), dtype=torch.bfloat16, device="cuda")
    cos, sin = torch.ones((n, 64), device="cuda"), torch.zeros((n, 64), device="cuda")
    torch.cuda.synchronize()
    for other in (side, side.cuda_stream):
        with T._cache(n_kv_heads=4, n_q_heads=4) as cache:
            cache.step([0], [n], stream=other)
            cache.append(0, kv, kv, stream=other)
            side.synchronize()
            mine = [torch.full((n, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
            seen = [torch.empty_like(x) for x in mine]
            places = {x.data_ptr() for x in mine}
            _busy()
            for x, y in zip(mine, seen):
                y.copy_(x)
            del mine, x
            if call == "append":
                out = (cache.append(0, kv, kv, cos, sin, Q=kv, stream=other),)
            elif call == "attend":
                out = (cache.attend(0, kv, stream=other),)
            else:
                out = cache.read(0, stream=other)
            assert not places & {x.data_ptr() for x in out}
            side.synchronize()
            assert all((x == 1).all() for x in out)
            torch.cuda.synchronize()
            assert all((y == 7).all() for y in seen)
            del out


def test_the_default_stream_by_its_number():
    with T._cache() as cache, torch.cuda.stream(torch.cuda.Stream()):
        kv = torch.ones((3, 2, 128), dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        cache.step([0], [3], stream=0)
        cache.append(0, kv, kv, stream=0)
        k, v = cache.read(0, stream=0)
        torch.cuda.synchronize()
        assert (k == 1).all() and (v == 1).all()


def test_scales_that_fp32_does_not_hold_are_refused():
    """A positive scale that is 0 in fp32 is not the default."""
    from paper_2605_09681_gb300 import FkError
    kv = torch.ones((3, 2, 128), dtype=torch.bfloat16, device="cuda")
    with T._cache(n_q_heads=2) as cache:
        cache.step([0], [3])
        cache.append(0, kv, kv)
        for scale in (1e-50, 1e-46, 5e-324, float("nan"), -1.0, 0.0):
            with pytest.raises(ValueError):
                cache.attend(0, kv, scale=scale)
        for scale in (1e39, float("inf")):
            with pytest.raises(FkError):
                cache.attend(0, kv, scale=scale)
        assert (cache.attend(0, kv, scale=1e-40) == 1).all()


@pytest.mark.parametrize("heads,asks", [(1, 2 ** 31 - 1), (1, 2 ** 30), (8, 2 ** 27), (64, 2 ** 24 + 5)])
def test_steps_of_more_query_rows_than_the_kernels_count_are_refused(heads, asks):
    """Rows (queries times heads) and positions are counted in 32 bits, with room for a tile and a window beside them: below 2^30."""
    from paper_2605_09681_gb300 import FkError
    with T._cache(n_q_heads=heads, n_kv_heads=1) as cache:
        for seqs, nq in (([0], [asks]), ([0, 1], [asks - 7, 7])):
            with pytest.raises(FkError) as e:
                cache.step(seqs, [1] * len(seqs), nq)
            assert e.value.name == "FK_ERR_ARG"
        cache.step([0], [1], [2 ** 30 // heads - 1])
        assert cache.length(0) == 1
