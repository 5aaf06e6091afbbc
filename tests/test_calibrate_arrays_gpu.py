"""What the calibration times: operators on arrays that no cache holds."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2504_14145_amd import calibrate, ops


def test_a_timed_call_does_not_find_its_arrays_in_the_caches(monkeypatch):
    """Between two calls on the same array there are 2^29 bytes of others, or the timed
    run is over."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    seen = {}
    for name in ("linear", "linear_backward", "group_norm", "group_norm_backward"):
        def record(*a, _f=getattr(ops, name), _name=name, **k):
            seen.setdefault(_name, []).append((a[0].data_ptr(), a[0].numel() * a[0].element_size()))
            return _f(*a, **k)
        monkeypatch.setattr(ops, name, record)
    for tokens in (200, 60000):
        seen.clear()
        samples = calibrate.measure([(4096, 4096)], [tokens], tp=4, repeats=2)
        assert len(samples) == 6 and all(s.seconds > 0 for s in samples)
        assert len(seen) == 4
        for name, calls in seen.items():
            last = calls[-10:]      # the last timed run
            for i, (p, size) in enumerate(last):
                again = [j for j in range(i + 1, 10) if last[j][0] == p]
                assert not again or sum(n for _, n in last[i:again[0]]) >= 1 << 28, name
