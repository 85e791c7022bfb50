"""The binding's own checks of the 8-bit cache's arguments, on the CPU: only the call into the library is replaced."""
import numpy as np
import pytest

from paper_2608_27128_amd import binding


class Lib:
    """Takes the calls' arguments down, as ctypes would hand them over."""

    def __init__(self):
        self.sent = {}

    def __getattr__(self, name):
        if not name.startswith("twinkv_"):
            raise AttributeError(name)
        types = binding.SIGNATURES[name][1]

        def call(*args):
            self.sent[name] = [a if x is None else getattr(x(a), "value", a) if isinstance(a, int) else a
                               for x, a in zip(types, args)]
            return 0
        return call


@pytest.fixture
def lib(monkeypatch):
    L = Lib()
    monkeypatch.setattr(binding, "_lib", L)
    monkeypatch.setattr(binding, "_launch", lambda dev, name, *args: getattr(L, name)(*args))
    monkeypatch.setattr(binding, "_stream", lambda dev: None)
    return L


def cache(H=2, rows=64, d=64, at=None):
    """A Cache8 of host memory (its constructor takes memory of a GPU only); `at`: its four arrays."""
    import torch
    C = rows // 32 * 32
    c = object.__new__(binding.Cache8)
    made = (torch.zeros((H, C, d), dtype=torch.int8), torch.zeros((H, C // 32), dtype=torch.uint8),
            torch.zeros((H, C // 8, d, 8), dtype=torch.int8), torch.zeros((H, C // 32), dtype=torch.uint8))
    c.k_codes, c.k_scales, c.v_codes, c.v_scales = made if at is None else at
    c.cu_rows, c.n_heads, c.n_seqs, c.d, c.device = np.array([0, C]), H, 1, d, made[0].device
    c._handle, c._scales = None, H * (C // 32)
    c._at = tuple(x.data_ptr() for x in (c.k_codes, c.k_scales, c.v_codes, c.v_scales))
    return c


def evict(c, to, *args, **kw):
    import torch
    return binding.cache8_evict(c, torch.zeros((2, 1), dtype=torch.int32), torch.zeros((2, 64)), 10, to, *args, **kw)


@pytest.mark.parametrize("sink,recent,want", [(4, 64, (4, 64)), (0, 1 << 32, (0, 2 ** 31 - 1)), (1 << 32, 0, (2 ** 31 - 1, 0)),
                                              ((1 << 32) + 7, 1 << 40, (2 ** 31 - 1, 2 ** 31 - 1)),
                                              (np.int64(1 << 33), 2 ** 31 - 1, (2 ** 31 - 1, 2 ** 31 - 1))])
def test_evict_protects_any_number_of_rows(lib, sink, recent, want):
    """More than 32 bits of first or last rows are all of them, not what the low bits say."""
    evict(cache(), cache(), sink, recent)
    assert tuple(lib.sent["twinkv_cache8_evict"][5:7]) == want


@pytest.mark.parametrize("sink,recent", [(-1, 0), (0, -1), (-(1 << 32), 4), (4, -(1 << 40))])
def test_evict_refuses_negative_numbers_of_rows(lib, sink, recent):
    with pytest.raises(ValueError, match="negative"):
        evict(cache(), cache(), sink, recent)
    assert "twinkv_cache8_evict" not in lib.sent


def test_evict_refuses_caches_that_overlap(lib):
    """Arrays of the two caches in one buffer: from every start, against their bytes listed one by one."""
    import torch
    H, rows, d = 2, 64, 64
    codes, scales = H * rows * d, H * rows // 32
    buf = torch.zeros(8 * codes, dtype=torch.int8)

    def placed(k, v, s):
        """Codes at k and v, scales at s and behind them."""
        u8 = buf.view(torch.uint8)
        return cache(H, rows, d, (buf[k:k + codes].view(H, rows, d), u8[s:s + scales].view(H, -1),
                                  buf[v:v + codes].view(H, rows // 8, d, 8), u8[s + scales:s + 2 * scales].view(H, -1)))
    a = placed(codes, 3 * codes, 5 * codes)
    mine = [(codes, 2 * codes), (3 * codes, 4 * codes), (5 * codes, 5 * codes + 2 * scales)]
    refused = kept = 0
    starts = sorted({x + y for x in (0, codes, 2 * codes, 3 * codes, 4 * codes) for y in (-codes, -1, 0, 1, codes // 2)})
    for k in starts:
        for v in (6 * codes, 2 * codes + 5):
            for s in (7 * codes, 5 * codes - scales, 5 * codes + scales, 5 * codes + 2 * scales, 5 * codes - 2 * scales):
                if k < 0:
                    continue
                b = placed(k, v, s)
                spans = mine + [(k, k + codes), (v, v + codes), (s, s + 2 * scales)]
                taken = np.zeros(len(buf), dtype=np.int32)
                for x, y in spans:
                    taken[x:y] += 1
                if taken.max() > 1:
                    refused += 1
                    for pair in ((a, b), (b, a)):
                        with pytest.raises(ValueError, match="overlap"):
                            evict(*pair)
                else:
                    kept += 1
                    evict(a, b)
    assert refused > 20 and kept > 5
    with pytest.raises(ValueError, match="overlap"):
        evict(a, a)
    assert cache(2, 0, 64)._spans() == []  # no rows: nothing to share


def test_binding_refuses_inputs_that_require_a_gradient(lib):
    """The calls that fill a cache or move its weights, whose gradient would be lost without a word; under no_grad they
    go on."""
    import torch
    c, to = cache(), cache()
    x = torch.zeros((2, 32, 64), dtype=torch.bfloat16)
    y, m = x.clone().requires_grad_(), torch.zeros((2, 32), requires_grad=True)
    ones, n = torch.ones((2, 32), dtype=torch.uint8), torch.zeros((2, 1), dtype=torch.int32)
    w = torch.zeros((2, 64), requires_grad=True)
    for call in (lambda: binding.cache8_compact(y, x, ones, c), lambda: binding.cache8_compact(x, y, ones, c),
                 lambda: binding.cache8_compact(x, x, ones, c, token_mass=m), lambda: binding.cache8_append(y, x, c, n),
                 lambda: binding.cache8_append(x, y, c, n), lambda: binding.cache8_evict(c, n, w, 10, to)):
        with pytest.raises(ValueError, match="gradient"):
            call()
    with torch.no_grad():
        binding.cache8_evict(c, n, w, 10, to)
    assert "twinkv_cache8_evict" in lib.sent and "twinkv_cache8_append" not in lib.sent
