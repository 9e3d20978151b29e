"""What the entry points around the step refuse, checked before they look at the device.  No kernel runs here."""
import ctypes as C

import pytest

from paper_2501_02379_amd import tgrad as T

BAD = T.TGRAD_ERR_INVALID_ARG


def _tensors(n=2, **change):
    t = (T.tgrad_tensor * n)()
    for i in range(n):
        t[i] = T.tgrad_tensor(100, 4096, None, 8192, 12288, 16384, T.TGRAD_BF16, T.TGRAD_F32, 1.0, 0.0)
    for k, v in change.items():
        setattr(t[n - 1], k, v)
    return t


def test_group_sizes_grow_with_tensors_and_pieces():
    lib = T.load()
    size = C.c_size_t(0)
    got = []
    for n, numel in ((1, 0), (1, 1 << 26), (1000, 100)):
        t = (T.tgrad_tensor * n)()
        for i in range(n):
            t[i].numel = numel
        assert lib.tgrad_group_query_size(t, n, C.byref(size)) == T.TGRAD_OK
        got.append(size.value)
    assert 0 < got[0] < got[1] and got[0] < got[2]
    assert all(g % 256 == 0 for g in got)


@pytest.mark.parametrize("numel,n,expected", [(-1, 1, BAD), (1 << 41, 1, T.TGRAD_ERR_UNSUPPORTED), (1 << 40, 3, None),
                                              (1 << 40, 9000, T.TGRAD_ERR_UNSUPPORTED), (1, 0, BAD), (1, -3, BAD)])
def test_group_query_refusals(numel, n, expected):
    size = C.c_size_t(0)
    t = (T.tgrad_tensor * max(n, 1))()
    for i in range(max(n, 1)):
        t[i].numel = numel
    assert T.load().tgrad_group_query_size(t, n, C.byref(size)) == (T.TGRAD_OK if expected is None else expected)


@pytest.mark.parametrize("change", [
    {"numel": -1}, {"grad": None}, {"grad": 4097}, {"grad_dtype": 5}, {"grad_dtype": -1}, {"param_dtype": 9},
    {"param_dtype": T.TGRAD_C64}, {"param": 8194}, {"exp_avg": 12290}, {"exp_avg_sq": 16385}, {"exp_avg": None}, {"exp_avg_sq": None},
    {"param": None}, {"exp_avg": 16384}, {"param": 4096}, {"out": 4097}, {"lr_scale": float("nan")}, {"lr_scale": -1.0},
    {"weight_decay": float("inf")}, {"weight_decay": -0.1},
])
def test_bad_tensors_are_refused(change):
    h = C.c_void_p(None)
    assert T.load().tgrad_group_init(C.byref(h), _tensors(**change), 2, 256, None) == BAD and not h


def test_group_null_and_misaligned_arguments():
    lib = T.load()
    h = C.c_void_p(None)
    hyper = T.tgrad_adamw(1e-3, 0.9, 0.999, 1e-8, 0)
    assert lib.tgrad_group_init(None, _tensors(), 2, 256, None) == BAD
    assert lib.tgrad_group_init(C.byref(h), None, 2, 256, None) == BAD
    assert lib.tgrad_group_init(C.byref(h), _tensors(), 2, None, None) == BAD
    assert lib.tgrad_group_init(C.byref(h), _tensors(), 2, 264, None) == BAD
    assert lib.tgrad_group_query_size(_tensors(), 2, None) == BAD
    assert lib.tgrad_group_bind(None, _tensors()) == BAD
    assert lib.tgrad_group_grad_norm(None, 1.0, None, 256) == BAD
    assert lib.tgrad_group_clip(None, 1.0, None, 256) == BAD
    assert lib.tgrad_group_scale(None, 256) == BAD
    assert lib.tgrad_group_adamw(None, C.byref(hyper), 0, None) == BAD
    assert lib.tgrad_group_destroy(None) == BAD


def _logits(**change):
    d = T.tgrad_logits(4096, 8, 100, 104, 8192, T.TGRAD_BF16, 1.0)
    for k, v in change.items():
        setattr(d, k, v)
    return C.byref(d)


BAD_LOGITS = [{"data": None}, {"data": 4097}, {"targets": None}, {"targets": 8196}, {"rows": -1}, {"rows": 1 << 31}, {"vocab": 0},
              {"vocab": 1 << 31}, {"row_stride": 99}, {"row_stride": 1 << 62}, {"dtype": T.TGRAD_C64}, {"dtype": 5},
              {"temperature": 0.0}, {"temperature": -1.0}, {"temperature": float("nan")}, {"temperature": float("inf")},
              {"temperature": 1e-45}]


@pytest.mark.parametrize("change", BAD_LOGITS)
def test_bad_logits_are_refused(change):
    lib = T.load()
    pol, pref = T.tgrad_policy(0.2, 0.2, 0.1), T.tgrad_preference(0.1, 0.0)
    assert lib.tgrad_token_logprobs(_logits(**change), 256, 512, None) == BAD
    assert lib.tgrad_token_logprobs_backward(_logits(**change), 256, 512, 1024, 200, None) == BAD
    assert lib.tgrad_policy_loss(_logits(**change), C.byref(pol), 256, 256, 256, None, None, 512, 1024, None, None, 0, None) == BAD
    assert lib.tgrad_preference_loss(_logits(**change), C.byref(pref), 2, 256, 256, 256, None, 512, 1024, 2048, None, None, 0,
                                     None) == BAD


def test_loss_arguments_are_checked():
    lib = T.load()
    nan, inf = float("nan"), float("inf")

    def policy(p=(0.2, 0.2, 0.1), weight=256, adv=256, old=256, ref=None, dloss=None, ws=512, stats=1024, logp=None, dx=None, st=0):
        h = T.tgrad_policy(*p)
        return lib.tgrad_policy_loss(_logits(), C.byref(h), weight, adv, old, ref, dloss, ws, stats, logp, dx, st, None)

    def preference(p=(0.1, 0.0), pairs=2, start=256, weight=256, ref=256, dloss=None, ws=512, loss=1024, rewards=2048, logp=None,
                   dx=None, st=0):
        h = T.tgrad_preference(*p)
        return lib.tgrad_preference_loss(_logits(), C.byref(h), pairs, start, weight, ref, dloss, ws, loss, rewards, logp, dx, st,
                                         None)

    for p in ((-0.1, 0.2, 0.1), (1.1, 0.2, 0.1), (0.2, -0.1, 0.1), (0.2, inf, 0.1), (nan, 0.2, 0.1), (0.2, 0.2, nan), (0.2, 0.2, inf)):
        assert policy(p) == BAD
    for change in ({"weight": None}, {"adv": None}, {"old": None}, {"old": 258}, {"ref": 258}, {"dloss": 257}, {"ws": None},
                   {"ws": 516}, {"stats": None}, {"logp": 2}, {"dx": 4098, "st": 99}, {"dx": 4099, "st": 100},
                   {"dx": 4096, "st": 100}):                                   # in place, but at another stride
        assert policy(**change) == BAD
    for p in ((0.0, 0.0), (-1.0, 0.0), (nan, 0.0), (inf, 0.0), (0.1, -0.1), (0.1, 0.6), (0.1, nan)):
        assert preference(p) == BAD
    for change in ({"pairs": 0}, {"pairs": -1}, {"pairs": 1 << 30}, {"start": None}, {"start": 260}, {"weight": None}, {"ref": None},
                   {"ref": 258}, {"dloss": 257}, {"ws": None}, {"ws": 516}, {"loss": None}, {"rewards": None}, {"logp": 2},
                   {"dx": 4098, "st": 99}, {"dx": 4096, "st": 100}):
        assert preference(**change) == BAD
    h = T.tgrad_policy(0.2, 0.2, 0.1)
    assert lib.tgrad_policy_loss(_logits(), None, 256, 256, 256, None, None, 512, 1024, None, None, 0, None) == BAD
    assert lib.tgrad_policy_loss(None, C.byref(h), 256, 256, 256, None, None, 512, 1024, None, None, 0, None) == BAD
    assert lib.tgrad_preference_loss(_logits(), None, 2, 256, 256, 256, None, 512, 1024, 2048, None, None, 0, None) == BAD
    for logp, lse in ((2, 256), (256, 2)):
        assert lib.tgrad_token_logprobs(_logits(), logp, lse, None) == BAD
    for lse, dlogp, dx, st in ((None, 256, 512, 100), (256, None, 512, 100), (256, 256, None, 100), (256, 256, 512, 99),
                               (256, 256, 4096, 100), (258, 256, 512, 100)):
        assert lib.tgrad_token_logprobs_backward(_logits(), lse, dlogp, dx, st, None) == BAD


def test_loss_scratch_sizes():
    lib = T.load()
    n = C.c_size_t(0)
    for rows, pairs in ((-1, 0), (1 << 31, 0), (1, -1), (1, 1 << 30)):
        assert lib.tgrad_loss_query_size(rows, pairs, C.byref(n)) == BAD
    assert lib.tgrad_loss_query_size(1, 1, None) == BAD
    sizes = []
    for rows, pairs in ((0, 0), (1000, 0), (1000, 10)):
        assert lib.tgrad_loss_query_size(rows, pairs, C.byref(n)) == T.TGRAD_OK
        sizes.append(n.value)
    assert 0 < sizes[0] <= sizes[1] and sizes[2] > 0


def test_bindings_refuse_tensors_that_do_not_fit():
    import torch

    from paper_2501_02379_amd import group, losses
    x, y, w = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    with pytest.raises(T.TgradError):                                          # not on a GPU
        losses.tgrad_token_logprobs(x, y)
    with pytest.raises(T.TgradError):
        losses.tgrad_policy_loss(x, y, w, w, w)
    with pytest.raises(T.TgradError):
        group.Group([])
    with pytest.raises(T.TgradError):
        group.Group([x])


def test_a_factor_on_another_gpu_is_refused():
    """The library is not reached: a pointer to another GPU's memory would be read by every later step."""
    from types import SimpleNamespace as N

    import torch

    class Scale:
        dtype, device = torch.float32, torch.device("cuda", 1)
        numel, is_neg, data_ptr = (lambda self: 1), (lambda self: False), (lambda self: 4096)
        get_device = lambda self: 1  # noqa: E731

    reached = []
    ctx = N(lib=N(tgrad_set_grad_scale=lambda *a: reached.append(a) or T.TGRAD_ERR_INVALID_ARG), handle=None,
            state_buf=N(get_device=lambda: 0))
    with pytest.raises(T.TgradError):
        T.Context.tgrad_set_grad_scale(ctx, Scale())
    assert not reached
