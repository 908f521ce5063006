"""What adloco_round's binding makes of the batches that the callback returns: every block is read as its kind in the list of
blocks says, and a batch that does not fit it is refused before the library sees its address.  The library and the GPU
tensors are stand-ins: nothing is launched (no GPU needed)."""
import pytest
import torch

import paper_2508_18182_amd as A
from paper_2508_18182_amd import binding as bind

B, T, D, N = 3, 5, 8, 8 + 4 * 6


class OnGpu:
    """A host tensor that says that it lives on a GPU."""
    is_cuda = True

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)


def gpu(*shape, dtype=torch.float32):
    return OnGpu(torch.zeros(shape, dtype=dtype))


@pytest.fixture
def batch(monkeypatch):
    """Calls adloco_round with a batch for [block of `kind`, linear block]; the descriptors that the library would get."""
    def run(kind, first, linear=None):
        seen = []

        class Lib:
            @staticmethod
            def adloco_round(h, cfg, arr, k, tmpl, n, size, cb, reports, stream):
                rc = cb(arr[0].user, 0, 0, 0, B, None, tmpl, n, None)
                seen.extend((d.delta, d.delta_row_stride, d.a, d.flags) for d in tmpl)
                return 5 if rc else 0

        class Ctx:
            device, _h = 0, None

            @staticmethod
            def _check(rc):
                assert rc == 0

        monkeypatch.setattr(bind, "load_library", lambda: Lib)
        monkeypatch.setattr(bind, "_stream_ptr", lambda stream: None)
        trainer = dict(theta_outer=gpu(N), momentum=gpu(N), b_req=B, acc=gpu(2, dtype=torch.float64), uid=0, per_sample_sqnorm=gpu(8),
                       workers=[dict(theta=gpu(N), exp_avg=gpu(N), exp_avg_sq=gpu(N), grad=gpu(N), step=0)])
        cfg = dict(T=T, dtype=A.ADLOCO_BF16, inner_steps=1, n_switch=2, merge_w=0, nesterov=1, b_max=8, b_cap=64, eta=0.3,
                   lr_inner=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1, lr_outer=0.7, mu_outer=0.9)
        linear = linear or dict(a=gpu(B, T, 6, dtype=torch.bfloat16), delta=gpu(B, T, 4, dtype=torch.bfloat16))
        A.adloco_round(Ctx, cfg, [trainer], [dict(kind=kind, d_out=D), dict(d_in=6, d_out=4)], lambda *a: [first, linear])
        return seen
    return run


def test_each_kind_gets_what_it_reads(batch):
    delta, x, sums = gpu(B, T, D, dtype=torch.bfloat16), gpu(B, T, D, dtype=torch.bfloat16), gpu(B, D)
    assert batch("vector", dict(delta=delta))[0] == (delta.data_ptr(), D, None, A.ADLOCO_KIND_VECTOR)
    assert batch("vector", dict(delta=delta, x=x))[0] == (delta.data_ptr(), D, x.data_ptr(), A.ADLOCO_KIND_VECTOR)
    assert batch("vector", dict(delta=delta, sums=None))[0][0] == delta.data_ptr()
    assert batch("sample_sums", dict(sums=sums))[0] == (sums.data_ptr(), D, None, A.ADLOCO_KIND_SAMPLE_SUMS)


def test_samples_of_sums_may_be_a_stride_apart(batch):
    wide = gpu(B, D + 5)
    sums = OnGpu(wide.t[:, 2:2 + D])
    assert batch("sample_sums", dict(sums=sums))[0][:2] == (sums.data_ptr(), D + 5)


def test_sums_of_one_column(batch, monkeypatch):
    monkeypatch.setitem(globals(), "D", 1)
    monkeypatch.setitem(globals(), "N", 1 + 4 * 6)
    sums = OnGpu(torch.zeros(1, B).t())                                      # (torch calls it contiguous)
    assert batch("sample_sums", dict(sums=sums))[0][:2] == (sums.data_ptr(), 1)


@pytest.mark.parametrize("kind,first", [
    ("vector", dict(sums=gpu(B, D))),                                        # T rows a sample would be read of one
    ("vector", dict(delta=gpu(B, T, D, dtype=torch.bfloat16), sums=gpu(B, D))),
    ("sample_sums", dict(delta=gpu(B, T, D, dtype=torch.bfloat16))),         # 16-bit rows read as fp32 sums
    ("sample_sums", dict(delta=gpu(B, 1, D))),
    ("sample_sums", dict(sums=gpu(B, D, dtype=torch.bfloat16))),
    ("sample_sums", dict(sums=gpu(B, D + 1))),                               # rows of another width
    ("sample_sums", dict(sums=gpu(B + 1, D))),
    ("sample_sums", dict(sums=gpu(B * D))),
    ("sample_sums", dict(sums=OnGpu(torch.zeros(D).expand(B, D)))),          # every sample the same row
    ("sample_sums", dict(sums=OnGpu(torch.zeros(D, B).t()))),
    ("sample_sums", dict(sums=torch.zeros(B, D))),                           # in host memory
])
def test_a_batch_that_is_not_of_its_blocks_kind_is_refused(batch, kind, first):
    with pytest.raises(ValueError, match="block 0"):
        batch(kind, first)


def test_sums_for_a_linear_block_are_refused(batch):
    with pytest.raises(ValueError, match="block 1"):
        batch("vector", dict(delta=gpu(B, T, D, dtype=torch.bfloat16)), linear=dict(sums=gpu(B, 4)))
