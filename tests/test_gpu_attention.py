"""Attention through a window with first tokens that stay visible, and its learned bias, forward and backward, against 64 bits."""
import pytest
import torch

import attention_reference as ref
from paper_2403_04206_amd import grawa

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


class Case:
    """Tensors of a call, and the call."""

    def __init__(self, K, N, Sq, Sk, H, G, D, dtype, seed=0, buckets=0, far=0, lengths=None, starts=None, shift=3, fused=False, **kinds):
        gen = generator(seed)
        self.K, self.N, self.Sq, self.Sk, self.H, self.G, self.D, self.dtype = K, N, Sq, Sk, H, G, D, dtype
        if fused:
            row = ref.make((K, N, Sq, (H + 2 * G) * D), dtype, gen)
            self.q, self.k, self.v = (t.unflatten(3, (-1, D)) for t in row.split([H * D, G * D, G * D], dim=3))
            back = torch.full_like(row, 7.0)
            self.dq, self.dk, self.dv = (t.unflatten(3, (-1, D)) for t in back.split([H * D, G * D, G * D], dim=3))
        else:
            self.q = ref.make((K, N, Sq, H, D), dtype, gen)
            self.k, self.v = (ref.make((K, N, Sk, G, D), dtype, gen) for _ in range(2))
            self.dq, self.dk, self.dv = (torch.full_like(t, 7.0) for t in (self.q, self.k, self.v))
        self.do = ref.make((K, N, Sq, H, D), dtype, gen)
        self.o = torch.full_like(self.do, 7.0)
        self.lse = torch.full((K, N, H, Sq), 7.0, device="cuda")
        self.bias = self.dbias = self.bucket_of = None
        self.starts = None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda").view(K, N)
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda").view(K, N)
        if buckets:
            self.bucket_of = grawa.log_buckets(buckets, far)
            rows = [torch.zeros((K, shift + H * buckets + 11), device="cuda", dtype=dtype) for _ in range(2)]
            self.rows, (self.bias, self.dbias) = rows, [r[:, shift:shift + H * buckets].view(K, H, buckets) for r in rows]
            self.bias.copy_(ref.make((K, H, buckets), dtype, gen))
        self.kinds = kinds
        self.plan = grawa.AttentionPlan(K, N, max(Sq, Sk), H, G, D, dtype=dtype, buckets=buckets, bucket_of=self.bucket_of, **kinds)

    def places(self):
        return dict(bias=self.bias, lengths=self.lengths, starts=self.starts)

    def forward(self, lse=True):
        self.plan.attention(self.q, self.k, self.v, self.o, lse_out=self.lse if lse else None, **self.places())

    def backward(self, accumulate=False):
        self.plan.attention_backward(self.do, self.q, self.k, self.v, self.o, self.lse, self.dq, self.dk, self.dv, dbias=self.dbias, accumulate=accumulate,
                                     **self.places())

    def want(self, do=True):
        return ref.attention(self.q, self.k, self.v, self.dtype, bias=self.bias, bucket_of=self.bucket_of, lengths=self.lengths, starts=self.starts,
                             do=self.do if do else None, **self.kinds)

    def check(self, train=True):
        self.forward(lse=train)
        if train:
            self.backward()
        torch.cuda.synchronize()
        worst = {}
        for name, (value, off) in self.want(train).items():
            if name == "lse" and not train:
                continue
            worst[name] = ref.check(getattr(self, name), value, off, name)
        print("[case] worst shares of the bounds", {n: "%.3f" % w for n, w in worst.items()}, flush=True)
        self.plan.destroy()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [8, 16, 40, 64, 72, 96, 128])
def test_widths(D, dtype):
    Case(2, 1, 150, 150, 2, 1, D, dtype, seed=D).check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("S", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 400])
def test_lengths(S, dtype):
    Case(1, 2, S, S, 2, 2, 64, dtype, seed=S, fused=True).check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 2), (32, 0), (33, 31), (64, 4), (100, 65), (128, 128), (129, 1), (300, 7), (1000, 3), (20, 200), (7, 1 << 40)])
def test_windows(window, sinks, dtype):
    Case(1, 1, 290, 290, 3, 1, 64, dtype, seed=window + sinks, window=window, sinks=sinks).check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("buckets,far,window,sinks", [(2, 3, 0, 0), (8, 20, 0, 0), (32, 128, 0, 0), (19, 77, 50, 3), (64, 900, 0, 0), (32, 128, 90, 70), (256, 1000, 0, 0)])
def test_bias(buckets, far, window, sinks, dtype):
    Case(2, 2, 270, 270, 2, 1, 64, dtype, seed=buckets, buckets=buckets, far=far, window=window, sinks=sinks).check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 104])
@pytest.mark.parametrize("biased", [False, True])
def test_padded_batches(D, biased, dtype):
    kinds = dict(buckets=16, far=40) if biased else {}
    Case(2, 4, 200, 200, 4, 2, D, dtype, seed=D, lengths=[200, 0, 1, 137, 64, 65, -3, 1000], starts=[0] * 8, window=77, sinks=2, **kinds).check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Sq,H,G,D", [(1, 1, 1, 64), (1, 4, 4, 64), (1, 32, 4, 128), (1, 64, 1, 64), (3, 6, 2, 80), (7, 16, 16, 64), (33, 2, 1, 64), (130, 4, 2, 128), (16, 5, 1, 64)])
@pytest.mark.parametrize("biased", [False, True])
def test_tokens_over_a_cache(Sq, H, G, D, biased, dtype):
    Sk = 700
    lengths = [700, 1, 2, Sq, 129, 333, 0, 512]
    kinds = dict(buckets=32, far=128) if biased else {}
    for window, sinks in ((0, 0), (200, 4)):
        Case(2, 4, Sq, Sk, H, G, D, dtype, seed=Sq + H, lengths=lengths, starts=[n - Sq for n in lengths], window=window, sinks=sinks, **kinds).check(train=False)


@pytest.mark.parametrize("dtype", DTYPES)
def test_gradients_of_a_chunk_over_a_cache(dtype):
    Case(1, 3, 70, 300, 4, 2, 64, dtype, seed=1, lengths=[300, 40, 250], starts=[230, -30, 180], window=90, sinks=5, buckets=8, far=60).check()


@pytest.mark.parametrize("dtype", DTYPES)
def test_default_place_is_the_end_of_the_keys(dtype):
    Case(1, 2, 5, 100, 2, 1, 64, dtype, seed=2).check()
    Case(1, 1, 100, 60, 2, 1, 64, dtype, seed=3).check()       # more queries than keys: the first 40 stand below 0 and see nothing


@pytest.mark.parametrize("dtype", DTYPES)
def test_long_sequences_share_their_keys_among_blocks(dtype):
    Case(1, 1, 1, 9000, 4, 2, 64, dtype, seed=3).check(train=False)
    Case(1, 1, 40, 5000, 8, 2, 128, dtype, seed=4, window=3001, sinks=9).check(train=False)
    Case(1, 1, 1500, 1500, 2, 1, 64, dtype, seed=5, window=100, sinks=3).check()
    Case(1, 1, 1500, 1500, 1, 1, 128, dtype, seed=6, window=100, sinks=200, buckets=12, far=300).check()
