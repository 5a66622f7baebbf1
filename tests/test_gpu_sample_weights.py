"""How exact the weights of sampling are: of two tokens with logits x and 0, the first stays if
exp(x / temperature) is at least min_p, and its weight lies within a few 2^-51 of that.

Bound: aug.h's 2^-51 + 2^-(s+1) = 1.5 * 2^-51 for two tokens (s = 51); min_p, a float32 above 1/2, is a
multiple of 2^-24 and is met as it is. Cases are further from the border than that, and nearer than 2^-49."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_sample import _run  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

# logit, temperature, min_p, whether it stays: float32 values, most with 32 x log2(e) / temperature half way between integers
CASES = [
    (-0.1541569083929062, 0.5699783563613892, 0.7630276679992676, True), (-0.09326106309890747, 0.7862573266029358, 0.8881506323814392, True),
    (-0.18411242961883545, 1.301867961883545, 0.8681231141090393, True), (-0.7822906970977783, 1.7619683742523193, 0.6414738893508911, True),
    (-0.33181580901145935, 1.2279478311538696, 0.763211727142334, True), (-0.1516110599040985, 1.2662384510040283, 0.8871569037437439, True),
    (-0.08190987259149551, 0.6923753023147583, 0.8884270787239075, True), (-0.17218142747879028, 1.7518715858459473, 0.9063912034034729, True),
    (-0.15645775198936462, 1.6101458072662354, 0.9074018001556396, True), (-0.08448772877454758, 1.1093648672103882, 0.926669180393219, True),
    (-0.4267430305480957, 1.4601609706878662, 0.7465762495994568, True), (-0.20333150029182434, 1.7007094621658325, 0.8873135447502136, True),
    (-0.4311923384666443, 0.9272396564483643, 0.628117561340332, False), (-0.1689692735671997, 1.1942687034606934, 0.8680695295333862, False),
    (-0.24872726202011108, 0.5882777571678162, 0.6552058458328247, False), (-0.07673089951276779, 0.7876657247543335, 0.9071789383888245, False),
    (-0.3440750241279602, 1.678794026374817, 0.814685046672821, False), (-0.707158625125885, 1.5913975238800049, 0.641232430934906, False),
    (-0.5651650428771973, 1.8031448125839233, 0.7309333682060242, False), (-0.028993602842092514, 0.535499095916748, 0.9472965002059937, False),
]


def test_weights_at_the_floor():
    x = torch.tensor([[c[0], 0.0] for c in CASES], device="cuda")
    settings = [dict(temperature=t, min_p=p) for _, t, p, _ in CASES]
    tokens, probs = _run(x, [0.0] * len(CASES), settings)
    for (logit, t, p, stays), token, prob in zip(CASES, tokens, probs):
        logit, t, p = (np.longdouble(np.float32(v)) for v in (logit, t, p))
        w = np.exp(logit / t)
        assert 1.5 * 2.0 ** -51 < abs(w - p) < 2.0 ** -49 and (w >= p) == stays          # the case itself
        assert token == (0 if stays else 1), (float(logit), float(t), float(p), token)
        share = w / (1 + w) if stays else 1.0
        assert abs(prob - share) <= share * (2.0 ** -24 + 2.0 ** -48)
