"""Arguments that the entry points of the softmax layer refuse before any device work (no GPU needed)."""
import ctypes

from paper_1802_09113_amd import binding
from paper_1802_09113_amd.binding import SSN_E_INVALID_ARG, SSN_E_UNSUPPORTED, SSN_OK

P = ctypes.c_void_p


def rows(**kw):
    d = binding.ssn_rows(4, 100, binding.SSN_F32, 0, 64, 100, None, 0, 64, 1, 0, None)
    for name, v in kw.items():
        setattr(d, name, v)
    return d


def forward(d, logp=64, k_out=64):
    return binding.lib().ssn_logprobs(ctypes.byref(d), P(logp), None, None, None, P(k_out), P(k_out), None, 0)


def test_log_probabilities():
    L = binding.lib()
    size = ctypes.c_int64()
    assert L.ssn_logprobs(None, None, None, None, None, None, None, None, 0) == SSN_E_INVALID_ARG
    assert L.ssn_logprobs_workspace(None, ctypes.byref(size)) == SSN_E_INVALID_ARG
    assert L.ssn_logprobs_workspace(ctypes.byref(rows()), None) == SSN_E_INVALID_ARG
    for bad in (dict(n=-1), dict(C=0), dict(C=1, reference=1), dict(reference=2), dict(dtype=4), dict(dtype=-1), dict(Z=None), dict(Z=66),
                dict(ldz=99), dict(m=-1), dict(k=-1), dict(C=3, k=4), dict(labels=None), dict(labels=66), dict(allowed=64, ld_allowed=3), dict(allowed=66, ld_allowed=4), dict(allowed=64, ld_allowed=-4)):
        assert forward(rows(**bad)) == SSN_E_INVALID_ARG, bad
    for bad in (dict(C=1 << 31), dict(n=1 << 31), dict(m=65), dict(k=65)):
        assert forward(rows(**bad)) == SSN_E_UNSUPPORTED, bad
    assert forward(rows(), logp=None) == SSN_E_INVALID_ARG
    assert forward(rows(), logp=66) == SSN_E_INVALID_ARG
    assert forward(rows(dtype=binding.SSN_F64), logp=68) == SSN_E_INVALID_ARG
    assert forward(rows(k=2), k_out=66) == SSN_E_INVALID_ARG
    assert forward(rows(k=2), k_out=None) == SSN_E_INVALID_ARG
    assert forward(rows(n=0, Z=None, labels=None)) == SSN_OK
    size.value = 5
    assert L.ssn_logprobs_workspace(ctypes.byref(rows(n=0)), ctypes.byref(size)) == SSN_OK and size.value == 0


def test_their_gradient():
    L = binding.lib()

    def grad(d, logp=64, maxpart=64, logpart=64, entropy=64, dlogp=64, dlse=None, dentropy=None, dZ=128, ld=100):
        return L.ssn_logprobs_grad(ctypes.byref(d), P(logp), P(maxpart), P(logpart), P(entropy), P(dlogp), P(dlse), P(dentropy), P(dZ), ld)

    for bad in (dict(logp=None), dict(maxpart=None), dict(logpart=None), dict(dlogp=None), dict(dZ=None), dict(dZ=130), dict(ld=99),
                dict(entropy=None, dentropy=64), dict(dZ=64, ld=101), dict(dlse=66), dict(maxpart=65)):
        assert grad(rows(), **bad) == SSN_E_INVALID_ARG, bad
    assert grad(rows(ldz=50)) == SSN_E_INVALID_ARG
    assert grad(rows(m=65)) == SSN_E_UNSUPPORTED
    assert grad(rows(n=0), dZ=None) == SSN_OK


def test_weights_in_4_bits():
    L = binding.lib()

    def quantize(dtype=binding.SSN_F32, W=64, sj=20, sc=1, **kw):
        b = binding.ssn_q4(100, 20, 32, 0, 64, 64)
        for name, v in kw.items():
            setattr(b, name, v)
        return L.ssn_q4_quantize(ctypes.byref(b), dtype, P(W), sj, sc, None)

    for bad in (dict(p=0), dict(K=0), dict(group=16), dict(group=0), dict(reserved=1), dict(packed=None), dict(scales=None), dict(packed=72),
                dict(scales=66), dict(W=None), dict(W=66), dict(dtype=9), dict(sj=0), dict(sc=0)):
        assert quantize(**bad) == SSN_E_INVALID_ARG, bad
    assert quantize(p=1 << 31) == SSN_E_UNSUPPORTED and quantize(K=1 << 31) == SSN_E_UNSUPPORTED
    assert L.ssn_q4_quantize(None, 0, None, 1, 1, None) == SSN_E_INVALID_ARG

    b, size = binding.ssn_q4(100, 20, 32, 0, 64, 64), ctypes.c_int64()
    assert L.ssn_q4_margins_workspace(None, 0, 1, ctypes.byref(size)) == SSN_E_INVALID_ARG
    assert L.ssn_q4_margins_workspace(ctypes.byref(b), 0, 1, None) == SSN_E_INVALID_ARG
    assert L.ssn_q4_margins_workspace(ctypes.byref(b), 0, -1, ctypes.byref(size)) == SSN_E_INVALID_ARG
    assert L.ssn_q4_margins_workspace(ctypes.byref(b), 7, 1, ctypes.byref(size)) == SSN_E_INVALID_ARG
    assert L.ssn_q4_margins_workspace(ctypes.byref(b), binding.SSN_F64, 1, ctypes.byref(size)) == SSN_E_UNSUPPORTED
    assert L.ssn_q4_margins_workspace(ctypes.byref(b), 0, 1 << 19, ctypes.byref(size)) == SSN_E_UNSUPPORTED
    size.value = 5
    assert L.ssn_q4_margins_workspace(ctypes.byref(b), 0, 0, ctypes.byref(size)) == SSN_OK and size.value == 0
    assert L.ssn_q4_margins(None, 0, 1, None, 0, 0, None, 0, None, 0, None) == SSN_E_INVALID_ARG

    def margins(dtype=0, n=2, X=64, ldx=100, zdtype=0, Z=64, ldz=20, **kw):
        b = binding.ssn_q4(100, 20, 32, 0, 64, 64)
        for name, v in kw.items():
            setattr(b, name, v)
        return L.ssn_q4_margins(ctypes.byref(b), dtype, n, P(X), ldx, zdtype, P(Z), ldz, None, 0, None)

    for bad in (dict(packed=None), dict(packed=72), dict(scales=None), dict(scales=68), dict(X=None), dict(X=66), dict(Z=None), dict(Z=65),
                dict(ldx=99), dict(ldz=19), dict(zdtype=binding.SSN_F16), dict(zdtype=binding.SSN_F64), dict(n=-1), dict(group=96)):
        assert margins(**bad) == SSN_E_INVALID_ARG, bad
    assert margins(dtype=binding.SSN_F64) == SSN_E_UNSUPPORTED
    assert margins(n=0, X=None, Z=None, packed=None) == SSN_OK
