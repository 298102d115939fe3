"""What q8_quantize_rows, q8_linear and policy_sample refuse, and the empty calls they accept, before any device work."""
import ctypes as C

import paper_2111_01264_amd as P

LIB = C.CDLL(P.LIB_PATH)
for _name in ("q8_quantize_rows", "q8_linear", "policy_sample", "policy_sample_workspace"):
    getattr(LIB, _name).restype, getattr(LIB, _name).argtypes = P.EXPORTS[_name]
LIB.dqn_last_error.restype = C.c_char_p
A = 0x1000   # an address that is never touched: every call below ends on the host


def call(fn, order, good, **bad):
    assert set(bad) <= set(order)
    return getattr(LIB, fn)(*[{**good, **bad}[k] for k in order])


QUANT = "x type ldx rows cols q ldq scale values ldv stream".split()
QUANT_GOOD = dict(x=A, type=1, ldx=8, rows=2, cols=8, q=A, ldq=8, scale=A, values=None, ldv=0, stream=None)


def test_quantize_refusals():
    for bad in (dict(type=3), dict(type=-1), dict(rows=-1), dict(cols=-1), dict(rows=P.Q8_QUANTIZE_MAX_ROWS + 1), dict(cols=P.Q8_QUANTIZE_MAX_COLS + 1, ldx=1 << 31, ldq=1 << 31), dict(x=None), dict(scale=None),
                dict(q=None), dict(ldx=7), dict(ldq=7), dict(values=A, ldv=7), dict(x=A + 1), dict(type=0, x=A + 2), dict(scale=A + 2), dict(values=A + 1, ldv=8)):
        assert call("q8_quantize_rows", QUANT, QUANT_GOOD, **bad) == P.DQN_EINVAL, bad
        assert b"q8_quantize_rows" in LIB.dqn_last_error()
    assert call("q8_quantize_rows", QUANT, QUANT_GOOD, rows=0, x=None, scale=None, q=None) == P.DQN_OK


LINEAR = "x ldx sx w ldw sw bias relu M N K y type ldy stream".split()
LINEAR_GOOD = dict(x=A, ldx=16, sx=A, w=A, ldw=16, sw=A, bias=None, relu=0, M=2, N=4, K=16, y=A, type=0, ldy=4, stream=None)


def test_linear_refusals():
    for bad in (dict(type=3), dict(M=-1), dict(N=-1), dict(K=-1), dict(K=P.Q8_LINEAR_MAX_K + 1, ldx=1 << 20, ldw=1 << 20), dict(M=P.Q8_LINEAR_MAX_ROWS + 1),
                dict(N=P.Q8_LINEAR_MAX_ROWS + 1, ldy=1 << 20), dict(x=None), dict(w=None), dict(sx=None), dict(sw=None), dict(y=None), dict(ldx=15), dict(ldw=15), dict(ldy=3),
                dict(y=A + 2), dict(sx=A + 1), dict(sw=A + 2), dict(bias=A + 2), dict(type=1, y=A + 1)):
        assert call("q8_linear", LINEAR, LINEAR_GOOD, **bad) == P.DQN_EINVAL, bad
        assert b"q8_linear" in LIB.dqn_last_error()
    assert call("q8_linear", LINEAR, LINEAR_GOOD, M=0, x=None, y=None) == P.DQN_OK
    assert call("q8_linear", LINEAR, LINEAR_GOOD, N=0, w=None, y=None) == P.DQN_OK


SAMPLE = "scores type ld rows n temperature top_k top_p min_p u index logp work work_bytes stream".split()
SAMPLE_GOOD = dict(scores=A, type=0, ld=18, rows=2, n=18, temperature=None, top_k=None, top_p=None, min_p=None, u=A, index=A, logp=None, work=None, work_bytes=0, stream=None)


def test_sample_refusals():
    for bad in (dict(type=7), dict(rows=-1), dict(n=-1), dict(n=P.POLICY_SAMPLE_MAX_N + 1, ld=1 << 23), dict(rows=P.POLICY_SAMPLE_MAX_ROWS + 1), dict(scores=None), dict(u=None),
                dict(index=None), dict(ld=17), dict(scores=A + 2), dict(type=2, scores=A + 1), dict(temperature=A + 1), dict(top_k=A + 2), dict(top_p=A + 3), dict(min_p=A + 1),
                dict(u=A + 2), dict(index=A + 2), dict(logp=A + 2), dict(work=A + 8)):
        assert call("policy_sample", SAMPLE, SAMPLE_GOOD, **bad) == P.DQN_EINVAL, bad
        assert b"policy_sample" in LIB.dqn_last_error()
    assert call("policy_sample", SAMPLE, SAMPLE_GOOD, rows=0, scores=None, u=None, index=None) == P.DQN_OK


def test_sample_workspace_is_asked_for():
    for rows, n in ((1, 131072), (1, 1 << 22), (7, 50021), (512, 18), (0, 5), (-1, 5), (5, -1), (1, P.POLICY_SAMPLE_MAX_N + 1)):
        need = P.policy_sample_workspace(rows, n)
        assert need >= 0 and (need == 0 or 0 < rows and 0 < n <= P.POLICY_SAMPLE_MAX_N)
        if need:
            big = dict(rows=rows, n=n, ld=n)
            assert call("policy_sample", SAMPLE, SAMPLE_GOOD, **big) == P.DQN_EINVAL
            assert call("policy_sample", SAMPLE, SAMPLE_GOOD, **big, work=A, work_bytes=need - 1) == P.DQN_EINVAL
            assert b"work" in LIB.dqn_last_error()
