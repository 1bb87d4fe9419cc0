// What the attention translation units share (GPU code only; everything has internal linkage).
#pragma once
#include "fq_attn_rules.h"
#include "fq_internal.h"

namespace fq {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

template <int DT> struct Stored;
template <> struct Stored<FQ_F32> { typedef float type; };
template <> struct Stored<FQ_F16> { typedef _Float16 type; };
template <> struct Stored<FQ_BF16> { typedef __bf16 type; };

constexpr float SLACK = 8.0f;   // accumulators are rescaled only when a maximum has grown by more than a factor 2^8
constexpr float LOG2E = 1.44269504088896340736f;

}  // namespace
}  // namespace fq
