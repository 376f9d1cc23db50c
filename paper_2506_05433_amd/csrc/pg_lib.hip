// The library's one translation unit: the grouped-attention calls with their host helpers, then the calls beside them.
#include <initializer_list>

#include "pg_attn.hip"
#include "pg_linear.hpp"
#include "pg_policy.hpp"

#include "pg_linear_api.hpp"
#include "pg_policy_api.hpp"
